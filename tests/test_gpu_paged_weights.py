"""How weights enter the second product of bf16 and 8-bit rows: as the sum of two bf16 numbers, the second to nearest.

The first part is the largest bf16 number below the weight, what is left is at most 2^-7 of the weight's power of two and
loses half a step of its own eight digits: 2^-16 of the weight.  Seen through values that cancel all the rest."""
import math

import numpy as np
import pytest
import torch

from paged_cases import DEV, normal

pytestmark = pytest.mark.gpu

LN2 = float(np.float32(math.log(2.0)))      # logits in powers of two
BOTH = pytest.mark.parametrize("wide", [False, True])
WIDE = 2000


def _codes(x, one=0x38):
    """Numbers as codes of +-1 and scales."""
    return torch.where(x < 0, one | 0x80, one).to(torch.uint8), x.abs()


def _pool(cache, k0, v):
    """A page of 16 positions per row: k0, v [R][16] are the keys' first element and the values, the same in all columns."""
    import paper_2502_17599_amd as pkg
    R, d = k0.shape[0], 64
    k = torch.zeros((R, 1, 16, d), dtype=torch.float32, device=DEV)
    if cache == "fp8":
        kc, ks = _codes(k0)
        codes = torch.zeros(k.shape, dtype=torch.uint8, device=DEV)
        codes[:, 0, :, 0] = kc
        vc, vs = _codes(v)
        return pkg.PagePool(codes, vc[:, None, :, None].expand(-1, -1, -1, d).contiguous(), ks[:, None].contiguous(), vs[:, None].contiguous())
    k[:, 0, :, 0] = k0
    return pkg.PagePool(k.bfloat16(), v[:, None, :, None].expand(-1, -1, -1, d).bfloat16().contiguous())


@BOTH
@pytest.mark.parametrize("G", [1, 2, 4, 5, 8, 16])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_weights_lose_less_than_half_a_step_of_sixteen_digits(cache, G, wide):
    """Row r: one position with the weight w = 2^x_r and the value 1, three with the weight 1 whose values add up to -w.  The
    result is what the weight lost, over 3 + w.  Beside 2^-16 w there are the exponential (two roundings of the argument, below 1,
    and one step of the result: 2^-22 w) and the four products' sums (2^-23), and the output's rounding (2^-8 of it)."""
    import paper_2502_17599_amd as pkg
    print(f"\n[weights] {cache} G={G} wide={wide}", flush=True)
    x = -torch.arange(1, 257, dtype=torch.float64) / 256                    # numbers that bf16 holds
    w = torch.exp(LN2 * x)
    parts, left = [], w.clone()
    for _ in range(3):
        parts.append(left.bfloat16().double())
        left = left - parts[-1]
    k0, v = torch.zeros(256, 16), torch.zeros(256, 16)
    k0[:, 0], v[:, 0] = x.float(), 1.0
    for i, p in enumerate(parts):
        v[:, 1 + i] = -p.float()
    pool = _pool(cache, k0.to(DEV), v.to(DEV))
    table = torch.full((256, WIDE if wide else 1), -1, dtype=torch.int32, device=DEV)
    table[:, 0] = torch.arange(256, device=DEV)
    lens = torch.full((256,), 4, dtype=torch.int32, device=DEV)
    q = torch.zeros((256, G, 64), dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 1.0
    out = pkg.PagedDecoder(pool, 256, G, table.shape[1], softmax_scale=LN2)(q, table, lens).double().cpu()
    want = (left / (3 + w))[:, None, None]
    tol = ((2.0 ** -16 + 2.0 ** -22) * w + 2.0 ** -23)[:, None, None] / (3 + w)[:, None, None]
    tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    err = (out - want).abs()
    assert (err <= tol).all(), float((err / tol).max())
    # to nearest: the losses go both ways.  Each is spread over +-2^-16 w (2^-16.8 w rms at most), so that five deviations of the
    # mean of 256 are 2^-18.5; cut off, they would all go down, by 2^-17 on average.
    mean = float((out[:, 0, 0] * (3 + w) / w).mean())
    assert abs(mean) <= 2.0 ** -18.5


@BOTH
@pytest.mark.parametrize("G", [1, 8, 16])
def test_infinite_values_of_small_weights(G, wide):
    """Weights down to 2^-100 have a second part that is a normal number: an infinity shows."""
    import paper_2502_17599_amd as pkg
    x = -torch.cat([torch.arange(120, 201) / 2.0, torch.arange(1, 100) / 64.0])      # numbers that bf16 holds
    R = len(x)
    k0, v = torch.zeros(R, 16), torch.ones(R, 16)
    k0[:, 1] = x
    v[:, 1] = float("inf")
    pool = _pool("bf16", k0.to(DEV), v.to(DEV))
    pool.v_pages[:, :, 1, 5] = float("-inf")
    pool.v_pages[:, :, 1, 6:] = 1.0
    table = torch.full((R, WIDE if wide else 1), -1, dtype=torch.int32, device=DEV)
    table[:, 0] = torch.arange(R, device=DEV)
    lens = torch.full((R,), 2, dtype=torch.int32, device=DEV)
    q = torch.zeros((R, G, 64), dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 1.0
    out = pkg.PagedDecoder(pool, R, G, table.shape[1], softmax_scale=LN2)(q, table, lens)
    assert (out[..., :5] == float("inf")).all() and (out[..., 5] == float("-inf")).all() and torch.isfinite(out[..., 6:]).all()
