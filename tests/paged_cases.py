"""Inputs and tolerances of the paged cache's tests."""
import math

import numpy as np
import torch

from oracle import fp8_oracle

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}     # half a step of the type, relative


def wide(t):
    return t.detach().to(torch.float64).cpu().numpy()


def normal(seed, *shape, dtype="f32"):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(DT[dtype]).to(DEV)


def make_pool(kind, n_pages, heads, page, d, seed=0, joint=False):
    """A pool of random contents; ``joint``: K and V pages next to each other."""
    import paper_2502_17599_amd as pkg
    if kind == "fp8":
        g = torch.Generator().manual_seed(seed)
        codes = [torch.randint(0, 256, (n_pages, heads, page, d), generator=g, dtype=torch.uint8) for _ in range(2)]
        codes = [torch.where((c & 127) == 127, c - 1, c).to(DEV) for c in codes]      # no NaN
        scales = [(torch.rand(n_pages, heads, page, generator=g) * 0.01 + 0.001).to(DEV) for _ in range(2)]
        return pkg.PagePool(*codes, *scales)
    if joint:
        both = normal(seed, n_pages, 2, heads, page, d, dtype=kind)
        return pkg.PagePool(both[:, 0], both[:, 1])
    return pkg.PagePool(normal(seed, n_pages, heads, page, d, dtype=kind), normal(seed + 1, n_pages, heads, page, d, dtype=kind))


def values(pool):
    """(K, V) pages in 64 bits."""
    if pool.k_scales is None:
        return wide(pool.k_pages), wide(pool.v_pages)
    table = fp8_oracle.e4m3_decode_table()
    return tuple(table[c.cpu().numpy()] * wide(s)[..., None] for c, s in ((pool.k_pages, pool.k_scales), (pool.v_pages, pool.v_scales)))


def make_table(lens, page, n_pages, seed=0, width=None):
    """Distinct pages in random order for rows of these lengths; -7 behind them."""
    held = [-(-n // page) for n in lens]
    order = np.random.default_rng(seed).permutation(n_pages)[:sum(held)]
    assert len(order) == sum(held)
    table, at = np.full((len(lens), width or max(1, max(held))), -7, np.int32), 0
    for r, n in enumerate(held):
        table[r, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)


def attention_tolerance(ref, v, logit, n, d, dtype):
    """fp32 sums of d products (error sqrt(d) roundings of the logit, which the weight takes over relatively) and of n terms
    spread over 64 lane groups and joins; bf16 kernels split a weight in two parts (2^-15 of it lost at most) and round
    the output once."""
    fp32 = 2.0 ** -23 * (math.sqrt(d) + math.sqrt(n / 64) + 8) * (1 + logit)
    return (fp32 + (2.0 ** -15 if dtype == "bf16" else 0.0)) * np.abs(v).max() + STEP[dtype] * np.abs(ref)
