"""Rotary positions against the oracle in 64 bits.

Tolerance: an element is a c - b s of one pair.  The angle in turns is rounded to fp32 (half a step of at most 1/2 turn:
2^-25 turns = 3.2 * 2^-24 rad), sine and cosine are good to 2 steps of their value (2^-23 .. 2^-22), two products and a sum
round once each (2^-24 each): together less than 2^-20 of |a| + |b|, of which an output in bf16 loses half a step more.
The angle's product in 64 bits has an error of 2^-52 turns per turn: 2^-52 * 2^31 * 2 pi < 2^-18 for the largest positions
with a frequency of 1, counted where positions are that large."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paged_cases import DEV, DT, STEP, normal, wide

pytestmark = pytest.mark.gpu


def _plan(rot, axes, interleaved, seed):
    import paper_2502_17599_amd as pkg
    half = rot // 2
    freq = torch.pow(torch.tensor(1e4, dtype=torch.float64), -torch.arange(half, dtype=torch.float64) / half)
    axis = torch.from_numpy(np.random.default_rng(seed).integers(0, axes, half).astype(np.uint8))
    return pkg.RotaryPlan(freq.to(DEV), axis.to(DEV) if axes > 1 else None, axes, interleaved), freq.numpy(), axis.numpy() if axes > 1 else None


def _check(name, got, x, pos, freq, axis, interleaved, inverse, dtype, angle=0.0):
    want = P.rotate(wide(x), pos, freq, axis, interleaved, inverse)
    half = len(freq)
    size = np.abs(wide(x))
    partner = size.copy()
    i = np.arange(half) * 2 if interleaved else np.arange(half)
    j = i + 1 if interleaved else i + half
    partner[..., i], partner[..., j] = size[..., j], size[..., i]
    tol = (2.0 ** -20 + angle) * (size + partner) + STEP[dtype] * np.abs(want)
    tol[..., 2 * half:] = 0.0
    err = np.abs(wide(got) - want)
    assert (err <= tol).all(), (name, float((err - tol).max()))


@pytest.mark.parametrize("T,Hq,Hk,d,dtype,rot,axes,interleaved,inverse", [
    (1, 1, 1, 64, "f32", 64, 1, False, False), (1, 28, 4, 128, "bf16", 128, 3, False, False), (7, 3, 1, 128, "f32", 128, 4, True, False),
    (129, 4, 4, 64, "bf16", 32, 2, False, True), (33, 5, 1, 128, "bf16", 18, 3, False, False), (50, 8, 2, 64, "f32", 6, 1, False, True),
    (1000, 7, 1, 128, "bf16", 96, 3, True, True), (257, 2, 2, 128, "f32", 2, 2, False, False), (65, 32, 8, 128, "bf16", 126, 3, True, False),
    (4100, 6, 2, 64, "bf16", 64, 3, False, False)])
def test_against_the_oracle(T, Hq, Hk, d, dtype, rot, axes, interleaved, inverse):
    import paper_2502_17599_amd as pkg
    print(f"\n[rotary] T={T} {Hq}/{Hk} d={d} {dtype} rot={rot} axes={axes} interleaved={interleaved} inverse={inverse}", flush=True)
    rope, freq, axis = _plan(rot, axes, interleaved, T)
    pos = np.random.default_rng(T).integers(0, 200000, size=(axes, T)).astype(np.int32)
    p = torch.from_numpy(pos).to(DEV)
    q, k = normal(1, T, Hq, d, dtype=dtype), normal(2, T, Hk, d, dtype=dtype)
    qo, ko = pkg.meda_rotary(q, k, p, rope, inverse=inverse)
    _check("q", qo, q, pos, freq, axis, interleaved, inverse, dtype)
    _check("k", ko, k, pos, freq, axis, interleaved, inverse, dtype)
    # from the fused projection, head by head, and in place: the same bits
    qkv = torch.cat([q, k, k], 1).contiguous()
    q2, k2 = (torch.full((h, T, d), 7.0, dtype=DT[dtype], device=DEV) for h in (Hq, Hk))
    pkg.meda_rotary(qkv[:, :Hq], qkv[:, Hq:Hq + Hk], p, rope, q2.transpose(0, 1), k2.transpose(0, 1), inverse=inverse)
    assert torch.equal(q2.transpose(0, 1), qo) and torch.equal(k2.transpose(0, 1), ko)
    a, b = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    pkg.meda_rotary(a, b, p, rope, a, b, inverse=inverse)
    assert torch.equal(a, qo) and torch.equal(b, ko) and torch.equal(qkv[:, Hq + Hk:], k)
    # queries alone
    alone, none = pkg.meda_rotary(q, None, p, rope, inverse=inverse)
    assert none is None and torch.equal(alone, qo)


def test_far_and_negative_positions():
    import paper_2502_17599_amd as pkg
    rope, freq, _ = _plan(128, 1, False, 0)
    pos = np.array([[-1, 0, 2 ** 31 - 1, -2 ** 31, 131071, -131072]], np.int32)
    q = normal(3, 6, 2, 128)
    out, _ = pkg.meda_rotary(q, None, torch.from_numpy(pos).to(DEV), rope)
    _check("q", out, q, pos, freq, None, False, False, "f32", angle=2.0 ** -18)
    assert torch.equal(out[1], q[1])


def test_inverse_is_the_gradient():
    """<g, R x> = <R^T g, x> in 64 bits of fp32 outputs, for random directions: each side rounds 2^-20 per pair."""
    import paper_2502_17599_amd as pkg
    rope, freq, axis = _plan(96, 3, False, 5)
    T, H, d = 40, 3, 128
    pos = torch.randint(0, 5000, (3, T), dtype=torch.int32, generator=torch.Generator().manual_seed(1)).to(DEV)
    x, g = normal(4, T, H, d), normal(5, T, H, d)
    y, _ = pkg.meda_rotary(x, None, pos, rope)
    dx, _ = pkg.meda_rotary(g, None, pos, rope, inverse=True)
    a, b = (wide(g) * wide(y)).sum(), (wide(dx) * wide(x)).sum()
    assert abs(a - b) <= 2 * 2.0 ** -20 * 2 * np.abs(wide(g) * np.abs(wide(x)).max()).sum()
    # and by differences of the forward pass, one element at a time
    for at in ((0, 0, 3), (17, 1, 51), (39, 2, 95), (5, 0, 127)):
        h = 0.5
        hi, lo = x.clone(), x.clone()
        hi[at] += h; lo[at] -= h
        diff = ((wide(pkg.meda_rotary(hi, None, pos, rope)[0]) - wide(pkg.meda_rotary(lo, None, pos, rope)[0])) * wide(g)).sum() / (2 * h)
        # the pair's two outputs, 2^-20 of their inputs each, on both sides
        assert abs(diff - wide(dx)[at]) <= 4 * 2.0 ** -20 * (np.abs(wide(x[at[0], at[1]])).max() + h) * 2 * np.abs(wide(g[at[0], at[1]])).max() / h


def test_infinities_stay_in_their_pair_and_nothing_is_done_for_no_tokens():
    import paper_2502_17599_amd as pkg
    for interleaved in (False, True):
        rope, _, _ = _plan(32, 1, interleaved, 0)
        x = normal(6, 2, 1, 64, dtype="bf16")
        x[0, 0, 40] = float("inf"); x[0, 0, 63] = float("nan"); x[1, 0, 3] = float("-inf")
        pos = torch.tensor([5, 7], dtype=torch.int32, device=DEV)
        out, _ = pkg.meda_rotary(x, None, pos, rope)
        assert torch.isinf(out[0, 0, 40]) and torch.isnan(out[0, 0, 63]) and torch.isfinite(out[0, 0, :40]).all()
        bad = ~torch.isfinite(out[1, 0])
        assert sorted(torch.nonzero(bad).flatten().tolist()) == ([2, 3] if interleaved else [3, 19])
        empty, _ = pkg.meda_rotary(x[:0], None, pos[:0], rope)
        assert empty.shape == (0, 1, 64)


def test_refusals():
    import paper_2502_17599_amd as pkg
    rope, _, _ = _plan(64, 1, False, 0)
    q, pos = normal(1, 8, 2, 64), torch.zeros(8, dtype=torch.int32, device=DEV)
    for bad in (dict(positions=pos[:4]), dict(positions=pos.long()), dict(positions=pos.cpu()), dict(k=q.bfloat16()), dict(k=q[:, :, :32]),
                dict(q=q[:, :, ::2]), dict(q_out=q[1:]), dict(q_out=q.bfloat16()),
                dict(q=normal(1, 8, 2, 32)), dict(k_out=q)):
        args = dict(q=q, k=None, positions=pos, rope=rope, q_out=None, k_out=None)
        args.update(bad)
        with pytest.raises(ValueError):
            pkg.meda_rotary(**args)
    buf = normal(2, 9 * 2 * 64 + 64)
    a, b = buf[:8 * 128].view(8, 2, 64), buf[128:9 * 128].view(8, 2, 64)
    with pytest.raises(ValueError, match="overlaps"):
        pkg.meda_rotary(a, None, pos, rope, b)
    odd = torch.empty(8 * 130, device=DEV).as_strided((8, 2, 64), (130, 64, 1))
    with pytest.raises(ValueError, match="16 bytes"):
        pkg.meda_rotary(odd, None, pos, rope)
