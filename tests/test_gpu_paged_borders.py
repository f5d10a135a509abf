"""Every position counts once, wherever the work is cut: at borders of units, waves, shares, loads of page numbers, pages.

With q = 0 all n positions of a row weigh the same and the values are +-1 at random, so a result times n is a whole number, the
sum S of n signs in each column.  Weights of 1 and sums of signs are exact in fp32 (S stays far below 2^15, the parts of a weight in bf16
are multiples of 2^-8), so what is left is the quotient and the output's rounding: 2^-24 and half a step of S.  A position left
out, or counted twice, changes every column by 1: it shows in those whose S is below 100 (bf16: 2^-8 * 100 < 0.4)."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paged_cases import DEV, STEP

pytestmark = pytest.mark.gpu


def _sign_pool(cache, n_pages, Hkv, page, d, rng):
    """Pages of keys of any value and values +-1; the values as numbers."""
    import paper_2502_17599_amd as pkg
    v = rng.integers(0, 2, size=(n_pages, Hkv, page, d)).astype(np.int8) * 2 - 1
    if cache == "fp8":
        codes = torch.from_numpy(np.where(v < 0, 0xB8, 0x38).astype(np.uint8)).to(DEV)
        k = torch.from_numpy(rng.integers(0, 126, size=v.shape).astype(np.uint8)).to(DEV)
        one = torch.ones(v.shape[:3], device=DEV)
        return pkg.PagePool(k, codes, one * 0.01, one), v
    dt = torch.float32 if cache == "f32" else torch.bfloat16
    return pkg.PagePool(torch.from_numpy(rng.normal(size=v.shape).astype(np.float32)).to(dt).to(DEV), torch.from_numpy(v).to(dt).to(DEV)), v


def _check(lens, Hq, Hkv, d, cache, page, n_pages, width=None, missing=(), seed=0):
    import paper_2502_17599_amd as pkg
    print(f"\n[borders] R={len(lens)} max={max(lens)} {Hq}/{Hkv} d={d} {cache} page={page} width={width}", flush=True)
    rng = np.random.default_rng(seed)
    pool, v = _sign_pool(cache, n_pages, Hkv, page, d, rng)
    sums = v.sum(2, dtype=np.int64)
    R, W = len(lens), width or max(1, max(P.blocks(n, page) for n in lens))
    table = rng.integers(0, n_pages, size=(R, W)).astype(np.int32)       # (pages may be shared: their order differs)
    for r, b in missing:
        table[r, b] = -1
    dt = "f32" if cache == "f32" else "bf16"
    q = torch.zeros((R, Hq, d), dtype=pool.row_dtype, device=DEV)
    out = pkg.PagedDecoder(pool, R, Hq, W)(q, torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV))
    out = out.double().cpu().numpy().reshape(R, Hkv, Hq // Hkv, d)
    for r, n in enumerate(lens):
        full, rest = divmod(n, page)
        held = table[r, :full][table[r, :full] >= 0]
        count, want = len(held) * page, sums[held].sum(0)
        if rest and table[r, full] >= 0:
            count, want = count + rest, want + v[table[r, full], :, :rest].sum(1, dtype=np.int64)
        if count == 0:
            assert (out[r] == 0).all(), r
            continue
        assert np.abs(want).max() < 2 ** 15
        if dt == "bf16":
            assert (np.abs(want).min(-1) < 100).all(), "the signs tell nothing"
        err = np.abs(out[r] * count - want[:, None])
        assert (err <= (STEP[dt] + 2.0 ** -22) * np.abs(want)[:, None]).all(), (r, n, float(err.max()))


MANY = [[33, 1, 700, 5, 0, 0, 64, 2100, 31, 1, 1, 1, 900, 12], [1] * 300 + [5000] + [1] * 300, [17] * 1000, [4096, 4095, 1, 4097],
        [1 + (r * 13) % 40 for r in range(900)] + [9000, 0, 0, 33000, 5000], [3000] + [0] * 150 + [2999], [700] + [0] * 60 + [1, 650]]


@pytest.mark.parametrize("cache", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("i", range(len(MANY)))
def test_many_rows(cache, i):
    _check(MANY[i], 4, 2, 64, cache, 16, 500, seed=i, width=max(512, -(-max(MANY[i]) // 16)))


@pytest.mark.parametrize("lens,Hq,Hkv,d,cache,page", [
    ([20000], 8, 1, 128, "bf16", 64), ([9001], 28, 4, 128, "bf16", 16), ([15000, 1, 0, 3000], 8, 2, 128, "fp8", 128), ([12345], 4, 4, 128, "f32", 32),
    ([777] * 40, 7, 1, 128, "bf16", 256), ([40 * i for i in range(60)], 12, 3, 128, "fp8", 32), ([30011, 4], 32, 2, 64, "bf16", 64),
    ([30011, 4], 32, 2, 64, "fp8", 16), ([30011, 4], 32, 2, 128, "f32", 16)])
def test_few_long_rows(lens, Hq, Hkv, d, cache, page):
    _check(lens, Hq, Hkv, d, cache, page, 400, seed=len(lens))


@pytest.mark.parametrize("cache", ["bf16", "fp8", "f32"])
def test_waves_that_load_page_numbers_many_times(cache):
    """Rows of 55000 to 60000 positions, some of whose blocks name no page."""
    lens = [int(n) for n in np.random.default_rng(5).integers(55000, 60001, size=64)]
    lens[7], lens[8] = 60000, 59985
    _check(lens, 4, 2, 64, cache, 16, 300, width=3750, missing=[(3, 1000), (40, 17)] + [(5, b) for b in range(3000, 3010)], seed=6)


@pytest.mark.parametrize("cache", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_short_tables(cache, page):
    """Every length up to some blocks, and a missing first, middle and last page, in one launch and in shares."""
    lens = list(range(0, 200)) + [255, 256, 257, 300]
    for width in (None, 2000):
        _check(lens, 6, 2, 128, cache, page, 40, width=width, missing=[(150, 0), (199, 100 // page), (203, (300 - 1) // page)], seed=page)
