"""Attention over pages against the oracle in 64 bits (tolerances: paged_cases.attention_tolerance)."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paged_cases import DEV, DT, attention_tolerance, make_pool, make_table, normal, values, wide

pytestmark = pytest.mark.gpu


def _check(out, q, pool, table, lens, scale=0.0, rows=None):
    dt = "f32" if pool.row_dtype == torch.float32 else "bf16"
    k, v = values(pool)
    tab, ln, qs, got = table.cpu().numpy(), lens.cpu().numpy(), wide(q), wide(out)
    d = q.shape[-1]
    s = scale or d ** -0.5
    for r in range(len(ln)) if rows is None else rows:
        ref = P.attention(qs[r:r + 1], k, v, tab[r:r + 1], ln[r:r + 1], s)[0]
        n = int(ln[r])
        if n <= 0:
            assert (got[r] == 0).all(), r
            continue
        kk = P.gather(k, tab[r], min(n, tab.shape[1] * k.shape[2]))
        logit = max([np.abs(qs[r, h] @ kk[h // (q.shape[1] // kk.shape[0])].T).max() * s if kk.shape[1] else 0 for h in range(q.shape[1])])
        tol = attention_tolerance(ref, v, logit, n, d, dt)
        err = np.abs(got[r] - ref)
        assert (err <= tol).all(), (r, n, float((err / tol).max()))


def _run(lens, Hq, Hkv, d, cache, page, joint=False, seed=0, scale=0.0, spare=2, width=None, rows=None):
    import paper_2502_17599_amd as pkg
    print(f"\n[paged attention] R={len(lens)} max={max(lens)} {Hq}/{Hkv} d={d} {cache} page={page} joint={joint}", flush=True)
    n_pages = sum(-(-n // page) for n in lens) + spare
    pool = make_pool(cache, n_pages, Hkv, page, d, seed=seed, joint=joint)
    table, ln = make_table(lens, page, n_pages, seed=seed, width=width)
    q = normal(seed + 9, len(lens), Hq, d, dtype="f32" if cache == "f32" else "bf16")
    out = pkg.PagedDecoder(pool, len(lens), Hq, table.shape[1], softmax_scale=scale)(q, table, ln)
    _check(out, q, pool, table, ln, scale, rows)
    return pool, table, ln, q, out


# Tables that cannot hold long rows are served by a workgroup per row and kv head, wider ones in shares: both are tested.
WIDE = 2000
BOTH = pytest.mark.parametrize("wide", [False, True])


def _widen(table, wide):
    return torch.nn.functional.pad(table, (0, WIDE - table.shape[1]), value=-7) if wide else table


@BOTH
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 9, 16])
@pytest.mark.parametrize("cache,d", [("bf16", 128), ("bf16", 64), ("fp8", 128), ("fp8", 64), ("f32", 128), ("f32", 64)])
def test_groups_and_types(G, cache, d, wide):
    _run([1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 0, 2], 2 * G, 2, d, cache, 16, seed=G, width=WIDE if wide else None)


@BOTH
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("cache", ["bf16", "fp8", "f32"])
def test_page_sizes_and_ends_inside_a_page(page, cache, wide):
    lens = [page - 1, page, page + 1, 1, 0, 2 * page - 15, 2 * page + 16, 3 * page + 17]
    _run(lens, 6, 3, 128 if cache != "f32" else 64, cache, page, joint=cache != "fp8", seed=page, width=WIDE if wide else None)


@pytest.mark.parametrize("lens,Hq,Hkv,cache,page", [
    ([20000], 8, 1, "bf16", 64), ([9001], 28, 4, "bf16", 16), ([15000, 1, 0, 3000], 8, 2, "fp8", 128), ([12345], 4, 4, "f32", 32),
    ([777] * 40, 7, 1, "bf16", 256), ([40 * i for i in range(60)], 12, 3, "fp8", 32)])
def test_work_cut_over_many_workgroups(lens, Hq, Hkv, cache, page):
    _run(lens, Hq, Hkv, 128, cache, page, seed=len(lens), rows=range(0, len(lens), max(1, len(lens) // 8)))


def test_many_rows():
    """More rows than the first search holds one each, most of them empty."""
    lens = [0] * 1500
    for r in range(0, 1500, 11):
        lens[r] = 1 + (r * 7) % 90
    _run(lens, 4, 2, 64, "bf16", 16, rows=range(0, 1500, 50))


@BOTH
def test_all_rows_empty(wide):
    import paper_2502_17599_amd as pkg
    pool = make_pool("bf16", 2, 2, 16, 64)
    table, lens = _widen(torch.full((3, 4), -1, dtype=torch.int32, device=DEV), wide), torch.zeros(3, dtype=torch.int32, device=DEV)
    dec = pkg.PagedDecoder(pool, 3, 4, table.shape[1])
    dec.out.fill_(7.0)
    assert (dec(normal(1, 3, 4, 64, dtype="bf16"), table, lens) == 0).all()


@BOTH
@pytest.mark.parametrize("cache", ["bf16", "fp8", "f32"])
def test_what_lies_behind_the_end_does_not_count(cache, wide):
    """NaN and infinities behind the last position, in pages nobody holds and in their scales; page numbers behind the held
    blocks that name no page; lengths past the table or below zero."""
    import paper_2502_17599_amd as pkg
    lens = [5, 33, 130, 64]
    pool, table, ln, q, out = _run(lens, 4, 2, 128, cache, 32, seed=3, spare=4, width=WIDE if wide else None)
    held = np.zeros((pool.n_pages, 32), bool)
    tab = table.cpu().numpy()
    for r, n in enumerate(lens):
        for i in range(n):
            held[tab[r, i // 32], i % 32] = True
    free = torch.from_numpy(~held).to(DEV)[:, None, :].expand(-1, 2, -1)
    want = out.clone()
    if cache == "fp8":
        pool.k_pages[free] = 127; pool.v_pages[free] = 255                      # NaN codes
        pool.k_scales[free] = float("inf"); pool.v_scales[free] = float("nan")
    else:
        pool.k_pages[free] = float("nan"); pool.v_pages[free] = float("inf")
    dec = pkg.PagedDecoder(pool, 4, 4, table.shape[1])
    assert torch.equal(dec(q, table, ln), want)
    wild = table.clone()
    wild[wild < 0] = 2 ** 31 - 1
    assert torch.equal(dec(q, wild, ln), want)
    over = ln.clone()
    over[0] = -3
    zeroed = dec(q, table, over)
    assert (zeroed[0] == 0).all()
    if cache != "fp8":      # what the oracle reads has no NaN
        pool.k_pages[free] = 0; pool.v_pages[free] = 0
    else:
        pool.k_pages[free] = 0; pool.v_pages[free] = 0; pool.k_scales[free] = 1; pool.v_scales[free] = 1
    _check(zeroed, q, pool, table, over)


@BOTH
@pytest.mark.parametrize("cache", ["bf16", "fp8", "f32"])
def test_missing_pages_are_left_out(cache, wide):
    import paper_2502_17599_amd as pkg
    lens, page = [200, 64, 33, 1, 400], 16
    n_pages = 60
    pool = make_pool(cache, n_pages, 2, page, 64, seed=5)
    table, ln = make_table(lens, page, n_pages, seed=5)
    table[0, 3] = -1; table[0, 4] = n_pages; table[1, 0] = 2 ** 31 - 1; table[2, 2] = -2 ** 31; table[3, 0] = -1; table[4, 24] = -9
    q = normal(4, 5, 6, 64, dtype="f32" if cache == "f32" else "bf16")
    table = _widen(table, wide)
    out = pkg.PagedDecoder(pool, 5, 6, table.shape[1])(q, table, ln)
    _check(out, q, pool, table, ln)
    assert (out[3] == 0).all()


def test_length_past_the_table_is_clamped():
    import paper_2502_17599_amd as pkg
    pool, table, ln, q, out = _run([64, 48], 4, 2, 64, "bf16", 16, seed=6)
    table[1, 3] = table[0, 0]
    got = pkg.PagedDecoder(pool, 2, 4, 4)(q, table, torch.tensor([10 ** 9, 2 ** 31 - 1], dtype=torch.int32, device=DEV))
    _check(got, q, pool, table, torch.tensor([64, 64], dtype=torch.int32, device=DEV))


@BOTH
@pytest.mark.parametrize("cache", ["bf16", "f32"])
def test_extreme_values(cache, wide):
    """Logits far apart, all equal, at the bottom of the range; infinite values and keys."""
    import paper_2502_17599_amd as pkg
    dt = DT[cache]
    page, n = 16, 48
    pool = make_pool(cache, 6, 1, page, 64, seed=7)
    table, lens = make_table([n, n], page, 6, seed=7, width=WIDE if wide else 3)
    tab, W = table.cpu().numpy(), table.shape[1]
    q = torch.zeros(2, 1, 64, dtype=dt, device=DEV)
    out = pkg.PagedDecoder(pool, 2, 1, W)(q, table, lens)
    _check(out, q, pool, table, lens)                                    # equal logits: the mean
    q[0, 0, 0] = 1e30
    pool.k_pages[..., 0] = -1e8
    _check(pkg.PagedDecoder(pool, 2, 1, W)(q, table, lens), q, pool, table, lens)     # every logit near -1e37, all equal
    pool.k_pages[tab[0, 1], 0, 5, 0] = 1.0
    got = pkg.PagedDecoder(pool, 2, 1, W)(q, table, lens)
    assert torch.equal(got[0, 0], pool.v_pages[tab[0, 1], 0, 5])                       # one key takes everything
    pool.k_pages[tab[0, 0], 0, :, 0] = float("-inf")                                   # no weight at all
    assert torch.equal(pkg.PagedDecoder(pool, 2, 1, W)(q, table, lens)[0, 0], pool.v_pages[tab[0, 1], 0, 5])
    q[1] = normal(8, 1, 64, dtype=cache)
    pool.k_pages[..., 0] = 0
    pool.v_pages[tab[1, 0], 0, 3, 10] = float("inf")
    pool.v_pages[tab[1, 2], 0, 3, 11] = float("-inf")
    got = pkg.PagedDecoder(pool, 2, 1, W)(q, table, lens)[1, 0]
    assert got[10] == float("inf") and got[11] == float("-inf") and torch.isfinite(got[torch.arange(64, device=DEV) // 2 != 5]).all()
    pool.k_pages[tab[1, 1], 0, 2, 7] = float("nan")
    assert torch.isnan(pkg.PagedDecoder(pool, 2, 1, W)(q, table, lens)[1]).all()


@BOTH
def test_strides_and_outputs(wide):
    """Rows of one layer out of a table of several, queries inside a fused projection, an output of the caller's."""
    import paper_2502_17599_amd as pkg
    L, N, page = 3, 4, 32
    lens = [20, 33, 0, 64, 7, 90, 100, 1, 65, 31, 32, 128]
    pool, table, ln, q, out = _run(lens, 4, 2, 128, "bf16", page, seed=11, width=WIDE if wide else None)
    for l in range(L):
        dec = pkg.PagedDecoder(pool, N, 4, table.shape[1])
        qkv = torch.full((N, 8, 128), 9.0, dtype=torch.bfloat16, device=DEV)
        qkv[:, :4] = q[l::L]
        res = torch.full((N, 2, 4, 128), 5.0, dtype=torch.bfloat16, device=DEV)
        dec(qkv[:, :4], table[l::L], ln[l::L], res[:, 1])
        _check(res[:, 1], qkv[:, :4], pool, table[l::L], ln[l::L])
        assert (res[:, 0] == 5).all()


def test_shared_pages():
    """Rows may read the same pages (a common prefix)."""
    import paper_2502_17599_amd as pkg
    pool = make_pool("bf16", 9, 2, 16, 64, seed=1)
    table = torch.tensor([[0, 1, 2, 3], [0, 1, 2, 4], [0, 1, 2, 3]], dtype=torch.int32, device=DEV)
    lens = torch.tensor([64, 55, 40], dtype=torch.int32, device=DEV)
    q = normal(3, 3, 4, 64, dtype="bf16")
    _check(pkg.PagedDecoder(pool, 3, 4, 4)(q, table, lens), q, pool, table, lens)


def test_offsets_past_32_bits():
    """A pool of more than 4 GiB whose last pages are used: byte offsets of 33 bits, element offsets of 32."""
    import paper_2502_17599_amd as pkg
    page, heads, d = 256, 8, 128
    n_pages = (5 << 30) // (page * heads * d * 2)
    k = torch.empty((n_pages, heads, page, d), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    pool = pkg.PagePool(k, v)
    used = [n_pages - 1, n_pages // 2 + 3, 0]
    small = make_pool("bf16", 3, heads, page, d, seed=2)
    for i, p in enumerate(used):
        k[p], v[p] = small.k_pages[i], small.v_pages[i]
    lens = torch.tensor([2 * page + 40, 100], dtype=torch.int32, device=DEV)
    table = torch.tensor([used, used], dtype=torch.int32, device=DEV)
    near = torch.tensor([[0, 1, 2]] * 2, dtype=torch.int32, device=DEV)
    q = normal(5, 2, 16, d, dtype="bf16")
    got, want = pkg.PagedDecoder(pool, 2, 16, 3)(q, table, lens), pkg.PagedDecoder(small, 2, 16, 3)(q, near, lens)
    assert torch.equal(got, want)
    new = normal(6, 2, heads, d, dtype="bf16")
    pkg.meda_paged_append(pool, new, new, torch.tensor([(n_pages - 1) * page + 77, (n_pages // 2) * page], device=DEV))
    assert torch.equal(k[n_pages - 1, :, 77], new[0]) and torch.equal(v[n_pages // 2, :, 0], new[1])


def test_same_bits_every_time():
    import paper_2502_17599_amd as pkg
    pool, table, ln, q, out = _run([5000, 3, 700, 0, 64], 8, 2, 128, "bf16", 64, seed=12, rows=[1])
    dec = pkg.PagedDecoder(pool, 5, 8, table.shape[1])
    first = dec(q, table, ln).clone()
    for _ in range(5):
        dec.workspace.fill_(255)       # what the workspace held does not matter
        assert torch.equal(dec(q, table, ln), first)


def test_refusals():
    import paper_2502_17599_amd as pkg
    pool, table, ln, q, out = _run([20, 33], 4, 2, 64, "bf16", 16)
    W = table.shape[1]
    dec = pkg.PagedDecoder(pool, 2, 4, W)
    for args in ((q.float(), table, ln), (q[:1], table, ln), (q, table.long(), ln), (q, table[:1], ln), (q, table, ln[:1]), (q, table, ln.cpu()),
                 (q, table[:, :1], ln), (q.transpose(0, 1), table, ln), (q, table, ln, q), (q, table, ln, q.float())):
        with pytest.raises(ValueError):
            dec(*args)
    for args in ((pool, 2, 3, W), (pool, 0, 4, W), (pool, 2, 4, 0), (pool, 2, 34, W), (pool, 2, 4, W, torch.float32)):
        with pytest.raises(pkg.MedaError):
            pkg.PagedDecoder(*args)
    with pytest.raises(pkg.MedaError):
        pkg.PagedDecoder(pool, 2, 4, W, softmax_scale=-1.0)


@pytest.mark.parametrize("width", [None, 4000])
@pytest.mark.parametrize("cache,G", [("bf16", 4), ("bf16", 16), ("fp8", 7), ("f32", 5)])
def test_short_rows_in_short_and_wide_tables(width, cache, G):
    """The same rows where the table says that they are short (a workgroup per row and kv head) and where it could hold long
    ones (shares): rows of one wave's units, of all waves', and none."""
    lens = [0, 1, 16, 31, 32, 33, 64, 100, 128, 129, 160, 200, 255, 256, 257, 300] * 3
    _run(lens, 2 * G, 2, 128, cache, 16, seed=G, width=width, rows=range(16))
    _run(lens[5:10], 3 * G, 3, 64, cache, 16, seed=G + 1, width=width)     # few pairs


def test_many_waves_in_one_pair_and_one_wave_over_many_pairs():
    """Shares that begin and end inside pairs, pairs that end inside a wave's part, pairs of one unit."""
    for seed, lens in ((1, [33, 1, 700, 5, 0, 0, 64, 2100, 31, 1, 1, 1, 900, 12]), (2, [1] * 300 + [5000] + [1] * 300), (3, [17] * 1000), (4, [4096, 4095, 1, 4097])):
        _run(lens, 4, 2, 64, "bf16", 16, seed=seed, width=512, rows=range(0, len(lens), max(1, len(lens) // 40)))
        _run(lens, 4, 2, 64, "f32", 16, seed=seed, width=512, rows=range(0, len(lens), max(1, len(lens) // 40)))


@pytest.mark.parametrize("cache", ["bf16", "fp8", "f32"])
def test_long_walks_of_one_wave(cache):
    """So many positions that every wave walks over more units than one load of page numbers covers.  The rows read the same
    few pages over and over (pages may be shared), each in an order of its own; some of their blocks name no page."""
    import paper_2502_17599_amd as pkg
    R, Hkv, page, n_pages, width = 64, 2, 16, 300, 3750
    pool = make_pool(cache, n_pages, Hkv, page, 64, seed=21)
    rng = np.random.default_rng(22)
    table = rng.integers(0, n_pages, size=(R, width)).astype(np.int32)
    table[3, 1000] = -1; table[5, 3000:3010] = n_pages; table[40, 17] = 2 ** 31 - 1
    lens = rng.integers(55000, width * page + 1, size=R).astype(np.int32)
    lens[7] = width * page
    t, n = torch.from_numpy(table).to(DEV), torch.from_numpy(lens).to(DEV)
    q = normal(23, R, 2 * Hkv, 64, dtype="f32" if cache == "f32" else "bf16")
    _check(pkg.PagedDecoder(pool, R, 2 * Hkv, width)(q, t, n), q, pool, t, n, rows=(0, 3, 5, 7, 31, 40, 63))


def test_long_rows_among_many_short_ones():
    """More (row, kv head) pairs than workgroups, some of them cut: the join goes by shares."""
    lens = [1 + (r * 13) % 40 for r in range(900)]
    lens[5], lens[400], lens[899] = 9000, 33000, 5000
    _run(lens, 4, 2, 64, "bf16", 16, seed=31, rows=[0, 4, 5, 6, 200, 399, 400, 401, 898, 899])


@pytest.mark.parametrize("R,Hkv", [(6, 2), (450, 2)])
def test_nothing_is_kept_from_the_call_before(R, Hkv):
    """One decoder over long rows, short ones, none and long ones again: as a new one gives them, bit by bit."""
    import paper_2502_17599_amd as pkg
    page, n_pages, width = 16, 200, 1500
    pool = make_pool("bf16", n_pages, Hkv, page, 64, seed=41)
    rng = np.random.default_rng(42)
    table = torch.from_numpy(rng.integers(0, n_pages, size=(R, width)).astype(np.int32)).to(DEV)
    q = normal(43, R, 2 * Hkv, 64, dtype="bf16")
    kept = pkg.PagedDecoder(pool, R, 2 * Hkv, width)
    for most in (width * page, 30, 3000, 0, 500, width * page):
        lens = torch.from_numpy(rng.integers(0, most + 1, size=R).astype(np.int32)).to(DEV)
        if most == 3000:
            lens[R // 2:] = 0
        got, want = kept(q, table, lens).clone(), pkg.PagedDecoder(pool, R, 2 * Hkv, width)(q, table, lens)
        assert torch.equal(got, want), most
        _check(got, q, pool, table, lens, rows=(0, R // 2, R - 1))
