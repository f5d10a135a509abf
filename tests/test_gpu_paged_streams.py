"""Calls on a given stream, and the memory that decoders and caches keep when such a stream is still at work."""
import numpy as np
import pytest
import torch

from paged_cases import DEV, make_pool, make_table, normal
from test_gpu_paged_rows import _cache

pytestmark = pytest.mark.gpu

BUSY = 30_000_000     # cycles: some milliseconds at least


def _late(side, *pairs):
    """Keeps the stream busy, then copies there: whoever reads the targets on another stream finds what they held before."""
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
        for to, value in pairs:
            to.copy_(value)


def test_attention_on_a_given_stream():
    import paper_2502_17599_amd as pkg
    lens, page = [700, 33, 0, 4000], 16
    pool = make_pool("bf16", 400, 2, page, 64, seed=1)
    table, ln = make_table(lens, page, 400, seed=2)
    q = normal(3, 4, 8, 64, dtype="bf16")
    dec = pkg.PagedDecoder(pool, 4, 8, table.shape[1])
    want = dec(q, table, ln).clone()
    side, late = torch.cuda.Stream(), torch.zeros_like(q)
    for out in (None, torch.zeros_like(q)):
        late.zero_()
        torch.cuda.synchronize()
        _late(side, (late, q))
        got = dec(late, table, ln, out, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_page_update_on_a_given_stream():
    import paper_2502_17599_amd as pkg
    R, page = 70, 16

    def state():
        return (torch.zeros(R, dtype=torch.int32, device=DEV), torch.full((R, 5), -1, dtype=torch.int32, device=DEV),
                torch.arange(200, dtype=torch.int32, device=DEV), torch.tensor([7, 200], dtype=torch.int64, device=DEV),
                torch.zeros((R, 2), dtype=torch.int64, device=DEV), torch.zeros(R, dtype=torch.int32, device=DEV))
    new = torch.from_numpy(np.random.default_rng(1).integers(0, 60, R).astype(np.int32)).to(DEV)
    want, got = state(), state()
    for s, n, stream in ((want, new, None), (got, torch.zeros_like(new), torch.cuda.Stream())):
        if stream is not None:
            _late(stream, (n, new))
        lens, table, ring, free, slots, granted = s
        pkg.meda_page_update(lens, n, table, ring, free, page, slots=slots, granted=granted, stream=stream)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_store_on_a_given_stream():
    import paper_2502_17599_amd as pkg
    lens, page, side = [5, 300, 77], 16, torch.cuda.Stream()
    cc, _ = _cache([lens], 2, 64, "bf16", False, 5)
    rows = cc.k_out.clone()
    pools = [make_pool("bf16", 40, 2, page, 64, seed=6) for _ in range(2)]
    table, ln = make_table(lens, page, 40, seed=7)
    pkg.meda_paged_store(pools[0], cc, table, ln)
    torch.cuda.synchronize()
    cc.k_out.zero_()
    _late(side, (cc.k_out, rows))
    pkg.meda_paged_store(pools[1], cc, table, ln, stream=side)
    torch.cuda.synchronize()
    for a, b in zip((pools[0].k_pages, pools[0].v_pages), (pools[1].k_pages, pools[1].v_pages)):
        assert torch.equal(a, b)


def _given_away(side, kept):
    """Whether new tensors of the current stream lie in the memory of those that were dropped; the side stream is still busy."""
    ranges = [(t.data_ptr(), t.numel() * t.element_size()) for t in kept]
    kept.clear()
    new = [torch.empty(n, dtype=torch.uint8, device=DEV) for _, n in ranges]
    assert side is None or not side.query()
    hit = any(a < t.data_ptr() + t.numel() and t.data_ptr() < a + n for a, n in ranges for t in new)
    torch.cuda.synchronize()
    return hit


@pytest.mark.parametrize("given", [True, False])
def test_a_dropped_decoders_memory_is_kept_until_its_stream_is_done(given):
    import paper_2502_17599_amd as pkg
    torch.cuda.empty_cache()
    pool = make_pool("bf16", 40, 2, 16, 64, seed=1)
    table, ln = make_table([300, 100], 16, 40, width=2000)
    q, side = normal(2, 2, 8, 64, dtype="bf16"), torch.cuda.Stream()
    dec = pkg.PagedDecoder(pool, 2, 8, 2000)
    dec(q, table, ln)
    torch.cuda.synchronize()
    _late(side)
    if given:
        dec(q, table, ln, stream=side)
    else:
        with torch.cuda.stream(side):
            dec(q, table, ln)
    kept = [dec.workspace, dec.out]
    del dec
    assert not _given_away(side, kept)


def test_a_dropped_caches_memory_is_kept_until_its_stream_is_done():
    import paper_2502_17599_amd as pkg
    for work in (lambda c: c.step(), lambda c: c.append(0, x[:, :2], x[:, :2]), lambda c: c.attend(1, x, torch.empty_like(x)), lambda c: c.release([1])):
        torch.cuda.empty_cache()
        x, side = normal(3, 40, 4, 64, dtype="f32").bfloat16(), torch.cuda.Stream()
        cache = pkg.PagedCache(40, 2, 4, 2, 64, max_len=4000, n_pages=300, page_size=16)
        cache.step()
        torch.cuda.synchronize()
        _late(side)
        with torch.cuda.stream(side):
            work(cache)
        kept = [cache.pool.k_pages, cache.pool.v_pages, cache.table, cache.lens, cache.granted, cache.slots, cache.free_ring, cache.free_state]
        del cache
        assert not _given_away(side, kept)


def test_what_a_call_was_lent_is_kept_until_its_stream_is_done():
    """Every tensor of a call on a given stream is dropped right after it, while the stream is still busy."""
    import paper_2502_17599_amd as pkg
    T, H, D, page, n = 300, 4, 64, 16, 40

    def rope():
        return pkg.RotaryPlan(torch.ones(D // 2, dtype=torch.float64, device=DEV), torch.zeros(D // 2, dtype=torch.uint8, device=DEV), 2)

    def rotary(side):
        plan = rope()
        t = [normal(1, T, H, D), normal(2, T, H, D), torch.zeros((2, T), dtype=torch.int32, device=DEV), torch.empty(T, H, D, device=DEV), torch.empty(T, H, D, device=DEV)]
        return t + [plan.inv_freq, plan.axis], lambda: pkg.meda_rotary(t[0], t[1], t[2], plan, t[3], t[4], stream=side)

    def append(side):
        plan, pool = rope(), make_pool("fp8", n, H, page, D)
        t = [normal(i, T, H, D, dtype="bf16") for i in range(4)] + [torch.arange(T, device=DEV), torch.zeros((2, T), dtype=torch.int32, device=DEV)]
        return t + [plan.inv_freq, plan.axis, *pool.tensors], lambda: pkg.meda_paged_append(pool, t[0], t[1], t[4], t[2], t[5], plan, t[3], stream=side)

    def store(side):
        pool = make_pool("f32", n, H, page, D)
        cc, _ = _cache([[300]], H, D, "f32", False, 3)
        table, lens = make_table([300], page, n)
        return [cc.k_out, cc.v_out, cc.layer_len, cc.layer_off, table, lens, *pool.tensors], lambda: pkg.meda_paged_store(pool, cc, table, lens, stream=side)

    def attention(side):
        pool = make_pool("fp8", n, H, page, D)
        table, lens = make_table([300, 200], page, n)
        q = normal(4, 2, 2 * H, D, dtype="bf16")
        out, dec = torch.empty_like(q), pkg.PagedDecoder(pool, 2, 2 * H, table.shape[1])
        return [q, out, table, lens, dec.workspace, *pool.tensors], lambda: dec(q, table, lens, out, stream=side)

    def update(side):
        R = 64
        t = [torch.zeros(R, dtype=torch.int32, device=DEV) for _ in range(4)] + [torch.zeros((R, 9), dtype=torch.int32, device=DEV),
             torch.arange(900, dtype=torch.int32, device=DEV), torch.tensor([0, 900], device=DEV), torch.zeros(2, dtype=torch.int64, device=DEV),
             torch.zeros((R, 3), dtype=torch.int64, device=DEV), torch.zeros(pkg.meda_page_update_workspace_bytes(R), dtype=torch.uint8, device=DEV)]
        return t, lambda: pkg.meda_page_update(t[0], t[1], t[4], t[5], t[6], page, t[2], t[7], t[8], t[3], t[9], side)

    for make in (rotary, append, store, attention, update):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        kept, call = make(None)                   # on the current stream: what is dropped serves its next tensors
        call()
        kept = list(kept)
        del call
        assert _given_away(None, kept), make.__name__
        torch.cuda.empty_cache()
        side = torch.cuda.Stream()
        kept, call = make(side)
        call()                                    # (loads the kernel before the stream is made busy)
        torch.cuda.synchronize()
        kept, call = make(side)
        torch.cuda.synchronize()
        _late(side)
        call()
        kept = list(kept)
        del call
        assert not _given_away(side, kept), make.__name__
