"""The operators together, as a serving program uses them: prompts are rotated, compressed, admitted to pages, and decoded
token by token beside other sequences, eagerly, from a captured graph, on another stream."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paged_cases import DEV, attention_tolerance, normal, values, wide
from workloads import generate, get_workload, variant

pytestmark = pytest.mark.gpu


def _prompts(n, L, Hq, Hkv, d, dtype, T, W, budget, seed):
    """n prompts of a video with text: q, k rotated on three axes and compressed."""
    import paper_2502_17599_amd as pkg
    base = variant(get_workload("tiny"), n_layers=L, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, dtype=dtype, window=W, total_budget=budget)
    seqs = [generate(variant(base, seed=seed + i)) for i in range(n)]
    half = d // 2
    rope = pkg.RotaryPlan(torch.pow(torch.tensor(1e4, dtype=torch.float64), -torch.arange(half, dtype=torch.float64) / half).to(DEV),
                          (torch.arange(half) * 3 // half).to(torch.uint8).to(DEV), 3)
    T = base.seq_len
    pos = torch.stack([torch.arange(T), torch.arange(T) // 64, torch.arange(T) % 64]).to(torch.int32).to(DEV)
    q, k, v = (torch.stack([s[x] for s in seqs]).to(DEV) for x in ("q", "k", "v"))
    for i in range(n):
        for l in range(L):     # head by head in place: [H][T][d] as rows of tokens
            kt, qt = k[i, l].transpose(0, 1), q[i, l].transpose(0, 1)
            pkg.meda_rotary(qt, None, pos[:, T - W:], rope, qt)
            pkg.meda_rotary(kt, None, pos, rope, kt)
    cache = pkg.meda_compress(q, k, v, torch.stack([s["mask"] for s in seqs]).to(DEV), budget)
    return rope, cache, T


def _reference(cache, l, q):
    k, v = values(cache.pool)
    table, lens = cache.table[l::cache.n_layers].cpu().numpy(), cache.lens[l::cache.n_layers].cpu().numpy()
    ref = P.attention(wide(q), k, v, table, lens)
    dt = "f32" if q.dtype == torch.float32 else "bf16"
    # of the rows held (the rest of a new pool is memory as it was found)
    k, v = (np.concatenate([P.gather(x, table[r], int(lens[r])).reshape(-1, q.shape[-1]) for r in range(len(lens))]) for x in (k, v))
    logit = np.linalg.norm(wide(q), axis=-1).max() * np.linalg.norm(k, axis=-1).max() * q.shape[-1] ** -0.5
    return ref, attention_tolerance(ref, v, logit, int(lens.max()) + 1, q.shape[-1], dt)


@pytest.mark.parametrize("dtype,pages,page", [("f32", torch.float32, 16), ("bf16", torch.bfloat16, 64), ("bf16", torch.uint8, 32)])
def test_serving_loop(dtype, pages, page):
    import paper_2502_17599_amd as pkg
    print(f"\n[serving] {dtype} {pages} page={page}", flush=True)
    L, Hq, Hkv, d, N = 3, 8, 2, 64, 4
    budget = 3 * 150
    rope, compressed, T = _prompts(2, L, Hq, Hkv, d, dtype, 0, 32, budget, 40)
    cache = pkg.PagedCache(N, L, Hq, Hkv, d, max_len=T + 100, n_pages=400, page_size=page, dtype=pages, rope=rope)
    granted = cache.admit(1, compressed)
    assert torch.equal(granted, compressed.layer_len)
    assert cache.lens.view(N, L)[0].tolist() == [0] * L
    # the pages hold the compressed rows
    kp, vp = values(cache.pool)
    for i in range(2):
        one = compressed.sequence(i)
        for l in range(L):
            k_l, v_l, _ = one.layer(l)
            row, n = cache.table[(1 + i) * L + l].cpu().numpy(), int(one.layer_len[l])
            for pages_of, rows in ((kp, k_l), (vp, v_l)):
                got, want = P.gather(pages_of, row, n), wide(rows)
                if pages == torch.uint8:
                    codes, scales = pkg.meda_quantize_fp8(rows.reshape(-1, d).contiguous())
                    want = wide(pkg.meda_dequantize_fp8(codes, scales, torch.float32)).reshape(want.shape)
                    assert np.allclose(got, want, rtol=2.0 ** -23, atol=0)      # the dequantised product rounds once
                else:
                    assert np.array_equal(got, want)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q0 = normal(0, N, Hq, d, dtype=dtype)
    for l in range(L):
        ref, tol = _reference(cache, l, q0)
        assert (np.abs(wide(cache.attend(l, q0)) - ref) <= tol).all()

    active = torch.tensor([1, 1, 1, 0], dtype=torch.int32, device=DEV)     # sequence 0 starts from nothing
    for step in range(20):
        got = cache.step(active)
        assert got.tolist() == [[1] * L, [1] * L, [1] * L, [0] * L]
        pos = torch.stack([torch.tensor([step, T + step, T + step, 0])] * 3).to(torch.int32).to(DEV)
        for l in range(L):
            x = normal(1000 + 10 * step + l, N, Hq + 2 * Hkv, d, dtype=dtype)
            q = cache.append(l, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], x[:, :Hq], pos)
            out = cache.attend(l, q)
            if step in (0, 1, 15, 16, 19):
                assert torch.equal(q, pkg.meda_rotary(x[:, :Hq], None, pos, rope)[0])
                ref, tol = _reference(cache, l, q)
                assert (np.abs(wide(out) - ref) <= tol).all(), (step, l)
    assert cache.lens.view(N, L)[0].tolist() == [20] * L
    # the rows appended last are those of the last tokens
    k_new = pkg.meda_rotary(x[:, Hq:Hq + Hkv], None, pos, rope)[0]
    if pages != torch.uint8:
        kp, _ = values(cache.pool)
        n = int(cache.lens.view(N, L)[1, L - 1])
        assert np.array_equal(P.gather(kp, cache.table[L + L - 1].cpu().numpy(), n)[:, -1], wide(k_new)[1])
    # pages come back, all of them
    held = int(((cache.lens + page - 1) // page).sum())
    assert int(cache.free_state[1]) == 400 - held
    cache.release([0, 1, 2, 3])
    assert int(cache.free_state[1]) == 400 and (cache.lens == 0).all()
    assert sorted(cache.free_ring.tolist()) == list(range(400))
    assert (cache.attend(0, q0) == 0).all()


def test_refused_rows_change_nothing():
    """Pages for one prompt and a bit: the rows of the other hold nothing and its caches are written nowhere; a step grants all
    layers of a sequence room or none, and what was refused can be asked for again."""
    import paper_2502_17599_amd as pkg
    L, Hq, Hkv, d, N, page = 3, 4, 2, 64, 2, 16
    rope, compressed, T = _prompts(2, L, Hq, Hkv, d, "f32", 0, 32, 3 * 100, 50)
    need = ((compressed.layer_len + page - 1) // page).view(-1)
    n_pages = int(need[:4].sum())                                 # those of one more layer, too few for the second prompt
    cache = pkg.PagedCache(N, L, Hq, Hkv, d, max_len=T, n_pages=n_pages, page_size=page, dtype=torch.float32)
    cache.pool.k_pages.fill_(3.0); cache.pool.v_pages.fill_(3.0)
    granted = cache.admit(0, compressed).reshape(-1)
    assert torch.equal(granted[:3], compressed.layer_len.view(-1)[:3]) and (granted[3:] == 0).all()
    assert torch.equal(cache.lens, granted) and int(cache.free_state[1]) == int(need[3])
    kp, _ = values(cache.pool)
    for l in range(L):
        k_l, _, _ = compressed.sequence(0).layer(l)
        assert np.array_equal(P.gather(kp, cache.table[l].cpu().numpy(), int(cache.lens[l])), wide(k_l))
    held = set(cache.table[0, :int(need[0])].tolist()) | set(cache.table[1, :int(need[1])].tolist()) | set(cache.table[2, :int(need[2])].tolist())
    free = [p for p in range(n_pages) if p not in held]
    assert len(free) == int(need[3]) and (cache.pool.k_pages[free] == 3.0).all()
    # as many steps of both as the pages allow: the second sequence starts from nothing and needs a page per layer at once
    x = normal(1, N, Hkv, d)
    refused = 0
    for step in range(3 * page * int(need[3])):
        lens, left = cache.lens.view(N, L).clone(), int(cache.free_state[1])
        before = cache.pool.k_pages.clone()
        got = cache.step()
        want, left_now = [], left
        for n in lens.tolist():
            ask = sum(m % page == 0 for m in n)
            fits = max(n) < cache.max_blocks * page and ask <= left_now
            want.append([int(fits)] * L)
            left_now -= ask if max(n) < cache.max_blocks * page else 0
        assert got.tolist() == want, step
        assert torch.equal(cache.lens.view(N, L), lens + got)
        cache.append(2, x, x)
        slots = cache.slots[2::L, 0].tolist()
        assert [t >= 0 for t in slots] == [bool(w[2]) for w in want]
        changed = (cache.pool.k_pages != before).flatten(1).any(1).nonzero().flatten().tolist()
        assert set(changed) <= {t // page for t in slots if t >= 0}
        cache.pool.k_pages.copy_(before)
        refused += want.count([0] * L)
        if refused >= 3:
            break
    assert refused >= 3
    cache.release([0])
    assert cache.step(torch.tensor([0, 1], device=DEV)).tolist() == [[0] * L, [1] * L]      # asked for again, with room


def test_graph_replays_and_streams():
    """The body of the loop captured: every replay against an eager twin, with eager work between the replays; the same on a
    stream of its own."""
    import paper_2502_17599_amd as pkg
    L, Hq, Hkv, d, N = 2, 6, 2, 128, 3
    rope, compressed, T = _prompts(1, L, Hq, Hkv, d, "bf16", 0, 32, 2 * 200, 60)
    x = [normal(70 + l, N, Hq + 2 * Hkv, d, dtype="bf16") for l in range(L)]
    pos = torch.zeros((3, N), dtype=torch.int32, device=DEV)
    active = torch.tensor([1, 0, 1], dtype=torch.int32, device=DEV)

    def make():
        cache = pkg.PagedCache(N, L, Hq, Hkv, d, max_len=T, n_pages=120, page_size=16, rope=rope)
        cache.pool.k_pages.zero_(); cache.pool.v_pages.zero_()
        cache.admit(2, compressed)
        return cache, [torch.zeros((N, Hq, d), dtype=torch.bfloat16, device=DEV) for _ in range(2 * L)]

    def body(cache, outs):
        cache.step(active)
        for l in range(L):
            cache.append(l, x[l][:, Hq:Hq + Hkv], x[l][:, Hq + Hkv:], x[l][:, :Hq], pos, outs[l])
            cache.attend(l, outs[l], outs[L + l])

    (twin, t_out), (cache, c_out), (other, o_out) = make(), make(), make()
    body(twin, t_out); body(cache, c_out)           # also loads every code object before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body(cache, c_out)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        body(other, o_out)
    torch.cuda.synchronize()                        # (what follows changes x on the first stream)
    for i in range(40):                             # across several page boundaries
        pos.fill_(i)
        for t in x:
            t.mul_(-1.0)
        torch.cuda.synchronize()
        body(twin, t_out)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            body(other, o_out)
        torch.cuda.synchronize()
        for name in ("lens", "table", "free_ring", "free_state", "slots", "granted"):
            assert torch.equal(getattr(cache, name), getattr(twin, name)) and torch.equal(getattr(other, name), getattr(twin, name)), (i, name)
        for a, b, c in zip(t_out, c_out, o_out):
            assert torch.equal(a, b) and torch.equal(a, c), i
        assert torch.equal(cache.pool.k_pages, twin.pool.k_pages) and torch.equal(cache.pool.v_pages, other.pool.v_pages)
    assert twin.lens.view(N, L)[:, 0].tolist()[:2] == [41, 0]


def test_one_sequence_equals_the_ragged_step():
    """A compressed cache in pages and as the pass wrote it: the same attention, up to the rounding of fp32 sums."""
    import paper_2502_17599_amd as pkg
    L, Hq, Hkv, d = 4, 8, 4, 64
    _, compressed, T = _prompts(1, L, Hq, Hkv, d, "f32", 0, 32, 4 * 120, 80)
    one = compressed.sequence(0)
    q = normal(5, L, Hq, d)
    want = pkg.meda_decode_attention(q, one)
    cache = pkg.PagedCache(1, L, Hq, Hkv, d, max_len=T, n_pages=60, page_size=16, dtype=torch.float32)
    cache.admit(0, compressed)
    got = torch.cat([cache.attend(l, q[l:l + 1]).clone() for l in range(L)])
    assert np.abs(wide(got) - wide(want)).max() <= 2e-6 * np.abs(wide(one.v_out)).max()
    every = pkg.PagedDecoder(cache.pool, L, Hq, cache.max_blocks)(q, cache.table, cache.lens)       # all layers in one call
    assert np.abs(wide(every) - wide(want)).max() <= 2e-6 * np.abs(wide(one.v_out)).max()


def test_refusals():
    import paper_2502_17599_amd as pkg
    L, Hq, Hkv, d = 2, 4, 2, 64
    _, compressed, T = _prompts(1, L, Hq, Hkv, d, "f32", 0, 32, 2 * 100, 90)
    for bad in (dict(n_seqs=0), dict(n_layers=0), dict(page_size=17), dict(max_len=0), dict(n_seqs=32769), dict(max_len=1 << 35), dict(n_pages=0)):
        with pytest.raises(ValueError):
            pkg.PagedCache(**dict(dict(n_seqs=1, n_layers=L, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, max_len=T, n_pages=9), **bad))
    cache = pkg.PagedCache(1, L, Hq, Hkv, d, max_len=T, n_pages=40, page_size=16, dtype=torch.float32)
    for call in (lambda: cache.admit(1, compressed), lambda: cache.admit(-1, compressed), lambda: cache.release([1]), lambda: cache.release([-1]),
                 lambda: cache.step(torch.ones(2, device=DEV)), lambda: cache.step(torch.ones(1)), lambda: cache.attend(L, normal(1, 1, Hq, d)),
                 lambda: cache.attend(-1, normal(1, 1, Hq, d)), lambda: cache.append(5, normal(1, 1, Hkv, d), normal(1, 1, Hkv, d)),
                 lambda: cache.attend(0, normal(1, 2, Hq, d))):
        with pytest.raises(ValueError):
            call()
    three = pkg.PagedCache(2, L + 1, Hq, Hkv, d, max_len=T, n_pages=40, page_size=16, dtype=torch.float32)
    with pytest.raises(ValueError):
        three.admit(0, compressed)


def _state(cache):
    return [getattr(cache, name).clone() for name in ("lens", "table", "free_ring", "free_state")] + [cache.pool.k_pages.clone()]


def test_a_cache_that_does_not_fit_is_refused_before_anything_changes():
    import dataclasses
    import paper_2502_17599_amd as pkg
    L, Hq, Hkv, d = 2, 4, 2, 64
    rope, compressed, T = _prompts(1, L, Hq, Hkv, d, "f32", 0, 32, 2 * 100, 95)
    cache = pkg.PagedCache(1, L, Hq, Hkv, d, max_len=T, n_pages=40, page_size=16, dtype=torch.float32, rope=rope)
    cache.pool.k_pages.zero_()
    cache.admit(0, compressed)
    before = _state(cache)
    half = dataclasses.replace(compressed, k_out=compressed.k_out.to(torch.bfloat16))
    heads = dataclasses.replace(compressed, n_kv_heads=Hkv + 1)
    x = normal(1, 1, Hkv, d)
    for call in (lambda: cache.admit(0, half), lambda: cache.admit(0, heads),
                 lambda: cache.append(0, x, x),                         # the cache rotates: by which positions?
                 lambda: cache.append(0, x, x, normal(2, 1, Hq, d))):
        with pytest.raises(ValueError):
            call()
    assert all(torch.equal(a, b) for a, b in zip(before, _state(cache)))


def test_output_over_queries_is_refused():
    """The decoder's own output as the next call's queries, as they lie and one row further."""
    import paper_2502_17599_amd as pkg
    R, Hq, Hkv, d = 3, 4, 2, 64
    pool = pkg.PagePool.empty(4, Hkv, 16, d, torch.float32)
    table = torch.zeros((R, 1), dtype=torch.int32, device=DEV)
    lens = torch.zeros(R, dtype=torch.int32, device=DEV)
    dec = pkg.PagedDecoder(pool, R, Hq, 1)
    two = torch.zeros((R + 1, Hq, d), dtype=torch.float32, device=DEV)
    with pytest.raises(ValueError):
        dec(dec(two[:R], table, lens), table, lens)
    with pytest.raises(ValueError):
        dec(two[1:], table, lens, two[:R])
    assert (dec(two[:R], table, lens, torch.ones_like(two[:R])) == 0).all()


def _stream_of(t):
    """The stream whose memory holds a tensor."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]


def test_outputs_made_for_a_stream_come_from_its_memory():
    """Memory of the current stream could still be in use there when a call on another stream writes to it."""
    import paper_2502_17599_amd as pkg
    T, H, d = 33, 2, 64
    side = torch.cuda.Stream()
    rope = pkg.RotaryPlan(torch.ones(d // 2, dtype=torch.float64, device=DEV))
    x, pos = normal(1, T, H, d), torch.arange(T, dtype=torch.int32, device=DEV)
    pool = pkg.PagePool.empty(4, H, 16, d, torch.float32)
    want = pkg.meda_rotary(x, x, pos, rope)[0]
    side.wait_stream(torch.cuda.current_stream())
    q, k = pkg.meda_rotary(x, x, pos, rope, stream=side)
    a = pkg.meda_paged_append(pool, x, x, torch.arange(T, device=DEV), x, pos, rope, stream=side)
    torch.cuda.synchronize()
    for t in (q, k, a):
        assert _stream_of(t) == side.cuda_stream and torch.equal(t, want)


def test_two_streams_at_once():
    """Two caches, each on a stream of its own and nothing between them, against the same work one after the other."""
    import paper_2502_17599_amd as pkg
    L, Hq, Hkv, d, N, steps = 2, 8, 2, 64, 40, 12
    x = [normal(200 + i, N, Hq + 2 * Hkv, d, dtype="bf16") for i in range(2)]

    def make():
        cache = pkg.PagedCache(N, L, Hq, Hkv, d, max_len=4000, n_pages=N * L * 3, page_size=16)
        return cache, torch.zeros((steps, L, N, Hq, d), dtype=torch.bfloat16, device=DEV)

    def work(cache, outs, y):
        for s in range(steps):
            cache.step()
            for l in range(L):
                cache.append(l, y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:])
                cache.attend(l, y[:, :Hq], outs[s, l])

    alone, together = [make() for _ in range(2)], [make() for _ in range(2)]
    for i in range(2):
        work(*alone[i], x[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            work(*together[i], x[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(alone[i][1], together[i][1])
        assert torch.equal(alone[i][0].lens, together[i][0].lens) and torch.equal(alone[i][0].table, together[i][0].table)
