"""Random sessions of a paged cache against lists of rows: prompts come and go, sequences grow by a token at a time, pages run
out, layers are appended in part.  The model keeps for every (sequence, layer) the k and v rows it should hold, in 64 bits."""
import numpy as np
import pytest
import torch

from oracle.decode_oracle import attend
from paged_cases import DEV, DT, attention_tolerance, normal, wide
from test_gpu_paged_rows import _cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,N,L,Hq,Hkv,d,page,n_pages,seed", [
    ("bf16", 5, 3, 6, 2, 64, 16, 60, 0), ("f32", 3, 2, 4, 4, 128, 32, 14, 1), ("bf16", 70, 1, 16, 1, 128, 16, 200, 2), ("f32", 2, 5, 7, 1, 64, 64, 12, 3), ("bf16", 5, 3, 6, 2, 64, 16, 12, 4)])
def test_sessions(dtype, N, L, Hq, Hkv, d, page, n_pages, seed):
    import paper_2502_17599_amd as pkg
    print(f"\n[session] {dtype} N={N} L={L} {Hq}/{Hkv} d={d} page={page} pages={n_pages}", flush=True)
    rng = np.random.default_rng(seed)
    max_len = 150
    cache = pkg.PagedCache(N, L, Hq, Hkv, d, max_len=max_len, n_pages=n_pages, page_size=page, dtype=DT[dtype])
    blocks = lambda n: -(-n // page)                                     # noqa: E731
    most = blocks(max_len) * page
    rows = [[(np.zeros((0, Hkv, d)), np.zeros((0, Hkv, d))) for _ in range(L)] for _ in range(N)]

    def free():
        return n_pages - sum(blocks(len(k)) for seq in rows for k, _ in seq)

    def empty():
        return [(np.zeros((0, Hkv, d)), np.zeros((0, Hkv, d))) for _ in range(L)]

    refused = 0
    for turn in range(60):
        what = rng.choice(["admit", "step", "step", "step", "step", "release"])
        if what == "release":
            gone = [int(s) for s in rng.permutation(N)[:int(rng.integers(0, max(2, N // 3)))]]
            cache.release(gone)
            for s in gone:
                rows[s] = empty()
        elif what == "admit":
            n = int(rng.integers(1, min(N, 3) + 1))
            first = int(rng.integers(0, N - n + 1))
            total = int(rng.integers(L, 60 * L))
            lens = [[int(x) for x in rng.multinomial(total, np.ones(L) / L)] for _ in range(n)]
            cc, off = _cache(lens, Hkv, d, dtype, True, 100 + turn)
            got = cache.admit(first, cc).tolist()
            k_all, v_all = wide(cc.k_out), wide(cc.v_out)
            for i in range(n):
                rows[first + i] = empty()
            left, wanted = free(), 0
            for i in range(n):
                need = sum(blocks(x) for x in lens[i])
                fits = max(lens[i]) <= most
                wanted += need if fits else 0
                ok = fits and (need == 0 or wanted <= left)
                assert got[i] == (lens[i] if ok else [0] * L), turn
                refused += not ok
                if ok:
                    for l in range(L):
                        o, x = int(off[i, l]) * Hkv, lens[i][l]
                        rows[first + i][l] = tuple(np.moveaxis(a[o:o + x * Hkv].reshape(Hkv, x, d), 0, 1) for a in (k_all, v_all))
        else:
            active = rng.random(N) < 0.8
            left, wanted, want = free(), 0, []
            for s in range(N):
                lens = [len(k) for k, _ in rows[s]]
                fits = max(lens) + 1 <= most
                need = sum(x % page == 0 for x in lens) if active[s] and fits else 0
                wanted += need
                ok = bool(active[s]) and fits and (need == 0 or wanted <= left)
                refused += bool(active[s]) and not ok
                want.append(ok)
            got = cache.step(torch.from_numpy(active).to(DEV))
            assert got.tolist() == [[int(w)] * L for w in want], turn
            gone = int(rng.integers(0, N)) if turn % 5 == 0 else -1          # ends between the step and its appends
            if gone >= 0:
                cache.release([gone])
                rows[gone], want[gone] = empty(), False
            for l in range(L):
                x = normal(1000 * turn + l, N, 2 * Hkv, d, dtype=dtype)
                cache.append(l, x[:, :Hkv], x[:, Hkv:])
                x = wide(x)
                for s in range(N):
                    if want[s]:
                        k, v = rows[s][l]
                        rows[s][l] = (np.concatenate([k, x[s:s + 1, :Hkv]]), np.concatenate([v, x[s:s + 1, Hkv:]]))
        assert cache.lens.view(N, L).tolist() == [[len(k) for k, _ in seq] for seq in rows], turn
        assert int(cache.free_state[1]) == free(), turn
        l = int(rng.integers(0, L))
        q = normal(7 * turn, N, Hq, d, dtype=dtype)
        out, qs = wide(cache.attend(l, q)), wide(q)
        for s in range(N) if N < 10 else rng.permutation(N)[:8]:
            k, v = rows[s][l]
            if not len(k):
                assert (out[s] == 0).all(), (turn, s)
                continue
            ref = np.stack([attend(qs[s, h], k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)]) for h in range(Hq)])
            logit = max(np.abs(k[:, h // (Hq // Hkv)] @ qs[s, h]).max() for h in range(Hq)) * d ** -0.5
            assert (np.abs(out[s] - ref) <= attention_tolerance(ref, v, logit, len(k), d, dtype)).all(), (turn, s)
    assert refused or n_pages >= N * L                     # (a page for every layer)
    held = set()
    lens, table = cache.lens.tolist(), cache.table.cpu().numpy()
    for r, n in enumerate(lens):
        mine = table[r, :blocks(n)].tolist()
        assert not held & set(mine) and len(set(mine)) == len(mine)
        held |= set(mine)
    head, count = cache.free_state.tolist()
    ring = cache.free_ring.tolist()
    assert held | {ring[(head + i) % n_pages] for i in range(count)} == set(range(n_pages)) and len(held) + count == n_pages
