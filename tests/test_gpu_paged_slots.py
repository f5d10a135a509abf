"""Slots of a step whose sequences are released or replaced before their tokens are appended."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paged_cases import DEV, normal, values, wide
from test_gpu_paged_serving import _prompts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", ["release", "admit"])
def test_a_released_sequence_writes_into_nobodys_pages(how):
    """Sequence 0 is given a page per layer by a step and ends before the appends; the pages go to a prompt, which takes all
    there are.  What the layers then append for sequence 0 is written nowhere."""
    import paper_2502_17599_amd as pkg
    L, Hq, Hkv, d, page = 3, 4, 2, 64, 16
    _, compressed, T = _prompts(1, L, Hq, Hkv, d, "f32", 0, 32, L * 100, 130)
    need = int(((compressed.layer_len + page - 1) // page).sum())
    cache = pkg.PagedCache(3, L, Hq, Hkv, d, max_len=T, n_pages=need + L, page_size=page, dtype=torch.float32)
    cache.pool.k_pages.zero_(); cache.pool.v_pages.zero_()
    assert cache.step(torch.tensor([1, 0, 1], device=DEV)).tolist() == [[1] * L, [0] * L, [1] * L]
    kept = cache.slots[2 * L:].clone()
    if how == "release":
        cache.release([0])
        to = 1
    else:
        to = 0
    assert torch.equal(cache.admit(to, compressed), compressed.layer_len)
    assert int(cache.free_state[1]) == 0 and torch.equal(cache.slots[2 * L:], kept) and (cache.slots[:2 * L] == -1).all()
    x = normal(7, 3, Hkv, d)
    for l in range(L):
        cache.append(l, x, x)
    kp, vp = values(cache.pool)
    one = compressed.sequence(0) if compressed.layer_len.dim() == 2 else compressed
    for l in range(L):
        row, n = cache.table[to * L + l].cpu().numpy(), int(compressed.layer_len.reshape(-1)[l])
        for pages_of, rows in zip((kp, vp), one.layer(l)[:2]):
            assert np.array_equal(P.gather(pages_of, row, n), wide(rows))
        # the sequence that goes on has its token
        assert np.array_equal(P.gather(kp, cache.table[2 * L + l].cpu().numpy(), 1)[:, 0], wide(x)[2])


def test_a_wrong_sequence_changes_nothing():
    import paper_2502_17599_amd as pkg
    cache = pkg.PagedCache(2, 2, 4, 2, 64, max_len=64, n_pages=8, page_size=16)
    cache.step()
    before = [t.clone() for t in (cache.slots, cache.lens, cache.table, cache.free_ring, cache.free_state)]
    for seqs in ([0, 2], (1, -1), range(3)):
        with pytest.raises(ValueError):
            cache.release(seqs)
    for a, b in zip(before, (cache.slots, cache.lens, cache.table, cache.free_ring, cache.free_state)):
        assert torch.equal(a, b)
    cache.release(s for s in (1, 1))       # named twice
    assert cache.lens.tolist() == [1, 1, 0, 0] and int(cache.free_state[1]) == 6 and (cache.slots[2:] == -1).all() and (cache.slots[:2] >= 0).all()
