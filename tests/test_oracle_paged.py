"""The oracle of the paged cache, pinned: pages are conserved and never held twice, rotations against complex numbers,
their group property and differences, attention over shuffled pages against attention over contiguous rows."""
import numpy as np
import pytest

from oracle import paged_oracle as P
from oracle.decode_oracle import attend


@pytest.mark.parametrize("page,n_pages,seed", [(16, 40, 0), (64, 9, 1), (32, 3, 2), (16, 1, 3)])
def test_pages_are_conserved_and_held_once(page, n_pages, seed):
    rng = np.random.default_rng(seed)
    R, width = 7, 6
    lens, table = np.zeros(R, np.int32), np.full((R, width), -1, np.int32)
    ring, state = rng.permutation(n_pages).astype(np.int32), np.array([n_pages // 2, n_pages])
    for _ in range(60):
        new = rng.choice([-1, 0, 1, 1, page // 2, 3 * page], size=R)
        before = lens.copy()
        lens, table, ring, state, slots, granted = P.page_update(lens, new, table, ring, state, page, 2)
        held = [int(x) for r in range(R) for x in table[r, :P.blocks(int(lens[r]), page)]]
        free = [int(ring[(state[0] + i) % n_pages]) for i in range(state[1])]
        assert sorted(held + free) == list(range(n_pages))
        for r in range(R):
            assert granted[r] in (new[r], 0) and lens[r] == (0 if new[r] < 0 else before[r] + max(0, granted[r]))
            assert (slots[r] >= 0).sum() == min(2, max(0, granted[r]))


def test_rows_granted_together_are_a_whole_or_nothing():
    table, ring = np.full((4, 3), -1), np.arange(5)
    lens, table, ring, state, slots, granted = P.page_update([0, 0, 0, 0], [16, 17, 16, 17], table, ring, [0, 5], 16, 1, rows_per_seq=2)
    assert granted.tolist() == [16, 17, 0, 0] and lens.tolist() == [16, 17, 0, 0] and state.tolist() == [3, 2]
    assert table[0, 0] == 0 and table[1, :2].tolist() == [1, 2] and (table[2:] == -1).all()
    # the first sequence asks for more than a table holds and needs no pages then; a row of the second has ended
    lens, table, ring, state, slots, granted = P.page_update(lens, [1, 48, 3, -1], table, ring, state, 16, 1, rows_per_seq=2)
    assert granted.tolist() == [0, 0, 3, -1] and lens.tolist() == [16, 17, 3, 0] and state.tolist() == [4, 1] and slots[2, 0] == 3 * 16


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_product_of_complex_numbers(interleaved):
    rng = np.random.default_rng(4)
    T, H, d, half = 5, 3, 16, 6
    x, pos = rng.normal(size=(T, H, d)), rng.integers(-50, 50, size=(2, T))
    freq, axis = 1.0 / 10.0 ** np.arange(half), np.array([0, 1, 0, 1, 1, 0])
    y = P.rotate(x, pos, freq, axis, interleaved)
    i = np.arange(half) * 2 if interleaved else np.arange(half)
    j = i + 1 if interleaved else i + half
    z = (x[:, :, i] + 1j * x[:, :, j]) * np.exp(1j * pos[axis].T * freq)[:, None]
    assert np.allclose(y[:, :, i], z.real, atol=1e-14) and np.allclose(y[:, :, j], z.imag, atol=1e-14)
    assert np.array_equal(y[:, :, 2 * half:], x[:, :, 2 * half:])
    assert np.allclose(P.rotate(y, pos, freq, axis, interleaved, inverse=True), x, atol=1e-14)
    assert np.allclose(P.rotate(P.rotate(x, pos, freq, axis, interleaved), pos, freq, axis, interleaved),
                       P.rotate(x, 2 * pos, freq, axis, interleaved), atol=1e-13)


def test_inverse_rotation_is_the_gradient_by_differences():
    rng = np.random.default_rng(5)
    T, H, d = 2, 1, 8
    x, g, pos, freq = rng.normal(size=(T, H, d)), rng.normal(size=(T, H, d)), np.array([[3, 17]]), np.array([1.0, 0.3, 0.1])
    grad = P.rotate(g, pos, freq, inverse=True)
    for at in np.ndindex(x.shape):
        e = np.zeros_like(x); e[at] = 1e-5
        diff = ((P.rotate(x + e, pos, freq) - P.rotate(x - e, pos, freq)) * g).sum() / 2e-5
        assert abs(diff - grad[at]) < 1e-9


def test_attention_over_shuffled_pages_is_attention_over_contiguous_rows():
    rng = np.random.default_rng(6)
    page, Hkv, d, lens = 16, 2, 8, [0, 1, 16, 17, 61]
    n_pages = 12
    k, v = rng.normal(size=(2, n_pages, Hkv, page, d))
    order, table, at = rng.permutation(n_pages), np.full((5, 4), -1), 0
    for r, n in enumerate(lens):
        for b in range(P.blocks(n, page)):
            table[r, b] = order[at]; at += 1
    q = rng.normal(size=(5, 6, d))
    out = P.attention(q, k, v, table, lens)
    assert np.array_equal(out[0], np.zeros((6, d)))
    assert np.allclose(out[1], np.repeat(v[table[1, 0]][:, 0], 3, axis=0))
    rows_k = np.concatenate([k[p][1] for p in table[4]])[:61]
    rows_v = np.concatenate([v[p][1] for p in table[4]])[:61]
    assert np.allclose(out[4, 3], attend(q[4, 3], rows_k, rows_v))
    table[4, 1] = n_pages      # a page that does not exist: its positions are left out
    keep = np.r_[0:16, 32:61]
    assert np.allclose(P.attention(q, k, v, table, lens)[4, 3], attend(q[4, 3], rows_k[keep], rows_v[keep]))
