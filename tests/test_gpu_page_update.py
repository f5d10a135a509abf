"""Block tables, slot maps and free pages against the oracle: whole numbers, so they have to be equal."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paged_cases import DEV

pytestmark = pytest.mark.gpu


def _dev(x, dtype):
    return torch.tensor(np.asarray(x), dtype=dtype, device=DEV)


class State:
    def __init__(self, R, width, n_pages, seed, head=0):
        rng = np.random.default_rng(seed)
        self.lens, self.table = np.zeros(R, np.int32), np.full((R, width), -1, np.int32)
        self.ring, self.state = rng.permutation(n_pages).astype(np.int32), np.array([head % n_pages, n_pages], np.int64)

    def step(self, new, page, max_new, in_place, per=1):
        import paper_2502_17599_amd as pkg
        print(f"\n[page update] R={len(new)} pages={len(self.ring)} page={page} max_new={max_new} in_place={in_place}", flush=True)
        lens, table, ring, state = (_dev(self.lens, torch.int32), _dev(self.table, torch.int32), _dev(self.ring, torch.int32),
                                    _dev(self.state, torch.int64))
        R = len(new)
        slots = torch.full((R, max_new), 99, dtype=torch.int64, device=DEV)
        granted = torch.full((R,), 99, dtype=torch.int32, device=DEV)
        lens_out = None if in_place else torch.full_like(lens, 99)
        state_out = None if in_place else torch.full_like(state, 99)
        pkg.meda_page_update(lens, _dev(new, torch.int32), table, ring, state, page, lens_out, state_out, slots, granted,
                             rows_per_seq=per)
        want = P.page_update(self.lens, new, self.table, self.ring, self.state, page, max_new, per)
        got = (lens if in_place else lens_out, table, ring, state if in_place else state_out, slots, granted)
        for name, g, w in zip(("lens", "table", "ring", "state", "slots", "granted"), got, want):
            assert np.array_equal(g.cpu().numpy(), w), name
        if not in_place:
            assert np.array_equal(lens.cpu().numpy(), self.lens) and np.array_equal(state.cpu().numpy(), self.state)
        self.lens, self.table, self.ring, self.state = want[:4]


@pytest.mark.parametrize("R,width,n_pages,page,max_new,seed", [
    (1, 1, 1, 16, 1, 0), (1, 5, 7, 16, 3, 1), (7, 6, 20, 16, 2, 2), (64, 9, 300, 32, 1, 3), (65, 12, 200, 64, 40, 4),
    (512, 30, 4000, 64, 1, 5), (1023, 5, 2000, 128, 0, 6), (1025, 4, 2500, 256, 5, 7), (2500, 7, 9000, 16, 1, 8), (6, 700, 2600, 16, 3000, 9)])
def test_random_histories(R, width, n_pages, page, max_new, seed):
    rng = np.random.default_rng(seed)
    s = State(R, width, n_pages, seed, head=int(rng.integers(n_pages)))
    for i in range(6):
        most = width * page
        new = rng.choice([-1, 0, 1, 1, 1, page, page + 1, max(1, most // 3), most + 1], size=R)
        if i == 0:
            new = rng.integers(0, max(2, min(most, 2 * page * n_pages // R)), size=R)   # a first filling that may not fit
        s.step(new, page, max_new, in_place=bool(i & 1))


@pytest.mark.parametrize("R,per,width,n_pages,page,max_new,seed", [
    (2, 2, 3, 4, 16, 1, 0), (64, 32, 9, 120, 16, 1, 1), (96, 3, 6, 200, 32, 40, 2), (66, 66, 5, 200, 16, 2, 3), (512, 32, 12, 2500, 16, 1, 4),
    (2048, 2, 4, 3000, 16, 1, 5), (2050, 41, 4, 3000, 16, 3, 6), (4096, 32, 5, 6000, 32, 1, 7), (6, 2, 700, 900, 16, 3000, 8)])
def test_rows_granted_together(R, per, width, n_pages, page, max_new, seed):
    rng = np.random.default_rng(seed)
    s = State(R, width, n_pages, seed, head=int(rng.integers(n_pages)))
    some, none = 0, 0
    for i in range(8):
        new = np.repeat(rng.choice([-1, 0, 1, 1, 1, page // 2, page + 1], size=R // per), per)
        odd = rng.random(R) < 0.5 / per                         # rows that ask for something else than their sequence
        new[odd] = rng.choice([-1, 0, 2, page, width * page + 1], size=int(odd.sum()))
        if i == 0:
            new = rng.integers(0, max(2, min(width * page, 2 * page * n_pages // R)), size=R)
        before = s.lens.copy()
        s.step(new, page, max_new, in_place=bool(i & 1), per=per)
        grown = ((s.lens > before) == (new > 0)).reshape(-1, per)[(new > 0).reshape(-1, per).any(1)]
        asked = (new > 0).reshape(-1, per)[(new > 0).reshape(-1, per).any(1)]
        for g, a in zip(grown, asked):                          # all that asked, or none of them
            assert g[a].all() or not g[a].any()
            some, none = some + bool(g[a].all()), none + (not g[a].any())
    assert some and none


def test_refusals_in_row_order_and_pages_given_back_serve_the_next_call():
    s = State(5, 4, 6, 0)
    s.step([64, 32, 0, 0, 0], 16, 1, True)             # all six pages held
    assert s.state[1] == 0
    s.step([-1, 1, 0, 1, 0], 16, 1, True)              # four come back, but not for this call
    assert s.lens.tolist() == [0, 32, 0, 0, 0] and s.state[1] == 4
    s.step([17, 1, 16, 0, 0], 16, 2, False)            # two, one, one: all fit
    assert s.lens.tolist() == [17, 33, 16, 0, 0]
    s.step([1, 1, 1, 1, 15], 16, 1, True)              # rows 2 and 3 need a page that is not there, the others do not
    assert s.lens.tolist() == [18, 34, 16, 0, 0]


def test_ring_state_and_lengths_out_of_range_are_clamped():
    """Numbers that no call of the library writes: nothing is read or written out of bounds."""
    import paper_2502_17599_amd as pkg
    ring, table = torch.arange(8, dtype=torch.int32, device=DEV), torch.full((3, 4), -1, dtype=torch.int32, device=DEV)
    lens, state = _dev([-5, 10 ** 6, 3], torch.int32), _dev([-9, 10 ** 12], torch.int64)
    granted = torch.zeros(3, dtype=torch.int32, device=DEV)
    pkg.meda_page_update(lens, _dev([16, 1, 2], torch.int32), table, ring, state, 16, granted=granted)
    assert granted.tolist() == [16, 0, 2] and lens.tolist() == [16, 64, 5]
    assert state.tolist() == [0, 7] and table[0].tolist() == [7, -1, -1, -1]


def test_no_slots_and_no_granted():
    import paper_2502_17599_amd as pkg
    ring, table = torch.arange(8, dtype=torch.int32, device=DEV), torch.full((1, 4), -1, dtype=torch.int32, device=DEV)
    lens, state = _dev([0], torch.int32), _dev([0, 8], torch.int64)
    pkg.meda_page_update(lens, _dev([40], torch.int32), table, ring, state, 16)
    assert lens.tolist() == [40] and table.tolist() == [[0, 1, 2, -1]] and state.tolist() == [3, 5]
