"""Slot maps of the largest size: indexes at the end of the range of int."""
import pytest
import torch

from paged_cases import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [True, False])
def test_as_many_slots_as_a_row_can_have(in_place):
    """2^31 - 1 columns (17 GB): a row is granted 40 positions, every other column says so."""
    import paper_2502_17599_amd as pkg
    print(f"\n[page update] max_new=2^31-1 in_place={in_place}", flush=True)
    ring = torch.tensor([5, 3, 4, 1, 2, 0, 6, 7], dtype=torch.int32, device=DEV)
    table = torch.full((1, 4), -1, dtype=torch.int32, device=DEV)
    lens, new = (torch.tensor([n], dtype=torch.int32, device=DEV) for n in (0, 40))
    state = torch.tensor([0, 8], dtype=torch.int64, device=DEV)
    slots = torch.full((1, 2 ** 31 - 1), 99, dtype=torch.int64, device=DEV)
    out = {} if in_place else dict(lens_out=torch.zeros_like(lens), free_state_out=torch.zeros_like(state))
    pkg.meda_page_update(lens, new, table, ring, state, 16, slots=slots, **out)
    assert table.tolist() == [[5, 3, 4, -1]] and out.get("lens_out", lens).tolist() == [40]
    assert out.get("free_state_out", state).tolist() == [3, 5]
    assert slots[0, :40].tolist() == [p * 16 + i for p in (5, 3, 4) for i in range(16)][:40]
    rest = slots[0, 40:]
    for part in rest.split(1 << 28):
        assert bool((part == -1).all())
    del slots, rest, part
    torch.cuda.empty_cache()
