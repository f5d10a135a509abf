"""Compressed caches that the store would not take: `admit` refuses them while the sequences still hold what they held."""
import dataclasses

import pytest
import torch

from paged_cases import DEV
from test_gpu_paged_rows import _cache
from test_gpu_paged_serving import _state

pytestmark = pytest.mark.gpu


def test_refused_before_anything_changes():
    import paper_2502_17599_amd as pkg
    L, Hkv, d = 3, 2, 64
    cc, _ = _cache([[40, 17, 60]], Hkv, d, "f32", False, 1)
    cache = pkg.PagedCache(2, L, 4, Hkv, d, max_len=64, n_pages=40, page_size=16, dtype=torch.float32)
    cache.pool.k_pages.zero_()
    assert cache.admit(0, cc).tolist() == [[40, 17, 60]]
    cache.step()
    before = _state(cache) + [cache.slots.clone()]
    rows = cc.k_out.shape[0]
    odd = torch.zeros(rows * d + 2, device=DEV)[2:].view(rows, d)           # 8 bytes behind a border of 16
    for bad in (dict(k_out=odd), dict(v_out=odd), dict(k_out=cc.k_out.clone().requires_grad_()), dict(v_out=cc.v_out * torch.ones(1, device=DEV, requires_grad=True))):
        with pytest.raises(ValueError):
            cache.admit(0, dataclasses.replace(cc, **bad))
    assert all(torch.equal(a, b) for a, b in zip(before, _state(cache) + [cache.slots]))
    with torch.no_grad():
        assert cache.admit(1, dataclasses.replace(cc, k_out=cc.k_out.clone().requires_grad_())).tolist() == [[40, 17, 60]]


def test_tables_too_large_for_a_store():
    """A table of 2^27 positions can be attended over a layer at a time; all its layers in one store are past its numbers."""
    import paper_2502_17599_amd as pkg
    L, Hkv, d = 32, 8, 64
    cc, _ = _cache([[5] * L], Hkv, d, "bf16", False, 1)
    cache = pkg.PagedCache(1, L, Hkv, Hkv, d, max_len=1 << 27, n_pages=64, page_size=256)
    cache.pool.k_pages.zero_()
    assert cache.step().tolist() == [[1] * L]
    before = _state(cache)
    with pytest.raises(ValueError, match="positions"):
        cache.admit(0, cc)
    assert all(torch.equal(a, b) for a, b in zip(before, _state(cache)))
