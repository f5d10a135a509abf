"""Scales of the logits that are finite and are not in the unit of the kernels' exponential (no GPU needed: the plan refuses)."""
import ctypes

import numpy as np
import pytest

import paper_2502_17599_amd as pkg
from paper_2502_17599_amd import _lib as L
from test_paged_abi import FAKE, INVALID, _attend, _params, _pool, ATT, lib   # noqa: F401


@pytest.mark.parametrize("scale", [3e38, 2.5e38, float(np.finfo(np.float32).max)])
def test_scales_past_the_range_are_refused(lib, scale):   # noqa: F811
    assert _attend(lib, dict(softmax_scale=scale)) == INVALID
    p, pool = _params(L.MedaPagedParams, ATT, dict(softmax_scale=scale)), _pool()
    assert lib.meda_paged_workspace_bytes(ctypes.byref(pool), ctypes.byref(p)) == 0


@pytest.mark.parametrize("scale", [0.0, 1e-40, 1.0, 2.3e38])
def test_scales_in_range_have_a_plan(lib, scale):   # noqa: F811
    p, pool = _params(L.MedaPagedParams, ATT, dict(softmax_scale=scale)), _pool()
    assert lib.meda_paged_workspace_bytes(ctypes.byref(pool), ctypes.byref(p)) > 0
    assert _attend(lib, dict(softmax_scale=scale), ws=None) == 4     # all that is missing is a workspace
