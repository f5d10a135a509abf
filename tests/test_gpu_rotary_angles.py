"""Sines and cosines of a rotation are those of the angle in 64 bits, also where they are near zero.

Pairs (1, 0) become (cos, sin).  The library's sine and cosine are good to 2 steps of their value (2^-22 of it), the two
corrections round once (2^-24): below 2^-21 of the value.  The number of turns has an error of three roundings, 3 * 2^-53 of
it: 2 pi * 3200 * 3 * 2^-53 < 2^-37 rad for 20000 rad."""
import numpy as np
import pytest
import torch

from paged_cases import DEV, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("freq", [1.0, 0.7310585786300049, 1.0 / 3.0])
def test_sines_and_cosines_to_a_few_roundings_of_their_value(freq, inverse, interleaved):
    import paper_2502_17599_amd as pkg
    T, half = 20001, 1
    rope = pkg.RotaryPlan(torch.tensor([freq], dtype=torch.float64, device=DEV), interleaved=interleaved)
    pos = torch.arange(T, dtype=torch.int32) - T // 2
    x = torch.zeros((T, 1, 64), device=DEV)
    x[..., 0] = 1.0
    x[..., 2] = 5.0                                        # behind the pair: as it is
    out = wide(pkg.meda_rotary(x, None, pos.to(DEV), rope, inverse=inverse)[0])[:, 0]
    angle = pos.double().numpy() * freq
    for got, want in ((out[:, 0], np.cos(angle)), (out[:, half], np.sin(angle) * (-1.0 if inverse else 1.0))):
        err = np.abs(got - want)
        assert (err <= 2.0 ** -21 * np.abs(want) + 2.0 ** -37).all(), float((err - 2.0 ** -21 * np.abs(want)).max())
    assert np.array_equal(out[:, 2:], wide(x)[:, 0, 2:])
