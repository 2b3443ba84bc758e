"""The oracle of the vocabulary operators at the ends of the numbers' range."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import vocab as ov


@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_a_rest_that_a_finite_mask_holds(tau):
    """All words beside the record lie at the lowest value: they share the mass outside it alike, and the gradient adds up to nothing."""
    z = np.full(12, -3.3e38)
    z[4], z[7] = 1.0, 2.5
    t, at = np.array([1.0, 2.0]), np.array([4, 7])
    lse = float(np.log(np.exp(t / tau).sum() / 0.9))  # a tenth outside
    _, grad, size = ov.distill(z, t, at, t_lse=lse, temperature=tau)
    others = np.delete(grad, at)
    assert np.allclose(others, -tau * 0.1 / 10, rtol=1e-12) and abs(grad.sum()) < 1e-12 and (np.abs(grad) <= size + 1e-15).all()
