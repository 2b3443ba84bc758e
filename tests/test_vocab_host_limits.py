"""Limits of the vocabulary operators' arguments; nothing here reaches a GPU."""
from __future__ import annotations

import pytest
from test_vocab_host import ALL, P, SHAPE, _calls, _shape

OF_A_CALL = ALL - {"sample"}  # (sampling has its temperatures on the GPU, any number)


@pytest.mark.parametrize("temperature", [2.0**-128, 1e-39, 1e-45, 0.999 * 2.0**-127])
def test_temperatures_whose_reciprocal_is_no_fp32_number_are_refused(temperature):
    assert _calls(_shape(), names=OF_A_CALL, temperature=temperature) == {name: SHAPE for name in OF_A_CALL}
    assert _calls(_shape(n=0, held=0), None, names=OF_A_CALL, temperature=temperature) == {name: SHAPE for name in OF_A_CALL}


@pytest.mark.parametrize("temperature", [2.0**-127, 2.0**-126, 3e38])
def test_the_least_and_largest_temperatures_are_taken(temperature):
    assert _calls(_shape(n=0, held=0), None, names=OF_A_CALL, temperature=temperature) == {name: 0 for name in OF_A_CALL}
