"""Scales that the attention refuses, without a GPU (refusals come before any HIP call)."""
import math

import pytest
from test_host_serve import ALIGN, PARAM, attend, descriptor


@pytest.mark.parametrize("scale", [math.inf, -math.inf, math.nan, 3.0e38, -2.4e38])
def test_a_scale_that_is_no_number_in_powers_of_two(scale):
    """Scores are taken to powers of two: scale * log2(e) has to be a number too."""
    assert attend(descriptor(scale=scale, workspace=0x100080)) == PARAM


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45, 2.3e38])
def test_a_scale_that_is_one(scale):
    """(The next check behind the scale's refuses these calls.)"""
    assert attend(descriptor(scale=scale, workspace=0x100080)) == ALIGN
