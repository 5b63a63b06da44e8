"""Calls of the target-side entry points that have no sound result: temperatures without a finite step, outputs over what
the call reads or writes elsewhere.  On a host without a GPU: nothing is launched."""
import ctypes as C
import math

import pytest

from paper_2609_24197_amd import hspec
from test_target_abi_cpu import FAKE, SHAPE, UNSUPPORTED, WORKSPACE, _chunk, _lib, _verify

WS = 1 << 50


@pytest.mark.parametrize("name", ["temperature", "draft_temperature"])
@pytest.mark.parametrize("value", [math.inf, 0.0, -1.0, math.nan, 1e-45])
def test_temperatures_without_a_finite_step(name, value):
    """log2(e) / T has to be positive and finite: with 0, masked logits give 0 x infinity."""
    assert _verify(**{name: value}) == SHAPE
    assert b"temperature" in _lib().hspec_last_error()
