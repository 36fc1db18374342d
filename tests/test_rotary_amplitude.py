"""Amplitudes that fp32 does not hold to its precision are refused: turned elements would lose digits, or all become zeros."""
import ctypes as c

import pytest

from paper_2207_08822_amd import fxp
from tests.test_abi import load
from tests.test_serve_abi import BIG, cache, rotation, step

SMALLEST = 2.0 ** -126


@pytest.fixture(scope="module")
def L():
    load()
    return fxp.lib()


@pytest.mark.parametrize("amplitude", [1e-300, 1e-46, 1e-40, SMALLEST * (1 - 2.0 ** -52)])
def test_too_small(L, amplitude):
    rope = rotation(amplitude=amplitude)
    assert L.fxp_rotary(rope, 0, 1, 2, 4, 2, 64, BIG, 512, 128, 64, BIG, 0, BIG, 512, 128, 64, None) == -10
    assert L.fxp_kv_append_rotary(cache(), step(), rope, 1, BIG, 128, 64, BIG, 128, 64, BIG, 256, 64, 4, BIG, 256, 64, None) == -10
    with pytest.raises(fxp.FxpError, match="amplitude"):
        fxp.Rotary(8, amplitude=amplitude)


def test_the_smallest_is_allowed(L):
    assert c.c_float(SMALLEST).value == SMALLEST
    assert L.fxp_rotary(rotation(amplitude=SMALLEST), 0, 1, 0, 4, 2, 64, BIG, 512, 128, 64, BIG, 0, BIG, 512, 128, 64, None) == 0      # nothing to do
    assert L.fxp_rotary(rotation(amplitude=0.99e30), 0, 1, 0, 4, 2, 64, BIG, 512, 128, 64, BIG, 0, BIG, 512, 128, 64, None) == 0
