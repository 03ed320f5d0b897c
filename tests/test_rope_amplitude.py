"""Amplitudes are applied in binary32: one that is infinite or zero there is refused.  Host arithmetic only."""
import ctypes as C

import pytest

from paper_2401_09135_b200 import binding as B
from test_ops_host_decoder import rope, rope_desc


@pytest.mark.parametrize("amplitude", [1e39, -1e39, 1e300, 1e-46, -1e-300])
def test_amplitudes_that_binary32_does_not_hold(amplitude):
    assert rope(desc=rope_desc(amplitude=amplitude)) == B.E_ARG
    assert B.lib().alsgd_rope_frequencies(rope_desc(amplitude=amplitude), (C.c_double * 32)()) == B.E_ARG


@pytest.mark.parametrize("amplitude", [3e38, -3e38, 1e-38, 1e-44, 0.5])
def test_amplitudes_that_it_holds(amplitude):
    assert B.lib().alsgd_rope_frequencies(rope_desc(amplitude=amplitude), (C.c_double * 32)()) == B.OK
