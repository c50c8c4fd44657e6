"""Limits of the operators' C ABI that need no GPU: sizes whose outputs are only partly empty."""

import pytest

from paper_1905_11722_amd import rcdp
from tests import ops_abi as abi
from tests.test_ops_host import NONE, scan


@pytest.mark.parametrize("missing", ["dB", "dC"])
def test_a_scan_without_channels_still_has_gradients_of_b_and_c(missing):
    a = scan(width=0, u=NONE, dt=NONE, dy=NONE, du=NONE, ddt=NONE, y=NONE, **{missing: None})
    assert abi.library().rc_scan_backward(a, None) == rcdp.E_ARG
    a.batch = 0
    assert abi.library().rc_scan_backward(a, None) == 0
