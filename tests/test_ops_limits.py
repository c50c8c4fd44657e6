"""Limits of the operators' C ABI that need no GPU: sizes whose outputs are only partly empty, sizes
beyond a launch's (fewer than 2^32 threads), which are refused before anything is enqueued, alignment."""

import pytest

from paper_1905_11722_amd import rcdp
from tests import ops_abi as abi
from tests.test_ops_host import NONE, X, conv, norm, scan, view


@pytest.mark.parametrize("missing", ["dB", "dC"])
def test_a_scan_without_channels_still_has_gradients_of_b_and_c(missing):
    a = scan(width=0, u=NONE, dt=NONE, dy=NONE, du=NONE, ddt=NONE, y=NONE, **{missing: None})
    assert abi.library().rc_scan_backward(a, None) == rcdp.E_ARG
    a.batch = 0
    assert abi.library().rc_scan_backward(a, None) == 0


# 256 threads a workgroup (512 from 17 states on): 2^24 workgroups are too many
BEYOND = [
    ("rc_conv_forward", conv, dict(batch=2 ** 26, length=32, width=1024)),
    ("rc_conv_backward", conv, dict(batch=2 ** 26, length=32, width=1024)),
    ("rc_conv_backward", conv, dict(batch=1, length=1, width=2 ** 25, taps=7, dweight=X)),
    ("rc_scan_forward", scan, dict(batch=2 ** 24, length=1, width=64, groups=1)),
    ("rc_scan_forward", scan, dict(batch=2 ** 23, length=1, width=64, groups=1, states=17)),
    ("rc_scan_backward", scan, dict(batch=2 ** 24, length=1, width=64, groups=1)),
    # its kernels of channels fit, the one of sums over them does not: 2^32 (token, group, value) sums
    ("rc_scan_backward", scan, dict(batch=16, length=2 ** 18, width=64, groups=8, states=64)),
]


@pytest.mark.parametrize("call,make,change", BEYOND, ids=lambda v: v if isinstance(v, str) else None)
def test_sizes_beyond_a_launch(call, make, change):
    assert getattr(abi.library(), call)(make(**change), None) == rcdp.E_OVERFLOW


@pytest.mark.parametrize("call,make,change", [
    ("rc_conv_backward", conv, dict(batch=1, length=1, width=2 ** 25 - 2, taps=7, dweight=X)),
    ("rc_scan_backward", scan, dict(batch=2 ** 24 - 1, length=1, width=64, groups=1)),
    ("rc_scan_backward", scan, dict(batch=16, length=2 ** 18 - 64, width=64, groups=8, states=64)),
], ids=["conv", "scan", "sums"])
def test_sizes_just_within(call, make, change):
    """The next check refuses them: no scratch is given."""
    assert getattr(abi.library(), call)(make(**change), None) == rcdp.E_SCRATCH


def test_tokens_beyond_a_launch():
    lib = abi.library()
    a = abi.ConvStepArgs(dtype=0, activation=1, batch=2 ** 24, width=512, taps=4, num_slots=2 ** 24, x=view(),
                         y=view(), state=view(), weight=X)
    assert lib.rc_conv_step(a, None) == rcdp.E_OVERFLOW
    b = abi.ScanStepArgs(dtype=0, batch=2 ** 24, width=1, states=4, groups=1, num_slots=2 ** 24, u=view(),
                         dt=view(), B=view(), C=view(), y=view(), A=X, state=X)
    assert lib.rc_scan_step(b, None) == rcdp.E_OVERFLOW


@pytest.mark.parametrize("off", [1, 2, 3])
def test_scratch_and_kept_states_are_aligned_to_a_float(off):
    lib = abi.library()
    for call, make, names in (("conv_backward", conv, ["workspace"]), ("scan_forward", scan, ["workspace", "kept"]),
                              ("scan_backward", scan, ["workspace", "kept"]), ("norm_backward", norm, ["workspace"])):
        for name in names:
            assert getattr(lib, "rc_" + call)(make(**{name: X + off}), None) == rcdp.E_ARG
