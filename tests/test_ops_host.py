"""The operators' C ABI and binding without a GPU: the header is plain C and
agrees with the binding's structs, every declared call is exported, and bad
arguments are refused before any device call."""

import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_1905_11722_amd import ops, rcdp
from tests import ops_abi as abi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "rc_ops.h")
STRUCTS = {"rc_conv_args": abi.ConvArgs, "rc_conv_step_args": abi.ConvStepArgs,
           "rc_scan_args": abi.ScanArgs, "rc_scan_step_args": abi.ScanStepArgs,
           "rc_norm_args": abi.NormArgs}


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = re.findall(r"^int (rc_\w+)\(", text, flags=re.M)
    assert len(names) >= 12
    lib = rcdp.load_library()
    for name in names:
        assert hasattr(lib, name), name


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no C compiler")
def test_header_is_plain_c_and_matches_the_binding(tmp_path):
    lines = []
    for name, struct in STRUCTS.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        for field, _ in struct._fields_:
            lines.append(f'printf("{name}.{field} %zu\\n", offsetof({name}, {field}));')
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "rc_ops.h"\nint main(void) {\n' + "\n".join(lines)
                   + "\nreturn 0; }\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I",
                           os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    said = dict(line.split() for line in subprocess.check_output([str(exe)], text=True).splitlines())
    for name, struct in STRUCTS.items():
        assert int(said[name]) == ctypes.sizeof(struct), name
        for field, _ in struct._fields_:
            assert int(said[f"{name}.{field}"]) == getattr(struct, field).offset, (name, field)


X = 0x1000          # stands for a device pointer; no call below gets as far as using it


def view(data=X):
    return abi.View(data, 64, 8)


def conv(**kw):
    a = abi.ConvArgs(dtype=1, activation=1, batch=2, length=8, width=8, taps=4, x=view(), y=view(),
                      weight=X, dy=view(), dx=view())
    return set_all(a, kw)


def scan(**kw):
    a = abi.ScanArgs(dtype=1, batch=2, length=8, width=8, states=16, groups=2, u=view(), dt=view(),
                      B=view(), C=view(), y=view(), A=X, kept=X, dy=view(), du=view(), ddt=view(),
                      dB=X, dC=X, dA=X)
    return set_all(a, kw)


def norm(**kw):
    a = abi.NormArgs(dtype=1, gate_activation=1, rows=4, width=8, eps=1e-5, block=view(),
                      residual=view(), out=view(), normed=view(), pre_weight=X, stats=X,
                      dblock=view(), dresidual=view())
    return set_all(a, kw)


def set_all(a, kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return a


NONE = abi.View()
BAD = [
    ("rc_conv_forward", conv, dict(dtype=3)), ("rc_conv_forward", conv, dict(dtype=-1)),
    ("rc_conv_forward", conv, dict(param_dtype=2)), ("rc_conv_forward", conv, dict(activation=2)),
    ("rc_conv_forward", conv, dict(taps=0)), ("rc_conv_forward", conv, dict(taps=9)),
    ("rc_conv_forward", conv, dict(batch=-1)), ("rc_conv_forward", conv, dict(width=-8)),
    ("rc_conv_forward", conv, dict(length=-1)), ("rc_conv_forward", conv, dict(weight=None)),
    ("rc_conv_forward", conv, dict(x=NONE)), ("rc_conv_forward", conv, dict(y=NONE)),
    ("rc_conv_backward", conv, dict(dy=NONE)), ("rc_conv_backward", conv, dict(dx=NONE)),
    ("rc_conv_forward", conv, dict(length=2 ** 30 + 1)), ("rc_conv_forward", conv, dict(width=2 ** 30 + 8)),
    ("rc_scan_forward", scan, dict(length=2 ** 30 + 1)), ("rc_scan_forward", scan, dict(width=2 ** 30 + 8)),
    ("rc_scan_forward", scan, dict(states=0)), ("rc_scan_forward", scan, dict(states=65)),
    ("rc_scan_forward", scan, dict(groups=3)), ("rc_scan_forward", scan, dict(groups=0)),
    ("rc_scan_forward", scan, dict(A=None)), ("rc_scan_forward", scan, dict(B=NONE)),
    ("rc_scan_forward", scan, dict(y=NONE)), ("rc_scan_backward", scan, dict(kept=None)),
    ("rc_scan_backward", scan, dict(dA=None)), ("rc_scan_backward", scan, dict(z=view())),
    ("rc_scan_backward", scan, dict(D=X)), ("rc_scan_backward", scan, dict(dt_bias=X)),
    ("rc_scan_backward", scan, dict(dB=None)),
    ("rc_norm_forward", norm, dict(width=16385)), ("rc_norm_forward", norm, dict(rows=-1)),
    ("rc_norm_forward", norm, dict(gate_activation=0)), ("rc_norm_forward", norm, dict(residual=NONE)),
    ("rc_norm_forward", norm, dict(residual_dtype=2)), ("rc_norm_forward", norm, dict(normed=NONE)),
    ("rc_norm_forward", norm, dict(out=NONE)), ("rc_norm_forward", norm, dict(block=NONE, scale=X)),
    ("rc_norm_forward", norm, dict(block=NONE, pre_weight=None)),
    ("rc_norm_backward", norm, dict(stats=None)), ("rc_norm_backward", norm, dict(dblock=NONE)),
    ("rc_norm_backward", norm, dict(gate=view())),
]


@pytest.mark.parametrize("call,make,change", BAD, ids=lambda v: v if isinstance(v, str) else None)
def test_bad_arguments(call, make, change):
    assert getattr(abi.library(), call)(make(**change), None) == rcdp.E_ARG


def test_null_and_scratch():
    lib = abi.library()
    n = ctypes.c_uint64()
    for call in ("conv_forward", "conv_backward", "conv_step", "scan_forward", "scan_backward",
                 "scan_step", "norm_forward", "norm_backward"):
        assert getattr(lib, "rc_" + call)(None, None) == rcdp.E_ARG
    for call in ("conv_backward_workspace", "scan_kept_bytes", "scan_forward_workspace",
                 "scan_backward_workspace", "norm_backward_workspace"):
        assert getattr(lib, "rc_" + call)(None, n) == rcdp.E_ARG
    # a scratch that is too small is refused before any work
    a = conv(dweight=X)
    assert lib.rc_conv_backward_workspace(a, n) == 0 and n.value > 0
    a.workspace, a.workspace_bytes = X, n.value - 1
    assert lib.rc_conv_backward(a, None) == rcdp.E_SCRATCH
    a = scan()
    assert lib.rc_scan_backward_workspace(a, n) == 0 and n.value > 0
    a.workspace, a.workspace_bytes = X, n.value - 1
    assert lib.rc_scan_backward(a, None) == rcdp.E_SCRATCH
    a = norm(dpre_weight=X)
    assert lib.rc_norm_backward_workspace(a, n) == 0 and n.value > 0
    a.workspace, a.workspace_bytes = X, n.value - 1
    assert lib.rc_norm_backward(a, None) == rcdp.E_SCRATCH


def test_step_arguments():
    lib = abi.library()
    a = abi.ConvStepArgs(dtype=0, activation=1, batch=3, width=8, taps=4, num_slots=2, x=view(),
                          y=view(), state=view(), weight=X)
    assert lib.rc_conv_step(a, None) == rcdp.E_ARG                 # fewer slots than rows
    a.slots, a.weight = X, None
    assert lib.rc_conv_step(a, None) == rcdp.E_ARG
    b = abi.ScanStepArgs(dtype=0, batch=3, width=8, states=4, groups=1, num_slots=2, u=view(),
                          dt=view(), B=view(), C=view(), y=view(), A=X, state=X)
    assert lib.rc_scan_step(b, None) == rcdp.E_ARG
    b.slots, b.state = X, None
    assert lib.rc_scan_step(b, None) == rcdp.E_ARG


def test_empty_calls_do_nothing():
    lib = abi.library()
    assert lib.rc_conv_forward(conv(batch=0), None) == 0
    assert lib.rc_conv_forward(conv(width=0), None) == 0
    assert lib.rc_scan_forward(scan(batch=0), None) == 0
    assert lib.rc_norm_forward(norm(rows=0), None) == 0
    assert lib.rc_norm_backward(norm(width=0), None) == 0


def test_no_cpu_path():
    x = torch.randn(1, 4, 8)
    with pytest.raises(ValueError):
        ops.causal_conv(x, torch.randn(8, 4))
    with pytest.raises(ValueError):
        ops.selective_scan(x, x, -torch.rand(8, 4), torch.randn(1, 4, 4), torch.randn(1, 4, 4))
    with pytest.raises(ValueError):
        ops.norm_residual(x, x)
