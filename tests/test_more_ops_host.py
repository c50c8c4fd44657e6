"""The linear-attention operators' C ABI and binding without a GPU: struct layouts, refusals of bad
arguments, scratch and sizes before any device call; the references of the GPU tests among themselves."""

import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_1905_11722_amd import ops, rcdp
from tests import more_ops_abi as abi
from tests import more_ops_reference as ref
from tests.ops_abi import View

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"rc_heads": abi.Heads, "rc_delta_args": abi.DeltaArgs, "rc_delta_step_args": abi.DeltaStepArgs,
           "rc_qk_args": abi.QkArgs, "rc_dropout_args": abi.DropoutArgs}


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no C compiler")
def test_header_matches_the_structs(tmp_path):
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
NONE, NO_HEADS = View(), abi.Heads()


def heads(data=X):
    return abi.Heads(data, 1024, 64, 8)


def view(data=X):
    return View(data, 64, 8)


def set_all(a, kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def delta(**kw):
    a = abi.DeltaArgs(dtype=1, batch=2, length=40, key_heads=2, heads=4, key=16, value=24, scale=0.25,
                      q=heads(), k=heads(), v=heads(), o=heads(), g=view(), beta=view(), kept=X, do_=heads(),
                      dq=heads(), dk=heads(), dv=heads(), dg=X, dbeta=X)
    return set_all(a, kw)


def step(**kw):
    a = abi.DeltaStepArgs(dtype=1, batch=3, key_heads=2, heads=4, key=16, value=24, num_slots=3, scale=0.25,
                          q=heads(), k=heads(), v=heads(), o=heads(), g=view(), beta=view(), state=X,
                          state_slot=4 * 16 * 24)
    return set_all(a, kw)


def qk(**kw):
    a = abi.QkArgs(dtype=1, norm=1, batch=2, length=9, heads=4, key_heads=2, channels=32, rotated=16, eps=1e-6,
                   q=heads(), k=heads(), q_out=heads(), k_out=heads(), q_weight=X, k_weight=X, inv_freq=X,
                   dq_out=heads(), dk_out=heads(), dq=heads(), dk=heads())
    return set_all(a, kw)


def dropout(**kw):
    a = abi.DropoutArgs(dtype=1, out_dtype=1, rows=4, width=24, p=0.25, seed=1, x=view(), out=view())
    return set_all(a, kw)


BAD = [("rc_delta_" + call, delta, change) for call in ("forward", "backward") for change in (
    dict(dtype=3), dict(dtype=-1), dict(batch=-1), dict(length=-1), dict(length=2 ** 30 + 1), dict(key=0),
    dict(key=257), dict(value=0), dict(value=257), dict(heads=-1), dict(key_heads=3), dict(key_heads=0),
    dict(key_heads=-2), dict(heads=0), dict(q=NO_HEADS), dict(k=NO_HEADS), dict(v=NO_HEADS), dict(beta=NONE),
    dict(kept=X + 2), dict(workspace=X + 1))] + [
    ("rc_delta_forward", delta, dict(o=NO_HEADS)),
    ("rc_delta_backward", delta, dict(do_=NO_HEADS)), ("rc_delta_backward", delta, dict(dq=NO_HEADS)),
    ("rc_delta_backward", delta, dict(dk=NO_HEADS)), ("rc_delta_backward", delta, dict(dv=NO_HEADS)),
    ("rc_delta_backward", delta, dict(dg=None)), ("rc_delta_backward", delta, dict(g=NONE)),
    ("rc_delta_backward", delta, dict(dbeta=None)), ("rc_delta_backward", delta, dict(kept=None))] + [
    ("rc_delta_step", step, change) for change in (
        dict(dtype=4), dict(batch=-1), dict(key=0), dict(key=257), dict(value=0), dict(value=300),
        dict(key_heads=3), dict(heads=0), dict(num_slots=-1), dict(num_slots=2), dict(state=None), dict(state=X + 2),
        dict(q=NO_HEADS), dict(beta=NONE), dict(o=NO_HEADS))] + [
    ("rc_qk_" + call, qk, change) for call in ("forward", "backward") for change in (
        dict(dtype=3), dict(param_dtype=2), dict(norm=3), dict(norm=-1), dict(batch=-1), dict(length=-1),
        dict(length=2 ** 30 + 1), dict(heads=-1), dict(key_heads=-1), dict(channels=0), dict(channels=257),
        dict(rotated=-2), dict(rotated=34), dict(rotated=15), dict(inv_freq=None), dict(q=NO_HEADS),
        dict(k=NO_HEADS))] + [
    ("rc_qk_forward", qk, dict(q_out=NO_HEADS)), ("rc_qk_forward", qk, dict(k_out=NO_HEADS)),
    ("rc_qk_backward", qk, dict(dq=NO_HEADS)), ("rc_qk_backward", qk, dict(dk=NO_HEADS)),
    ("rc_qk_backward", qk, dict(q_weight=None, dq_weight=X)),
    ("rc_qk_backward", qk, dict(k_weight=None, dk_weight=X)),
    ("rc_qk_backward", qk, dict(workspace=X + 3))] + [
    ("rc_dropout_" + call, dropout, change) for call in ("forward", "backward") for change in (
        dict(dtype=3), dict(out_dtype=2), dict(rows=-1), dict(width=-1), dict(p=-0.1), dict(p=1.1),
        dict(p=float("nan")), dict(x=NONE), dict(out=NONE))] + [
    ("rc_dropout_forward", dropout, dict(out_dtype=0))]


@pytest.mark.parametrize("call,make,change", BAD, ids=lambda v: v if isinstance(v, str) else None)
def test_bad_arguments(call, make, change):
    assert getattr(abi.library(), call)(make(**change), None) == rcdp.E_ARG


def test_null():
    lib, n = abi.library(), ctypes.c_uint64()
    for call in ("delta_forward", "delta_backward", "delta_step", "qk_forward", "qk_backward", "dropout_forward",
                 "dropout_backward"):
        assert getattr(lib, "rc_" + call)(None, None) == rcdp.E_ARG
    for call, make in (("delta_kept_bytes", delta), ("delta_forward_workspace", delta),
                       ("delta_backward_workspace", delta), ("qk_backward_workspace", qk)):
        assert getattr(lib, "rc_" + call)(None, n) == rcdp.E_ARG
        assert getattr(lib, "rc_" + call)(make(), None) == rcdp.E_ARG


@pytest.mark.parametrize("call,size,make", [
    ("rc_delta_forward", "rc_delta_forward_workspace", delta),
    ("rc_delta_backward", "rc_delta_backward_workspace", delta),
    ("rc_qk_backward", "rc_qk_backward_workspace", lambda: qk(dq_weight=X))])
def test_scratch_that_is_too_small(call, size, make):
    lib, n, a = abi.library(), ctypes.c_uint64(), make()
    assert getattr(lib, size)(a, n) == 0 and n.value > 0
    assert getattr(lib, call)(a, None) == rcdp.E_SCRATCH
    a.workspace, a.workspace_bytes = X, n.value - 1
    assert getattr(lib, call)(a, None) == rcdp.E_SCRATCH


@pytest.mark.parametrize("call,make,change", [
    ("rc_delta_forward", delta, dict(batch=2 ** 24, heads=4)),
    ("rc_delta_forward", delta, dict(batch=2 ** 16, length=2 ** 13)),
    ("rc_delta_backward", delta, dict(batch=2 ** 16, length=2 ** 13)),
    ("rc_delta_backward", delta, dict(batch=2 ** 15, length=2 ** 13, heads=1, key_heads=1, key=129)),
    ("rc_delta_step", step, dict(batch=2 ** 24, num_slots=2 ** 24)),
    ("rc_delta_step", step, dict(batch=2 ** 28, heads=32, num_slots=2 ** 28)),
    ("rc_delta_forward", delta, dict(batch=2 ** 31 - 1, heads=2 ** 31 - 2, length=2 ** 30)),
    ("rc_qk_forward", qk, dict(heads=2 ** 31 - 1)), ("rc_qk_backward", qk, dict(key_heads=2 ** 31 - 1)),
    ("rc_dropout_forward", dropout, dict(rows=2 ** 40, width=2 ** 40)),
    ("rc_dropout_backward", dropout, dict(rows=2 ** 40, width=2 ** 40))],
    ids=lambda v: v if isinstance(v, str) else None)
def test_sizes_beyond_a_launch(call, make, change):
    assert getattr(abi.library(), call)(make(**change), None) == rcdp.E_OVERFLOW


def test_empty_calls_do_nothing():
    lib = abi.library()
    assert lib.rc_delta_forward(delta(batch=0), None) == 0
    assert lib.rc_delta_forward(delta(heads=0, key_heads=0), None) == 0
    assert lib.rc_delta_backward(delta(batch=0), None) == 0
    assert lib.rc_delta_step(step(batch=0), None) == 0
    assert lib.rc_qk_forward(qk(length=0), None) == 0
    assert lib.rc_qk_forward(qk(heads=0, key_heads=0), None) == 0
    assert lib.rc_qk_backward(qk(batch=0), None) == 0
    assert lib.rc_dropout_forward(dropout(rows=0), None) == 0
    assert lib.rc_dropout_backward(dropout(width=0), None) == 0


def test_no_cpu_path():
    x, g = torch.randn(1, 4, 2, 8), torch.zeros(1, 4, 2)
    with pytest.raises(ValueError):
        ops.gated_delta(x, x, x, g, g)
    with pytest.raises(ValueError):
        ops.gated_delta_step(torch.zeros(1, 2, 8, 8), x[:, 0], x[:, 0], x[:, 0], g[:, 0], g[:, 0])
    with pytest.raises(ValueError):
        ops.qk_norm(x, x)
    with pytest.raises(ValueError):
        ops.dropout(x, 0.5, 1)
    with pytest.raises(ValueError):
        ops.dropout(x, 0.5, 1.5)
    with pytest.raises(ValueError):
        ops.dropout(x, 0.5, 1 << 64)
    with pytest.raises(ValueError):
        ops.qk_norm(x, x, norm="max")


def test_philox_known_answers():
    """The published test vectors of Philox4x32-10."""
    f = 0xFFFFFFFF
    assert ref.philox([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert ref.philox([f] * 4, [f] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert ref.philox([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0]) == [
        0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_the_delta_rule_stores_and_corrects():
    """What the definition is for: with beta 1 and keys of length one, the state returns the last value
    written for a key, and an orthogonal key's value stays."""
    torch.manual_seed(0)
    basis = torch.linalg.qr(torch.randn(4, 4, dtype=torch.float64))[0]
    k = basis[[0, 1, 0]][None, :, None]
    v = torch.randn(1, 3, 1, 5, dtype=torch.float64)
    one = torch.ones(1, 3, 1, dtype=torch.float64)
    _, S = ref.gated_delta(k, k, v, None, one, scale=1.0)
    torch.testing.assert_close(basis[0] @ S[0, 0], v[0, 2, 0])
    torch.testing.assert_close(basis[1] @ S[0, 0], v[0, 1, 0])


def test_sizes_beyond_a_launch_have_no_scratch():
    n = ctypes.c_uint64()
    far = delta(batch=2 ** 31 - 1, heads=2 ** 31 - 2, length=2 ** 30)
    for call in ("kept_bytes", "forward_workspace", "backward_workspace"):
        assert getattr(abi.library(), "rc_delta_" + call)(far, n) == rcdp.E_OVERFLOW
    assert abi.library().rc_qk_backward_workspace(qk(heads=2 ** 31 - 1), n) == rcdp.E_OVERFLOW
