"""The linear-attention operators' structs and calls of include/rc_ops.h through ctypes."""

import ctypes

from tests import ops_abi as abi

_P, _i32, _i64, _u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64


class Heads(ctypes.Structure):
    _fields_ = [("data", _P), ("batch", _i64), ("time", _i64), ("head", _i64)]


def _fields(text):
    types = {"i32": _i32, "i64": _i64, "u64": _u64, "f32": ctypes.c_float, "f64": ctypes.c_double,
             "ptr": _P, "view": abi.View, "heads": Heads}
    out = []
    for line in text.strip().splitlines():
        kind, names = line.split(":")
        out += [(n, types[kind.strip()]) for n in names.split()]
    return out


class DeltaArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype batch length key_heads heads key value
        f32: scale
        heads: q k v o
        view: g beta
        ptr: state_in state_out lengths kept
        heads: do_ dq dk dv
        ptr: dg dbeta dstate_out dstate_in workspace
        u64: workspace_bytes""")


class DeltaStepArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype batch key_heads heads key value num_slots
        f32: scale
        heads: q k v o
        view: g beta
        ptr: state
        i64: state_slot
        ptr: slots""")


class QkArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype param_dtype norm interleaved batch length heads key_heads channels rotated
        f32: eps
        heads: q k q_out k_out
        ptr: q_weight k_weight inv_freq positions
        i64: positions_batch positions_time
        ptr: lengths
        heads: dq_out dk_out dq dk
        ptr: dq_weight dk_weight workspace
        u64: workspace_bytes""")


class DropoutArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype out_dtype
        i64: rows width
        f64: p
        i64: seed tag
        ptr: seed_device
        view: x residual out""")


_lib = None


def library():
    global _lib
    if _lib is None:
        lib = abi.library()
        for name, args in (("delta_forward", DeltaArgs), ("delta_backward", DeltaArgs),
                           ("delta_step", DeltaStepArgs), ("qk_forward", QkArgs), ("qk_backward", QkArgs),
                           ("dropout_forward", DropoutArgs), ("dropout_backward", DropoutArgs)):
            f = getattr(lib, "rc_" + name)
            f.restype, f.argtypes = ctypes.c_int, [ctypes.POINTER(args), _P]
        for name, args in (("delta_kept_bytes", DeltaArgs), ("delta_forward_workspace", DeltaArgs),
                           ("delta_backward_workspace", DeltaArgs), ("qk_backward_workspace", QkArgs)):
            f = getattr(lib, "rc_" + name)
            f.restype, f.argtypes = ctypes.c_int, [ctypes.POINTER(args), ctypes.POINTER(_u64)]
        _lib = lib
    return _lib
