"""The structs and calls of include/rc_ops.h through ctypes."""

import ctypes

from paper_1905_11722_amd import rcdp

_P, _i32, _i64, _u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64


class View(ctypes.Structure):
    _fields_ = [("data", _P), ("batch", _i64), ("time", _i64)]


def _fields(text):
    """Struct fields from 'type: names' lines, in the order of rc_ops.h."""
    types = {"i32": _i32, "i64": _i64, "u64": _u64, "f32": ctypes.c_float, "ptr": _P,
             "view": View}
    out = []
    for line in text.strip().splitlines():
        kind, names = line.split(":")
        out += [(n, types[kind.strip()]) for n in names.split()]
    return out


class ConvArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype param_dtype activation batch length width taps
        view: x y state_in state_out
        ptr: weight bias lengths
        view: dy dstate_out dx dstate_in
        ptr: dweight dbias workspace
        u64: workspace_bytes""")


class ConvStepArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype param_dtype activation batch width taps num_slots
        view: x y state
        ptr: weight bias slots""")


class ScanArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype softplus batch length width states groups
        view: u dt z B C y
        i64: B_group C_group
        ptr: A D dt_bias state_in state_out lengths kept
        view: dy du ddt dz
        ptr: dB dC dstate_out dA dD ddt_bias dstate_in workspace
        u64: workspace_bytes""")


class ScanStepArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype softplus batch width states groups num_slots
        view: u dt z B C y
        i64: B_group C_group
        ptr: A D dt_bias state
        i64: state_slot
        ptr: slots""")


class NormArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype residual_dtype param_dtype gate_activation rows width
        f32: eps
        view: block gate residual out normed
        ptr: post_weight scale pre_weight stats
        view: dout dnormed dblock dgate dresidual
        ptr: dpost_weight dscale dpre_weight workspace
        u64: workspace_bytes""")


_lib = None


def library():
    global _lib
    if _lib is None:
        lib = rcdp.load_library()
        for name, args in (("conv", ConvArgs), ("scan", ScanArgs), ("norm", NormArgs),
                           ("conv_step", ConvStepArgs), ("scan_step", ScanStepArgs)):
            step = name.endswith("_step")
            for call in ([name] if step else [name + "_forward", name + "_backward"]):
                f = getattr(lib, "rc_" + call)
                f.restype, f.argtypes = ctypes.c_int, [ctypes.POINTER(args), _P]
        for name, args in (("conv_backward_workspace", ConvArgs), ("scan_kept_bytes", ScanArgs),
                           ("scan_forward_workspace", ScanArgs),
                           ("scan_backward_workspace", ScanArgs),
                           ("norm_backward_workspace", NormArgs)):
            f = getattr(lib, "rc_" + name)
            f.restype, f.argtypes = ctypes.c_int, [ctypes.POINTER(args), ctypes.POINTER(_u64)]
        _lib = lib
    return _lib
