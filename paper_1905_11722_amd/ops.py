"""Sequence-model operators on the HIP library (``include/rc_ops.h``): the
nodes of a network whose recomputation ``rcdp`` plans.

* :func:`causal_conv` / :func:`causal_conv_step`: short causal convolution of
  every channel, with bias and SiLU;
* :func:`selective_scan` / :func:`selective_scan_step`: selective state space
  scan;
* :func:`norm_residual`: the norms before and after a block, fused with the
  block's gate and residual scale.

The whole-sequence forms are differentiable (once); the ``*_step`` forms take
one token of each sequence and update a pool of states in place.  Activations
are float32, bfloat16 or float16 on one GPU; sums, states and statistics are
held in 32 bits.  Work is enqueued on PyTorch's current stream of the
inputs' device, outputs and scratch come from PyTorch's allocator, nothing
synchronises.  As with torch's own operators, a tensor made on another stream has to
be ready on the current one, and recorded there if it is freed early.

Arguments that cannot be used raise ValueError before anything runs; errors of
the library raise ``rcdp.RcError``.  A tensor whose channels are not
contiguous is copied first; batch and time strides are free.  There is no CPU
fallback.
"""

from __future__ import annotations

import ctypes

import torch

from . import rcdp

__all__ = ["causal_conv", "causal_conv_step", "selective_scan", "selective_scan_step",
           "norm_residual", "MAX_TAPS", "MAX_STATES", "MAX_NORM_WIDTH"]

MAX_TAPS, MAX_STATES, MAX_NORM_WIDTH = 8, 64, 16384
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_ACTIVATIONS = {None: 0, "silu": 1, "sigmoid": 2}

_P, _i32, _i64, _u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64


class _View(ctypes.Structure):
    _fields_ = [("data", _P), ("batch", _i64), ("time", _i64)]


def _fields(text):
    """Struct fields from 'type: names' lines, in the order of rc_ops.h."""
    types = {"i32": _i32, "i64": _i64, "u64": _u64, "f32": ctypes.c_float, "ptr": _P,
             "view": _View}
    out = []
    for line in text.strip().splitlines():
        kind, names = line.split(":")
        out += [(n, types[kind.strip()]) for n in names.split()]
    return out


class _ConvArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype param_dtype activation batch length width taps
        view: x y state_in state_out
        ptr: weight bias lengths
        view: dy dstate_out dx dstate_in
        ptr: dweight dbias workspace
        u64: workspace_bytes""")


class _ConvStepArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype param_dtype activation batch width taps num_slots
        view: x y state
        ptr: weight bias slots""")


class _ScanArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype softplus batch length width states groups
        view: u dt z B C y
        i64: B_group C_group
        ptr: A D dt_bias state_in state_out lengths kept
        view: dy du ddt dz
        ptr: dB dC dstate_out dA dD ddt_bias dstate_in workspace
        u64: workspace_bytes""")


class _ScanStepArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype softplus batch width states groups num_slots
        view: u dt z B C y
        i64: B_group C_group
        ptr: A D dt_bias state
        i64: state_slot
        ptr: slots""")


class _NormArgs(ctypes.Structure):
    _fields_ = _fields("""
        i32: dtype residual_dtype param_dtype gate_activation rows width
        f32: eps
        view: block gate residual out normed
        ptr: post_weight scale pre_weight stats
        view: dout dnormed dblock dgate dresidual
        ptr: dpost_weight dscale dpre_weight workspace
        u64: workspace_bytes""")


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = rcdp.load_library()
        for name, args in (("conv", _ConvArgs), ("scan", _ScanArgs), ("norm", _NormArgs),
                           ("conv_step", _ConvStepArgs), ("scan_step", _ScanStepArgs)):
            step = name.endswith("_step")
            for call in ([name] if step else [name + "_forward", name + "_backward"]):
                f = getattr(lib, "rc_" + call)
                f.restype, f.argtypes = ctypes.c_int, [ctypes.POINTER(args), _P]
        for name, args in (("conv_backward_workspace", _ConvArgs), ("scan_kept_bytes", _ScanArgs),
                           ("scan_forward_workspace", _ScanArgs),
                           ("scan_backward_workspace", _ScanArgs),
                           ("norm_backward_workspace", _NormArgs)):
            f = getattr(lib, "rc_" + name)
            f.restype, f.argtypes = ctypes.c_int, [ctypes.POINTER(args), ctypes.POINTER(_u64)]
        _lib = lib
    return _lib


def _call(name, args, device):
    """Enqueue a library call on the current stream of the tensors' device."""
    f = getattr(_library(), name)
    if device.index == torch.cuda.current_device():
        st = f(args, torch.cuda.current_stream().cuda_stream)
    else:
        with torch.cuda.device(device):
            st = f(args, torch.cuda.current_stream().cuda_stream)
    if st:
        raise rcdp.RcError(st, name)


def _bytes(name, args, device):
    n = _u64()
    with torch.cuda.device(device):
        st = getattr(_library(), name)(args, n)
    if st:
        raise rcdp.RcError(st, name)
    return n.value


def _scratch(name, args, device):
    n = _bytes(name, args, device)
    w = torch.empty(n, dtype=torch.uint8, device=device)
    args.workspace, args.workspace_bytes = w.data_ptr(), n
    return w


# ------------------------------------------------------------------ arguments


def _require(ok, what):
    if not ok:
        raise ValueError(what)


def _tensor(name, t, shape, dtype, device):
    """t after its checks: a GPU tensor of that shape and type (or one of several types)."""
    _require(isinstance(t, torch.Tensor), f"{name} must be a tensor")
    _require(tuple(t.shape) == tuple(shape),
             f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    types = dtype if isinstance(dtype, tuple) else (dtype,)
    _require(t.dtype in types, f"{name} must be {' or '.join(str(d) for d in types)}, not {t.dtype}")
    _require(t.device == device, f"{name} must be on {device}, not on {t.device}")
    return t


def _main(name, t, dims):
    """The tensor that gives sizes, type and device."""
    _require(isinstance(t, torch.Tensor), f"{name} must be a tensor")
    _require(t.is_cuda, f"{name} must be on a GPU: there is no CPU path")
    _require(t.dim() == dims, f"{name} must have {dims} dimensions, not {t.dim()}")
    _require(t.dtype in _DTYPES, f"{name} must be float32, bfloat16 or float16, not {t.dtype}")
    _require(all(n < 2 ** 31 for n in t.shape), f"{name} is too large")


def _rows(t):
    """t with contiguous channels: itself, or a copy."""
    return t if t is None or t.stride(-1) == 1 or t.shape[-1] <= 1 else t.contiguous()


def _view(t):
    """A (batch, time, channel) or (batch, channel) tensor as an rc_view."""
    if t is None:
        return _View()
    s = t.stride()
    return _View(t.data_ptr(), s[0], s[1] if len(s) > 2 else 0)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _activation(name, value, allowed):
    _require(value in allowed, f"{name} must be one of {allowed}, not {value!r}")
    return _ACTIVATIONS[value]


def _check_lengths(lengths, batch, device):
    if lengths is None:
        return None
    return _tensor("lengths", lengths, (batch,), torch.int32, device).contiguous()


def _check_slots(slots, batch, num_slots, device):
    if slots is None:
        _require(num_slots >= batch, f"state has {num_slots} slots for {batch} rows")
        return None
    return _tensor("slots", slots, (batch,), torch.int32, device).contiguous()


def _params(named, shapes, dtype, device):
    """Parameters, contiguous, of one type: float32 or the activations'."""
    given = [t for t in named.values() if t is not None]
    kind = given[0].dtype if given and isinstance(given[0], torch.Tensor) else torch.float32
    _require(kind in (torch.float32, dtype),
             f"{next(iter(named))} must be torch.float32 or {dtype}, not {kind}")
    out = [None if t is None else _tensor(n, t, shapes[n], kind, device).contiguous()
           for n, t in named.items()]
    return out, _DTYPES[kind]


def _differentiated(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


# ---------------------------------------------------------------- convolution


def _conv_args(x, weight, bias, state, lengths, activation, param):
    b, n, d = x.shape
    return _ConvArgs(dtype=_DTYPES[x.dtype], param_dtype=param, activation=activation, batch=b,
                     length=n, width=d, taps=weight.shape[1], x=_view(x), state_in=_view(state),
                     weight=_ptr(weight), bias=_ptr(bias), lengths=_ptr(lengths))


def _conv_forward(x, weight, bias, state, lengths, activation, param, want_state):
    args = _conv_args(x, weight, bias, state, lengths, activation, param)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    args.y = _view(y)
    out = None
    if want_state:
        out = x.new_empty((x.shape[0], weight.shape[1] - 1, x.shape[2]))
        args.state_out = _view(out)
    _call("rc_conv_forward", args, x.device)
    return y, out


class _Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, state, lengths, activation, param, want_state):
        y, out = _conv_forward(x, weight, bias, state, lengths, activation, param, want_state)
        ctx.save_for_backward(x, weight, bias, state, lengths)
        ctx.how = activation, param
        ctx.set_materialize_grads(False)
        return y, out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dout):
        x, weight, bias, state, lengths = ctx.saved_tensors
        args = _conv_args(x, weight, bias, state, lengths, *ctx.how)
        dy = torch.zeros_like(x) if dy is None else _rows(dy)
        dout = _rows(dout)
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        args.dy, args.dstate_out, args.dx = _view(dy), _view(dout), _view(dx)
        dw = torch.empty_like(weight) if ctx.needs_input_grad[1] else None
        db = torch.empty_like(bias) if bias is not None and ctx.needs_input_grad[2] else None
        ds = None
        if state is not None and ctx.needs_input_grad[3]:
            ds = torch.empty(state.shape, dtype=x.dtype, device=x.device)
            args.dstate_in = _view(ds)
        args.dweight, args.dbias = _ptr(dw), _ptr(db)
        work = _scratch("rc_conv_backward_workspace", args, x.device) if dw is not None or db is not None else None
        _call("rc_conv_backward", args, x.device)
        del work
        return dx, dw, db, ds, None, None, None, None


def causal_conv(x, weight, bias=None, *, state=None, lengths=None, activation="silu",
                return_state=False):
    """Short causal convolution over time, each channel on its own.

    ``y[b, t, d] = act(bias[d] + sum_k weight[d, k] x[b, t - (K - 1) + k, d])``

    x: (batch, length, width).  weight: (width, K), 1 <= K <= 8, and bias:
    (width,), float32 or x's type.  state: (batch, K - 1, width) of x's type,
    the inputs before the first, oldest first (default: zeros).  lengths:
    int32 (batch,), where each sequence ends; what lies past it is not used,
    and is 0 in y.  activation: "silu" or None.

    Returns y, or with ``return_state`` (y, the state after each sequence).
    """
    _main("x", x, 3)
    b, _, d = x.shape
    _require(isinstance(weight, torch.Tensor) and weight.dim() == 2, "weight must be a (width, taps) tensor")
    k = weight.shape[1]
    _require(1 <= k <= MAX_TAPS, f"weight must have 1 to {MAX_TAPS} taps, not {k}")
    (weight, bias), param = _params({"weight": weight, "bias": bias},
                                    {"weight": (d, k), "bias": (d,)}, x.dtype, x.device)
    if state is not None:
        state = _rows(_tensor("state", state, (b, k - 1, d), x.dtype, x.device))
    lengths = _check_lengths(lengths, b, x.device)
    run = _Conv.apply if _differentiated(x, weight, bias, state) else _conv_forward
    y, out = run(_rows(x), weight, bias, state, lengths,
                         _activation("activation", activation, (None, "silu")), param, return_state)
    return (y, out) if return_state else y


def causal_conv_step(state, x, weight, bias=None, *, slots=None, activation="silu"):
    """:func:`causal_conv` for one token of each sequence.

    x: (batch, width).  state: (slots, K - 1, width) of x's type, a pool of
    running states; row i uses ``state[slots[i]]`` (slots: int32 (batch,),
    default 0, 1, ...) and shifts its token into it.  A row whose slot is
    outside the pool (-1, say) is padding: its y is 0 and no state changes.
    The slots of one call must differ.  Returns y: (batch, width).
    """
    _main("x", x, 2)
    b, d = x.shape
    _require(isinstance(weight, torch.Tensor) and weight.dim() == 2, "weight must be a (width, taps) tensor")
    k = weight.shape[1]
    _require(1 <= k <= MAX_TAPS, f"weight must have 1 to {MAX_TAPS} taps, not {k}")
    (weight, bias), param = _params({"weight": weight, "bias": bias},
                                    {"weight": (d, k), "bias": (d,)}, x.dtype, x.device)
    _require(isinstance(state, torch.Tensor) and state.dim() == 3, "state must have 3 dimensions")
    _tensor("state", state, (state.shape[0], k - 1, d), x.dtype, x.device)
    _require(state.stride(2) == 1 or d <= 1, "state must have contiguous channels")
    slots = _check_slots(slots, b, state.shape[0], x.device)
    x = _rows(x)
    y = torch.empty((b, d), dtype=x.dtype, device=x.device)
    _call("rc_conv_step", _ConvStepArgs(
        _DTYPES[x.dtype], param, _activation("activation", activation, (None, "silu")), b, d, k,
        state.shape[0], _view(x), _view(y), _view(state), _ptr(weight), _ptr(bias), _ptr(slots)),
        x.device)
    return y


# ----------------------------------------------------------------------- scan


def _bc(t):
    """B or C as (batch, length, groups, states) with contiguous states."""
    return t if t.stride(-1) == 1 or t.shape[-1] <= 1 else t.contiguous()


def _scan_args(u, dt, A, B, C, D, z, dt_bias, state, lengths, softplus):
    b, n, d = u.shape
    return _ScanArgs(dtype=_DTYPES[u.dtype], softplus=softplus, batch=b, length=n, width=d,
                     states=A.shape[1], groups=B.shape[2], u=_view(u), dt=_view(dt), z=_view(z),
                     B=_view(B), C=_view(C), B_group=B.stride(2), C_group=C.stride(2), A=_ptr(A),
                     D=_ptr(D), dt_bias=_ptr(dt_bias), state_in=_ptr(state), lengths=_ptr(lengths))


def _scan_forward(u, dt, A, B, C, D, z, dt_bias, state, lengths, softplus, want_state, keep=False):
    args = _scan_args(u, dt, A, B, C, D, z, dt_bias, state, lengths, softplus)
    y = torch.empty(u.shape, dtype=u.dtype, device=u.device)
    args.y = _view(y)
    out = kept = None
    if want_state:
        out = torch.empty((u.shape[0], *A.shape), dtype=torch.float32, device=u.device)
        args.state_out = _ptr(out)
    if keep:
        kept = torch.empty(_bytes("rc_scan_kept_bytes", args, u.device), dtype=torch.uint8,
                           device=u.device)
        args.kept = _ptr(kept)
    work = _scratch("rc_scan_forward_workspace", args, u.device)
    _call("rc_scan_forward", args, u.device)
    del work
    return (y, out, kept) if keep else (y, out)


class _Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, dt, A, B, C, D, z, dt_bias, state, lengths, softplus, want_state):
        y, out, kept = _scan_forward(u, dt, A, B, C, D, z, dt_bias, state, lengths, softplus,
                                     want_state, keep=True)
        ctx.save_for_backward(u, dt, A, B, C, D, z, dt_bias, state, lengths, kept)
        ctx.softplus = softplus
        ctx.set_materialize_grads(False)
        return y, out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dout):
        u, dt, A, B, C, D, z, dt_bias, state, lengths, kept = ctx.saved_tensors
        args = _scan_args(u, dt, A, B, C, D, z, dt_bias, state, lengths, ctx.softplus)
        dy = torch.zeros_like(u) if dy is None else _rows(dy)
        dout = None if dout is None else dout.contiguous()

        def like(t):
            return None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device)

        du, ddt, dA, dB, dC, dD, dz, dbias = (like(t) for t in (u, dt, A, B, C, D, z, dt_bias))
        ds = like(state) if ctx.needs_input_grad[8] else None
        args.kept = _ptr(kept)
        args.dy, args.du, args.ddt, args.dz = _view(dy), _view(du), _view(ddt), _view(dz)
        args.dB, args.dC, args.dstate_out = _ptr(dB), _ptr(dC), _ptr(dout)
        args.dA, args.dD, args.ddt_bias, args.dstate_in = _ptr(dA), _ptr(dD), _ptr(dbias), _ptr(ds)
        work = _scratch("rc_scan_backward_workspace", args, u.device)
        _call("rc_scan_backward", args, u.device)
        del work
        return du, ddt, dA, dB, dC, dD, dz, dbias, ds, None, None, None


def _scan_sizes(u, A, B, C, tokens):
    """(states, groups, B, C) after checks; B and C with a group dimension."""
    d, dev = u.shape[-1], u.device
    _require(isinstance(A, torch.Tensor) and A.dim() == 2, "A must be a (width, states) tensor")
    n = A.shape[1]
    _require(1 <= n <= MAX_STATES, f"A must have 1 to {MAX_STATES} states, not {n}")
    _tensor("A", A, (d, n), torch.float32, dev)
    _require(isinstance(B, torch.Tensor) and isinstance(C, torch.Tensor), "B and C must be tensors")
    if B.dim() == len(tokens) + 1:
        B = B.unsqueeze(-2)
    if C.dim() == len(tokens) + 1:
        C = C.unsqueeze(-2)
    _require(B.dim() == len(tokens) + 2, f"B must have {len(tokens) + 1} or {len(tokens) + 2} dimensions")
    g = B.shape[-2]
    _require(g >= 1 and d % g == 0, f"{g} groups of B do not divide {d} channels")
    _tensor("B", B, (*tokens, g, n), u.dtype, dev)
    _tensor("C", C, (*tokens, g, n), u.dtype, dev)
    return n, g, _bc(B), _bc(C)


def selective_scan(u, dt, A, B, C, D=None, z=None, dt_bias=None, *, softplus=False, state=None,
                   lengths=None, return_state=False):
    """Selective state space scan over time.

    With delta = softplus(dt + dt_bias) if ``softplus`` else dt + dt_bias, each
    channel d of group g keeps a state h of N numbers:

    ``h[n] = exp(delta A[d, n]) h[n] + delta u B[g, n]``,
    ``y = (sum_n h[n] C[g, n] + D[d] u) silu(z)``

    u, dt and z (optional gate): (batch, length, width).  A: (width, N),
    N <= 64, finite and not positive.  B, C: (batch, length, N), or (batch,
    length, groups, N) with groups dividing width.  D, dt_bias: (width,).
    state: (batch, width, N), the state before the first token (default:
    zeros).  A, D, dt_bias and state are float32, the rest of u's type.
    lengths: int32 (batch,), where each sequence ends; what lies past it is
    not used, and is 0 in y.

    Returns y, or with ``return_state`` (y, the float32 state after each
    sequence).  For its gradients the forward pass keeps the states of every few tokens;
    the backward pass computes those between again.
    """
    _main("u", u, 3)
    b, length, d = u.shape
    dev = u.device
    n, _, B, C = _scan_sizes(u, A, B, C, (b, length))
    dt = _rows(_tensor("dt", dt, u.shape, u.dtype, dev))
    if z is not None:
        z = _rows(_tensor("z", z, u.shape, u.dtype, dev))
    if D is not None:
        D = _tensor("D", D, (d,), torch.float32, dev).contiguous()
    if dt_bias is not None:
        dt_bias = _tensor("dt_bias", dt_bias, (d,), torch.float32, dev).contiguous()
    if state is not None:
        state = _tensor("state", state, (b, d, n), torch.float32, dev).contiguous()
    lengths = _check_lengths(lengths, b, dev)
    run = _Scan.apply if _differentiated(u, dt, A, B, C, D, z, dt_bias, state) else _scan_forward
    y, out = run(_rows(u), dt, A.contiguous(), B, C, D, z, dt_bias, state, lengths,
                 int(bool(softplus)), return_state)
    return (y, out) if return_state else y


def selective_scan_step(state, u, dt, A, B, C, D=None, z=None, dt_bias=None, *, softplus=False,
                        slots=None):
    """:func:`selective_scan` for one token of each sequence.

    u, dt, z: (batch, width); B, C: (batch, N) or (batch, groups, N).  state:
    float32 (slots, width, N), a pool of running states updated in place;
    slots as :func:`causal_conv_step`.  Returns y: (batch, width).
    """
    _main("u", u, 2)
    b, d = u.shape
    dev = u.device
    n, g, B, C = _scan_sizes(u, A, B, C, (b,))
    dt = _rows(_tensor("dt", dt, u.shape, u.dtype, dev))
    if z is not None:
        z = _rows(_tensor("z", z, u.shape, u.dtype, dev))
    if D is not None:
        D = _tensor("D", D, (d,), torch.float32, dev).contiguous()
    if dt_bias is not None:
        dt_bias = _tensor("dt_bias", dt_bias, (d,), torch.float32, dev).contiguous()
    _require(isinstance(state, torch.Tensor) and state.dim() == 3, "state must have 3 dimensions")
    _tensor("state", state, (state.shape[0], d, n), torch.float32, dev)
    _require(state[:1].is_contiguous(), "each slot of state must be contiguous")
    slots = _check_slots(slots, b, state.shape[0], dev)
    u, A = _rows(u), A.contiguous()
    y = torch.empty((b, d), dtype=u.dtype, device=dev)
    _call("rc_scan_step", _ScanStepArgs(
        _DTYPES[u.dtype], int(bool(softplus)), b, d, n, g, state.shape[0], _view(u), _view(dt),
        _view(z), _view(B), _view(C), _view(y), B.stride(1), C.stride(1), _ptr(A), _ptr(D),
        _ptr(dt_bias), _ptr(state), state.stride(0), _ptr(slots)), dev)
    return y


# ---------------------------------------------------------------------- norms


def _flat(t, rows):
    """(..., width) as rows: a view where strides allow it, else a copy."""
    return None if t is None else _rows(t.reshape(rows, t.shape[-1]))


def _norm_args(block, residual, gate, post, scale, pre, act, param, eps):
    rows, d = residual.shape
    x = block if block is not None else residual
    return _NormArgs(dtype=_DTYPES[x.dtype], residual_dtype=_DTYPES[residual.dtype],
                     param_dtype=param, gate_activation=act, rows=rows, width=d, eps=eps,
                     block=_view(block), gate=_view(gate), residual=_view(residual),
                     post_weight=_ptr(post), scale=_ptr(scale), pre_weight=_ptr(pre))


def _norm_forward(block, residual, gate, post, scale, pre, act, param, eps, keep=False):
    args = _norm_args(block, residual, gate, post, scale, pre, act, param, eps)
    dev = residual.device
    out = normed = stats = None
    if block is not None:
        out = torch.empty(residual.shape, dtype=residual.dtype, device=dev)
        args.out = _view(out)
    if pre is not None:
        main = block if block is not None else residual
        normed = torch.empty(residual.shape, dtype=main.dtype, device=dev)
        args.normed = _view(normed)
    if keep:
        stats = torch.empty((residual.shape[0], 2), dtype=torch.float32, device=dev)
        args.stats = _ptr(stats)
    _call("rc_norm_forward", args, dev)
    return (out, normed, stats) if keep else (out, normed)


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, block, residual, gate, post, scale, pre, act, param, eps):
        out, normed, stats = _norm_forward(block, residual, gate, post, scale, pre, act, param, eps,
                                           keep=True)
        ctx.save_for_backward(block, residual, gate, post, scale, pre, stats)
        ctx.how = act, param, eps
        ctx.set_materialize_grads(False)
        return out, normed

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dnormed):
        block, residual, gate, post, scale, pre, stats = ctx.saved_tensors
        args = _norm_args(block, residual, gate, post, scale, pre, *ctx.how)
        args.stats = _ptr(stats)

        def like(t, want=True):
            return torch.empty(t.shape, dtype=t.dtype, device=t.device) if t is not None and want else None

        need = ctx.needs_input_grad
        dout, dnormed = _rows(dout), _rows(dnormed)
        dblock, dresidual, dgate = like(block), like(residual), like(gate)
        dpost, dscale, dpre = like(post, need[3]), like(scale, need[4]), like(pre, need[5])
        args.dout, args.dnormed, args.dblock = _view(dout), _view(dnormed), _view(dblock)
        args.dgate, args.dresidual = _view(dgate), _view(dresidual)
        args.dpost_weight, args.dscale, args.dpre_weight = _ptr(dpost), _ptr(dscale), _ptr(dpre)
        work = _scratch("rc_norm_backward_workspace", args, residual.device)
        _call("rc_norm_backward", args, residual.device)
        del work
        return dblock, dresidual, dgate, dpost, dscale, dpre, None, None, None


def norm_residual(block, residual, gate=None, post_weight=None, scale=None, pre_weight=None, *,
                  gate_activation="silu", eps=1e-5):
    """The norm after a block and the norm before the next one, with the
    block's gate and residual scale:

    ``v = block * act(gate)``, ``p = v / rms(v) * post_weight``,
    ``out = residual + scale * p``, ``normed = out / rms(out) * pre_weight``

    with ``rms(x) = sqrt(mean(x^2) + eps)`` over the last dimension (at most
    16384 channels).  block and gate: (..., width), the residual of the same
    shape and of block's type or float32.  The weights and scale: (width,),
    float32 or block's type, each optional: without post_weight p is v,
    without pre_weight there is no normed.  block None: only the norm of the
    residual.  gate_activation: "silu" or "sigmoid".

    Returns (out, normed): out of the residual's type (the residual itself
    where block is None), normed of block's (or None).
    """
    _require(isinstance(residual, torch.Tensor), "residual must be a tensor")
    _require(residual.dim() >= 1, "residual must have a dimension of channels")
    main = block if block is not None else residual
    _main("block" if block is not None else "residual", main, residual.dim())
    d, dev, shape = residual.shape[-1], main.device, residual.shape
    _require(d <= MAX_NORM_WIDTH, f"at most {MAX_NORM_WIDTH} channels, not {d}")
    _tensor("residual", residual, main.shape, (main.dtype, torch.float32), dev)
    if block is None:
        _require(gate is None and post_weight is None and scale is None,
                 "gate, post_weight and scale belong to a block")
        _require(pre_weight is not None, "without a block, pre_weight is needed")
    if gate is not None:
        _tensor("gate", gate, shape, main.dtype, dev)
    act = _activation("gate_activation", gate_activation, ("silu", "sigmoid"))
    weights = {"post_weight": post_weight, "scale": scale, "pre_weight": pre_weight}
    (post, scale, pre), param = _params(weights, dict.fromkeys(weights, (d,)), main.dtype, dev)
    rows = residual.numel() // d if d else 0
    _require(rows < 2 ** 31, "too many rows")
    run = _Norm.apply if _differentiated(block, residual, gate, post, scale, pre) else _norm_forward
    out, normed = run(_flat(block, rows), _flat(residual, rows), _flat(gate, rows), post, scale,
                      pre, act, param, float(eps))
    out = residual if block is None else out.view(shape)
    return out, None if normed is None else normed.view(shape)
