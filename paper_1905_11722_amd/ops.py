"""Sequence-model operators on the HIP library (``include/rc_ops.h``): the
nodes of a network whose recomputation ``rcdp`` plans.

* :func:`causal_conv` / :func:`causal_conv_step`: short causal convolution of
  every channel, with bias and SiLU;
* :func:`selective_scan` / :func:`selective_scan_step`: selective state space
  scan;
* :func:`norm_residual`: the norms before and after a block, fused with the
  block's gate and residual scale.

The whole-sequence forms are differentiable (once, in reverse mode); the ``*_step`` forms take
one token of each sequence and update a pool of states in place, without
gradients: they refuse inputs that require one (call them under
``torch.no_grad()``).  Activations
are float32, bfloat16 or float16 on one GPU; sums, states and statistics are
held in 32 bits.  Work is enqueued on PyTorch's current stream of the
inputs' device, outputs and scratch come from PyTorch's allocator, nothing
synchronises.  As with torch's own operators, a tensor made on another stream has to
be ready on the current one, and recorded there if it is freed early.

Arguments that cannot be used raise ValueError (TypeError where a tensor is
expected and something else comes) before anything runs; errors of the library
raise ``rcdp.RcError``.  A tensor whose channels are not
contiguous is copied first; batch and time strides are free.  There is no CPU
fallback.
"""

from __future__ import annotations

import importlib

from . import rcdp

__all__ = ["causal_conv", "causal_conv_step", "selective_scan", "selective_scan_step",
           "norm_residual", "MAX_TAPS", "MAX_STATES", "MAX_NORM_WIDTH"]

MAX_TAPS, MAX_STATES, MAX_NORM_WIDTH = 8, 64, 16384
_CONV_ACTIVATIONS = {None: 0, "silu": 1}
_GATE_ACTIVATIONS = {"silu": 1, "sigmoid": 2}

_native = None


def load():
    """Load the binding's native part and the library under it; raises ImportError where
    they have not been built."""
    global _native
    if _native is None:
        import torch  # noqa: F401 - its libraries come first
        rcdp.load_library()
        _native = importlib.import_module("._ops", __package__)
    return _native


def _activation(name, value, allowed):
    try:
        return allowed[value]
    except (KeyError, TypeError):
        raise ValueError(f"{name} must be one of {tuple(allowed)}, not {value!r}") from None


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
    out = (_native or load()).causal_conv(
        x, weight, bias, state, lengths, _activation("activation", activation, _CONV_ACTIVATIONS),
        return_state)
    return (out[0], out[1]) if return_state else out[0]


def causal_conv_step(state, x, weight, bias=None, *, slots=None, activation="silu"):
    """:func:`causal_conv` for one token of each sequence.

    x: (batch, width).  state: (slots, K - 1, width) of x's type, a pool of
    running states; row i uses ``state[slots[i]]`` (slots: int32 (batch,),
    default 0, 1, ...) and shifts its token into it.  A row whose slot is
    outside the pool (-1, say) is padding: its y is 0 and no state changes.
    The slots of one call must differ, and those of the pool must not share
    memory.  Returns y: (batch, width).
    """
    return (_native or load()).causal_conv_step(
        state, x, weight, bias, slots, _activation("activation", activation, _CONV_ACTIVATIONS))


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
    sequence).  For its gradients the forward pass keeps the states of every
    16 tokens in 32 bits (states / 4 bytes for each token and channel); the
    backward pass computes those between again.
    """
    out = (_native or load()).selective_scan(u, dt, A, B, C, D, z, dt_bias, bool(softplus), state,
                                             lengths, return_state)
    return (out[0], out[1]) if return_state else out[0]


def selective_scan_step(state, u, dt, A, B, C, D=None, z=None, dt_bias=None, *, softplus=False,
                        slots=None):
    """:func:`selective_scan` for one token of each sequence.

    u, dt, z: (batch, width); B, C: (batch, N) or (batch, groups, N).  state:
    float32 (slots, width, N), a pool of running states updated in place;
    slots as :func:`causal_conv_step`.  Returns y: (batch, width).
    """
    return (_native or load()).selective_scan_step(state, u, dt, A, B, C, D, z, dt_bias,
                                                   bool(softplus), slots)


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
    return (_native or load()).norm_residual(
        block, residual, gate, post_weight, scale, pre_weight,
        _activation("gate_activation", gate_activation, _GATE_ACTIVATIONS), eps)
