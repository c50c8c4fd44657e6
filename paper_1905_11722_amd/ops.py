"""Sequence-model operators on the HIP library (``include/rc_ops.h``): the
nodes of a network whose recomputation ``rcdp`` plans.

* :func:`causal_conv` / :func:`causal_conv_step`: short causal convolution of
  every channel, with bias and SiLU;
* :func:`selective_scan` / :func:`selective_scan_step`: selective state space
  scan;
* :func:`norm_residual`: the norms before and after a block, fused with the
  block's gate and residual scale;
* :func:`gated_delta` / :func:`gated_delta_step`: gated delta rule, a linear
  attention;
* :func:`qk_norm`: the norms of its queries and keys for each head, with their
  rotation by position;
* :func:`dropout`: dropout whose mask is drawn again wherever it is needed.

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
import operator

from . import rcdp

__all__ = ["causal_conv", "causal_conv_step", "selective_scan", "selective_scan_step",
           "norm_residual", "gated_delta", "gated_delta_step", "qk_norm", "dropout",
           "MAX_TAPS", "MAX_STATES", "MAX_NORM_WIDTH", "MAX_HEAD"]

MAX_TAPS, MAX_STATES, MAX_NORM_WIDTH, MAX_HEAD = 8, 64, 16384, 256
_CONV_ACTIVATIONS = {None: 0, "silu": 1}
_GATE_ACTIVATIONS = {"silu": 1, "sigmoid": 2}
_QK_NORMS = {None: 0, "rms": 1, "l2": 2}

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


def gated_delta(q, k, v, g, beta, *, scale=None, state=None, lengths=None, return_state=False):
    """Gated delta rule over time: a linear attention whose state corrects what it holds for a key.

    Each head keeps a matrix S of key x value numbers:

    ``S = exp(g) S``, ``S = S + k (beta (v - S^T k))^T``, ``o = scale S^T q``

    q, k: (batch, length, key_heads, key), v: (batch, length, heads, value),
    key and value at most 256; key_heads divides heads, and head h takes q and k of
    head h // (heads // key_heads).  g (None: 0; not positive, -inf forgets
    everything before) and beta: (batch, length, heads), float32.  The state stays
    bounded where beta k^T k is at most 2, as with keys of length one (:func:`qk_norm` with
    ``norm="l2"``) and beta in (0, 1).  scale: default key ** -0.5.  state: float32
    (batch, heads, key, value), the one before the first token (default:
    zeros).  lengths: int32 (batch,), where each sequence ends; what lies past
    it is not used, and is 0 in o.

    Returns o, or with ``return_state`` (o, the float32 state after each
    sequence).  For its gradients the forward pass keeps the state of every 64
    tokens in 32 bits (of every 32 for keys above 128 and for more than 64 in float16 or float32)
    and what each token wrote, with key taken up to 32, 64, 128 or 256, value to a multiple of 32 and the
    length to one of those tokens: 4 key value bytes for each such block and 4 value bytes for each token, of each head.

    A number that is not finite (or a float32 above 3.39e38) makes its own token's results NaN and those that
    depend on it: outputs after it, and gradients on whichever side they go through the state.  All others are
    what they are without it.
    """
    out = (_native or load()).gated_delta(q, k, v, g, beta, _scale(scale, q), state, lengths, return_state)
    return (out[0], out[1]) if return_state else out[0]


def gated_delta_step(state, q, k, v, g, beta, *, scale=None, slots=None):
    """:func:`gated_delta` for one token of each sequence.

    q, k: (batch, key_heads, key), v: (batch, heads, value), g and beta: (batch,
    heads).  state: float32 (slots, heads, key, value), a pool of running states
    updated in place; slots as :func:`causal_conv_step`.  Returns o: (batch,
    heads, value).
    """
    return (_native or load()).gated_delta_step(state, q, k, v, g, beta, _scale(scale, q), slots)


def _scale(scale, q):
    """The scale of a linear attention's outputs."""
    if scale is not None:
        return float(scale)
    n = q.shape[-1] if getattr(q, "ndim", 0) else 0
    return n ** -0.5 if n else 1.0


def qk_norm(q, k, q_weight=None, k_weight=None, inv_freq=None, positions=None, *, norm="rms",
            eps=1e-6, interleaved=False, lengths=None):
    """Norms of queries and keys, each head on its own, with their rotation by position.

    ``y = x / sqrt(mean(x^2) + eps) * weight`` ("rms"), or by the sum in place
    of the mean ("l2": length one), or ``x * weight`` (None); then pair i of y
    is turned by ``position * inv_freq[i]``: channels i and i + R / 2 (2i and 2i +
    1 if ``interleaved``), R = 2 len(inv_freq).  Channels from R on are not turned.

    q: (batch, length, heads, channels), k: (batch, length, key_heads,
    channels), channels at most 256.  The weights: (channels,), float32 or q's
    type.  inv_freq: float32 (R / 2,), without a gradient (None: no rotation).  positions:
    int32 (batch, length), any (default: 0, 1, ..); angles are taken in 64 bits.
    lengths: int32 (batch,), where each sequence ends; what lies past it is
    not used, and is 0 in the results.  For single tokens length is 1 and positions
    say where they are.

    Returns (q, k).
    """
    out = (_native or load()).qk_norm(q, k, q_weight, k_weight, inv_freq, positions, lengths,
                                      _activation("norm", norm, _QK_NORMS), bool(interleaved), eps)
    return out[0], out[1]


def dropout(x, p, seed, *, tag=0, residual=None):
    """Dropout whose mask is never stored: ``residual + (kept ? x / (1 - p) : 0)``.

    Element i of x (in the order of a contiguous x) is kept where word i % 4 of
    Philox4x32-10 with key ``seed`` and counter (i // 4, ``tag``) is not below
    p 2^32 (rounded to a whole number).  The same seed and tag draw the same mask again, in the backward
    pass or where a node of a planned step is computed a second time; take
    another tag for each use in a model and another seed for each step.

    seed: an int, or an int64 tensor of one number on x's GPU, read when the
    kernel runs, so that a captured graph draws another mask once the tensor
    holds another number.  (The backward pass reads it again: between the two it must
    not change.)  tag: an int.  p: from 0 to 1.  residual: of x's shape, float32
    or x's type, which the result has then too.
    """
    number, where = (0, seed) if hasattr(seed, "data_ptr") else (_word("seed", seed), None)
    return (_native or load()).dropout(x, p, where, number, _word("tag", tag), residual)


def _word(name, value):
    """An int as 64 bits (int64 or uint64)."""
    try:
        value = operator.index(value)
    except TypeError:
        raise ValueError(f"{name} must be an int, not {value!r}") from None
    if not -(1 << 63) <= value < 1 << 64:
        raise ValueError(f"{name} must fit 64 bits")
    return value - (1 << 64) if value >= 1 << 63 else value
