"""Plain 64-bit implementations of the sequence-model operators, token by
token and tap by tap, differentiable by torch: what the kernels are held to."""

import torch


def silu(x):
    return x * torch.sigmoid(x)


def softplus(x):
    return torch.logaddexp(x, torch.zeros_like(x))


def causal_conv(x, weight, bias=None, state=None, lengths=None, activation="silu"):
    """(y, final state)."""
    batch, length, width = x.shape
    taps = weight.shape[1]
    ys, ends = [], []
    for i in range(batch):
        n = length if lengths is None else max(0, min(length, int(lengths[i])))
        head = state[i] if state is not None else x.new_zeros(taps - 1, width)
        seen = torch.cat([head, x[i, :n]])
        p = torch.zeros(n, width, dtype=x.dtype)
        for k in range(taps):
            p = p + weight[:, k] * seen[k:k + n]
        if bias is not None:
            p = p + bias
        if activation == "silu":
            p = silu(p)
        ys.append(torch.cat([p, x.new_zeros(length - n, width)]))
        ends.append(seen[n:])
    return torch.stack(ys) if ys else x.clone(), torch.stack(ends) if ends else None


def selective_scan(u, dt, A, B, C, D=None, z=None, dt_bias=None, soft=False, state=None,
                   lengths=None):
    """(y, final state); B and C are (batch, length, groups, states)."""
    batch, length, width = u.shape
    states, groups = A.shape[1], B.shape[2]
    ys, ends = [], []
    for i in range(batch):
        n = length if lengths is None else max(0, min(length, int(lengths[i])))
        h = state[i] if state is not None else u.new_zeros(width, states)
        rows = []
        for t in range(n):
            raw = dt[i, t] + (dt_bias if dt_bias is not None else 0.0)
            delta = softplus(raw) if soft else raw
            b = B[i, t].repeat_interleave(width // groups, 0)
            c = C[i, t].repeat_interleave(width // groups, 0)
            h = torch.exp(delta[:, None] * A) * h + (delta * u[i, t])[:, None] * b
            y = (h * c).sum(1)
            if D is not None:
                y = y + D * u[i, t]
            if z is not None:
                y = y * silu(z[i, t])
            rows.append(y)
        rows += [u.new_zeros(width)] * (length - n)
        ys.append(torch.stack(rows) if rows else u.new_zeros(0, width))
        ends.append(h)
    return torch.stack(ys), torch.stack(ends)


def norm_residual(block, residual, gate=None, post=None, scale=None, pre=None, act="silu",
                  eps=1e-5):
    """(out, normed or None)."""
    def rms(x):
        return torch.sqrt(x.square().mean(-1, keepdim=True) + eps)

    out = residual
    if block is not None:
        v = block
        if gate is not None:
            v = v * (silu(gate) if act == "silu" else torch.sigmoid(gate))
        if post is not None:
            v = v / rms(v) * post
        out = residual + (v if scale is None else scale * v)
    return out, None if pre is None else out / rms(out) * pre
