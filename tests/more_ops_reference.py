"""Plain 64-bit implementations of the linear-attention operators, token by
token, differentiable by torch, and Philox in Python integers."""

import torch


def live_tokens(lengths, batch, length):
    """(batch, length) truth values."""
    n = torch.full((batch,), length) if lengths is None else torch.as_tensor(lengths).clamp(0, length)
    return torch.arange(length)[None] < n[:, None]


def gated_delta(q, k, v, g=None, beta=None, scale=None, state=None, lengths=None):
    """(o, final state)."""
    batch, length, heads, value = v.shape
    key, per = q.shape[3], heads // q.shape[2]
    scale = key ** -0.5 if scale is None else scale
    live = live_tokens(lengths, batch, length)
    S = v.new_zeros(batch, heads, key, value) if state is None else state
    out = []
    for t in range(length):
        on = live[:, t, None, None, None]
        kt, qt = (torch.where(on[..., 0], x[:, t], 0).repeat_interleave(per, 1) for x in (k, q))
        vt = torch.where(on[..., 0], v[:, t], 0)
        bt = torch.where(on[..., 0, 0], beta[:, t], 0)
        D = S if g is None else torch.exp(torch.where(on[..., 0, 0], g[:, t], 0))[..., None, None] * S
        w = bt[..., None] * (vt - (kt[..., None] * D).sum(-2))
        S = torch.where(on, D + kt[..., None] * w[..., None, :], S)
        out.append(torch.where(on[..., 0], scale * (qt[..., None] * S).sum(-2), 0))
    return (torch.stack(out, 1) if out else torch.zeros_like(v)), S


def qk_norm(q, k, q_weight=None, k_weight=None, inv_freq=None, positions=None, norm="rms", eps=1e-6,
            interleaved=False, lengths=None):
    batch, length = q.shape[:2]
    live = live_tokens(lengths, batch, length)[..., None, None]
    at = torch.arange(length).expand(batch, length) if positions is None else positions
    out = []
    for x, w in ((q, q_weight), (k, k_weight)):
        x = torch.where(live, x, 0)
        if norm == "rms":
            x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
        elif norm == "l2":
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) + eps)
        if w is not None:
            x = x * w
        if inv_freq is not None:
            m = len(inv_freq)
            angle = at.double()[..., None, None] * inv_freq.double()
            if interleaved:
                a, b = x[..., 0:2 * m:2], x[..., 1:2 * m:2]
            else:
                a, b = x[..., :m], x[..., m:2 * m]
            a, b = a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()
            both = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
            x = torch.cat([both, x[..., 2 * m:]], -1)
        out.append(torch.where(live, x, 0))
    return out


def philox(counter, key):
    """Philox4x32-10 of Salmon, Moraes, Dror and Shaw (2011): four words from four and two."""
    mask = 0xFFFFFFFF
    c, k = list(counter), list(key)
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [q >> 32 ^ c[1] ^ k[0], q & mask, p >> 32 ^ c[3] ^ k[1], p & mask]
        k = [k[0] + 0x9E3779B9 & mask, k[1] + 0xBB67AE85 & mask]
    return c


def kept(n, p, seed, tag=0):
    """The first n elements' truth values: kept."""
    mask, words = 0xFFFFFFFF, []
    for i in range(-(-n // 4)):
        words += philox([i & mask, i >> 32, tag & mask, tag >> 32 & mask], [seed & mask, seed >> 32 & mask])
    return torch.tensor([w >= round(p * 2 ** 32) for w in words[:n]])
