"""The measured cases of the operators of ``paper_1905_11722_amd/ops.py``: the
short causal convolution, the selective state space scan and the fused norms
with gate and residual scale, for training, for prompts and for single tokens.

A case names an operator, a call and its sizes:

* ``conv`` / ``scan`` / ``norm``: the operator;
* ``call``: ``forward`` (a prompt: outputs and, for conv and scan, the state
  after it), ``train`` (outputs and the gradient of every input) or ``step``
  (one token of each sequence, states kept in a pool and updated in place);
* ``dtype``: type of the activations; parameters are 32-bit;
* ``batch``, ``length``, ``width`` and, for the scan, ``states`` per channel
  and ``groups`` of channels that share B and C; ``taps`` of the convolution;
  ``rows`` of the norm;
* ``ragged``: sequences end at lengths of their own inside the padded batch.

Where ``own`` is false the operators run in their plain form: elementary torch
operations in 32 bits, rounded once at the end.
"""

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5

# -------------------------------------------------------------------- cases


def listed():
    return [
        # a prompt through the convolution of a wide layer
        {"name": "conv prompt", "op": "conv", "call": "forward", "dtype": "bf16", "batch": 2,
         "length": 4096, "width": 4096, "taps": 4, "ragged": False},
        # a training batch of sequences of their own lengths
        {"name": "conv train ragged", "op": "conv", "call": "train", "dtype": "bf16", "batch": 8,
         "length": 2047, "width": 2048, "taps": 4, "ragged": True},
        # one token of each running sequence, states picked from a pool
        {"name": "conv step", "op": "conv", "call": "step", "dtype": "f16", "batch": 48,
         "width": 2048, "taps": 4},
        # a training batch, the usual number of states
        {"name": "scan train", "op": "scan", "call": "train", "dtype": "bf16", "batch": 8,
         "length": 2048, "width": 2048, "states": 16, "groups": 1, "ragged": False},
        # one long prompt
        {"name": "scan prompt", "op": "scan", "call": "forward", "dtype": "bf16", "batch": 1,
         "length": 16384, "width": 2048, "states": 16, "groups": 1, "ragged": False},
        # a small odd-sized layer in 32 bits, B and C shared by groups of channels
        {"name": "scan train odd", "op": "scan", "call": "train", "dtype": "f32", "batch": 3,
         "length": 777, "width": 200, "states": 12, "groups": 2, "ragged": True},
        # many states per channel
        {"name": "scan train wide", "op": "scan", "call": "train", "dtype": "f16", "batch": 2,
         "length": 1000, "width": 1024, "states": 64, "groups": 1, "ragged": False},
        # the next token of one sequence: latency
        {"name": "scan step one", "op": "scan", "call": "step", "dtype": "bf16", "batch": 1,
         "width": 1024, "states": 16, "groups": 1},
        # the next token of many sequences
        {"name": "scan step many", "op": "scan", "call": "step", "dtype": "bf16", "batch": 256,
         "width": 4096, "states": 16, "groups": 1},
        # the norms between two blocks while tokens are generated: latency
        {"name": "norm tokens", "op": "norm", "call": "forward", "dtype": "bf16", "rows": 16,
         "width": 2048, "gate": True, "wide_residual": True},
        # the norms between two blocks of a training batch, a 32-bit residual stream
        {"name": "norm train", "op": "norm", "call": "train", "dtype": "bf16", "rows": 16384,
         "width": 4096, "gate": True, "wide_residual": True},
        # an odd width, no gate, the residual stream in 16 bits
        {"name": "norm train odd", "op": "norm", "call": "train", "dtype": "f16", "rows": 1003,
         "width": 1001, "gate": False, "wide_residual": False},
    ]


def _spread(rng, lo, hi):
    """A whole number from lo..hi, even over its logarithm, odd ones among them."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng, lo, hi):
    """Mostly a multiple of 64, as layers have it, else any number."""
    n = _spread(rng, lo, hi)
    return n if rng.random() < 0.35 else max(64, n // 64 * 64)


def draw(rng):
    op = rng.choice(["conv", "scan", "scan", "norm"])
    top = {c["name"]: work(c) for c in listed()}
    most_bytes = max(w["bytes"] for w in top.values())
    most_flops = max(w["flops"] for w in top.values())
    while True:
        c = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
        c["call"] = rng.choice(["forward", "train"] if op == "norm" else ["forward", "train", "step"])
        if op == "norm":
            c.update(rows=_spread(rng, 1, 16384), width=_width(rng, 64, 8192),
                     gate=rng.random() < 0.6, wide_residual=rng.random() < 0.6)
            if c["width"] == 3072:
                continue
        else:
            c.update(batch=_spread(rng, 1, 256 if c["call"] == "step" else 16),
                     width=_width(rng, 64, 4096))
            if c["width"] == 3072:
                continue
            if c["call"] != "step":
                c.update(length=_spread(rng, 16, 16384), ragged=rng.random() < 0.4)
                if c["length"] == 3072:
                    continue
            if op == "conv":
                c["taps"] = rng.choice([2, 3, 4, 4, 4, 5, 8])
            else:
                c["groups"] = 2 if c["width"] % 2 == 0 and rng.random() < 0.25 else 1
                c["states"] = rng.choice([16, 16, 16, 8, 32, 64, rng.randint(1, 64)])
        w = work(c)
        # the plain scan holds several tensors of one value per state
        if w["bytes"] <= most_bytes and w["flops"] <= most_flops:
            return c


# ------------------------------------------------------------------- inputs


def _lengths(case, r, device):
    """Sequence lengths of a ragged batch: one of them full, one of them empty
    where there are enough, the others anything."""
    n, top = case["batch"], case["length"]
    v = torch.randint(1, top + 1, (n,), generator=r, device=device, dtype=torch.int32)
    v[0] = top
    if n > 2:
        v[1] = 0
    return v


def _slots(case, r, device):
    """Where each row's state lies in a pool somewhat larger than the batch;
    one row of a larger batch is padding (-1)."""
    n = case["batch"]
    slots = torch.randperm(n + n // 8 + 1, generator=r, device=device)[:n].to(torch.int32)
    if n > 8:
        slots[n // 2] = -1
    return slots


def prepare(case, seed, device="cuda"):
    r = torch.Generator(device=device)
    r.manual_seed(seed)
    t = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(shape, generator=r, device=device) * scale).to(dtype)

    def uniform(lo, hi, *shape):
        return lo + (hi - lo) * torch.rand(shape, generator=r, device=device)

    s = {"case": case}
    if case["op"] == "norm":
        n, d = case["rows"], case["width"]
        rt = torch.float32 if case["wide_residual"] else t
        s.update(block=normal(n, d), residual=normal(n, d, scale=2.0, dtype=rt),
                 gate=normal(n, d) if case["gate"] else None,
                 post_weight=uniform(0.5, 1.5, d), pre_weight=uniform(0.5, 1.5, d),
                 scale=uniform(0.05, 0.5, d))
        if case["call"] == "train":
            s.update(d_residual=normal(n, d, dtype=rt), d_normed=normal(n, d))
        return s
    b, d = case["batch"], case["width"]
    rows = (b,) if case["call"] == "step" else (b, case["length"])
    s["lengths"] = _lengths(case, r, device) if case.get("ragged") else None
    s["slots"] = _slots(case, r, device) if case["call"] == "step" else None
    pool = b + b // 8 + 1 if case["call"] == "step" else b
    if case["op"] == "conv":
        k = case["taps"]
        s.update(x=normal(*rows, d), weight=normal(d, k, scale=k ** -0.5, dtype=torch.float32),
                 bias=uniform(-0.5, 0.5, d), state=normal(pool, k - 1, d))
    else:
        n, g = case["states"], case["groups"]
        # softplus(dt + dt_bias) is about 0.001 .. 0.1 and decays are -1 .. -n, as these layers start out
        step = torch.exp(uniform(math.log(1e-3), math.log(1e-1), d))
        s.update(u=normal(*rows, d), dt=normal(*rows, d, scale=0.5), z=normal(*rows, d),
                 A=-torch.arange(1, n + 1, device=device).float() * uniform(0.8, 1.25, d, n),
                 B=normal(*rows, g, n), C=normal(*rows, g, n), D=uniform(0.5, 1.5, d),
                 dt_bias=step + torch.log(-torch.expm1(-step)),
                 state=normal(pool, d, n, scale=0.3, dtype=torch.float32))
    if case["call"] == "train":
        s["dy"] = normal(*rows, d)
    return s


# --------------------------------------------------------------- plain forms


def _valid(lengths, length, device):
    """(batch or 1, length, 1) truth values: the token is before its sequence's end."""
    t = torch.arange(length, device=device)[None, :, None]
    return t >= 0 if lengths is None else t < lengths[:, None, None]


def _silu_and_slope(x):
    sig = 1 / (1 + torch.exp(-x))
    return x * sig, sig * (1 + x * (1 - sig))


def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-torch.abs(x)))


def _conv_plain(s, train):
    x, w, b = s["x"].float(), s["weight"], s["bias"]
    k, length = w.shape[1], x.shape[1]
    ok = _valid(s["lengths"], length, x.device)
    x = torch.where(ok, x, 0)
    full = torch.cat([s["state"].float(), x], 1)
    taps = full.unfold(1, k, 1)                                # (batch, length, width, k)
    act, slope = _silu_and_slope((taps * w).sum(-1) + b)
    y = torch.where(ok, act, 0)
    # the last k - 1 inputs before each sequence's end
    ends = torch.full((x.shape[0],), length, device=x.device) if s["lengths"] is None else s["lengths"]
    at = ends[:, None] + torch.arange(k - 1, device=x.device)
    if not train:
        return {"y": y.to(s["x"].dtype),
                "state": torch.gather(full, 1, at.long()[:, :, None].expand(-1, -1, x.shape[2])).to(s["x"].dtype)}
    dp = torch.where(ok, s["dy"].float(), 0) * slope
    pad = torch.nn.functional.pad(dp, (0, 0, k - 1, k - 1))    # dp before and after the sequence is 0
    dfull = (pad.unfold(1, k, 1) * w.flip(1)).sum(-1)          # of every input and of the state
    return {"y": y.to(s["x"].dtype), "dx": torch.where(ok, dfull[:, k - 1:], 0).to(s["x"].dtype),
            "dweight": (taps * dp[..., None]).sum((0, 1)), "dbias": dp.sum((0, 1)),
            "dstate": dfull[:, :k - 1].to(s["x"].dtype)}


def _recurrence(a, b):
    """h_t = a_t h_{t-1} + b_t over dimension 0 from h = 0: pairs of steps
    make one step of half the length, whose results are every other h."""
    n = a.shape[0]
    if n == 1:
        return b
    even = n // 2 * 2
    half = _recurrence(a[1:even:2] * a[0:even:2], a[1:even:2] * b[0:even:2] + b[1:even:2])
    h = torch.empty_like(b)
    h[0] = b[0]
    h[1::2] = half
    h[2::2] = a[2::2] * half[:(n - 1) // 2] + b[2::2]
    return h


def _scan_plain(s, train):
    t = s["u"].dtype
    u, dt, z = (s[k].float().transpose(0, 1) for k in ("u", "dt", "z"))    # time first
    length, batch, d = u.shape
    A = s["A"]
    n, g = A.shape[1], s["B"].shape[2]
    ok = _valid(s["lengths"], length, u.device).transpose(0, 1)
    u, z, raw = (torch.where(ok, v, 0) for v in (u, z, dt + s["dt_bias"]))
    delta = torch.where(ok, _softplus(raw), 0)

    def channels(v):
        """B or C for every channel: (length, batch, groups, 1, n)."""
        return torch.where(ok[..., None], v.float().transpose(0, 1), 0)[:, :, :, None]

    def grouped(v):
        """(length, batch, d) as (length, batch, groups, d / groups, 1)."""
        return v.reshape(length, batch, g, d // g, 1)

    B, C, shape = channels(s["B"]), channels(s["C"]), (length, batch, g, d // g, n)
    a = torch.exp(delta[..., None] * A).reshape(shape)
    b = grouped(delta * u) * B
    h0 = s["state"].reshape(shape[1:])
    b[0] += a[0] * h0
    h = _recurrence(a, b)
    del b
    y = (h * C).sum(-1).reshape(u.shape) + s["D"] * u
    act, slope = _silu_and_slope(z)
    out = torch.where(ok, y * act, 0).transpose(0, 1).to(t)
    if not train:
        return {"y": out, "state": h[-1].reshape(batch, d, n)}
    dout = torch.where(ok, s["dy"].float().transpose(0, 1), 0)
    dy = dout * act
    # g_t = C_t dy_t + a_{t+1} g_{t+1}: the same recurrence, backwards in time
    after = torch.cat([a[1:], torch.ones_like(a[:1])]).flip(0)
    grad = _recurrence(after, (C * grouped(dy)).flip(0)).flip(0)
    del after
    dB = (grad * grouped(delta * u)).sum(3)
    dC = (h * grouped(dy)).sum(3)
    dinput = (grad * B).sum(-1).reshape(u.shape)
    grad *= a                                                   # of the state before the token
    dstate = grad[0].reshape(batch, d, n).clone()
    grad *= torch.cat([h0[None], h[:-1]])                       # of delta A
    grad = grad.reshape(length, batch, d, n)
    ddelta = u * dinput + (grad * A).sum(-1)
    draw_ = torch.where(ok, ddelta / (1 + torch.exp(-raw)), 0)

    def back(v):
        return torch.where(ok, v, 0).transpose(0, 1).to(t)

    return {"y": out, "du": back(delta * dinput + s["D"] * dy), "ddt": back(draw_),
            "dA": (grad * delta[..., None]).sum((0, 1)), "dB": dB.transpose(0, 1).to(t),
            "dC": dC.transpose(0, 1).to(t), "dD": (dy * u).sum((0, 1)), "dz": back(dout * y * slope),
            "ddt_bias": draw_.sum((0, 1)), "dstate": dstate}


def _conv_step_plain(s):
    x, w = s["x"], s["weight"]
    ok = s["slots"] >= 0
    at = s["slots"][ok].long()
    taps = torch.cat([s["state"][at], x[ok][:, None]], 1)
    act, _ = _silu_and_slope((taps.float() * w.t()).sum(1) + s["bias"])
    y = torch.zeros_like(x)
    y[ok] = act.to(x.dtype)
    s["state"][at] = taps[:, 1:]
    return {"y": y, "state": s["state"]}


def _scan_step_plain(s):
    ok = s["slots"] >= 0
    at = s["slots"][ok].long()
    u, dt, z, B, C = (s[k][ok].float() for k in ("u", "dt", "z", "B", "C"))
    d, n = s["A"].shape
    delta = _softplus(dt + s["dt_bias"])

    def channels(v):
        return v[:, :, None].expand(-1, -1, d // v.shape[1], -1).reshape(-1, d, n)

    h = torch.exp(delta[..., None] * s["A"]) * s["state"][at] + (delta * u)[..., None] * channels(B)
    out = ((h * channels(C)).sum(-1) + s["D"] * u) * _silu_and_slope(z)[0]
    y = torch.zeros_like(s["u"])
    y[ok] = out.to(y.dtype)
    s["state"][at] = h
    return {"y": y, "state": s["state"]}


def _norm_plain(s, train):
    u, r = s["block"].float(), s["residual"].float()
    d = u.shape[1]
    act, slope = _silu_and_slope(s["gate"].float()) if s["gate"] is not None else (1.0, None)
    v = u * act
    rv = torch.rsqrt((v * v).sum(1, keepdim=True) / d + EPS)
    p = v * rv * s["post_weight"]
    out = r + s["scale"] * p
    ro = torch.rsqrt((out * out).sum(1, keepdim=True) / d + EPS)
    unit = out * ro
    y = {"residual": out.to(s["residual"].dtype), "normed": (unit * s["pre_weight"]).to(s["block"].dtype)}
    if not train:
        return y
    dn = s["d_normed"].float()
    e = dn * s["pre_weight"]
    dr = s["d_residual"].float() + ro * (e - unit * ((e * unit).sum(1, keepdim=True) / d))
    dp = dr * s["scale"]
    e = dp * s["post_weight"]
    vn = v * rv
    dv = rv * (e - vn * ((e * vn).sum(1, keepdim=True) / d))
    y.update(dblock=(dv * act).to(s["block"].dtype), dresidual=dr.to(s["residual"].dtype),
             dgate=(dv * u * slope).to(s["block"].dtype) if slope is not None else None,
             dpost_weight=(dp * vn).sum(0), dscale=(dr * p).sum(0), dpre_weight=(dn * unit).sum(0))
    return y


# ----------------------------------------------------------------------- run


def _own(s):
    from paper_1905_11722_amd import ops

    op, call = s["case"]["op"], s["case"]["call"]
    if call == "step":
        if op == "conv":
            y = ops.causal_conv_step(s["state"], s["x"], s["weight"], s["bias"], slots=s["slots"])
        else:
            y = ops.selective_scan_step(s["state"], s["u"], s["dt"], s["A"], s["B"], s["C"], s["D"],
                                        s["z"], s["dt_bias"], softplus=True, slots=s["slots"])
        return {"y": y, "state": s["state"]}
    if op == "norm":
        names = ["block", "residual", "gate", "post_weight", "scale", "pre_weight"]
        call_of = lambda v: ops.norm_residual(*v, eps=EPS)  # noqa: E731
    elif op == "conv":
        names = ["x", "weight", "bias", "state"]
        call_of = lambda v: ops.causal_conv(  # noqa: E731
            *v[:3], state=v[3], lengths=s["lengths"], return_state=call == "forward")
    else:
        names = ["u", "dt", "A", "B", "C", "D", "z", "dt_bias", "state"]
        call_of = lambda v: ops.selective_scan(  # noqa: E731
            *v[:8], softplus=True, state=v[8], lengths=s["lengths"], return_state=call == "forward")
    if call == "forward":
        y = call_of([s[k] for k in names])
        return dict(zip(("residual", "normed") if op == "norm" else ("y", "state"), y))
    inputs = {k: s[k].detach().requires_grad_() for k in names if s[k] is not None}
    y = call_of([inputs.get(k) for k in names])
    if op == "norm":
        out, dout = dict(zip(("residual", "normed"), y)), [s["d_residual"], s["d_normed"]]
    else:
        out, dout = {"y": y}, [s["dy"]]
    grads = torch.autograd.grad(list(out.values()), list(inputs.values()), dout)
    out = {k: v.detach() for k, v in out.items()}
    out.update({"d" + k: v for k, v in zip(inputs, grads)})
    if op == "norm":
        out.setdefault("dgate", None)
    return out


def run(state):
    if own:
        return _own(state)
    op, call = state["case"]["op"], state["case"]["call"]
    if call == "step":
        return _conv_step_plain(state) if op == "conv" else _scan_step_plain(state)
    plain = {"conv": _conv_plain, "scan": _scan_plain, "norm": _norm_plain}[op]
    return plain(state, call == "train")


# ---------------------------------------------------------------------- work


def work(case):
    """Each input read once and each output written once; for the scan one
    exponential and six more operations for each token, channel and state,
    and sixteen more for its gradients."""
    e = 4 if case["dtype"] == "f32" else 2
    train = case["call"] == "train"
    d = case["width"]
    if case["op"] == "norm":
        n = case["rows"] * d
        r = 4 if case["wide_residual"] else e
        gates = 2 if case["gate"] else 1
        moved = n * (gates * e + r) + n * (r + e) + 12 * d
        if train:
            moved += n * (r + e) + n * (gates * e + r) + 12 * d
        return {"bytes": moved, "flops": n * (40 if train else 12)}
    tokens = case["batch"] * (1 if case["call"] == "step" else case["length"])
    n = tokens * d
    if case["op"] == "conv":
        k = case["taps"]
        held = case["batch"] * (k - 1) * d * e
        moved = n * e * (4 if train else 2) + 2 * held + 4 * d * (k + 1) * (2 if train else 1)
        return {"bytes": moved, "flops": n * (6 * k + 16 if train else 2 * k + 6)}
    ns, g = case["states"], case["groups"]
    held = 4 * case["batch"] * d * ns
    moved = (4 * n + 2 * tokens * g * ns) * e + 2 * held + 4 * d * (ns + 2)
    if train:
        moved += (4 * n + 2 * tokens * g * ns) * e + 4 * d * (ns + 2)
    return {"bytes": moved, "flops": n * (ns * (7 + (16 if train else 0)) + (60 if train else 20))}


# --------------------------------------------------------------------- exact


def exact(case, seed):
    """The operators' definitions in 64 bits: token by token, tap by tap, and
    for conv and norm with gradients from differentiating the definition."""
    def conv(v):
        x, w = v["x"], v["weight"]
        length, k = x.shape[1], w.shape[1]
        ends = v["lengths"].tolist() if v["lengths"] is not None else [length] * x.shape[0]
        ys, states = [], []
        for i, n in enumerate(ends):
            seen = torch.cat([v["state"][i], x[i, :n]])
            p = v["bias"] + sum(w[:, j] * seen[j:j + n] for j in range(k))
            ys.append(torch.cat([p * torch.sigmoid(p), torch.zeros_like(x[i, n:])]))
            states.append(seen[n:])
        return {"y": torch.stack(ys), "state": torch.stack(states)}

    def norm(v):
        block, r = v["block"], v["residual"]
        if v["gate"] is not None:
            block = block * v["gate"] * torch.sigmoid(v["gate"])
        p = block / torch.sqrt(block.pow(2).mean(1, keepdim=True) + EPS) * v["post_weight"]
        out = r + v["scale"] * p
        return {"residual": out,
                "normed": out / torch.sqrt(out.pow(2).mean(1, keepdim=True) + EPS) * v["pre_weight"]}

    def scan(v, train):
        u, dt, z, A = v["u"], v["dt"], v["z"], v["A"]
        batch, length, d = u.shape
        n, g = A.shape[1], v["B"].shape[2]
        dev = u.device
        ends = v["lengths"] if v["lengths"] is not None else torch.full((batch,), length, device=dev)
        raw = dt + v["dt_bias"]
        delta = torch.nn.functional.softplus(raw, threshold=100.0)
        group = torch.arange(d, device=dev) // (d // g)

        def live(t):
            return (ends > t)[:, None]

        h = v["state"].clone()
        kept = [h]
        y = torch.zeros_like(u)
        for t in range(length):
            new = torch.exp(delta[:, t, :, None] * A) * h + (delta[:, t] * u[:, t])[..., None] * v["B"][:, t, group]
            h = torch.where(live(t)[..., None], new, h)
            y[:, t] = torch.where(live(t), (h * v["C"][:, t, group]).sum(-1) + v["D"] * u[:, t], 0)
            if train:
                kept.append(h)
        sig = torch.sigmoid(z)
        out = y * z * sig
        if not train:
            return {"y": out, "state": h}
        ok = torch.arange(length, device=dev)[None, :, None] < ends[:, None, None]
        dout = torch.where(ok, v["dy"], 0.0)
        dy = dout * z * sig
        gh = torch.zeros_like(h)
        du, ddt, dA = torch.zeros_like(u), torch.zeros_like(u), torch.zeros_like(A)
        dB, dC = torch.zeros_like(v["B"]), torch.zeros_like(v["C"])
        for t in reversed(range(length)):
            m = live(t)
            a = torch.where(m[..., None], torch.exp(delta[:, t, :, None] * A), 1.0)
            step = torch.where(m, delta[:, t], 0.0)
            gh = gh + dy[:, t, :, None] * v["C"][:, t, group]
            dC[:, t] = (dy[:, t, :, None] * kept[t + 1]).reshape(batch, g, d // g, n).sum(2)
            dB[:, t] = (gh * (step * u[:, t])[..., None]).reshape(batch, g, d // g, n).sum(2)
            through = (gh * v["B"][:, t, group]).sum(-1)
            via = gh * a * kept[t]
            dA += (via * step[..., None]).sum(0)
            du[:, t] = step * through + v["D"] * dy[:, t]
            ddt[:, t] = torch.where(m, (u[:, t] * through + (via * A).sum(-1)) * torch.sigmoid(raw[:, t]), 0.0)
            gh = gh * a
        return {"y": out, "du": du, "ddt": ddt, "dA": dA, "dB": dB, "dC": dC, "dD": (dy * u).sum((0, 1)),
                "dz": dout * y * sig * (1 + z * (1 - sig)), "ddt_bias": ddt.sum((0, 1)), "dstate": gh}

    def conv_step(v):
        y = torch.zeros_like(v["x"])
        for i, slot in enumerate(v["slots"].tolist()):
            if slot >= 0:
                seen = torch.cat([v["state"][slot], v["x"][i:i + 1]])
                p = v["bias"] + (seen * v["weight"].t()).sum(0)
                y[i] = p * torch.sigmoid(p)
                v["state"][slot] = seen[1:]
        return {"y": y, "state": v["state"]}

    def scan_step(v):
        y = torch.zeros_like(v["u"])
        d, g = v["A"].shape[0], v["B"].shape[1]
        group = torch.arange(d, device=y.device) // (d // g)
        for i, slot in enumerate(v["slots"].tolist()):
            if slot >= 0:
                delta = torch.nn.functional.softplus(v["dt"][i] + v["dt_bias"], threshold=100.0)
                h = (torch.exp(delta[:, None] * v["A"]) * v["state"][slot]
                     + (delta * v["u"][i])[:, None] * v["B"][i, group])
                z = v["z"][i]
                y[i] = ((h * v["C"][i, group]).sum(-1) + v["D"] * v["u"][i]) * z * torch.sigmoid(z)
                v["state"][slot] = h
        return {"y": y, "state": v["state"]}

    s = prepare(case, seed)
    call = case["call"]
    v = {k: x.double() if isinstance(x, torch.Tensor) and x.is_floating_point() else x
         for k, x in s.items()}
    if call == "step":
        return (conv_step if case["op"] == "conv" else scan_step)(v)
    if case["op"] == "scan":
        return scan(v, call == "train")
    names = {"conv": ["x", "weight", "bias", "state"],
             "norm": ["block", "residual", "gate", "post_weight", "scale", "pre_weight"]}[case["op"]]
    names = [k for k in names if v[k] is not None]
    if call == "train":
        for k in names:
            v[k].requires_grad_()
    out = (conv if case["op"] == "conv" else norm)(v)
    if call == "train":
        if case["op"] == "conv":
            out.pop("state")
        given = [v["dy"]] if case["op"] == "conv" else [v["d_residual"], v["d_normed"]]
        grads = torch.autograd.grad(list(out.values()), [v[k] for k in names], given)
        out.update({"d" + k: x for k, x in zip(names, grads)})
        if case["op"] == "norm":
            out.setdefault("dgate", None)
    return {k: x.detach() if x is not None else None for k, x in out.items()}
