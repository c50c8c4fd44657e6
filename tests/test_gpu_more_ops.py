"""The linear-attention operators on the GPU against plain 64-bit implementations: every type, odd
sizes, head layouts, strides, ragged and empty sequences, gradients, single tokens, streams and graphs.

Tolerances are those of the other operators' tests: a 16-bit result is off by half a unit in its
last place, and 2e-5 of the larger of its size and the results' root mean square for what 32-bit sums
leave.  For the delta rule that covers sums of up to 256 + 256 + 64 terms (a
few tens of units of 2^-24, rounding errors being of either sign) that pass through the
states of a handful of chunks without growing: with keys of length at most one and beta in [0, 2] no
state's part grows from token to token."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1905_11722_amd import ops  # noqa: E402
from tests import more_ops_reference as ref  # noqa: E402
from tests import ops_reference as old  # noqa: E402
from tests.test_gpu_ops import DEV, DTYPES, Inputs, check, compare_grads  # noqa: E402


def int32(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device=DEV)


# ----------------------------------------------------------------- delta rule

DELTA = [  # dtype, batch, length, key_heads, heads, key, value, parts (g, s: state), lengths
    ("f32", 2, 37, 2, 4, 16, 24, "gs", None),
    ("bf16", 2, 70, 2, 2, 64, 64, "gs", (70, 33)),
    ("f16", 3, 65, 1, 3, 32, 48, "gs", (65, 0, 32)),
    ("f32", 1, 1, 1, 1, 1, 1, "gs", None),
    ("bf16", 1, 1, 1, 2, 128, 128, "gs", None),
    ("f32", 2, 32, 1, 1, 3, 5, "g", (32, 31)),
    ("f32", 1, 33, 2, 2, 33, 17, "s", None),
    ("bf16", 1, 64, 1, 2, 100, 70, "gs", (63,)),
    ("f16", 1, 96, 2, 2, 129, 33, "gs", (95,)),
    ("bf16", 1, 40, 1, 1, 256, 256, "gs", None),
    ("f32", 1, 40, 1, 2, 256, 130, "gs", (39,)),
    ("f16", 1, 31, 1, 1, 255, 1, "g", None),
    ("bf16", 2, 130, 1, 4, 128, 96, "gs", (130, 97)),
    ("f32", 1, 200, 1, 1, 64, 15, "gs", None),
    ("f32", 3, 66, 1, 2, 40, 65, "gs", (0, 0, 66)),
    # few heads and many chunks: the length is cut into segments
    ("f32", 1, 700, 1, 1, 16, 8, "gs", None),
    ("bf16", 2, 1100, 1, 2, 128, 64, "gs", (1100, 530)),
    ("f16", 3, 600, 1, 1, 64, 33, "gs", (599, 0, 1)),
    ("bf16", 1, 1290, 1, 1, 200, 40, "g", (1285,)),
    ("f32", 1, 530, 1, 2, 96, 100, "gs", None),
]


def delta_inputs(dtype, batch, length, key_heads, heads, key, value, parts, seed=4):
    x = Inputs(seed, DTYPES[dtype])
    for name, n, c in (("q", key_heads, key), ("k", key_heads, key), ("v", heads, value)):
        x.add(name, batch, length, n, c)
    for name in ("q", "k"):                      # of length one, as closely as the type has it
        t = x.cpu[name]
        x.put(name, (t / t.norm(dim=-1, keepdim=True)).to(DTYPES[dtype]))
    if "g" in parts:
        x.add("g", batch, length, heads, lo=-1.5, hi=0.0, dtype=torch.float32)
    x.add("beta", batch, length, heads, lo=0.05, hi=1.0, dtype=torch.float32)
    if "s" in parts:
        x.add("state", batch, heads, key, value, scale=0.5, dtype=torch.float32)
    return x


def run_delta(x, lengths=None, scale=None):
    def args(d):
        return [d.get(n) for n in ("q", "k", "v", "g", "beta")]

    outs = ops.gated_delta(*args(x.gpu), scale=scale, state=x.gpu.get("state"), lengths=int32(lengths),
                           return_state=True)
    return outs, ref.gated_delta(*args(x.cpu), scale=scale, state=x.cpu.get("state"), lengths=lengths)


@pytest.mark.parametrize("case", DELTA, ids=lambda c: "-".join(map(str, c[:7])))
def test_delta(case):
    *sizes, lengths = case
    x = delta_inputs(*sizes)
    if lengths is not None:                      # what lies past the ends is not a number
        with torch.no_grad():
            for i, e in enumerate(lengths):
                for n in ("q", "k", "v", "g", "beta"):
                    if n in x.gpu:
                        x.gpu[n][i, e:] = float("nan")
                        x.cpu[n][i, e:] = 0
    x.grads()
    outs, wants = run_delta(x, lengths)
    for n, o, w in zip(("o", "state"), outs, wants):
        check(o, w, n)
    compare_grads(x, outs, wants)


def test_delta_two_segments():
    """The least length that is cut in two; the plain form's 4100 steps run on the GPU too, in 64 bits."""
    x, ends = delta_inputs("bf16", 2, 4100, 8, 16, 66, 97, "gs"), (4100, 2000)
    with torch.no_grad():
        for n in ("q", "k", "v", "g", "beta"):
            x.gpu[n][1, ends[1]:] = float("nan")
            x.cpu[n][1, ends[1]:] = 0
    x.grads()
    names = ("q", "k", "v", "g", "beta")
    outs = ops.gated_delta(*[x.gpu[n] for n in names], state=x.gpu["state"], lengths=int32(ends), return_state=True)
    with torch.device(DEV):
        wants = ref.gated_delta(*[x.cpu[n].to(DEV) for n in names], state=x.cpu["state"].to(DEV), lengths=ends)
    wants = [w.cpu() for w in wants]
    for n, o, w in zip(("o", "state"), outs, wants):
        check(o, w, n)
    compare_grads(x, outs, wants)


@pytest.mark.parametrize("batch,length,key_heads,heads", [(64, 512, 1, 2), (16, 500, 2, 8)])
def test_delta_heads_that_share_a_key_head(batch, length, key_heads, heads):
    """So many blocks that one workgroup has all of a key head's heads, or some of them."""
    x = delta_inputs("f32", batch, length, key_heads, heads, 8, 8, "g")
    x.grads()
    outs, wants = run_delta(x)
    check(outs[0], wants[0], "o")
    compare_grads(x, outs[:1], wants[:1])


@pytest.mark.parametrize("key,value,length", [(16, 8, 90), (100, 33, 700)])
def test_delta_scratch_aligned_to_a_float(key, value, length):
    """Scratch and what is kept need no more than a float's alignment."""
    from tests import more_ops_abi as abi
    import ctypes
    lib, n = abi.library(), ctypes.c_uint64()
    x = delta_inputs("bf16", 1, length, 1, 1, key, value, "g")
    g = {k: t.contiguous() for k, t in x.gpu.items()}
    o, do = torch.empty_like(g["v"]), torch.randn_like(g["v"])
    back = {k: torch.empty_like(t) for k, t in g.items()}

    def heads(t):
        return abi.Heads(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))

    def view(t):
        return abi.abi.View(t.data_ptr(), t.stride(0), t.stride(1))

    a = abi.DeltaArgs(dtype=1, batch=1, length=length, key_heads=1, heads=1, key=key, value=value, scale=0.2,
                      q=heads(g["q"]), k=heads(g["k"]), v=heads(g["v"]), o=heads(o), g=view(g["g"]),
                      beta=view(g["beta"]), do_=heads(do), dq=heads(back["q"]), dk=heads(back["k"]),
                      dv=heads(back["v"]), dg=back["g"].data_ptr(), dbeta=back["beta"].data_ptr())
    buffers = []

    def floats(call):
        assert getattr(lib, call)(a, n) == 0
        buffers.append(torch.empty(n.value // 4 + 8, device=DEV))
        return buffers[-1].data_ptr() + 4, n.value

    got = []
    for _ in range(2):
        a.kept, _ = floats("rc_delta_kept_bytes")
        a.workspace, a.workspace_bytes = floats("rc_delta_forward_workspace")
        assert lib.rc_delta_forward(a, None) == 0
        a.workspace, a.workspace_bytes = floats("rc_delta_backward_workspace")
        assert lib.rc_delta_backward(a, None) == 0
        torch.cuda.synchronize()
        got.append([t.clone() for t in (o, *back.values())])
    leaves = [t.detach().requires_grad_() for t in g.values()]
    want = ops.gated_delta(*leaves, scale=0.2)
    for w, first, second in zip((want, *torch.autograd.grad(want, leaves, do)), *got):
        assert torch.equal(w, first) and torch.equal(w, second)


@pytest.mark.parametrize("of", ["o", "state"])
def test_delta_gradient_of_one_output(of):
    x = delta_inputs("f32", 2, 50, 1, 2, 20, 30, "gs")
    x.grads()
    outs, wants = run_delta(x, (50, 20))
    i = ("o", "state").index(of)
    compare_grads(x, [outs[i]], [wants[i]])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_delta_forgets(dtype):
    """Tokens that forget everything (-infinity, or a number whose exp is 0), that keep everything, and
    strong decays before weak ones: what comes after is as exact as without them."""
    x = delta_inputs(dtype, 2, 90, 1, 2, 32, 40, "gs")
    g = x.cpu["g"].clone() * 0.01
    g[0, 3, 0] = g[0, 40, 1] = float("-inf")
    g[1, 5, 0] = -1e30
    g[1, 33:60, 1] = -90.0
    g[1, 64, 0] = -500.0
    g[0, 70:75] = 0.0
    x.put("g", g.float())
    x.grads()
    outs, wants = run_delta(x)
    for n, o, w in zip(("o", "state"), outs, wants):
        check(o, w, n)
    # (exp's own derivative at -infinity is 0 times infinity in the reference: 0)
    rng = torch.Generator().manual_seed(5)
    vs = [torch.randn(w.shape, generator=rng).to(o.dtype) for o, w in zip(outs, wants)]
    names = list(x.gpu)
    got = torch.autograd.grad(outs, [x.gpu[n] for n in names], [v.to(DEV) for v in vs])
    want = torch.autograd.grad(wants, [x.cpu[n] for n in names], [v.double() for v in vs])
    for n, a, b in zip(names, got, want):
        check(a, torch.nan_to_num(b), "d" + n)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_delta_equal_keys(dtype):
    """One key over and over with beta 1 (each token replaces the last value), beta 0 (nothing is
    written), beta 2 (the value is mirrored), keys of zeros."""
    x = delta_inputs(dtype, 1, 70, 1, 4, 16, 8, "s")
    k = torch.zeros(1, 70, 1, 16)
    k[..., 3] = 1.0
    k[0, 50:55] = 0.0
    x.put("k", k.to(DTYPES[dtype]))
    beta = torch.ones(1, 70, 4)
    beta[..., 1] = 0.0
    beta[..., 2] = 2.0
    beta[0, ::3, 3] = 0.0
    x.put("beta", beta)
    x.grads()
    outs, wants = run_delta(x)
    for n, o, w in zip(("o", "state"), outs, wants):
        check(o, w, n)
    compare_grads(x, outs, wants)


@pytest.mark.parametrize("key_heads", [1, 4])
def test_delta_nothing_past_an_end(key_heads):
    """What the last tokens of a sequence hold reaches neither the tokens past its end nor other sequences."""
    x = delta_inputs("f32", 2, 70, key_heads, 4, 24, 20, "gs")
    x.gpu["v"].detach()[0, 42, 1] = float("nan")
    x.gpu["q"].detach()[0, 40, 0] = float("inf")
    leaves = [x.gpu[n].detach().requires_grad_() for n in ("q", "k", "v", "g", "beta")]
    o = ops.gated_delta(*leaves, state=x.gpu["state"].detach(), lengths=int32([43, 70]))
    for g, t in zip(torch.autograd.grad(o, leaves, torch.ones_like(o)), leaves):
        assert g[0].isnan().any() or t is leaves[2]
        assert not g[0, 43:].any() and g[1].isfinite().all() and g[1].any()
    assert not o[0, 43:].any() and o[1].isfinite().all()


def test_delta_layouts():
    """Slices of one projection, heads before tokens, an expanded gradient, a scale."""
    torch.manual_seed(3)
    b, n, h, d, e = 2, 45, 3, 24, 20
    wide = torch.randn(b, n, h * (2 * d + e), device=DEV) * 0.2
    q, k, v = (t.unflatten(-1, (h, -1)) for t in wide.split([h * d, h * d, h * e], -1))
    g, beta = -torch.rand(b, h, n, device=DEV).transpose(1, 2), torch.rand(b, n, 2 * h, device=DEV)[..., ::2]
    for args in ((q, k, v), [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v)],
                 [t.transpose(2, 3).contiguous().transpose(2, 3) for t in (q, k, v)]):
        leaves = [t.detach().requires_grad_() for t in (*args, g, beta)]
        o = ops.gated_delta(*leaves, scale=0.7)
        cpu = [t.detach().cpu().double().requires_grad_() for t in leaves]
        want, _ = ref.gated_delta(*cpu, scale=0.7)
        check(o, want, "o")
        for a, w in zip(torch.autograd.grad(o.sum(), leaves), torch.autograd.grad(want.sum(), cpu)):
            check(a, w, "gradient")


def test_delta_empty():
    for shape in ((0, 5, 2), (2, 0, 2), (2, 5, 0)):
        q, v = torch.randn(*shape[:2], min(shape[2], 1), 8, device=DEV), torch.randn(*shape, 6, device=DEV)
        beta = torch.rand(shape, device=DEV)
        s = torch.randn(shape[0], shape[2], 8, 6, device=DEV)
        leaves = [t.requires_grad_() for t in (q, v, beta, s)]
        o, end = ops.gated_delta(q, q, v, None, beta, state=s, return_state=True)
        assert o.shape == v.shape and end.shape == s.shape
        if not shape[1]:
            assert torch.equal(end, s)
            ds, = torch.autograd.grad(end, s, torch.ones_like(end), retain_graph=True)
            assert torch.equal(ds, torch.ones_like(s))
        for t, g in zip(leaves, torch.autograd.grad(o.sum() + end.sum(), leaves, allow_unused=True)):
            assert g is None or g.shape == t.shape


def test_delta_lengths_outside_the_batch():
    """Lengths are clamped to [0, length]."""
    x = delta_inputs("f32", 3, 20, 1, 1, 8, 8, "gs").gpu

    def run(n):
        return ops.gated_delta(x["q"], x["k"], x["v"], x["g"], x["beta"], state=x["state"], lengths=int32(n),
                               return_state=True)

    for a, b in zip(run([-5, 1000, 20]), run([0, 20, 20])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,batch,key_heads,heads,key,value", [
    ("f32", 3, 2, 4, 10, 12), ("bf16", 5, 1, 3, 128, 128), ("f16", 1, 1, 1, 1, 1), ("bf16", 2, 2, 2, 256, 256),
    ("f32", 2, 1, 2, 33, 65), ("f16", 4, 2, 2, 65, 31), ("bf16", 2, 1, 1, 200, 3)])
def test_delta_step(dtype, batch, key_heads, heads, key, value):
    x = delta_inputs(dtype, batch, 6, key_heads, heads, key, value, "gs")
    pool = torch.randn(batch + 3, heads, key, value, device=DEV)
    slots = torch.randperm(batch + 3, device=DEV)[:batch].to(torch.int32)
    pool[slots.long()] = x.gpu["state"]
    before = pool.clone()
    c = x.cpu
    whole = ref.gated_delta(c["q"], c["k"], c["v"], c["g"], c["beta"], state=c["state"])
    for t in range(6):
        o = ops.gated_delta_step(pool, *[x.gpu[n][:, t] for n in ("q", "k", "v", "g", "beta")], slots=slots)
        check(o, whole[0][:, t], f"o {t}")
    check(pool[slots.long()], whole[1], "state")
    rest = torch.ones(batch + 3, dtype=torch.bool, device=DEV)
    rest[slots.long()] = False
    assert torch.equal(pool[rest], before[rest])


def test_delta_step_parts_and_padding():
    """Without g, with a scale and a wider pool's rows, -infinity; padded rows of anything."""
    x = delta_inputs("f32", 2, 1, 1, 2, 8, 12, "s")
    c, wide = x.cpu, torch.zeros(3, 2 * 8 * 12 + 5, device=DEV)
    pool = wide.as_strided((3, 2, 8, 12), (wide.shape[1], 96, 12, 1))
    pool[:2] = x.gpu["state"]
    want = ref.gated_delta(c["q"], c["k"], c["v"], None, c["beta"], 0.3, c["state"])
    o = ops.gated_delta_step(pool, *[x.gpu[n][:, 0] for n in ("q", "k", "v")], None, x.gpu["beta"][:, 0], scale=0.3)
    check(o, want[0][:, 0], "o")
    check(pool[:2], want[1], "state")
    nan = [torch.full(s, float("nan"), device=DEV) for s in ((3, 1, 8), (3, 1, 8), (3, 2, 12), (3, 2), (3, 2))]
    before = wide.clone()
    o = ops.gated_delta_step(pool, *nan, slots=int32([-1, 3, 2 ** 31 - 1]))
    assert not o.any() and torch.equal(wide, before)
    clear = torch.full((2, 2), float("-inf"), device=DEV)
    o = ops.gated_delta_step(pool, *[x.gpu[n][:, 0] for n in ("q", "k", "v")], clear, x.gpu["beta"][:, 0])
    want = ref.gated_delta(c["q"], c["k"], c["v"], None, c["beta"])
    check(o, want[0][:, 0], "o after forgetting")
    check(pool[:2], want[1], "state after forgetting")


# ----------------------------------------------------------- queries and keys

QK = [  # dtype, batch, length, heads, key_heads, channels, rotated, norm, interleaved, weights, lengths
    ("f32", 2, 9, 4, 2, 32, 32, "rms", False, "f32", None),
    ("bf16", 2, 17, 3, 1, 128, 128, "rms", False, "f32", (17, 4)),
    ("f16", 3, 5, 2, 2, 64, 32, "l2", True, None, (5, 0, 1)),
    ("f32", 1, 1, 1, 1, 1, 0, "rms", False, "f32", None),
    ("bf16", 1, 33, 1, 5, 80, 48, "l2", True, "bf16", None),
    ("f32", 2, 6, 2, 1, 33, 20, "rms", False, "f32", (6, 5)),
    ("f16", 1, 7, 2, 2, 255, 254, "rms", True, "f16", None),
    ("f16", 1, 7, 2, 2, 251, 250, "rms", False, "f32", None),
    ("bf16", 1, 4, 40, 3, 256, 256, "rms", False, "f32", None),
    ("f32", 2, 8, 2, 2, 16, 16, None, False, None, (8, 3)),
    ("f32", 1, 8, 2, 2, 18, 2, None, True, "f32", None),
    ("bf16", 1, 8, 1, 1, 256, 2, "l2", False, None, None),
    ("f32", 1, 300, 5, 2, 10, 6, "rms", False, "f32", (290,)),
    ("f32", 2, 5, 3, 0, 24, 24, "rms", False, "f32", None),
]


def qk_inputs(dtype, batch, length, heads, key_heads, channels, weights, seed=6):
    x = Inputs(seed, DTYPES[dtype])
    x.add("q", batch, length, heads, channels)
    x.add("k", batch, length, key_heads, channels, scale=0.3)
    if weights:
        x.add("q_weight", channels, lo=0.5, hi=1.5, dtype=DTYPES[weights])
        x.add("k_weight", channels, lo=-1.5, hi=-0.5, dtype=DTYPES[weights])
    return x


def run_qk(x, freq, positions, lengths, **kw):
    def args(d):
        return [d.get(n) for n in ("q", "k", "q_weight", "k_weight")]

    outs = ops.qk_norm(*args(x.gpu), None if freq is None else freq.to(DEV),
                       None if positions is None else positions.to(DEV), lengths=int32(lengths), **kw)
    return outs, ref.qk_norm(*args(x.cpu), freq, positions, lengths=lengths, **kw)


@pytest.mark.parametrize("case", QK, ids=lambda c: "-".join(map(str, c[:9])))
def test_qk(case):
    dtype, batch, length, heads, key_heads, channels, rotated, norm, inter, weights, lengths = case
    x = qk_inputs(dtype, batch, length, heads, key_heads, channels, weights)
    freq = torch.rand(rotated // 2) ** 3 if rotated else None
    positions = torch.randint(0, 5000, (batch, length), dtype=torch.int32)
    if lengths is not None:
        for i, e in enumerate(lengths):
            for n in ("q", "k"):
                x.gpu[n][i, e:] = float("nan")
                x.cpu[n][i, e:] = 0
    x.grads()
    outs, wants = run_qk(x, freq, positions, lengths, norm=norm, interleaved=inter)
    for n, o, w in zip("qk", outs, wants):
        check(o, w, n)
    if channels > 1:
        compare_grads(x, outs, wants)
        return
    # One channel: dx = r (a - u m) with a the gradient of the unit vector u and m = mean(a u) = a u, and
    # 1 - u^2 is only eps r^2, a millionth.  a, u, m and the products are each within a few 2^-24 of
    # their sizes, so dx is off by a few 2^-24 of r |a| (1 + u^2), whatever is left of it: at most 16 of them.
    gs = [torch.full_like(o, 1.25) for o in outs]
    got = torch.autograd.grad(outs, list(x.gpu.values()), gs)
    want = torch.autograd.grad(wants, list(x.cpu.values()), [g.cpu().double() for g in gs])
    for n, g, w in zip(x.gpu, got, want):
        if n in "qk":
            size = 2 * 1.25 * (x.cpu[n + "_weight"] / x.cpu[n]).abs().max().item()
            assert (g.cpu().double() - w).abs().max().item() <= 16 * 2.0 ** -24 * size, n
        else:
            check(g, w, "d" + n)


@pytest.mark.parametrize("of", [0, 1])
def test_qk_gradient_of_one_output(of):
    x = qk_inputs("f32", 2, 7, 2, 3, 20, "f32")
    x.grads()
    outs, wants = run_qk(x, torch.rand(5), None, (7, 2))
    compare_grads(x, [outs[of]], [wants[of]])


def test_qk_far_positions():
    """Angles of the largest positions, before and behind: the product is taken in 64 bits, so the angle is
    exact to about 2^31 2^-52 turns."""
    x = qk_inputs("f32", 1, 6, 2, 1, 64, None)
    positions = torch.tensor([[2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, -1, 16777217, 0]], dtype=torch.int32)
    freq = 10000.0 ** (-torch.arange(32) / 32)
    outs, wants = run_qk(x, freq.float(), positions, None)
    for n, o, w in zip("qk", outs, wants):
        check(o, w, n)


def test_qk_rows_of_zeros():
    """eps alone under the root: zeros stay zeros, their gradient is finite and eps^-1/2 large."""
    x = qk_inputs("f32", 1, 3, 2, 2, 16, "f32")
    x.put("q", x.cpu["q"].float() * torch.tensor([0.0, 1.0, 0.0])[None, :, None, None])
    x.grads()
    for norm in ("rms", "l2"):
        outs, wants = run_qk(x, torch.rand(8), None, None, norm=norm)
        for n, o, w in zip("qk", outs, wants):
            check(o, w, n)
        compare_grads(x, outs, wants)


def test_qk_layouts():
    """Slices of one projection, heads before tokens, channels apart; positions of one row for all, expanded
    gradients."""
    torch.manual_seed(5)
    wide = torch.randn(2, 11, 7, 24, device=DEV)
    freq, at = torch.rand(12), torch.randint(0, 99, (1, 11), dtype=torch.int32)
    for q, k in ((wide[:, :, :4], wide[:, :, 4:6]),
                 [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (wide[:, :, :4], wide[:, :, 4:])],
                 [t.transpose(2, 3).contiguous().transpose(2, 3) for t in (wide[:, :, :4], wide[:, :, 4:])]):
        q, k = (t.detach().requires_grad_() for t in (q, k))
        outs = ops.qk_norm(q, k, None, None, freq.to(DEV), at.to(DEV).expand(2, 11))
        cq, ck = (t.detach().cpu().double().requires_grad_() for t in (q, k))
        wants = ref.qk_norm(cq, ck, None, None, freq, at.expand(2, 11))
        for o, w in zip(outs, wants):
            check(o, w, "output")
        for a, b in zip(torch.autograd.grad(outs[0].sum() + outs[1].sum(), [q, k]),
                        torch.autograd.grad(wants[0].sum() + wants[1].sum(), [cq, ck])):
            check(a, b, "gradient")


def test_qk_empty():
    w = torch.rand(8, device=DEV, requires_grad=True)
    for shape in ((0, 4, 2, 8), (2, 0, 2, 8), (2, 4, 0, 8)):
        q = torch.randn(shape, device=DEV, requires_grad=True)
        a, b = ops.qk_norm(q, q, w, w)
        assert a.shape == q.shape and b.shape == q.shape
        dq, dw = torch.autograd.grad(a.sum() + b.sum(), [q, w])
        assert dq.shape == q.shape and not dw.any()


# -------------------------------------------------------------------- dropout


def mask_of(shape, p, seed, tag=0):
    n = 1
    for s in shape:
        n *= s
    return ref.kept(n, p, seed, tag).reshape(shape)


DROPOUT = [  # dtype, shape, p, residual ("f32", "same" or None)
    ("f32", (5, 33), 0.3, None), ("bf16", (4, 64), 0.1, "f32"), ("f16", (3, 7, 11), 0.5, "same"),
    ("bf16", (1, 1), 0.5, None), ("f16", (1000,), 0.25, None), ("f32", (2, 8), 0.9, "same"),
    ("bf16", (), 0.5, "same"), ("bf16", (13, 24), 0.0, "f32"), ("f16", (13, 24), 1.0, "f32"),
    ("f32", (7, 1), 0.2, None), ("f16", (9, 1031), 0.4, "f32"),
]


@pytest.mark.parametrize("case", DROPOUT, ids=lambda c: "-".join(map(str, c)))
def test_dropout(case):
    dtype, shape, p, residual = case
    x = Inputs(7, DTYPES[dtype])
    x.add("x", *shape)
    if residual:
        x.add("residual", *shape, dtype=torch.float32 if residual == "f32" else None)
    x.grads()
    seed, tag = 0x123456789ABCDEF, 77
    out = ops.dropout(x.gpu["x"], p, seed, tag=tag, residual=x.gpu.get("residual"))
    gain = mask_of(shape, p, seed, tag).double() * (1 / (1 - p) if p < 1 else 0.0)
    want = x.cpu["x"] * gain + (x.cpu["residual"] if residual else 0)
    assert out.dtype == (x.gpu["residual"] if residual else x.gpu["x"]).dtype
    check(out, want, "out")
    compare_grads(x, [out], [want])


def test_dropout_seeds():
    """Seeds and tags of 64 bits, negative or not, as ints and on the GPU; each draws a mask of its own."""
    x = torch.ones(40, 5, device=DEV)
    seen = set()
    for seed, tag in ((0, 0), (0, 1), (1, 0), (2 ** 32, 0), (0, 2 ** 32), (2 ** 64 - 1, 3), (-1, 2 ** 63),
                      (-2 ** 63, -2 ** 63)):
        out = ops.dropout(x, 0.5, seed, tag=tag).cpu() != 0
        assert torch.equal(out, mask_of((40, 5), 0.5, seed % 2 ** 64, tag % 2 ** 64))
        there = torch.tensor(seed - 2 ** 64 if seed >= 2 ** 63 else seed, device=DEV)
        assert torch.equal(ops.dropout(x, 0.5, there, tag=tag).cpu() != 0, out)
        seen.add(tuple(out.flatten().tolist()))
    assert len(seen) == 8


def test_dropout_layouts():
    """The mask goes by an element's place in a contiguous x, whatever the strides; gradients too."""
    seed = 5
    for d in (24, 17):
        wide = torch.randn(6, 9, 40, device=DEV)
        for x in (wide[..., 3:3 + d], wide[:, ::2, :d], wide.transpose(0, 1)[..., :d], wide[0, :, 5:5 + d],
                  wide.transpose(1, 2)[:, :d, :8]):
            r = torch.randn(x.shape[::-1], device=DEV).permute(*range(x.ndim)[::-1])
            leaf = x.detach().requires_grad_()
            out = ops.dropout(leaf, 0.5, seed, residual=r)
            keep = mask_of(x.shape, 0.5, seed)
            want = torch.where(keep, x.cpu().double() * 2, 0) + r.cpu().double()
            check(out, want, "out")
            g = torch.randn(x.shape[::-1], device=DEV).permute(*range(x.ndim)[::-1])
            dx, = torch.autograd.grad(out, leaf, g)
            check(dx, torch.where(keep, g.cpu().double() * 2, 0), "dx")
            dx, = torch.autograd.grad(ops.dropout(leaf, 0.5, seed).sum(), leaf)      # an expanded gradient
            assert torch.equal(dx.cpu() != 0, keep)


def test_dropout_what_is_dropped_is_zero():
    """Infinity and NaN in dropped places reach nothing."""
    keep = mask_of((8, 16), 0.5, 9)
    x = torch.where(keep, 1.0, torch.tensor(float("nan"))).to(DEV)
    assert torch.equal(ops.dropout(x, 0.5, 9).cpu(), keep * 2.0)
    assert not ops.dropout(torch.full_like(x, float("inf")), 1.0, 9).any()


def test_dropout_second_run_and_share():
    """A second run draws the same mask; the share that is kept is 1 - p within five standard deviations
    (sqrt(p (1 - p) / n)), and so is each of the four words' (of a quarter as many)."""
    x = torch.ones(1024, 1024, dtype=torch.bfloat16, device=DEV)
    for p in (0.1, 0.5):
        a = ops.dropout(x, p, 31)
        assert torch.equal(a, ops.dropout(x, p, 31))
        keep = (a != 0).float().reshape(-1, 4)
        spread = (p * (1 - p) / keep.numel()) ** 0.5
        assert abs(keep.mean().item() - (1 - p)) < 5 * spread
        assert (keep.mean(0) - (1 - p)).abs().max().item() < 10 * spread


def test_dropout_empty():
    for shape in ((0,), (0, 4), (4, 0)):
        x = torch.zeros(shape, device=DEV, requires_grad=True)
        out = ops.dropout(x, 0.5, 1, residual=torch.zeros(shape, device=DEV))
        assert out.shape == x.shape
        assert torch.autograd.grad(out.sum(), x)[0].shape == x.shape


# ------------------------------------------------------------- all of them


@pytest.mark.parametrize("op", ["delta", "qk"])
def test_gradient_against_differences(op):
    """<gradient, v> against (f(x + e v) - f(x - e v)) / 2e, all in 32 bits: the difference is off by
    e^2 f''' / 6 (e = 2^-7: about 1e-5 of f''') and by the rounding of f over 2e (2^-24 64 |f|): 1 % of the
    gradient's size covers both."""
    torch.manual_seed(8)
    if op == "delta":
        x = delta_inputs("f32", 2, 40, 1, 2, 12, 10, "gs")
        names = ["q", "k", "v", "g", "beta", "state"]
        f = lambda v: ops.gated_delta(*v[:5], state=v[5])  # noqa: E731
    else:
        x = qk_inputs("f32", 2, 10, 2, 2, 24, "f32")
        names = ["q", "k", "q_weight", "k_weight"]
        freq = torch.rand(9, device=DEV)
        f = lambda v: torch.cat(ops.qk_norm(*v, freq))  # noqa: E731
    xs = [x.gpu[n].requires_grad_() for n in names]
    weight = torch.randn_like(f(xs).detach())
    total = lambda v: (f(v).double() * weight).sum()  # noqa: E731
    grads = torch.autograd.grad(total(xs), xs)
    for i, (n, g) in enumerate(zip(names, grads)):
        v = [torch.randn_like(t) if j == i else torch.zeros_like(t) for j, t in enumerate(xs)]
        with torch.no_grad():
            hi, lo = (total([t.detach() + s * 2.0 ** -7 * d for t, d in zip(xs, v)]).item() for s in (1, -1))
        want = (g.double() * v[i]).sum().item()
        assert abs((hi - lo) * 64 - want) <= 0.01 * g.double().norm().item() + 1e-3, n


class Block:
    """A block of linear attention: convolution, norms and rotation of its q and k, delta rule,
    dropout onto the residual stream, and the norm before the next block."""

    def __init__(self, dtype, batch, length, heads=2, key=16, value=24, seed=12):
        self.h, self.dk, self.dv, self.batch, self.length = heads, key, value, batch, length
        self.width = heads * (2 * key + value)
        x = self.x = Inputs(seed, dtype)
        x.add("x", batch, length, self.width)
        x.add("w", self.width, 4, scale=0.5, dtype=torch.float32)
        x.add("g", batch, length, heads, lo=-1.0, hi=0.0, dtype=torch.float32)
        x.add("beta", batch, length, heads, lo=0.05, hi=1.0, dtype=torch.float32)
        x.add("r", batch, length, heads * value, dtype=torch.float32)
        x.add("pre", heads * value, lo=0.5, hi=1.5, dtype=torch.float32)
        x.grads()
        self.freq = 100.0 ** (-torch.arange(key // 2) / (key // 2))
        self.gpu_freq = self.freq.to(DEV)

    def split(self, u):
        n = [self.h * self.dk] * 2 + [self.h * self.dv]
        return [t.unflatten(-1, (self.h, -1)) for t in u.split(n, -1)]

    def run(self, p, kernels, seed=3, first=0, states=None):
        if kernels:
            u, conv = ops.causal_conv(p["x"], p["w"], return_state=True)
            q, k, v = self.split(u)
            q, k = ops.qk_norm(q, k, None, None, self.gpu_freq, norm="l2")
            o, S = ops.gated_delta(q, k, v, p["g"], p["beta"], return_state=True)
            r = ops.dropout(o.flatten(-2), 0.25, seed, residual=p["r"])
            return r, ops.norm_residual(None, r, pre_weight=p["pre"])[1], conv, S
        u, conv = old.causal_conv(p["x"], p["w"])
        q, k, v = self.split(u)
        q, k = ref.qk_norm(q, k, None, None, self.freq, norm="l2")
        o, S = ref.gated_delta(q, k, v, p["g"], p["beta"])
        y = o.flatten(-2)
        r = p["r"] + y * mask_of(y.shape, 0.25, seed).double() / 0.75
        return r, old.norm_residual(None, r, pre=p["pre"])[1], conv, S


def test_a_block_of_them():
    """As they would be used together, with gradients, in 32 bits against the chain of the references."""
    b = Block(torch.float32, 2, 50)
    outs, wants = b.run(b.x.gpu, True), b.run(b.x.cpu, False)
    for n, o, w in zip(("r", "normed", "conv", "state"), outs, wants):
        check(o, w, n)
    compare_grads(b.x, outs[:2], wants[:2])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_block_token_by_token(dtype):
    """A prompt and then single tokens give what the whole sequence gives.  In 16 bits the intermediate
    results of both ways are rounded from 32-bit values that differ by their noise: nearly all alike, a
    few by one unit (2^-7 of a value)."""
    b = Block(dtype, 2, 41)
    p = {n: t.detach() for n, t in b.x.gpu.items()}
    with torch.no_grad():
        _, _, conv_end, S_end = b.run(p, True)
        u = ops.causal_conv(p["x"], p["w"])
        q, k, v = b.split(u)
        q, k = ops.qk_norm(q, k, None, None, b.gpu_freq, norm="l2")
        whole = ops.gated_delta(q, k, v, p["g"], p["beta"])
        n = 33
        _, conv = ops.causal_conv(p["x"][:, :n], p["w"], return_state=True)
        _, S = ops.gated_delta(q[:, :n], k[:, :n], v[:, :n], p["g"][:, :n], p["beta"][:, :n], return_state=True)
        pool = torch.full((4, *S.shape[1:]), 7.0, device=DEV)
        slots = int32([2, 0])
        pool[slots.long()] = S
        for t in range(n, b.length):
            u = ops.causal_conv_step(conv, p["x"][:, t], p["w"])
            qt, kt, vt = b.split(u)
            at = torch.full((2, 1), t, dtype=torch.int32, device=DEV)
            qt, kt = ops.qk_norm(qt[:, None], kt[:, None], None, None, b.gpu_freq, at, norm="l2")
            o = ops.gated_delta_step(pool, qt[:, 0], kt[:, 0], vt, p["g"][:, t], p["beta"][:, t], slots=slots)
            tol = 1e-5 if dtype == torch.float32 else 2.0 ** -6
            torch.testing.assert_close(o.float(), whole[:, t].float(), rtol=tol, atol=tol)
    assert torch.equal(conv, conv_end)
    torch.testing.assert_close(pool[slots.long()], S_end, rtol=tol, atol=tol)
    assert (pool[1] == 7).all() and (pool[3] == 7).all()


def grads_of(b, seed):
    outs = b.run(b.x.gpu, True, seed=seed)[:2]
    grads = torch.autograd.grad(outs, list(b.x.gpu.values()), [torch.ones_like(o) for o in outs])
    return [o.detach() for o in outs] + list(grads)


def test_other_stream_and_repeats():
    """The same bits on another stream and in every repeat."""
    b = Block(torch.bfloat16, 2, 70)
    first = grads_of(b, 3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = grads_of(b, 3)
    torch.cuda.current_stream().wait_stream(s)
    for x, y, z in zip(first, other, grads_of(b, 3)):
        assert torch.equal(x, y) and torch.equal(x, z)


def test_graph_replays():
    """A captured forward and backward pass and a captured token give the eager results at every replay, with
    other work between them; the mask follows the seed's tensor."""
    b = Block(torch.bfloat16, 2, 70)
    seed = torch.tensor([1], device=DEV)
    pool = torch.randn(4, 2, 16, 24, device=DEV)
    slots = int32([3, -1])
    tok = [torch.randn(2, 2, n, device=DEV, dtype=torch.bfloat16) * 0.2 for n in (16, 16, 24)]
    gates = [-torch.rand(2, 2, device=DEV), torch.rand(2, 2, device=DEV)]

    def step():
        return ops.gated_delta_step(pool, *tok, *gates, slots=slots)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        grads_of(b, seed), step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = grads_of(b, seed)
        o = step()
    masks = []
    for k in range(4):
        with torch.no_grad():
            for t in b.x.gpu.values():
                t.mul_(1.0 - 0.01 * k)
            seed.fill_(100 + k)
            tok[0].copy_(torch.randn(2, 2, 16, device=DEV))
        state = pool.clone()
        want, wo = grads_of(b, seed), step()
        after = pool.clone()
        pool.copy_(state)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs, want):
            assert torch.equal(x, y), k
        assert torch.equal(o, wo) and torch.equal(pool, after)
        masks.append(outs[0].clone())
    assert not torch.equal(masks[0], masks[1])


def test_far_offsets():
    """Tokens whose offsets pass 2^31 elements: strided views of a large buffer."""
    d, n, step = 32, 40, 2 ** 30 // 16
    big = torch.zeros(step * n + 3 * d, dtype=torch.bfloat16, device=DEV)
    rows = torch.randn(n, 3 * d).to(torch.bfloat16) * 0.15
    x = big.as_strided((1, n, 3 * d), (0, step, 1))
    x.copy_(rows.to(DEV)[None])
    q, k, v = (t.unflatten(-1, (2, -1)) for t in x.split(d, -1))
    g, beta = -torch.rand(1, n, 2), torch.rand(1, n, 2)
    cq, ck, cv = (t.double().unflatten(-1, (2, -1))[None] for t in rows.split(d, -1))
    check(ops.gated_delta(q, k, v, g.to(DEV), beta.to(DEV)),
          ref.gated_delta(cq, ck, cv, g.double(), beta.double())[0], "o")
    freq = torch.rand(8)
    for a, w in zip(ops.qk_norm(q, k, None, None, freq.to(DEV)), ref.qk_norm(cq, ck, None, None, freq)):
        check(a, w, "qk")
    check(ops.dropout(x, 0.5, 3), rows.double()[None] * mask_of((1, n, 3 * d), 0.5, 3) * 2, "dropout")
    # elements past 2^32 of one dropout: their counters pass 2^30
    del big, x, q, k, v
    ones = torch.ones(1, dtype=torch.bfloat16, device=DEV).expand(2 ** 32 + 64).contiguous()
    tail = ops.dropout(ones, 0.5, 3)[-64:].cpu() != 0
    words = []
    for i in range(2 ** 30, 2 ** 30 + 16):
        words += ref.philox([i, 0, 0, 0], [3, 0])
    assert torch.equal(tail, torch.tensor([w >= 2 ** 31 for w in words]))
    # a pool's slot past 2^31 elements
    pool = torch.zeros(2 ** 25 + 2, 1, 8, 8, device=DEV)
    t = [c[:, 0, :1, :8] for c in (cq, ck, cv)]
    gb = [c[:, 0, :1] for c in (g, beta)]
    o = ops.gated_delta_step(pool, *[c.bfloat16().to(DEV) for c in t], *[c.to(DEV) for c in gb],
                             slots=int32([2 ** 25 + 1]))
    want = ref.gated_delta(*[c[:, None] for c in t], *[c.double()[:, None] for c in gb])
    check(o, want[0][:, 0], "token")
    check(pool[-1:], want[1], "slot")
    assert not pool[:2 ** 20].any()


def test_delta_many_tokens():
    """Queries and keys of 2^31 elements each, heads of one number: where everything before is forgotten, outputs
    and gradients are those of the tokens from there on, bit for bit."""
    n, h, tail = 2 ** 17, 128, 128
    q = torch.randn(1, n, h, 128, dtype=torch.bfloat16, device=DEV).mul_(0.08)
    k = q.flip(2)
    v, beta = (torch.rand(1, n, h, *c, dtype=t, device=DEV) for c, t in (((1,), torch.bfloat16), ((), torch.float32)))
    g = -beta
    g[:, -tail] = -float("inf")

    def run(from_):
        t = [x[:, from_:].requires_grad_() for x in (q.detach(), k.detach(), v.detach(), g.detach(), beta.detach())]
        o = ops.gated_delta(*t)
        d = torch.zeros_like(o)
        d[:, -tail:] = v.detach()[:, -tail:]
        return [o.detach()[:, -tail:]] + [x[:, -tail:].clone() for x in torch.autograd.grad(o, t, d)]

    few = run(n - tail)
    many = run(0)
    for a, b in zip(few, many):
        assert torch.equal(a, b) and a.any()


# ------------------------------------------------------------------- refusals


def test_refusals():
    b, n, h, d = 2, 5, 2, 8
    x = torch.randn(b, n, h, d, device=DEV)
    g = -torch.rand(b, n, h, device=DEV)
    pool = torch.zeros(2, h, d, d, device=DEV)
    t, gt = x[:, 0], g[:, 0]
    freq, at = torch.rand(4, device=DEV), torch.zeros(b, n, dtype=torch.int32, device=DEV)
    wide = torch.zeros(1, 3, 1, 257, device=DEV)
    one = torch.zeros(1, 3, 1, device=DEV)
    small = torch.zeros(1, 3, 1, 4, device=DEV)
    bad = [
        lambda: ops.gated_delta(x.cpu(), x, x, g, g),
        lambda: ops.gated_delta(x, x, x.cpu(), g, g),
        lambda: ops.gated_delta(x.double(), x.double(), x.double(), g, g),
        lambda: ops.gated_delta(x, x.half(), x, g, g),
        lambda: ops.gated_delta(x, x, x, g.half(), g),
        lambda: ops.gated_delta(x, x, x, g, g.bfloat16()),
        lambda: ops.gated_delta(x, x, x, g[:, :, :1], g),
        lambda: ops.gated_delta(x, x, x, g, g[:, :4]),
        lambda: ops.gated_delta(x, x, x[0], g, g),
        lambda: ops.gated_delta(x[0], x, x, g, g),
        lambda: ops.gated_delta(x, x[:, :, :1], x, g, g),
        lambda: ops.gated_delta(torch.cat([x, x[:, :, :1]], 2), torch.cat([x, x[:, :, :1]], 2), x, g, g),
        lambda: ops.gated_delta(x[..., :0], x[..., :0], x, g, g),
        lambda: ops.gated_delta(x, x, x[:, :, :0], g[:, :, :0], g[:, :, :0]),
        lambda: ops.gated_delta(x, x, x[..., :0], g, g),
        lambda: ops.gated_delta(wide, wide, small, one, one),
        lambda: ops.gated_delta(small, small, wide, one, one),
        lambda: ops.gated_delta(x, x, x, g, g, state=pool.half()),
        lambda: ops.gated_delta(x, x, x, g, g, state=pool[:, :, :4]),
        lambda: ops.gated_delta(x, x, x, g, g, lengths=torch.zeros(b, dtype=torch.int64, device=DEV)),
        lambda: ops.gated_delta_step(pool[:1], t, t, t, gt, gt),
        lambda: ops.gated_delta_step(pool.half(), t, t, t, gt, gt),
        lambda: ops.gated_delta_step(pool.transpose(2, 3), t, t, t, gt, gt),
        lambda: ops.gated_delta_step(pool[:1].expand(2, -1, -1, -1), t, t, t, gt, gt),
        lambda: ops.gated_delta_step(pool, t, t, t, gt, gt, slots=torch.zeros(b, dtype=torch.int64, device=DEV)),
        lambda: ops.gated_delta_step(pool, t, t, t.requires_grad_(), gt, gt),
        lambda: ops.qk_norm(x, x.half()),
        lambda: ops.qk_norm(x, x[..., :4]),
        lambda: ops.qk_norm(x[0], x),
        lambda: ops.qk_norm(x, x[0]),
        lambda: ops.qk_norm(x, x, freq[:2]),
        lambda: ops.qk_norm(x, x, torch.rand(d, device=DEV).half()),
        lambda: ops.qk_norm(x, x, torch.rand(d, device=DEV), torch.rand(d, device=DEV).bfloat16()),
        lambda: ops.qk_norm(x, x, None, None, torch.rand(5, device=DEV)),
        lambda: ops.qk_norm(x, x, None, None, freq.double()),
        lambda: ops.qk_norm(x, x, None, None, freq[None]),
        lambda: ops.qk_norm(x, x, None, None, freq.clone().requires_grad_()),
        lambda: ops.qk_norm(x, x, None, None, freq, at.long()),
        lambda: ops.qk_norm(x, x, None, None, freq, at[:1]),
        lambda: ops.qk_norm(x, x, norm="batch"),
        lambda: ops.qk_norm(wide, wide),
        lambda: ops.dropout(x, 1.5, 0),
        lambda: ops.dropout(x, -0.1, 0),
        lambda: ops.dropout(x, float("nan"), 0),
        lambda: ops.dropout(x.double(), 0.5, 0),
        lambda: ops.dropout(x, 0.5, 0, residual=x[:1]),
        lambda: ops.dropout(x.half(), 0.5, 0, residual=x.bfloat16()),
        lambda: ops.dropout(x, 0.5, torch.zeros(2, dtype=torch.int64, device=DEV)),
        lambda: ops.dropout(x, 0.5, torch.zeros(1, device=DEV)),
        lambda: ops.dropout(x, 0.5, torch.zeros(1, dtype=torch.int64)),
        lambda: ops.dropout(x, 0.5, None),
        lambda: ops.dropout(x, 0.5, 0, tag=0.5),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("not refused:", i)
    torch.cuda.synchronize()


def test_twice_differentiated_and_forward_mode_are_refused():
    x = torch.randn(1, 6, 2, 8, device=DEV, requires_grad=True)
    g = torch.rand(1, 6, 2, device=DEV)
    calls = [lambda x: ops.gated_delta(x, x, x, None, g), lambda x: ops.qk_norm(x, x)[0],
             lambda x: ops.dropout(x, 0.5, 1)]
    for f in calls:
        d, = torch.autograd.grad(f(x).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(d.sum(), x)
        with torch.autograd.forward_ad.dual_level():
            dual = torch.autograd.forward_ad.make_dual(x.detach(), torch.ones_like(x))
            with pytest.raises(NotImplementedError):
                f(dual)


def test_a_step_on_a_saved_state_is_seen():
    pool = torch.randn(2, 1, 8, 8, device=DEV)
    w = torch.randn(2, 1, 8, 8, device=DEV, requires_grad=True)
    y = (pool * w).sum()
    x, g = torch.randn(2, 1, 8, device=DEV), torch.rand(2, 1, device=DEV)
    with torch.no_grad():
        ops.gated_delta_step(pool, x, x, x, None, g)
    with pytest.raises(RuntimeError):
        y.backward()


def test_views_that_negate():
    """Lazily negated views are taken at their values."""
    x = torch.randn(1, 5, 2, 8, device=DEV) * 0.3
    g = torch.rand(1, 5, 2, device=DEV)
    neg = torch._neg_view(x)
    a = ops.gated_delta(neg, neg, neg, torch._neg_view(g), g)
    assert torch.equal(a, ops.gated_delta(-x, -x, -x, -g, g))
    for a, b in zip(ops.qk_norm(neg, neg), ops.qk_norm(-x, -x)):
        assert torch.equal(a, b)
    assert torch.equal(ops.dropout(neg, 0.5, 1, residual=neg), ops.dropout(-x, 0.5, 1, residual=-x))
    with pytest.raises(ValueError):
        ops.gated_delta_step(torch._neg_view(torch.zeros(1, 2, 8, 8, device=DEV)), x[:, 0], x[:, 0], x[:, 0],
                             None, g[:, 0])
