"""The sequence-model operators on the GPU against plain 64-bit
implementations: every type, odd sizes, strides, ragged and empty sequences, gradients,
single tokens, streams and graphs."""

import pytest
import torch

from tests import ops_reference as ref

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1905_11722_amd import ops  # noqa: E402

DEV = torch.device("cuda", 0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# The kernels compute in 32 bits and round once.  A 16-bit result is off by
# half a unit in its last place (2^-8 or 2^-11 of it, or half the smallest
# subnormal, 2^-25).  In 32 bits, sums of up to some thousand terms and a few
# approximate functions (each within 2^-23) leave about a hundred units of
# 2^-24 of the result's typical size: 2e-5 covers that several times.
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
F32_NOISE = 2e-5


def check(got, want, what):
    assert (got is None) == (want is None), what
    if got is None:
        return
    assert tuple(got.shape) == tuple(want.shape), what
    g, w = got.detach().cpu().double(), want.detach().double()
    if not g.numel():
        return
    rms = w.square().mean().sqrt()
    off = (g - w).abs()
    bound = 1.01 * ROUND[got.dtype] * w.abs() + F32_NOISE * torch.maximum(rms, w.abs()) + 2.0 ** -25
    assert torch.isfinite(g).all(), what
    worst = (off / bound).max().item()
    assert worst <= 1, f"{what}: {worst:.2f} times the bound, at {off.argmax().item()}"


class Inputs:
    """Random inputs on the GPU and their 64-bit copies on the CPU."""

    def __init__(self, seed, dtype):
        self.rng = torch.Generator().manual_seed(seed)
        self.dtype = dtype
        self.gpu, self.cpu = {}, {}

    def add(self, name, *shape, scale=1.0, dtype=None, lo=None, hi=None, shift=0.0):
        x = torch.randn(shape, generator=self.rng) * scale + shift
        if lo is not None:
            x = lo + (hi - lo) * torch.rand(shape, generator=self.rng)
        self.put(name, x.to(dtype or self.dtype))

    def put(self, name, x):
        self.gpu[name] = x.to(DEV)
        self.cpu[name] = x.double()

    def grads(self):
        for d in (self.gpu, self.cpu):
            for t in d.values():
                t.requires_grad_()

    def get(self, name):
        return self.gpu.get(name), self.cpu.get(name)


def compare_grads(x, outs, wants, seed=5):
    """Gradients of random weights of all outputs, kernels against reference."""
    rng = torch.Generator().manual_seed(seed)
    pairs = [(o, w) for o, w in zip(outs, wants) if o is not None and o.requires_grad]
    gs, ws = [], []
    for o, w in pairs:
        v = torch.randn(w.shape, generator=rng).to(o.dtype)
        gs.append(v.to(DEV))
        ws.append(v.double())
    names = list(x.gpu)
    got = torch.autograd.grad([o for o, _ in pairs], [x.gpu[n] for n in names], gs, allow_unused=True)
    want = torch.autograd.grad([w for _, w in pairs], [x.cpu[n] for n in names], ws, allow_unused=True)
    for n, g, w in zip(names, got, want):
        check(g, torch.zeros_like(x.cpu[n]) if w is None else w, "d" + n)


# ---------------------------------------------------------------- convolution

CONV = [  # dtype, batch, length, width, taps, state, bias, activation, lengths, param
    ("f32", 2, 37, 40, 4, True, True, "silu", None, "f32"),
    ("bf16", 3, 65, 264, 4, True, True, "silu", (65, 0, 2), "f32"),
    ("f16", 2, 130, 33, 3, False, True, "silu", (1, 130), "f16"),
    ("bf16", 1, 1, 8, 4, True, False, None, None, "bf16"),
    ("f32", 1, 5, 1, 8, True, True, "silu", (3,), "f32"),
    ("bf16", 2, 77, 513, 8, True, True, "silu", (77, 4), "bf16"),
    ("f16", 1, 9, 7, 1, False, True, "silu", None, "f32"),
    ("f32", 2, 40, 24, 2, True, True, None, (40, 39), "f32"),
    ("bf16", 2, 70, 72, 5, True, True, "silu", None, "f32"),
    ("f32", 1, 33, 16, 6, True, True, "silu", None, "f32"),
    ("f16", 2, 31, 20, 7, True, False, "silu", (31, 5), "f32"),
    ("bf16", 2, 2100, 16, 4, False, True, "silu", (2100, 1999), "f32"),
    ("f32", 3, 300, 36, 4, True, True, "silu", (300, 33, 100), "f32"),
    ("f16", 2, 260, 12, 8, True, True, "silu", (260, 7), "f16"),
    # the last load of a row moves back by one to seven channels
    ("bf16", 2, 35, 1031, 4, True, True, "silu", (35, 17), "f32"),
    ("f32", 2, 66, 521, 4, True, True, "silu", (66, 1), "f32"),
    ("f16", 1, 50, 9, 3, True, True, "silu", None, "f16"),
    ("bf16", 2, 40, 15, 4, True, True, None, None, "bf16"),
    ("bf16", 1, 40, 6, 2, True, True, "silu", None, "f32"),
    ("f32", 1, 12, 3, 4, True, True, "silu", (11,), "f32"),
]


def conv_inputs(dtype, batch, length, width, taps, state, bias, lengths, param, seed=1):
    x = Inputs(seed, DTYPES[dtype])
    x.add("x", batch, length, width)
    x.add("weight", width, taps, scale=0.5, dtype=DTYPES[param])
    if bias:
        x.add("bias", width, scale=0.3, dtype=DTYPES[param])
    if state:
        x.add("state", batch, taps - 1, width)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    return x, n


@pytest.mark.parametrize("case", CONV, ids=lambda c: "-".join(map(str, c[:5])))
def test_conv(case):
    dtype, batch, length, width, taps, state, bias, act, lengths, param = case
    x, n = conv_inputs(dtype, batch, length, width, taps, state, bias, lengths, param)
    if lengths is not None:                      # what lies past the ends is not a number
        with torch.no_grad():
            for i, e in enumerate(lengths):
                x.gpu["x"][i, e:] = float("nan")
                x.cpu["x"][i, e:] = 0
    x.grads()
    args = [x.gpu.get(k) for k in ("x", "weight", "bias")]
    outs = ops.causal_conv(*args, state=x.gpu.get("state"), lengths=n, activation=act,
                           return_state=True)
    wants = ref.causal_conv(x.cpu["x"], x.cpu["weight"], x.cpu.get("bias"), x.cpu.get("state"),
                            lengths, act)
    check(outs[0], wants[0], "y")
    check(outs[1], wants[1], "state")
    only = ops.causal_conv(*args, state=x.gpu.get("state"), lengths=n, activation=act)
    assert torch.equal(only, outs[0])
    with torch.no_grad():
        again = ops.causal_conv(*args, state=x.gpu.get("state"), lengths=n, activation=act)
    assert torch.equal(again, outs[0])
    compare_grads(x, outs, wants)


def test_conv_strides():
    """Rows of a wider tensor, a transposed one, misaligned starts."""
    wide = torch.randn(2, 30, 100, device=DEV)
    w = torch.randn(33, 4, device=DEV)
    for x in (wide[:, :, 3:36], wide.transpose(0, 1)[:, :, 1:34], wide.transpose(1, 2)[:, :33, :33].transpose(1, 2),
              wide[:, ::3, 5:38]):
        x = x[..., :33]
        if x.shape[-1] != 33:
            continue
        got = ops.causal_conv(x, w)
        check(got, ref.causal_conv(x.cpu().double(), w.cpu().double())[0], "y")


def test_conv_expanded_gradient():
    x = torch.randn(2, 9, 12, device=DEV, requires_grad=True)
    w = torch.randn(12, 4, device=DEV, requires_grad=True)
    got = torch.autograd.grad(ops.causal_conv(x, w).sum(), [x, w])
    xc, wc = x.detach().cpu().double().requires_grad_(), w.detach().cpu().double().requires_grad_()
    want = torch.autograd.grad(ref.causal_conv(xc, wc)[0].sum(), [xc, wc])
    check(got[0], want[0], "dx")
    check(got[1], want[1], "dw")


def test_conv_empty():
    w = torch.randn(8, 4, device=DEV, requires_grad=True)
    for shape in ((0, 5, 8), (2, 0, 8)):
        x = torch.randn(shape, device=DEV, requires_grad=True)
        y, s = ops.causal_conv(x, w, return_state=True)
        assert y.shape == x.shape and s.shape == (shape[0], 3, 8) and not s.any()
        dx, dw = torch.autograd.grad(y.sum(), [x, w])
        assert dx.shape == x.shape and not dw.any()


def test_conv_state_of_short_sequences():
    """Sequences shorter than the state, down to none: the state moves on by
    their tokens, and its gradient goes back through it."""
    x = Inputs(9, torch.float32)
    x.add("x", 4, 2, 8)
    x.add("weight", 8, 5)
    x.add("state", 4, 4, 8)
    x.grads()
    n = torch.tensor([0, 1, 2, 2], dtype=torch.int32, device=DEV)
    outs = ops.causal_conv(x.gpu["x"], x.gpu["weight"], state=x.gpu["state"], lengths=n, return_state=True)
    wants = ref.causal_conv(x.cpu["x"], x.cpu["weight"], None, x.cpu["state"], [0, 1, 2, 2])
    for o, w in zip(outs, wants):
        check(o, w, "output")
    compare_grads(x, outs, wants)
    empty = torch.zeros(4, 0, 8, device=DEV)
    s = x.gpu["state"]
    _, out = ops.causal_conv(empty, x.gpu["weight"], state=s, return_state=True)
    assert torch.equal(out, s)
    g, = torch.autograd.grad(out, s, torch.ones_like(out))
    assert torch.equal(g, torch.ones_like(g))


def test_lengths_outside_the_batch():
    """Lengths are clamped to [0, length]."""
    x = torch.randn(3, 20, 16, device=DEV)
    w, A = torch.randn(16, 4, device=DEV), -torch.rand(16, 4, device=DEV)
    bc = torch.randn(3, 20, 4, device=DEV)
    odd = torch.tensor([-5, 1000, 20], dtype=torch.int32, device=DEV)
    fair = torch.tensor([0, 20, 20], dtype=torch.int32, device=DEV)
    for f in (lambda n: ops.causal_conv(x, w, lengths=n, return_state=True),
              lambda n: ops.selective_scan(x, x, A, bc, bc, softplus=True, lengths=n, return_state=True)):
        for a, b in zip(f(odd), f(fair)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,batch,width,taps", [
    ("f32", 3, 10, 4), ("bf16", 5, 257, 4), ("f16", 1, 1, 2), ("bf16", 2, 64, 8), ("f32", 2, 6, 1)])
def test_conv_step(dtype, batch, width, taps):
    x, _ = conv_inputs(dtype, batch, 6, width, taps, True, True, None, "f32")
    pool = torch.randn(batch + 3, taps - 1, width, device=DEV).to(DTYPES[dtype])
    slots = torch.randperm(batch + 3, device=DEV)[:batch].to(torch.int32)
    pool[slots.long()] = x.gpu["state"]
    before = pool.clone()
    want = ref.causal_conv(x.cpu["x"], x.cpu["weight"], x.cpu["bias"], x.cpu["state"])
    for t in range(6):
        y = ops.causal_conv_step(pool, x.gpu["x"][:, t], x.gpu["weight"], x.gpu["bias"], slots=slots)
        check(y, want[0][:, t], f"y {t}")
    check(pool[slots.long()], want[1], "state")
    rest = torch.ones(batch + 3, dtype=torch.bool, device=DEV)
    rest[slots.long()] = False
    assert torch.equal(pool[rest], before[rest])


def test_conv_step_padding():
    pool = torch.randn(4, 3, 16, device=DEV)
    before = pool.clone()
    x = torch.full((3, 16), float("nan"), device=DEV)
    slots = torch.tensor([-1, 4, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    y = ops.causal_conv_step(pool, x, torch.randn(16, 4, device=DEV), slots=slots)
    assert not y.any() and torch.equal(pool, before)


# ----------------------------------------------------------------------- scan

SCAN = [  # dtype, batch, length, width, states, groups, parts, lengths
    ("f32", 2, 37, 10, 16, 1, "Dzbs", None),
    ("bf16", 2, 40, 70, 16, 1, "Dzbs", (40, 7)),
    ("f16", 3, 33, 12, 12, 2, "Dzbs", (33, 0, 17)),
    ("f32", 1, 1, 3, 1, 1, "Dzbs", None),
    ("f32", 2, 50, 6, 3, 3, "zb", (50, 49)),
    ("bf16", 1, 70, 65, 5, 1, "D", None),
    ("f32", 1, 35, 40, 8, 2, "s", (34,)),
    ("f16", 1, 64, 36, 17, 1, "Dzbs", None),
    ("f32", 2, 31, 20, 33, 1, "Dzb", (31, 16)),
    ("bf16", 1, 48, 24, 64, 2, "Dzbs", (47,)),
    ("f32", 1, 300, 5, 16, 1, "Dzbs", None),
    ("f32", 2, 600, 66, 16, 1, "Dzbs", (600, 333)),
    ("bf16", 1, 1030, 130, 4, 2, "Dzbs", None),
    # several chunks of the length, sequences that end inside, at and before one; every
    # number of states that changes the lanes; enough channels for one chunk
    ("f32", 3, 900, 68, 16, 1, "Dzbs", (900, 448, 130)),
    ("f16", 2, 500, 36, 40, 1, "Dzb", (500, 64)),
    ("bf16", 2, 400, 40, 24, 2, "Dzbs", (399, 0)),
    ("f32", 1, 260, 12, 2, 3, "zbs", (257,)),
    ("f32", 1, 210, 130, 7, 1, "Dzbs", None),
    ("bf16", 64, 33, 1024, 4, 1, "Dzb", None),
    ("bf16", 130, 20, 64, 64, 1, "Dz", None),
    # a last load of channels that moves back by one to three, each number of lanes
    ("f32", 2, 120, 71, 16, 1, "Dzbs", (120, 41)),
    ("bf16", 2, 75, 133, 10, 1, "Dzbs", (75, 0)),
    ("f16", 1, 50, 90, 16, 2, "Dzbs", None),
    ("f32", 2, 40, 78, 24, 1, "Dzbs", (40, 5)),
    ("bf16", 1, 70, 37, 40, 1, "Dzbs", (69,)),
    ("f32", 1, 40, 7, 3, 1, "Dzbs", None),
    # a workgroup for nearly every compute unit, several tiles
    ("bf16", 230, 100, 40, 16, 1, "Dzbs", None),
    ("f32", 120, 70, 70, 9, 1, "z", None),
]


def scan_inputs(dtype, batch, length, width, states, groups, parts, seed=2):
    x = Inputs(seed, DTYPES[dtype])
    x.add("u", batch, length, width)
    x.add("dt", batch, length, width, scale=0.5, shift=0.0 if "b" in parts else -2.0)
    x.add("A", width, states, dtype=torch.float32, lo=-states - 1.0, hi=-0.3)
    x.add("B", batch, length, groups, states)
    x.add("C", batch, length, groups, states)
    if "D" in parts:
        x.add("D", width, dtype=torch.float32)
    if "z" in parts:
        x.add("z", batch, length, width)
    if "b" in parts:
        x.add("dt_bias", width, dtype=torch.float32, lo=-6.0, hi=-2.0)
    if "s" in parts:
        x.add("state", batch, width, states, dtype=torch.float32)
    return x


def run_scan(x, lengths, n, return_state=True):
    kw = {k: x.gpu[k] for k in ("D", "z", "dt_bias", "state") if k in x.gpu}
    outs = ops.selective_scan(*(x.gpu[k] for k in ("u", "dt", "A", "B", "C")), **kw, softplus=True,
                              lengths=n, return_state=return_state)
    kw = {k: x.cpu[k] for k in ("D", "z", "dt_bias", "state") if k in x.cpu}
    return outs, ref.selective_scan(*(x.cpu[k] for k in ("u", "dt", "A", "B", "C")), **kw, soft=True,
                                    lengths=lengths)


@pytest.mark.parametrize("case", SCAN, ids=lambda c: "-".join(map(str, c[:7])))
def test_scan(case):
    dtype, batch, length, width, states, groups, parts, lengths = case
    x = scan_inputs(dtype, batch, length, width, states, groups, parts)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    if lengths is not None:
        with torch.no_grad():
            for name in ("u", "dt", "B", "C", "z"):
                for i, e in enumerate(lengths):
                    if name in x.gpu:
                        x.gpu[name][i, e:] = float("nan")
                        x.cpu[name][i, e:] = 0
    x.grads()
    outs, wants = run_scan(x, lengths, n)
    check(outs[0], wants[0], "y")
    check(outs[1], wants[1], "state")
    with torch.no_grad():
        again, _ = run_scan(x, lengths, n, return_state=False)
    check(again, wants[0], "y without gradients")
    compare_grads(x, outs, wants)


def test_scan_gradient_of_one_output():
    """Only y, or only the state, has a gradient."""
    x = scan_inputs("f32", 2, 21, 6, 8, 1, "Dzbs")
    x.grads()
    outs, wants = run_scan(x, None, None)
    for k in (0, 1):
        outs, wants = run_scan(x, None, None)
        o, w = outs[k], wants[k]
        v = torch.randn(w.shape).float()
        names = list(x.gpu)
        got = torch.autograd.grad(o, [x.gpu[m] for m in names], v.to(DEV), allow_unused=True)
        want = torch.autograd.grad(w, [x.cpu[m] for m in names], v.double(), allow_unused=True)
        for m, g, t in zip(names, got, want):
            check(g, torch.zeros_like(x.cpu[m]) if t is None else t, "d" + m)


def test_scan_raw_delta():
    """Without softplus, delta is dt + dt_bias as it stands, 0 included."""
    x = Inputs(4, torch.float32)
    x.add("u", 1, 30, 8)
    x.put("dt", torch.rand(1, 30, 8, generator=x.rng) * 0.2 * (torch.arange(30) % 3 > 0)[None, :, None])
    x.add("A", 8, 16, lo=-9.0, hi=-0.5)
    x.add("B", 1, 30, 1, 16)
    x.add("C", 1, 30, 1, 16)
    x.grads()
    got = ops.selective_scan(*(x.gpu[k] for k in ("u", "dt", "A", "B", "C")))
    want = ref.selective_scan(*(x.cpu[k] for k in ("u", "dt", "A", "B", "C")))[0]
    check(got, want, "y")
    compare_grads(x, [got], [want])


def test_scan_extreme_steps():
    """Steps from almost nothing to ones that forget the state at once."""
    x = Inputs(6, torch.float32)
    x.add("u", 1, 24, 8)
    x.put("dt", torch.linspace(-80, 80, 24)[None, :, None].expand(1, 24, 8).contiguous())
    x.add("A", 8, 4, lo=-9.0, hi=-0.5)
    x.add("B", 1, 24, 1, 4)
    x.add("C", 1, 24, 1, 4)
    x.grads()
    got = ops.selective_scan(*(x.gpu[k] for k in ("u", "dt", "A", "B", "C")), softplus=True)
    want = ref.selective_scan(*(x.cpu[k] for k in ("u", "dt", "A", "B", "C")), soft=True)[0]
    check(got, want, "y")
    compare_grads(x, [got], [want])


def test_scan_layouts():
    """Strided u, dt, z, B and C (slices of projections), and B, C without groups."""
    torch.manual_seed(0)
    b, n, d, s = 2, 45, 24, 16
    both = torch.randn(b, n, 2 * d, device=DEV)
    proj = torch.randn(b, n, 7 + 2 * s, device=DEV)
    dt = torch.randn(n, b, d, device=DEV).transpose(0, 1) * 0.3 - 2
    u, z = both[..., :d], both[..., d:]
    B, C = proj[..., 7:7 + s], proj[..., 7 + s:]
    A = -torch.rand(d, s, device=DEV) * 5 - 0.2
    got = ops.selective_scan(u, dt, A, B, C, z=z, softplus=True)
    c = [t.cpu().double() for t in (u, dt, A, B[:, :, None], C[:, :, None])]
    check(got, ref.selective_scan(*c, z=z.cpu().double(), soft=True)[0], "y")
    for t in (u, dt, B, C, z):
        t.requires_grad_() if t.is_leaf else None
    leaf = [t.detach().requires_grad_() for t in (u, dt, A, B, C, z)]
    cl = [t.detach().cpu().double().requires_grad_() for t in leaf]
    dy = torch.randn(b, n, d)
    gg = torch.autograd.grad(ops.selective_scan(*leaf[:5], z=leaf[5], softplus=True), leaf, dy.to(DEV))
    want = ref.selective_scan(*cl[:3], cl[3][:, :, None], cl[4][:, :, None], z=cl[5], soft=True)[0]
    for k, g, w in zip("u dt A B C z".split(), gg, torch.autograd.grad(want, cl, dy.double())):
        check(g, w, "d" + k)
    # the transposed layout is copied
    ut = u.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(ops.selective_scan(ut, dt, A, B, C, z=z, softplus=True), got)


def test_scan_empty():
    A = -torch.rand(8, 4, device=DEV)
    A.requires_grad_()
    for b, n in ((0, 5), (2, 0)):
        u = torch.randn(b, n, 8, device=DEV, requires_grad=True)
        bc = torch.randn(b, n, 4, device=DEV)
        h = torch.randn(b, 8, 4, device=DEV, requires_grad=True)
        y, out = ops.selective_scan(u, u.detach(), A, bc, bc, state=h, return_state=True)
        assert y.shape == u.shape and torch.equal(out, h)
        du, dA, dh = torch.autograd.grad([y, out], [u, A, h], [torch.zeros_like(y), torch.ones_like(out)])
        assert du.shape == u.shape and not dA.any() and torch.equal(dh, torch.ones_like(h))


@pytest.mark.parametrize("dtype,batch,width,states,groups", [
    ("f32", 3, 10, 16, 2), ("bf16", 5, 130, 16, 1), ("f16", 1, 3, 5, 1), ("bf16", 2, 65, 64, 1),
    ("f32", 2, 7, 1, 1), ("f32", 2, 24, 30, 3)])
def test_scan_step(dtype, batch, width, states, groups):
    x = scan_inputs(dtype, batch, 6, width, states, groups, "Dzbs")
    pool = torch.randn(batch + 3, width, states, device=DEV)
    slots = torch.randperm(batch + 3, device=DEV)[:batch].to(torch.int32)
    pool[slots.long()] = x.gpu["state"]
    before = pool.clone()
    _, want = run_scan(x, None, None)
    for t in range(6):
        y = ops.selective_scan_step(pool, *(x.gpu[k][:, t] for k in ("u", "dt")), x.gpu["A"],
                                    x.gpu["B"][:, t], x.gpu["C"][:, t], x.gpu["D"], x.gpu["z"][:, t],
                                    x.gpu["dt_bias"], softplus=True, slots=slots)
        check(y, want[0][:, t], f"y {t}")
    check(pool[slots.long()], want[1], "state")
    rest = torch.ones(batch + 3, dtype=torch.bool, device=DEV)
    rest[slots.long()] = False
    assert torch.equal(pool[rest], before[rest])


def test_scan_step_plain_parts():
    """No D, z, bias, softplus or slots; padding rows leave every state."""
    x = scan_inputs("f32", 3, 1, 9, 6, 1, "s")
    x.gpu["dt"].abs_()
    x.cpu["dt"].abs_()
    pool = x.gpu["state"].clone()
    y = ops.selective_scan_step(pool, x.gpu["u"][:, 0], x.gpu["dt"][:, 0], x.gpu["A"],
                                x.gpu["B"][:, 0, 0], x.gpu["C"][:, 0, 0])
    want = ref.selective_scan(*(x.cpu[k] for k in ("u", "dt", "A", "B", "C")), state=x.cpu["state"])
    check(y, want[0][:, 0], "y")
    check(pool, want[1], "state")
    before = pool.clone()
    slots = torch.tensor([-1, 3, -7], dtype=torch.int32, device=DEV)
    y = ops.selective_scan_step(pool, x.gpu["u"][:, 0], x.gpu["dt"][:, 0], x.gpu["A"],
                                x.gpu["B"][:, 0], x.gpu["C"][:, 0], slots=slots)
    assert not y.any() and torch.equal(pool, before)


# ---------------------------------------------------------------------- norms

NORM = [  # dtype, residual, rows, width, parts, gate activation, param
    ("f32", "f32", 5, 64, "bgpsn", "silu", "f32"),
    ("bf16", "f32", 9, 1001, "bgpsn", "silu", "f32"),
    ("bf16", "bf16", 33, 513, "bpsn", "silu", "bf16"),
    ("f16", "f32", 7, 7, "bgpsn", "sigmoid", "f32"),
    ("f16", "f16", 3, 2048, "bgn", "sigmoid", "f16"),
    ("bf16", "f32", 4, 4096, "bgps", "silu", "f32"),
    ("f32", "f32", 3, 4097, "bpn", "silu", "f32"),
    ("bf16", "bf16", 2, 16384, "bgpsn", "silu", "f32"),
    ("f32", "f32", 2, 9000, "bgpsn", "silu", "f32"),
    ("f32", "f32", 1, 1, "bgpsn", "silu", "f32"),
    ("bf16", "bf16", 6, 129, "n", "silu", "f32"),
    ("f32", "f32", 6, 700, "bg", "silu", "f32"),
    ("f32", "f32", 4, 300, "b", "silu", "f32"),
    ("bf16", "f32", 3001, 40, "bgpsn", "silu", "f32"),
    ("f16", "f16", 1400, 1030, "bpsn", "silu", "f32"),
    ("bf16", "f32", 40, 200, "bgpsn", "sigmoid", "f32"),
    ("bf16", "bf16", 300, 256, "bgpsn", "silu", "bf16"),
    ("bf16", "f32", 5, 5000, "bgpsn", "silu", "f32"),
    ("f32", "f32", 300, 8192, "bgpsn", "silu", "f32"),
    ("bf16", "f32", 3, 12345, "bgpsn", "silu", "f32"),
    # several rows a workgroup, the last load of a row moved back
    ("f32", "f32", 700, 1003, "bpsn", "silu", "f32"),
    ("bf16", "f32", 600, 4095, "bgpsn", "silu", "f32"),
    ("f16", "f16", 520, 5001, "bgps", "silu", "f16"),
    ("f32", "f32", 5000, 3, "bgpsn", "sigmoid", "f32"),
    ("bf16", "bf16", 800, 1000, "n", "silu", "f32"),
    ("f16", "f32", 550, 7001, "bgpsn", "silu", "f32"),
    ("f32", "f32", 9000, 9, "bg", "silu", "f32"),
]


def norm_inputs(dtype, residual, rows, width, parts, param, seed=3):
    x = Inputs(seed, DTYPES[dtype])
    if "b" in parts:
        x.add("block", rows, width)
    x.add("residual", rows, width, scale=2.0, dtype=DTYPES[residual])
    if "g" in parts:
        x.add("gate", rows, width)
    for k, name in (("p", "post"), ("s", "scale"), ("n", "pre")):
        if k in parts:
            x.add(name, width, dtype=DTYPES[param], lo=0.3, hi=1.5)
    return x


@pytest.mark.parametrize("case", NORM, ids=lambda c: "-".join(map(str, c[:5])))
def test_norm(case):
    dtype, residual, rows, width, parts, act, param = case
    x = norm_inputs(dtype, residual, rows, width, parts, param)
    if rows > 2 and "b" in parts:
        with torch.no_grad():                              # a row of nothing
            x.gpu["block"][1] = 0
            x.cpu["block"][1] = 0
    x.grads()
    keys = ("block", "residual", "gate", "post", "scale", "pre")
    outs = ops.norm_residual(*(x.gpu.get(k) for k in keys), gate_activation=act)
    wants = ref.norm_residual(*(x.cpu.get(k) for k in keys), act=act)
    check(outs[0], wants[0], "out")
    check(outs[1], wants[1], "normed")
    with torch.no_grad():
        again = ops.norm_residual(*(x.gpu.get(k) for k in keys), gate_activation=act)
    for a, o in zip(again, outs):
        assert (a is None and o is None) or torch.equal(a, o)
    if "b" not in parts:
        outs, wants = outs[1:], wants[1:]
    compare_grads(x, outs, wants)


def test_norm_one_gradient():
    """Only one of the two outputs is used."""
    keys = ("block", "residual", "gate", "post", "scale", "pre")
    for k in (0, 1):
        x = norm_inputs("f32", "f32", 5, 90, "bgpsn", "f32")
        x.grads()
        o = ops.norm_residual(*(x.gpu[m] for m in keys))[k]
        w = ref.norm_residual(*(x.cpu[m] for m in keys))[k]
        compare_grads(x, [o], [w])


def test_norm_shapes_and_strides():
    torch.manual_seed(1)
    x = torch.randn(2, 3, 4, 100, device=DEV)
    r = torch.randn(4, 3, 2, 100, device=DEV).transpose(0, 2)
    w = torch.rand(98, device=DEV)
    out, normed = ops.norm_residual(x[..., 1:99], r[..., 2:], pre_weight=w, post_weight=w)
    want = ref.norm_residual(x[..., 1:99].cpu().double(), r[..., 2:].cpu().double(), post=w.cpu().double(),
                             pre=w.cpu().double())
    check(out, want[0], "out")
    check(normed, want[1], "normed")
    empty, _ = ops.norm_residual(x[:0], r[:0])
    assert empty.shape == (0, 3, 4, 100)
    p = torch.rand(100, device=DEV, requires_grad=True)
    _, n = ops.norm_residual(None, x[:0], pre_weight=p)
    assert not torch.autograd.grad(n.sum(), p)[0].any()


def test_norm_not_finite():
    """A row with an infinity or a NaN spoils that row alone."""
    x, r = torch.randn(6, 300, device=DEV), torch.randn(6, 300, device=DEV)
    w = torch.rand(300, device=DEV)
    good = ops.norm_residual(x, r, post_weight=w, pre_weight=w)
    x[2, 5], r[4, 7] = float("inf"), float("nan")
    bad = ops.norm_residual(x, r, post_weight=w, pre_weight=w)
    keep = torch.tensor([0, 1, 3, 5], device=DEV)
    for g, b in zip(good, bad):
        assert torch.equal(g[keep], b[keep]) and not torch.isfinite(b[4, 7])


# -------------------------------------------------------------- all operators


def _directional(f, xs, vs, eps):
    with torch.no_grad():
        hi = f([x + eps * v for x, v in zip(xs, vs)])
        lo = f([x - eps * v for x, v in zip(xs, vs)])
    return ((hi - lo) / (2 * eps)).item()


@pytest.mark.parametrize("op", ["conv", "scan", "norm"])
def test_gradient_against_differences(op):
    """<gradient, v> against (f(x + e v) - f(x - e v)) / 2e, all in 32 bits: the
    difference is off by e^2 f''' / 6 (e = 2^-7: about 1e-5 of f''') and by the rounding of
    f over 2e (2^-24 64 |f|): 1 % of the gradient's size covers both."""
    torch.manual_seed(8)
    if op == "conv":
        x, _ = conv_inputs("f32", 2, 20, 12, 4, True, True, None, "f32")
        names = ["x", "weight", "bias", "state"]
        f = lambda v: ops.causal_conv(*v[:3], state=v[3])  # noqa: E731
        shape = (2, 20, 12)
    elif op == "scan":
        x = scan_inputs("f32", 2, 40, 6, 5, 1, "Dzbs")
        names = ["u", "dt", "A", "B", "C", "D", "z", "dt_bias", "state"]
        f = lambda v: ops.selective_scan(*v[:8], softplus=True, state=v[8])  # noqa: E731
        shape = (2, 40, 6)
    else:
        x = norm_inputs("f32", "f32", 6, 70, "bgpsn", "f32")
        names = ["block", "residual", "gate", "post", "scale", "pre"]
        f = lambda v: torch.cat(ops.norm_residual(*v))  # noqa: E731
        shape = (12, 70)
    weight = torch.randn(shape, device=DEV)
    total = lambda v: (f(v).double() * weight).sum()  # noqa: E731
    xs = [x.gpu[n].requires_grad_() for n in names]
    grads = torch.autograd.grad(total(xs), xs)
    for i, (n, g) in enumerate(zip(names, grads)):
        v = [torch.randn_like(t) if j == i else torch.zeros_like(t) for j, t in enumerate(xs)]
        d = _directional(total, [t.detach() for t in xs], v, 2.0 ** -7)
        want = (g.double() * v[i]).sum().item()
        assert abs(d - want) <= 0.01 * g.double().norm().item() + 1e-3, (n, d, want)


def _training_step():
    torch.manual_seed(11)
    b, n, d, s = 2, 70, 64, 16
    p = {"x": torch.randn(b, n, d, device=DEV, dtype=torch.bfloat16),
         "w": torch.randn(d, 4, device=DEV), "dt": torch.randn(b, n, d, device=DEV, dtype=torch.bfloat16),
         "A": -torch.rand(d, s, device=DEV) * 8 - 0.3,
         "B": torch.randn(b, n, s, device=DEV, dtype=torch.bfloat16),
         "C": torch.randn(b, n, s, device=DEV, dtype=torch.bfloat16),
         "r": torch.randn(b, n, d, device=DEV), "pw": torch.rand(d, device=DEV)}
    for t in p.values():
        t.requires_grad_()

    def run():
        u = ops.causal_conv(p["x"], p["w"])
        y = ops.selective_scan(u, p["dt"], p["A"], p["B"], p["C"], softplus=True)
        out, normed = ops.norm_residual(y, p["r"], post_weight=p["pw"], pre_weight=p["pw"])
        grads = torch.autograd.grad([out, normed], list(p.values()),
                                    [torch.ones_like(out), torch.ones_like(normed)])
        return [out.detach(), normed.detach(), *grads]
    return p, run


def test_other_stream_and_repeats():
    """The same bits on another stream and in every repeat."""
    _, run = _training_step()
    first = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = run()
    torch.cuda.current_stream().wait_stream(s)
    for a, b, c in zip(first, other, run()):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_graph_replays():
    """A captured forward and backward pass, and captured single tokens, give
    the eager results at every replay, with other work between them."""
    p, run = _training_step()
    pool = torch.randn(5, 64, 16, device=DEV)
    conv = torch.randn(5, 3, 64, device=DEV, dtype=torch.bfloat16)
    slots = torch.tensor([3, -1, 0], dtype=torch.int32, device=DEV)
    tok = torch.randn(3, 64, device=DEV, dtype=torch.bfloat16)
    bc = torch.randn(3, 16, device=DEV, dtype=torch.bfloat16)
    A, w = p["A"].detach(), p["w"].detach()

    def step():
        u = ops.causal_conv_step(conv, tok, w, slots=slots)
        return ops.selective_scan_step(pool, u, tok, A, bc, bc, softplus=True, slots=slots)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(), step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
        y = step()
    for k in range(4):
        with torch.no_grad():
            for t in p.values():
                t.mul_(1.0 + 0.01 * k)
            tok.copy_(torch.randn(3, 64, device=DEV))
        state = pool.clone(), conv.clone()
        want, wy = run(), step()
        after = pool.clone(), conv.clone()
        pool.copy_(state[0]), conv.copy_(state[1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), k
        assert torch.equal(y, wy) and torch.equal(pool, after[0]) and torch.equal(conv, after[1])


def test_far_offsets():
    """Rows whose offsets pass 2^31 elements: a strided view of a large buffer."""
    d, step = 32, 2 ** 30 // 16
    big = torch.zeros(2 ** 30 // 16 * 40 + d, dtype=torch.bfloat16, device=DEV)
    rows = torch.randn(40, d).to(torch.bfloat16)
    x = big.as_strided((1, 40, d), (0, step, 1))
    x.copy_(rows.to(DEV)[None])
    w = torch.randn(d, 4)
    check(ops.causal_conv(x, w.to(DEV)), ref.causal_conv(rows.double()[None], w.double())[0], "y")
    A = -torch.rand(d, 4) - 0.1
    got = ops.selective_scan(x, x, A.to(DEV), x[..., :4], x[..., 4:8], softplus=True)
    r = rows.double()[None]
    want = ref.selective_scan(r, r, A.double(), r[:, :, None, :4], r[:, :, None, 4:8], soft=True)[0]
    check(got, want, "scan")
    pw = torch.rand(d)
    _, n = ops.norm_residual(None, x[0], pre_weight=pw.to(DEV))
    check(n, ref.norm_residual(None, rows.double(), pre=pw.double())[1], "normed")


# ------------------------------------------------------------------- refusals


def test_refusals():
    x = torch.randn(2, 5, 8, device=DEV)
    w = torch.randn(8, 4, device=DEV)
    A, bc = -torch.rand(8, 4, device=DEV), torch.randn(2, 5, 4, device=DEV)
    n = torch.tensor([5, 2], dtype=torch.int32, device=DEV)
    bad = [
        lambda: ops.causal_conv(x.cpu(), w),
        lambda: ops.causal_conv(x.double(), w),
        lambda: ops.causal_conv(x[0], w),
        lambda: ops.causal_conv(x, w.cpu()),
        lambda: ops.causal_conv(x, w[:4]),
        lambda: ops.causal_conv(x, torch.randn(8, 9, device=DEV)),
        lambda: ops.causal_conv(x, w.half()),
        lambda: ops.causal_conv(x, w, w[:, 0].half()),
        lambda: ops.causal_conv(x, w, activation="relu"),
        lambda: ops.causal_conv(x, w, lengths=n.long()),
        lambda: ops.causal_conv(x, w, lengths=n[:1]),
        lambda: ops.causal_conv(x, w, state=torch.randn(2, 4, 8, device=DEV)),
        lambda: ops.causal_conv_step(torch.randn(1, 3, 8, device=DEV), x[:, 0], w),
        lambda: ops.causal_conv_step(torch.randn(2, 3, 8, device=DEV).half(), x[:, 0], w),
        lambda: ops.causal_conv_step(torch.randn(2, 8, 3, device=DEV).transpose(1, 2), x[:, 0], w),
        lambda: ops.selective_scan(x, x[:, :4], A, bc, bc),
        lambda: ops.selective_scan(x, x.half(), A, bc, bc),
        lambda: ops.selective_scan(x, x, A.half(), bc, bc),
        lambda: ops.selective_scan(x, x, -torch.rand(8, 65, device=DEV), bc, bc),
        lambda: ops.selective_scan(x, x, A, bc[:, :, None].expand(-1, -1, 3, -1), bc),
        lambda: ops.selective_scan(x, x, A, bc, bc[..., :3]),
        lambda: ops.selective_scan(x, x, A, bc, bc, state=torch.randn(2, 4, 8, device=DEV)),
        lambda: ops.selective_scan_step(torch.randn(1, 8, 4, device=DEV), x[:, 0], x[:, 0], A, bc[:, 0], bc[:, 0]),
        lambda: ops.selective_scan_step(torch.randn(2, 4, 8, device=DEV).transpose(1, 2), x[:, 0], x[:, 0], A,
                                        bc[:, 0], bc[:, 0]),
        lambda: ops.norm_residual(x, x[:1]),
        lambda: ops.norm_residual(x.half(), x.bfloat16()),
        lambda: ops.norm_residual(None, x),
        lambda: ops.norm_residual(None, x, gate=x, pre_weight=w[:, 0]),
        lambda: ops.norm_residual(x, x, post_weight=torch.rand(7, device=DEV)),
        lambda: ops.norm_residual(x, x, gate_activation="tanh"),
        lambda: ops.norm_residual(torch.randn(1, 16385, device=DEV), torch.randn(1, 16385, device=DEV)),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    torch.cuda.synchronize()


def test_twice_differentiated_is_refused():
    x = torch.randn(1, 6, 8, device=DEV, requires_grad=True)
    w = torch.randn(8, 4, device=DEV, requires_grad=True)
    g, = torch.autograd.grad(ops.causal_conv(x, w).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), w)
