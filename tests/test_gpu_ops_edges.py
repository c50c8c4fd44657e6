"""The sequence-model operators off the usual ground: states that autograd
has saved, derivatives that do not exist, pools that share memory or are too
large, views that negate, no channels, scratch aligned to a float only, values
that are not finite beside masked ones, and the walks that only large inputs take."""

import ctypes

import pytest
import torch
from torch.autograd import forward_ad

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1905_11722_amd import ops  # noqa: E402
from tests import ops_abi as abi  # noqa: E402
from tests import ops_reference as ref  # noqa: E402
from tests.test_gpu_ops import (F32_NOISE, ROUND, check, compare_grads, run_scan,  # noqa: E402
                                scan_inputs)

DEV = torch.device("cuda", 0)


def close(got, want, what):
    """The bound of tests/test_gpu_ops.py, which says where it comes from, on the GPU."""
    assert got.shape == want.shape, what
    w = want.detach()
    rms = w.square().mean().sqrt()
    bound = 1.01 * ROUND[got.dtype] * w.abs() + F32_NOISE * torch.maximum(rms, w.abs()) + 2.0 ** -25
    worst = ((got.detach().double() - w).abs() / bound).max().item()
    assert worst <= 1, f"{what}: {worst:.2f} times the bound"          # (and no NaN)


def token(op, pool, slots=None):
    """One token through a step form on a pool of states; its y."""
    x = torch.randn(2, 8, device=DEV)
    if op == "conv":
        return ops.causal_conv_step(pool, x, torch.randn(8, 4, device=DEV), slots=slots)
    bc = torch.randn(2, 4, device=DEV)
    return ops.selective_scan_step(pool, x, x, -torch.rand(8, 4, device=DEV), bc, bc, softplus=True,
                                   slots=slots)


def pool_of(op, slots=2):
    return torch.randn((slots, 3, 8) if op == "conv" else (slots, 8, 4), device=DEV)


@pytest.mark.parametrize("op", ["conv", "scan"])
def test_a_step_on_a_saved_state_is_seen(op):
    """A token that overwrites a state that a backward pass still needs makes
    that pass raise, as torch's own operators in place do."""
    pool = pool_of(op)
    version = pool._version
    x = torch.randn(2, 6, 8, device=DEV, requires_grad=True)
    if op == "conv":
        y = ops.causal_conv(x, torch.randn(8, 4, device=DEV), state=pool)
    else:
        bc = torch.randn(2, 6, 4, device=DEV)
        y = ops.selective_scan(x, x, -torch.rand(8, 4, device=DEV), bc, bc, softplus=True, state=pool)
    token(op, pool)
    assert pool._version > version
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    with torch.inference_mode():
        token(op, pool_of(op))                       # tensors without versions


def test_steps_have_no_gradients():
    """With gradients recorded, a token form refuses any input that requires one."""
    def leaf(*shape):
        return torch.rand(shape, device=DEV)

    conv = {"state": leaf(2, 3, 8), "x": leaf(2, 8), "weight": leaf(8, 4), "bias": leaf(8)}
    scan = {"state": leaf(2, 8, 4), "u": leaf(2, 8), "dt": leaf(2, 8), "A": -leaf(8, 4), "B": leaf(2, 4),
            "C": leaf(2, 4), "D": leaf(8), "z": leaf(2, 8), "dt_bias": leaf(8)}
    for f, args in ((ops.causal_conv_step, conv), (ops.selective_scan_step, scan)):
        for name in args:
            args[name].requires_grad_()
            before = args["state"].detach().clone()
            with pytest.raises(ValueError, match="no gradients"):
                f(**args)
            assert torch.equal(args["state"].detach(), before)
            with torch.no_grad():
                assert not f(**args).requires_grad
            args[name].requires_grad_(False)
        assert not f(**args).requires_grad


def test_forward_mode_is_refused():
    """A tangent of any input raises, with gradients recorded or not, rather than being dropped."""
    x, w, A = torch.randn(2, 5, 8, device=DEV), torch.randn(8, 4, device=DEV), -torch.rand(8, 4, device=DEV)
    bc, v = torch.randn(2, 5, 4, device=DEV), torch.rand(8, device=DEV)
    pool, h = pool_of("conv"), pool_of("scan")
    calls = [
        (lambda *a: ops.causal_conv(*a[:3], state=a[3]), [x, w, v, pool]),
        (lambda *a: ops.selective_scan(*a[:8], state=a[8]), [x, x, A, bc, bc, v, x, v, h]),
        (lambda *a: ops.norm_residual(*a)[0], [x, x, x, v, v, v]),
        (ops.causal_conv_step, [pool, x[:, 0], w, v]),
        (ops.selective_scan_step, [h, x[:, 0], x[:, 0], A, bc[:, 0], bc[:, 0], v, x[:, 0], v]),
    ]
    for f, args in calls:
        for i in range(len(args)):
            with forward_ad.dual_level():
                dual = list(args)
                dual[i] = forward_ad.make_dual(args[i], torch.ones_like(args[i]))
                with pytest.raises(NotImplementedError, match="forward-mode"):
                    f(*dual)
                with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
                    f(*dual)
        with forward_ad.dual_level():
            f(*args)
    for f, args in calls[:3]:
        y = f(args[0].requires_grad_(), *args[1:])
        y = y if isinstance(y, torch.Tensor) else y[0]
        with forward_ad.dual_level():
            dy = forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y))
            with pytest.raises(NotImplementedError, match="forward-mode"):
                torch.autograd.grad(y, args[0], dy)
        args[0].requires_grad_(False)


def test_pools_that_share_memory():
    """A pool whose states overlap is refused; strides that only interleave them are not."""
    flat = torch.randn(4096, device=DEV)
    conv = [(1, 0, 8), (2, 24, 0), (2, 7, 100), (2, 100, 7), (3, 20, 8), (40, 9, 50), (2, 23, 8), (1, 0, 7)]
    for slots, slot, row in conv:
        pool = flat.as_strided((slots, 3, 8), (slot, row, 1))
        at = [i * slot + k * row + c for i in range(slots) for k in range(3) for c in range(8)]
        n = torch.zeros(2, dtype=torch.int32, device=DEV) - 1          # no state is touched
        if len(set(at)) < len(at):
            with pytest.raises(ValueError, match="share memory"):
                token("conv", pool, n)
        else:
            token("conv", pool, n)
    for slots, slot in ((2, 0), (3, 31), (3, 32), (1, 0)):
        pool = flat.as_strided((slots, 8, 4), (slot, 4, 1))
        if slots > 1 and slot < 32:
            with pytest.raises(ValueError, match="share memory"):
                token("scan", pool, n)
        else:
            token("scan", pool, n)
    pool, other = flat.as_strided((4, 3, 8), (8, 32, 1)), flat.clone()   # slots between rows
    x, w = torch.randn(2, 8, device=DEV), torch.randn(8, 4, device=DEV)
    n = torch.tensor([3, 1], dtype=torch.int32, device=DEV)
    dense = pool.contiguous()
    assert torch.equal(ops.causal_conv_step(pool, x, w, slots=n), ops.causal_conv_step(dense, x, w, slots=n))
    assert torch.equal(pool, dense) and torch.equal(flat[96:], other[96:])


def test_pools_of_more_slots_than_an_index_reaches():
    """2^32 + 2 slots without rows (one tap): not taken for 2 of them."""
    pool = torch.empty(2 ** 32 + 2, 0, 8, device=DEV)
    x, w = torch.randn(2, 8, device=DEV), torch.randn(8, 1, device=DEV)
    for n in (torch.tensor([0, 5], dtype=torch.int32, device=DEV), None):
        with pytest.raises(ValueError, match="too many slots"):
            ops.causal_conv_step(pool, x, w, slots=n)


def test_views_that_negate():
    """Lazily negated views (the imaginary part of a conjugate) are taken at
    their values; a pool that is one is refused."""
    neg = torch._neg_view
    x, w, v = torch.randn(2, 5, 8, device=DEV), torch.randn(8, 4, device=DEV), torch.rand(8, device=DEV)
    A, bc, h = -torch.rand(8, 4, device=DEV), torch.randn(2, 5, 4, device=DEV), torch.randn(2, 8, 4, device=DEV)
    pool = torch.randn(2, 3, 8, device=DEV)
    calls = [
        (lambda *a: ops.causal_conv(*a[:3], state=a[3]), [x, w, v, pool]),
        (lambda *a: ops.selective_scan(*a[:8], state=a[8]), [x, x, A, bc, bc, v, x, v, h]),
        (lambda *a: torch.cat(ops.norm_residual(*a)), [x, x, x, v, v, v]),
        (lambda *a: ops.causal_conv_step(pool.clone(), *a), [x[:, 0], w, v]),
        (lambda *a: ops.selective_scan_step(h.clone(), *a), [x[:, 0], x[:, 0], A, bc[:, 0], bc[:, 0], v, x[:, 0], v]),
    ]
    for f, args in calls:
        want = f(*args)
        for i in range(len(args)):
            view = neg(args[i].neg())
            assert view.is_neg()
            assert torch.equal(f(*args[:i], view, *args[i + 1:]), want)
    lazy = neg(pool.neg())
    for op, p in (("conv", lazy), ("scan", neg(h.neg()))):
        with pytest.raises(ValueError, match="negates"):
            token(op, p)
    xs = x.clone().requires_grad_()
    want, = torch.autograd.grad(ops.causal_conv(xs, w), xs, x)
    got, = torch.autograd.grad(ops.causal_conv(xs, w), xs, neg(x.neg()))
    assert torch.equal(got, want)


@pytest.mark.parametrize("groups", [0, 2])
def test_scan_without_channels(groups):
    """No channels: nothing depends on B and C, whose gradients are zeros (not what
    their memory held)."""
    b, n, s = 3, 40, 5
    shape = (b, n, groups, s) if groups else (b, n, s)
    u = torch.zeros(b, n, 0, device=DEV, requires_grad=True)
    B, C = (torch.randn(shape, device=DEV, requires_grad=True) for _ in range(2))
    A = torch.zeros(0, s, device=DEV, requires_grad=True)
    h = torch.zeros(b, 0, s, device=DEV, requires_grad=True)
    y, out = ops.selective_scan(u, u, A, B, C, softplus=True, state=h, return_state=True)
    assert y.shape == u.shape and out.shape == h.shape
    old = [torch.full(shape, float("nan"), device=DEV) for _ in range(8)]
    del old
    grads = torch.autograd.grad([y, out], [B, C, u, A, h], [torch.ones_like(y), torch.ones_like(out)])
    for g, t in zip(grads, (B, C, u, A, h)):
        assert g.shape == t.shape and not g.any()
    for shape in ((0, 4, 0), (2, 0, 0)):
        u = torch.zeros(shape, device=DEV, requires_grad=True)
        B = torch.zeros(*shape[:2], s, device=DEV, requires_grad=True)
        g, = torch.autograd.grad(ops.selective_scan(u, u, A, B, B).sum(), B)
        assert g.shape == B.shape


@pytest.mark.parametrize("states,width", [(16, 70), (5, 64), (33, 33)])
def test_scratch_aligned_to_a_float(states, width):
    """Kept states and scratch 4, 8 and 12 bytes past an aligned address give the aligned ones' bits."""
    torch.manual_seed(4)
    b, n = 2, 300
    lib = abi.library()
    u, dt, z, dy = (torch.randn(b, n, width, device=DEV) for _ in range(4))
    B, C = torch.randn(b, n, states, device=DEV), torch.randn(b, n, states, device=DEV)
    A = -torch.rand(width, states, device=DEV)

    def view(t):
        return abi.View(t.data_ptr(), t.stride(0), t.stride(1))

    def floats(count, off):
        """(its memory, the address of `count` floats `off` floats past an aligned one)"""
        t = torch.zeros(count + 8, device=DEV)
        assert t.data_ptr() % 16 == 0
        return t, t.data_ptr() + 4 * off

    def run(off):
        out = [torch.full_like(t, 7) for t in (u, u, u, u, B, C, A)]
        y, du, ddt, dz, dB, dC, dA = out
        a = abi.ScanArgs(dtype=0, softplus=1, batch=b, length=n, width=width, states=states, groups=1, u=view(u),
                         dt=view(dt), z=view(z), B=view(B), C=view(C), y=view(y), A=A.data_ptr(), dy=view(dy),
                         du=view(du), ddt=view(ddt), dz=view(dz), dB=dB.data_ptr(), dC=dC.data_ptr(), dA=dA.data_ptr())
        size = ctypes.c_uint64()
        assert lib.rc_scan_kept_bytes(a, size) == 0
        kept, a.kept = floats(size.value // 4, off)
        stream = torch.cuda.current_stream().cuda_stream
        for call in ("forward", "backward"):
            assert getattr(lib, f"rc_scan_{call}_workspace")(a, size) == 0
            work, a.workspace = floats(size.value // 4 + 1, off)
            a.workspace_bytes = size.value
            assert getattr(lib, "rc_scan_" + call)(a, stream) == 0
        torch.cuda.synchronize()
        return out

    want = run(0)
    for off in (1, 2, 3):
        for g, w in zip(run(off), want):
            assert torch.equal(g, w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("taps", [1, 4, 8])
def test_conv_gradients_past_an_end(dtype, bad, taps):
    """A token that is not finite just before an end: the gradients past it are 0 all the same,
    and the other sequences' are what they were."""
    torch.manual_seed(2)
    x = torch.randn(3, 90, 24, device=DEV).to(dtype)
    w, s = torch.randn(24, taps, device=DEV), torch.randn(3, taps - 1, 24, device=DEV).to(dtype)
    n = torch.tensor([90, 41, 0], dtype=torch.int32, device=DEV)
    dy = torch.randn(3, 90, 24, device=DEV).to(dtype)

    def grads():
        leaf = [x.clone().requires_grad_(), s.clone().requires_grad_()]
        y, end = ops.causal_conv(leaf[0], w, state=leaf[1], lengths=n, return_state=True)
        return torch.autograd.grad([y, end], leaf, [dy, torch.ones_like(end)])

    good = grads()
    x[1, 40], s[2] = bad, bad
    got = grads()
    assert torch.equal(got[0][0], good[0][0]) and torch.equal(got[1][0], good[1][0])
    assert not got[0][1, 41:].any() and not got[0][2].any()
    assert torch.equal(got[1][2], torch.ones_like(got[1][2]))      # an empty sequence hands it on


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("states", [4, 16, 33])
def test_scan_gradients_past_an_end(dtype, bad, states):
    torch.manual_seed(3)
    d = 24
    u, dt, z, dy = (torch.randn(3, 90, d, device=DEV).to(dtype) for _ in range(4))
    B, C = (torch.randn(3, 90, states, device=DEV).to(dtype) for _ in range(2))
    A = -torch.rand(d, states, device=DEV)
    n = torch.tensor([90, 41, 0], dtype=torch.int32, device=DEV)

    def grads():
        leaf = [t.clone().requires_grad_() for t in (u, dt, B, C, z)]
        y = ops.selective_scan(leaf[0], leaf[1], A, leaf[2], leaf[3], z=leaf[4], softplus=True, lengths=n)
        return y, torch.autograd.grad(y, leaf, dy)

    _, good = grads()
    u[1, 40] = bad
    y, got = grads()
    assert not y[1, 41:].any() and not y[2].any()
    for name, a, b in zip("u dt B C z".split(), good, got):
        assert torch.equal(a[0], b[0]), name
        assert not b[1, 41:].any() and not b[2].any(), name


def conv_definition(x, w, bias, state, n):
    """y and the final state in 64 bits on the GPU; tokens past the ends are zeros in x."""
    taps, length = w.shape[1], x.shape[1]
    seen = torch.cat([state, x], 1)
    p = bias + sum(w[:, k] * seen[:, k:k + length] for k in range(taps))
    live = torch.arange(length, device=DEV)[None, :, None] < n[:, None, None]
    at = (n[:, None] + torch.arange(taps - 1, device=DEV)).long()[:, :, None].expand(-1, -1, x.shape[2])
    return torch.where(live, p * torch.sigmoid(p), 0.0), torch.gather(seen, 1, at)


@pytest.mark.parametrize("dtype,taps", [(torch.float32, k) for k in range(1, 9)]
                         + [(torch.bfloat16, 4), (torch.bfloat16, 5), (torch.float16, 8)])
def test_conv_long_walks(dtype, taps):
    """Enough rows that a thread walks over 16 forward and 32 backward, in groups that are loaded
    ahead (256 compute units); an odd width, sequences that end inside a walk, one without a token."""
    rng = torch.Generator(device=DEV).manual_seed(taps)
    b, length, d = 9, 2047, 2051

    def normal(*shape, t=dtype):
        return torch.randn(shape, generator=rng, device=DEV).to(t)

    n = torch.tensor([2047, 0, 1, 1023, 2046, 1500, 40, 2047, 7], dtype=torch.int32, device=DEV)
    dead = torch.arange(length, device=DEV)[None, :, None] >= n[:, None, None]
    x, dy, state = normal(b, length, d).masked_fill(dead, float("nan")), normal(b, length, d), normal(b, taps - 1, d)
    w, bias = normal(d, taps, t=torch.float32) * 0.5, normal(d, t=torch.float32) * 0.3
    dend = normal(b, taps - 1, d)
    leaf = [t.requires_grad_() for t in (x, w, bias, state)]
    y, end = ops.causal_conv(x, w, bias, state=state, lengths=n, return_state=True)
    got = torch.autograd.grad([y, end], leaf, [dy, dend])
    wide = [t.detach().double().masked_fill(dead, 0.0) if t is x else t.detach().double() for t in leaf]
    wide = [t.requires_grad_() for t in wide]
    wy, wend = conv_definition(*wide, n)
    want = torch.autograd.grad([wy, wend], wide, [dy.double(), dend.double()])
    close(y, wy, "y")
    if taps > 1:
        close(end, wend, "state")
    for name, g, v in zip(("dx", "dweight", "dbias", "dstate"), got, want):
        if g.numel():
            close(g, v, name)


@pytest.mark.parametrize("batch,length,width,states,groups", [
    (3, 300, 20, 16, 1), (3, 90, 70, 4, 1), (2, 150, 6, 8, 2), (2, 130, 36, 24, 1), (2, 100, 21, 40, 1),
    (260, 40, 40, 16, 1)])
def test_scan_without_a_gate(batch, length, width, states, groups):
    """No z, in 32 bits: one chunk and several, sequences that end inside a tile or have no token."""
    x = scan_inputs("f32", batch, length, width, states, groups, "Dbs")
    ends = [length, length - 23, 0][:batch] + [length] * (batch - 3)
    n = torch.tensor(ends, dtype=torch.int32, device=DEV)
    with torch.no_grad():
        for name in ("u", "dt", "B", "C"):
            for i, e in enumerate(ends):
                x.gpu[name][i, e:] = float("nan")
                x.cpu[name][i, e:] = 0
    x.grads()
    outs, wants = run_scan(x, ends, n)
    check(outs[0], wants[0], "y")
    check(outs[1], wants[1], "state")
    compare_grads(x, outs, wants)


@pytest.mark.parametrize("dtype,wide,width,gate", [
    (torch.bfloat16, True, 9001, True), (torch.float16, False, 9001, False), (torch.float32, True, 16384, True),
    (torch.bfloat16, False, 12288, True)])
def test_norm_long_walks(dtype, wide, width, gate):
    """Above 8192 channels with more rows than twice the compute units, so that each workgroup adds
    several rows' weight gradients, those in LDS among them, and the first of the rows to the last."""
    rng = torch.Generator(device=DEV).manual_seed(7)
    rows, rt = 1100, torch.float32 if wide else dtype

    def normal(*shape, t=dtype, scale=1.0):
        return (torch.randn(shape, generator=rng, device=DEV) * scale).to(t)

    def weight():
        return torch.rand(width, generator=rng, device=DEV) + 0.3

    args = [normal(rows, width), normal(rows, width, t=rt, scale=2.0), normal(rows, width) if gate else None,
            weight(), weight(), weight()]
    dout, dnormed = normal(rows, width, t=rt), normal(rows, width)
    args[0][5] = 0
    leaf = [t.requires_grad_() if t is not None else None for t in args]
    got = ops.norm_residual(*leaf)
    grads = torch.autograd.grad(got, [t for t in leaf if t is not None], [dout, dnormed])
    far = [t.detach().double().requires_grad_() if t is not None else None for t in leaf]
    want = ref.norm_residual(*far)
    wants = torch.autograd.grad(want, [t for t in far if t is not None], [dout.double(), dnormed.double()])
    names = [k for k, t in zip(("block", "residual", "gate", "post", "scale", "pre"), leaf) if t is not None]
    for k, g, w in zip(("out", "normed"), got, want):
        close(g, w, k)
    for k, g, w in zip(names, grads, wants):
        close(g, w, "d" + k)


@pytest.mark.parametrize("dtype,batch,width,states,groups", [
    (torch.bfloat16, 700, 1090, 16, 1), (torch.float32, 1100, 270, 16, 2), (torch.float16, 1030, 129, 40, 1),
    (torch.float32, 2100, 700, 3, 1)])
def test_scan_step_of_many_rows(dtype, batch, width, states, groups):
    """Two channels a thread (eight workgroups a compute unit and more), the second of them past the
    width for some; rows that are padding."""
    rng = torch.Generator(device=DEV).manual_seed(states)

    def normal(*shape, t=dtype, scale=1.0):
        return (torch.randn(shape, generator=rng, device=DEV) * scale).to(t)

    u, dt, z = normal(batch, width), normal(batch, width, scale=0.5), normal(batch, width)
    B, C = normal(batch, groups, states), normal(batch, groups, states)
    A = -torch.rand(width, states, generator=rng, device=DEV) * states - 0.3
    D, bias = normal(width, t=torch.float32), normal(width, t=torch.float32) - 3
    pool = normal(batch + 9, width, states, t=torch.float32)
    slots = torch.randperm(batch + 9, generator=rng, device=DEV)[:batch].to(torch.int32)
    slots[::50] = -1
    before = pool.double()
    y = ops.selective_scan_step(pool, u, dt, A, B, C, D, z, bias, softplus=True, slots=slots)
    on, at = slots >= 0, slots[slots >= 0].long()
    group = torch.arange(width, device=DEV) // (width // groups)
    raw = dt.double()[on] + bias.double()
    delta = torch.logaddexp(raw, torch.zeros_like(raw))
    h = (torch.exp(delta[..., None] * A.double()) * before[at]
         + (delta * u.double()[on])[..., None] * B.double()[on][:, group])
    want = torch.zeros(batch, width, dtype=torch.float64, device=DEV)
    want[on] = ((h * C.double()[on][:, group]).sum(-1) + D.double() * u.double()[on]) * ref.silu(z.double()[on])
    after = before.clone()
    after[at] = h
    close(y, want, "y")
    close(pool, after, "state")
    assert not y[~on].any()


@pytest.mark.parametrize("rows,width", [(6, 90), (5, 700), (4, 4096), (3, 5000), (3, 7001), (3, 9001)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_norm_gradients_without_the_second_norm(rows, width, bad):
    """Only the first output is used: the second norm has no part in the gradients, not
    even in a row whose residual is not finite."""
    rng = torch.Generator(device=DEV).manual_seed(5)
    args = [torch.randn(rows, width, generator=rng, device=DEV) for _ in range(3)]
    args += [torch.rand(width, generator=rng, device=DEV) + 0.3 for _ in range(3)]
    dout = torch.randn(rows, width, generator=rng, device=DEV)

    def grads(pre):
        leaf = [t.clone().requires_grad_() for t in args[:5 + pre]]
        out, _ = ops.norm_residual(*leaf)
        return torch.autograd.grad(out, leaf, dout)

    args[1][1, width // 2] = bad
    alone, both = grads(0), grads(1)
    for name, a, b in zip(("block", "residual", "gate", "post", "scale"), alone, both):
        assert torch.equal(a, b), name
    assert torch.equal(both[1], dout)
    assert not both[5].any()
