"""The linear-attention operators off the usual ground: no eps under a root beside padded tokens, views that
negate, numbers that are not finite beside those that are, lengths that are cut into segments."""

import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1905_11722_amd import ops  # noqa: E402
from tests import more_ops_abi as abi  # noqa: E402
from tests import more_ops_reference as ref  # noqa: E402
from tests import test_gpu_more_ops as usual  # noqa: E402
from tests.test_gpu_ops import DEV, check, compare_grads  # noqa: E402

# ----------------------------------------------------------- queries and keys


@pytest.mark.parametrize("dtype,channels,rotated,norm", [
    ("f32", 32, 16, "rms"), ("f32", 33, 20, "l2"), ("bf16", 128, 128, "l2"), ("f16", 20, 0, "rms")])
def test_qk_without_eps_beside_padded_tokens(dtype, channels, rotated, norm):
    """Rows of zeros have no unit vector, but those of padded tokens are nobody's: outputs and gradients are those
    of the tokens before each end.  The bound is that of the operator's other tests."""
    lengths = (9, 4, 0)
    x = usual.qk_inputs(dtype, 3, 9, 3, 2, channels, "f32")
    freq = torch.rand(rotated // 2) if rotated else None
    x.grads()
    names = ("q", "k", "q_weight", "k_weight")
    outs = ops.qk_norm(*[x.gpu[n] for n in names], None if freq is None else freq.to(DEV), norm=norm, eps=0.0,
                       lengths=usual.int32(lengths))
    live = [ref.qk_norm(x.cpu["q"][i:i + 1, :n], x.cpu["k"][i:i + 1, :n], x.cpu["q_weight"], x.cpu["k_weight"], freq,
                        norm=norm, eps=0.0) for i, n in enumerate(lengths)]
    wants = [torch.cat([torch.nn.functional.pad(t[j], (0, 0, 0, 0, 0, 9 - t[j].shape[1])) for t in live])
             for j in range(2)]
    for n, o, w in zip("qk", outs, wants):
        check(o, w, n)
    compare_grads(x, outs, wants)


# ------------------------------------------------------------ views that negate


def test_positions_and_seeds_that_negate():
    """Lazily negated views of whole numbers are taken at their values too."""
    x, freq = torch.randn(2, 5, 2, 8, device=DEV), torch.rand(4, device=DEV)
    at = torch.randint(1, 99, (2, 5), dtype=torch.int32, device=DEV)
    for a, b in zip(ops.qk_norm(x, x, None, None, freq, torch._neg_view(at)), ops.qk_norm(x, x, None, None, freq, -at)):
        assert torch.equal(a, b)
    seed = torch.tensor([5], device=DEV)
    x.requires_grad_()
    a, b = ops.dropout(x, 0.5, torch._neg_view(seed)), ops.dropout(x, 0.5, -5)
    assert torch.equal(a, b)
    for a, b in zip(*[torch.autograd.grad(y, x, torch.ones_like(y)) for y in (a, b)]):
        assert torch.equal(a, b)


# ------------------------------------------------------ numbers that are not finite

WILD = [  # dtype, batch, length, key_heads, heads, key, value, the token
    ("f32", 2, 100, 1, 2, 24, 20, 0), ("f32", 2, 100, 1, 2, 24, 20, 5), ("f32", 2, 100, 2, 2, 24, 20, 40),
    ("f32", 2, 100, 1, 2, 24, 20, 99), ("bf16", 2, 100, 1, 2, 24, 20, 17), ("bf16", 2, 100, 1, 2, 128, 64, 31),
    ("bf16", 1, 100, 1, 2, 128, 64, 63), ("f16", 1, 100, 1, 1, 64, 40, 64), ("f16", 2, 70, 1, 2, 128, 40, 20),
    ("f32", 1, 70, 1, 2, 200, 33, 37), ("bf16", 1, 70, 1, 2, 256, 72, 50), ("bf16", 1, 800, 1, 2, 64, 64, 500),
]


def wild_inputs(case, of, value):
    """(inputs, gradients of the outputs) with one number of `of` replaced."""
    *sizes, at = case
    x = usual.delta_inputs(*sizes, "gs")
    rng = torch.Generator().manual_seed(7)
    given = {"do": torch.randn(x.cpu["v"].shape, generator=rng).to(x.dtype),
             "dstate": torch.randn(x.cpu["state"].shape, generator=rng)}
    place = {"q": (0, at, 0, 3), "k": (0, at, 0, 3), "v": (0, at, 1 % sizes[4], 5), "g": (0, at, 0),
             "beta": (0, at, 0), "state": (0, 0, 3, 5), "do": (0, at, 0, 5), "dstate": (0, 0, 3, 5)}[of]
    for t in ([given[of]] if of in given else [x.gpu[of], x.cpu[of]]):
        t[place] = value
    return x, given


def wild_values(of):
    """(Infinity is not a decay, and its negative is one.)"""
    return [float("nan")] + [float("inf"), -float("inf")] * (of != "g")


def leaves_the_rest(got, want, own, what):
    """Not finite where `want` is not, and within the usual bound of it elsewhere; token `own` of the first sequence
    (None: no token) may be NaN."""
    got, want = got.detach().cpu(), want.detach()
    finite = want.isfinite()
    assert not got[~finite].isfinite().any(), what
    if own is not None:
        finite[0, own] = False
    check(got[finite], want[finite], what)


@pytest.mark.parametrize("of", ["q", "k", "v", "g", "beta", "state"])
@pytest.mark.parametrize("case", WILD, ids=lambda c: "-".join(map(str, c)))
def test_delta_outputs_beside_a_number_that_is_not_finite(case, of):
    """What depends on it by the definition, token by token in 64 bits, is not finite either, and all the rest is
    what it is."""
    for value in wild_values(of):
        x, _ = wild_inputs(case, of, value)
        (o, end), (want_o, want_end) = usual.run_delta(x)
        leaves_the_rest(o, want_o, None if of == "state" else case[-1], f"o, {value}")
        leaves_the_rest(end, want_end, None, f"state, {value}")


@pytest.mark.parametrize("of", ["q", "k", "v", "g", "beta", "state", "do", "dstate"])
@pytest.mark.parametrize("case", WILD, ids=lambda c: "-".join(map(str, c)))
def test_delta_gradients_beside_a_number_that_is_not_finite(case, of):
    """The same of the gradients."""
    for value in wild_values(of):
        x, given = wild_inputs(case, of, value)
        x.grads()
        outs, wants = usual.run_delta(x)
        d = list(given.values())
        got = torch.autograd.grad(outs, list(x.gpu.values()), [t.to(DEV) for t in d])
        want = torch.autograd.grad(wants, list(x.cpu.values()), [t.double() for t in d])
        for n, a, b in zip(x.gpu, got, want):
            leaves_the_rest(a, b, None if "state" in (n, of) or of == "dstate" else case[-1], f"d{n}, {value}")


def test_delta_many_numbers_that_are_not_finite():
    """Of several tokens, columns and heads the first (backward: the last) counts; a sequence without one is as without
    them, bit for bit."""
    def run(wild):
        x = usual.delta_inputs("bf16", 3, 90, 2, 4, 40, 48, "gs").gpu
        do = torch.randn(3, 90, 4, 48, generator=torch.Generator().manual_seed(3)).to(DEV).bfloat16()
        if wild:
            x["v"][0, [7, 50, 33], [0, 0, 2], [1, 1, 30]] = float("inf")
            x["k"][0, 60, 1] = float("nan")
            do[1, [10, 70], [1, 3], [0, 47]] = float("nan")
        leaves = [t.requires_grad_() for t in x.values()]
        o = ops.gated_delta(*[x[n] for n in ("q", "k", "v", "g", "beta")], state=x["state"])
        return [o.detach(), *torch.autograd.grad(o, leaves, do)]

    wild, tame = run(True), run(False)
    for a, b in zip(wild, tame):
        assert torch.equal(a[2], b[2])
    o, dq, dk, dv, dg, dbeta = wild[:6]
    want = torch.ones(90, 4, 48, dtype=torch.bool, device=DEV)      # finite
    want[7:, 0, 1] = want[33:, 2, 30] = False
    want[60:, 2:] = False
    assert torch.equal(o[0].isfinite(), want) and torch.equal(o[0][want], tame[0][0][want])
    assert torch.equal(o[1], tame[0][1])
    assert dv[1, :11, 1, 0].isnan().all() and dv[1, 11:, 1, 0].isfinite().all()
    assert dv[1, :71, 3, 47].isnan().all() and dv[1, 71:, 3, 47].isfinite().all()
    for t, head in ((dg, 1), (dbeta, 1)):
        assert t[1, :11, head].isnan().all() and t[1, 11:, head].isfinite().all()
    assert dk[1, 71:].isfinite().all() and dq[1, 71:].isfinite().all() and dq[1, :10].isfinite().all()


# -------------------------------------------------- lengths that are cut into segments

CUT = [  # dtype, batch, length, key_heads, heads, key, value, parts, lengths, segments
    ("f32", 1, 800, 1, 1, 16, 8, "gs", None, 3),
    ("f16", 3, 800, 1, 1, 30, 33, "gs", (799, 0, 300), 3),
    ("bf16", 2, 1030, 1, 2, 32, 96, "g", (1030, 31), 4),
    ("f16", 3, 900, 1, 1, 64, 33, "gs", (899, 1, 257), 3),
    ("f32", 1, 1100, 1, 2, 48, 64, "gs", (1095,), 4),
    ("bf16", 1, 800, 2, 2, 64, 64, "s", None, 3),
    ("f32", 1, 790, 1, 2, 96, 100, "gs", (790,), 3),
    ("f16", 2, 1050, 1, 1, 128, 40, "gs", (1050, 520), 4),
    ("bf16", 1, 1601, 1, 1, 200, 40, "g", (1597,), 3),
    ("f32", 2, 1540, 1, 1, 256, 24, "gs", (1540, 600), 3),
    ("f16", 1, 1540, 1, 2, 130, 70, "gs", None, 3),
]


def segments(dtype, batch, length, key_heads, heads, key, value):
    """Into how many segments a length is cut, from the scratch that it takes beside the chunks'."""
    lib, n = abi.library(), ctypes.c_uint64()

    def scratch(tokens):
        a = abi.DeltaArgs(dtype=("f32", "bf16", "f16").index(dtype), batch=batch, length=tokens, key_heads=key_heads,
                          heads=heads, key=key, value=value)
        assert lib.rc_delta_forward_workspace(a, n) == 0
        return n.value

    chunks = -(-length // 32) * scratch(32)                         # (one chunk is not cut)
    rows, columns = 32 if key <= 32 else 64 if key <= 64 else 128 if key <= 128 else 256, -(-value // 32) * 32
    each = 4 * batch * heads * rows * (rows + 2 * columns)
    more = scratch(length) - chunks
    assert more % each == 0
    return max(1, more // each)


@pytest.mark.parametrize("case", CUT, ids=lambda c: "-".join(map(str, c[:7])))
def test_delta_cut_into_segments(case):
    """Every width of keys and every type, ends in the first, in the last and in segments between; the bound is that
    of the operator's other tests."""
    *sizes, lengths, count = case
    assert segments(*sizes[:7]) == count
    x = usual.delta_inputs(*sizes)
    if lengths is not None:
        with torch.no_grad():
            for i, e in enumerate(lengths):
                for n in x.gpu:
                    if n != "state":
                        x.gpu[n][i, e:] = float("nan")
                        x.cpu[n][i, e:] = 0
    x.grads()
    outs, wants = usual.run_delta(x, lengths)
    for n, o, w in zip(("o", "state"), outs, wants):
        check(o, w, n)
    compare_grads(x, outs, wants)


@pytest.mark.parametrize("key,value,length", [(16, 8, 800), (100, 33, 800), (200, 40, 1540)])
def test_delta_cut_with_scratch_aligned_to_a_float(key, value, length):
    assert segments("bf16", 1, length, 1, 1, key, value) == 3
    usual.test_delta_scratch_aligned_to_a_float(key, value, length)
