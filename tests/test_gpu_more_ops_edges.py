"""The linear-attention operators off the usual ground: no eps under a root beside padded tokens, views that
negate."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1905_11722_amd import ops  # noqa: E402
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
