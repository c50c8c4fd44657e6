"""The linear attention of examples/sequence_model.py: a planned step, whose dropped nodes draw their
masks again, has the plain step's gradients; single tokens go on from a prompt."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from tests.test_gpu_example import example  # noqa: E402


def build(dtype=torch.float32):
    torch.manual_seed(3)
    model = example.DeltaModel(3, 128, dtype=dtype, p=0.2)
    x = torch.randn(2, 70, 128, device="cuda").to(dtype)
    return model, x, torch.randn(2, 70, 128, device="cuda")


@pytest.mark.parametrize("fraction", [0.0, 0.3, 1.0])
def test_planned_step(fraction):
    """In 32 bits each gradient is a sum over 140 tokens in another grouping at
    most (segments are differentiated apart): 1e-4 of its size covers that.  A mask drawn
    otherwise the second time would change a fifth of the values."""
    model, x, dy = build()
    graph, budget, schedule = example.plan(model, 2, 70, fraction)
    assert schedule.peak <= budget
    for seed in (1, 2):
        model.seed = seed
        loss, want = example.plain_step(model, x, dy)
        planned, got = example.planned_step(model, x, dy, schedule)
        assert torch.allclose(loss, planned, rtol=1e-5)
        for g, w in zip(got, want):
            assert (g is None) == (w is None)
            if w is not None:
                assert (g - w).norm() <= 1e-4 * w.norm() + 1e-6
        if seed == 2:
            assert loss != before
        before = loss


def test_tokens_after_a_prompt():
    """Single tokens and the whole sequence differ by rounding alone: 32 bits
    through 3 blocks, 1e-4."""
    model, x, _ = build()
    whole, _ = example.prompt(model, x)
    out, states = example.prompt(model, x[:, :43])
    assert torch.allclose(out, whole[:, :43], rtol=1e-4, atol=1e-4)
    for t in range(43, 70):
        out = example.token(model, x[:, t], states)
        assert (out - whole[:, t]).norm() <= 1e-4 * whole[:, t].norm()
