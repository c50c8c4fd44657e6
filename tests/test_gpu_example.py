"""The example of examples/sequence_model.py: the planned training step has
the plain step's gradients, and single tokens go on from a prompt."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location(
    "sequence_model", os.path.join(ROOT, "examples", "sequence_model.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def build(dtype):
    torch.manual_seed(3)
    model = example.Model(3, 64, dtype=dtype)
    x = torch.randn(2, 50, 64, device="cuda").to(dtype)
    return model, x, torch.randn(2, 50, 64, device="cuda")


@pytest.mark.parametrize("fraction", [0.0, 0.3, 1.0])
def test_planned_step(fraction):
    """In 32 bits each gradient is a sum over 100 tokens in another grouping at
    most (segments are differentiated apart): 1e-4 of its size covers that."""
    model, x, dy = build(torch.float32)
    graph, budget, schedule = example.plan(model, 2, 50, fraction)
    assert schedule.peak <= budget
    loss, want = example.plain_step(model, x, dy)
    planned, got = example.planned_step(model, x, dy, schedule)
    assert torch.allclose(loss, planned, rtol=1e-5)
    for g, w in zip(got, want):
        assert (g is None) == (w is None)
        if w is not None:
            assert (g - w).norm() <= 1e-4 * w.norm() + 1e-6


def test_tokens_after_a_prompt():
    """Single tokens and the whole sequence differ by rounding alone: 32 bits
    through 3 blocks, 1e-4."""
    model, x, _ = build(torch.float32)
    whole, _ = example.prompt(model, x)
    out, states = example.prompt(model, x[:, :43])
    assert torch.allclose(out, whole[:, :43], rtol=1e-4, atol=1e-4)
    for t in range(43, 50):
        out = example.token(model, x[:, t], states)
        assert (out - whole[:, t]).norm() <= 1e-4 * whole[:, t].norm()
