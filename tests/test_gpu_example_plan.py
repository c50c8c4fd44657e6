"""The planned step of examples/sequence_model.py does what its plan says:
what it computes again, how often, and in how much memory."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from tests.test_gpu_example import example  # noqa: E402


def build(blocks=4, width=256, batch=2, length=512, dtype=torch.bfloat16):
    torch.manual_seed(3)
    model = example.Model(blocks, width, dtype=dtype)
    x = torch.randn(batch, length, width, device="cuda").to(dtype)
    return model, x, torch.randn_like(x)


@pytest.mark.parametrize("fraction", [0.0, 0.1, 0.4, 1.0])
def test_a_planned_step_computes_again_what_its_plan_says(fraction):
    model, x, dy = build()
    graph, _, schedule = example.plan(model, 2, 512, fraction)
    step = example.Step(model, x, dy)
    example.planned_step(model, x, dy, schedule, step)
    last = schedule.seg.max()
    again = [v for v in range(graph.n) if not schedule.cached[v] and schedule.seg[v] < last]
    assert step.runs == [2 if v in again else 1 for v in range(graph.n)]
    counted = sum(graph.T[v] for v in again) + sum(graph.T[v] for v in range(graph.n) if schedule.seg[v] == last)
    assert counted == schedule.overhead
    assert not step.values and set(step.grads) <= {0}


@pytest.mark.parametrize("fraction", [0.0, 0.1, 0.4])
def test_a_planned_step_keeps_to_its_budget(fraction):
    """The most that is allocated at once, less the parameters' gradients, which no plan can drop
    (and which stay from one step to the next in a training loop)."""
    model, x, dy = build(blocks=6, width=512, batch=4, length=1024)
    _, budget, schedule = example.plan(model, 4, 1024, fraction)
    (_, grads), _, mib = example.measured(lambda: example.planned_step(model, x, dy, schedule))
    assert mib - sum(g.nbytes for g in grads) / 2 ** 20 <= budget / 1024
    _, _, plain = example.measured(lambda: example.plain_step(model, x, dy))
    assert mib < plain


def test_sizes_are_what_the_nodes_hold():
    """The scan's node holds its result and a 32-bit state every 16 tokens."""
    model, _, _ = build()
    graph = model.graph(2, 512)
    size = dict(zip(graph.ops, graph.M))
    tokens, inner = 2 * 512, model.inner
    assert size["scan"] >= (tokens * inner * 2 + tokens // 16 * inner * model.states * 4) // 1024
    assert size["conv"] >= tokens * inner * 2 // 1024
    assert size["project"] >= 2 * tokens * inner * 2 // 1024
