"""A sequence model trained under a memory budget, and then run token by token.

The model is a stack of residual blocks: projection, short causal
convolution, projection to the scan's steps and its B and C, selective state space
scan with a gate, projection back, and the norms after this block and before
the next one.  Its operators come from ``paper_1905_11722_amd.ops``, its plain
matrix products from PyTorch.

The training step is planned by ``paper_1905_11722_amd.rcdp``: every operation
of the step is a node with its forward time (measured, in tenths of a microsecond) and
its size in KiB (measured: its result and what its backward pass keeps beside that, the scan's
states every few tokens, say).  For a budget the solver returns the chain
of lower sets of least recomputation overhead, and the step runs its
canonical strategy (Section 3 of Kusumoto et al.): forward, the nodes on a segment's boundary
stay; in the backward pass each segment's other nodes are computed again from them.
(Those of the last segment need not be, though Eq. 1 counts them.)  The
gradients are those of the plain step.

Then the model reads a prompt and goes on token by token with the single-token forms,
from the states that the prompt left.

    python examples/sequence_model.py --blocks 8 --width 1024 --batch 4 --length 2048
"""

from __future__ import annotations

import argparse
import os
import statistics
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1905_11722_amd import ops, rcdp, workloads  # noqa: E402

NODES = ("project", "conv", "steps", "delta", "scan", "back", "join")      # of a block, in order


class Model:
    """The stack's parameters and the function of each node.

    width: channels of the residual stream; the block works on 2 * width
    channels with ``states`` states each, taps of the convolution, and
    steps of rank width / 16.
    """

    def __init__(self, blocks, width, states=16, taps=4, dtype=torch.bfloat16, device="cuda", seed=0):
        rng = torch.Generator(device=device).manual_seed(seed)
        inner, rank = 2 * width, max(1, width // 16)
        self.blocks, self.width, self.inner, self.states, self.rank = blocks, width, inner, states, rank
        self.taps, self.dtype = taps, dtype

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=rng, device=device) * rows ** -0.5).to(dtype)

        self.p = []
        for _ in range(blocks):
            decay = torch.arange(1, states + 1, device=device, dtype=torch.float32)
            self.p.append({
                "project": matrix(width, 2 * inner), "conv": matrix(taps, inner).t().float().contiguous(),
                "conv_bias": torch.zeros(inner, device=device), "steps": matrix(inner, rank + 2 * states),
                "dt": matrix(rank, inner), "dt_bias": torch.full((inner,), -4.0, device=device),
                "A": -decay.repeat(inner, 1), "D": torch.ones(inner, device=device),
                "back": matrix(inner, width), "post": torch.ones(width, device=device),
                "scale": torch.full((width,), 0.5, device=device), "pre": torch.ones(width, device=device)})
        for block in self.p:
            for t in block.values():
                t.requires_grad_()
        self.first = torch.ones(width, device=device).requires_grad_()

    def parameters(self):
        return [t for block in self.p for t in block.values()] + [self.first]

    @property
    def nodes(self):
        """Nodes of a step: the first norm, the blocks', the loss."""
        return self.blocks * len(NODES) + 2

    def place(self, node):
        """(block, kind) of a node; "start" and "loss" belong to no block."""
        if node in (0, self.nodes - 1):
            return None, "loss" if node else "start"
        block, kind = divmod(node - 1, len(NODES))
        return block, NODES[kind]

    def owned(self, node):
        """The parameters that a node takes."""
        block, kind = self.place(node)
        names = {"project": ["project"], "conv": ["conv", "conv_bias"], "steps": ["steps"], "delta": ["dt"],
                 "scan": ["dt_bias", "A", "D"], "back": ["back"], "join": ["post", "scale", "pre"]}
        return [self.first] if kind == "start" else [self.p[block][k] for k in names.get(kind, [])]

    def start(self, x):
        """(residual stream, normed) of the input."""
        return ops.norm_residual(None, x, pre_weight=self.first)

    def run(self, block, kind, values, state=None):
        """The value of a block's node from its predecessors' (with ``state``, the
        states of a prompt or of one token, in the order of `predecessors`)."""
        p, rank, n = self.p[block], self.rank, self.states
        if kind == "project":
            return values[0][1] @ p["project"]
        if kind == "conv":
            x = values[0][..., :self.inner]
            if state is None:
                return ops.causal_conv(x, p["conv"], p["conv_bias"])
            return ops.causal_conv_step(state[0], x, p["conv"], p["conv_bias"])
        if kind == "steps":
            return values[0] @ p["steps"]
        if kind == "delta":
            return values[0][..., :rank] @ p["dt"]
        if kind == "scan":
            u, steps, dt, z = *values[:3], values[3][..., self.inner:]
            B, C = steps[..., rank:rank + n], steps[..., rank + n:]
            if state is None:
                return ops.selective_scan(u, dt, p["A"], B, C, p["D"], z, p["dt_bias"], softplus=True)
            return ops.selective_scan_step(state[1], u, dt, p["A"], B, C, p["D"], z, p["dt_bias"],
                                           softplus=True)
        if kind == "back":
            return values[0] @ p["back"]
        return ops.norm_residual(values[0], values[1][0], post_weight=p["post"], scale=p["scale"],
                                 pre_weight=p["pre"])

    def predecessors(self, node):
        """Nodes whose values the node takes."""
        block, kind = self.place(node)
        if block is None:
            return [node - 1] if node else []
        first = 1 + block * len(NODES)
        return {"project": [first - 1], "conv": [first], "steps": [first + 1], "delta": [first + 2],
                "scan": [first + 1, first + 2, first + 3, first], "back": [first + 4],
                "join": [first + 5, first - 1]}[kind]

    def node(self, node, get, x=None, dy=None, state=None):
        """The value of a node of a step on input x with the loss <output, dy>."""
        block, kind = self.place(node)
        if kind == "start":
            return self.start(x)
        values = [get(v) for v in self.predecessors(node)]
        if kind == "loss":
            return (values[0][1] * dy).sum(dtype=torch.float32)
        return self.run(block, kind, values, None if state is None else state[block])

    def graph(self, batch, length):
        """The step's nodes with their times and sizes (workloads.Graph)."""
        cost = measure(self, batch, length)
        places = [self.place(v) for v in range(self.nodes)]
        succ = [[] for _ in places]
        for v in range(self.nodes):
            for u in self.predecessors(v):
                succ[u].append(v)
        kinds = [kind for _, kind in places]
        return workloads.Graph(self.nodes, [sorted(x) for x in succ], [cost[k][0] for k in kinds],
                               [cost[k][1] for k in kinds],
                               [k if b is None else f"{k}{b}" for b, k in places], kinds)


def _tensors(value):
    return list(value) if isinstance(value, tuple) else [value]


class _Port(torch.autograd.Function):
    """A predecessor's value on its way into a node: its gradient goes to
    ``grads``, and the node's graph holds nothing of the value itself."""

    @staticmethod
    def forward(ctx, token, value, grads, index):
        ctx.grads, ctx.index = grads, index
        return value.view_as(value)

    @staticmethod
    def backward(ctx, g):
        old = ctx.grads[ctx.index]
        ctx.grads[ctx.index] = g if old is None else old + g
        return None, None, None, None


class Step:
    """A training step whose nodes run one by one, each with an autograd graph
    of its own.  What a graph has to keep of its predecessors' values it takes
    from ``values`` in the backward pass, so that they may be dropped and
    computed again in between; what else it keeps is the node's."""

    def __init__(self, model, x, dy):
        self.model, self.x, self.dy = model, x, dy
        self.values, self.grads, self.params = {}, {}, {}
        self.runs = [0] * model.nodes
        self.token = torch.zeros((), device=x.device, requires_grad=True)

    def forward(self, v, record):
        """Run a node; with ``record`` so that `backward` can follow."""
        self.runs[v] += 1
        if not record:
            with torch.no_grad():
                self.values[v] = self.model.node(v, self.values.__getitem__, self.x, self.dy)
            return
        where = {t.untyped_storage().data_ptr(): (u, i) for u in self.model.predecessors(v)
                 for i, t in enumerate(_tensors(self.values[u]))}

        def pack(t):
            at = where.get(t.untyped_storage().data_ptr())
            if at is None:
                return t
            base = _tensors(self.values[at[0]])[at[1]]
            return at, t.size(), t.stride(), t.storage_offset() - base.storage_offset()

        def unpack(packed):
            if isinstance(packed, torch.Tensor):
                return packed
            (u, i), size, stride, offset = packed
            base = _tensors(self.values[u])[i].detach()
            return base.as_strided(size, stride, base.storage_offset() + offset)

        def get(u):
            value = self.values[u]
            grads = self.grads.setdefault(u, [None] * len(_tensors(value)))
            ports = tuple(t if t.data_ptr() == self.x.data_ptr() else _Port.apply(self.token, t.detach(), grads, i)
                          for i, t in enumerate(_tensors(value)))
            return ports if isinstance(value, tuple) else ports[0]

        with torch.enable_grad(), torch.autograd.graph.saved_tensors_hooks(pack, unpack):
            self.values[v] = self.model.node(v, get, self.x, self.dy)

    def backward(self, v):
        """Gradients of a recorded node's predecessors and parameters; its value goes."""
        outs = [(t, g) for t, g in zip(_tensors(self.values[v]), self.grads.pop(v)) if g is not None]
        owned = self.model.owned(v)
        got = torch.autograd.grad([t for t, _ in outs], owned + [self.token], [g for _, g in outs],
                                  allow_unused=True)
        self.params.update(zip(map(id, owned), got))
        del self.values[v]

    def result(self):
        return [self.params.get(id(p)) for p in self.model.parameters()]


@torch.no_grad()
def measure(model, batch, length, repeats=5):
    """{kind: (tenths of a microsecond forward, KiB)} of the step's nodes, from
    running the first block.  The size is that of what a recorded node holds or, if that is more, of
    its gradient and the scratch of its backward pass."""
    x = torch.randn(batch, length, model.width, device=model.first.device).to(model.dtype)
    step, last = Step(model, x, torch.randn_like(x)), model.nodes - 1
    order = list(range(1 + len(NODES))) + [last]
    cost = {}

    def pass_over():
        for v in order:
            before = torch.cuda.memory_allocated()
            step.forward(v, True)
            cost[v] = torch.cuda.memory_allocated() - before
            if v == len(NODES):                      # the last block's end, for the loss
                step.values[last - 1] = step.values[v]
        step.grads[last] = [torch.ones_like(step.values[last])]
        for v in reversed(order):
            if v == len(NODES) and last - 1 != v:
                step.grads[v] = step.grads.pop(last - 1)
                del step.values[last - 1]
            if v == 0:
                step.grads[v][0] = None
            result = step.values[v]                  # (not freed meanwhile)
            beside = cost[v] - sum(t.nbytes for t in _tensors(result) if t.data_ptr() != x.data_ptr())
            torch.cuda.reset_peak_memory_stats()
            step.backward(v)                         # its own gradient and `beside` are freed
            freed = torch.cuda.max_memory_allocated() - torch.cuda.memory_allocated()
            cost[v] = max(cost[v], freed - beside)
            del result

    pass_over()                                      # (libraries take their workspaces)
    pass_over()
    times = {}
    for v in order:
        step.forward(v, False)
        spans = []
        for _ in range(repeats):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            step.forward(v, False)
            end.record()
            end.synchronize()
            spans.append(start.elapsed_time(end))
        times[v] = statistics.median(spans)
        if v == len(NODES):
            step.values[last - 1] = step.values[v]
    return {model.place(v)[1]: (max(1, round(times[v] * 1e4)), max(1, -(-cost[v] // 1024))) for v in order}


def plain_step(model, x, dy):
    """Loss <output, dy> and the parameters' gradients, everything kept."""
    values = {}
    for v in range(model.nodes):
        values[v] = model.node(v, values.__getitem__, x, dy)
    return values[v].detach(), torch.autograd.grad(values[v], model.parameters(), allow_unused=True)


def planned_step(model, x, dy, schedule, step=None):
    """The same through the canonical strategy of a schedule (rcdp.Schedule)."""
    step = step or Step(model, x, dy)
    segments = [[] for _ in range(int(schedule.seg.max()) + 1)]
    for v, s in enumerate(schedule.seg):
        segments[int(s)].append(v)
    for nodes in segments[:-1]:
        for v in nodes:
            step.forward(v, bool(schedule.cached[v]))
        for v in nodes:
            if not schedule.cached[v]:
                del step.values[v]
    loss = None
    for nodes in reversed(segments):
        for v in nodes:
            if v not in step.values:
                step.forward(v, True)
        if loss is None:
            loss = step.values[nodes[-1]].detach()
            step.grads[nodes[-1]] = [torch.ones_like(loss)]
        for v in reversed(nodes):
            step.backward(v)
    return loss, step.result()


@torch.no_grad()
def prompt(model, x):
    """(normed output, the states after the prompt) of a prompt."""
    values, states, n = model.start(x), [], model.states
    for b in range(model.blocks):
        p = model.p[b]
        both = model.run(b, "project", [values])
        u, conv = ops.causal_conv(both[..., :model.inner], p["conv"], p["conv_bias"], return_state=True)
        steps = model.run(b, "steps", [u])
        B, C = steps[..., model.rank:model.rank + n], steps[..., model.rank + n:]
        y, scan = ops.selective_scan(u, model.run(b, "delta", [steps]), p["A"], B, C, p["D"],
                                     both[..., model.inner:], p["dt_bias"], softplus=True, return_state=True)
        states.append((conv, scan))
        values = model.run(b, "join", [model.run(b, "back", [y]), values])
    return values[1], states


@torch.no_grad()
def token(model, x, states):
    """The normed output of one token of each sequence; updates the states."""
    values = {}
    for v in range(model.nodes - 1):
        values[v] = model.node(v, values.__getitem__, x, state=states)
    return values[v][1]


def plan(model, batch, length, fraction):
    """(graph, budget, schedule) at a fraction of the way from the smallest
    feasible budget to the one that keeps everything."""
    graph = model.graph(batch, length)
    family = rcdp.Graph.create(graph).build_family("pruned")
    low, high = family.min_budget(), 2 * family.info["M_total"]
    budget = low + int((high - low) * fraction)
    solution = family.solve(budget, "tc")
    return graph, budget, solution.reconstruct()


def measured(step):
    """(result, milliseconds, MiB allocated beside what was) of the second of two runs of a step."""
    step()
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    e0, e1 = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    e0.record()
    result = step()
    e1.record()
    torch.cuda.synchronize()
    return result, e0.elapsed_time(e1), (torch.cuda.max_memory_allocated() - before) / 2 ** 20


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--blocks", type=int, default=8)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--length", type=int, default=2048)
    ap.add_argument("--fraction", type=float, default=0.0, help="of the way from the smallest budget")
    ap.add_argument("--tokens", type=int, default=16, help="of the length, one by one after the rest as a prompt")
    a = ap.parse_args()
    if not 1 <= a.tokens <= a.length:
        ap.error("--tokens must be at least 1 and at most the length")
    torch.manual_seed(1)
    model = Model(a.blocks, a.width)
    x = torch.randn(a.batch, a.length, a.width, device="cuda").to(model.dtype)
    dy = torch.randn_like(x)
    graph, budget, schedule = plan(model, a.batch, a.length, a.fraction)
    again = sum(graph.T[v] for v in range(graph.n)
                if not schedule.cached[v] and schedule.seg[v] < schedule.seg.max())
    print(f"{graph.n} nodes, {sum(graph.M) / 1024:.0f} MiB, {sum(graph.T) / 1e4:.2f} ms forward; budget "
          f"{budget / 1024:.0f} MiB: {len(schedule.chain)} segments, {int(schedule.cached.sum())} nodes kept "
          f"({schedule.cache_mem / 1024:.0f} MiB), {again / 1e4:.2f} ms computed again "
          f"({schedule.overhead / 1e4:.2f} with the last segment)")
    plain, ms, mib = measured(lambda: plain_step(model, x, dy))
    print(f"plain    step {ms:8.2f} ms, peak {mib:8.0f} MiB")
    planned, ms, mib = measured(lambda: planned_step(model, x, dy, schedule))
    grads = sum(g.nbytes for g in planned[1]) / 2 ** 20
    print(f"planned  step {ms:8.2f} ms, peak {mib:8.0f} MiB, {grads:.0f} of it the parameters' gradients")
    off = max(((p.float() - q.float()).norm() / p.float().norm()).item()
              for p, q in zip(plain[1], planned[1]) if p.norm() > 0)
    print(f"gradients differ by at most {off:.1e} of their size")
    out, states = prompt(model, x[:, :a.length - a.tokens])
    for t in range(a.length - a.tokens, a.length):
        out = token(model, x[:, t], states)
    whole, _ = prompt(model, x)
    off = ((out.float() - whole[:, -1].float()).norm() / whole[:, -1].float().norm()).item()
    print(f"{a.tokens} single tokens after the prompt: {off:.1e} off the whole sequence's last output")


if __name__ == "__main__":
    main()
