"""The operators of a language module's training step together: experts' MLPs behind a residual with dropout, and the loss over a vocabulary, forward
and back, eagerly and from a graph, against automatic differentiation in 64 bits (tolerances of whole layers: `tol`)."""
import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2605_18710_amd import binding as mb, synth
from helpers import from_dev, quantize, rel_l2, to_dev, tol

pytestmark = pytest.mark.gpu
T, h, f, E, V, P, SITE = 333, 128, 192, 5, 1003, 0.2, 7
OFFSETS = [0, 100, 100, 171, 300, 333]


class Step:
    """Buffers of one training step; run() makes its calls on the current stream."""

    def __init__(self, dtype, x, w1, w2, table, target):
        self.dtype = dtype
        self.x, self.w1, self.w2, self.table = (to_dev(v, dtype) for v in (x, w1, w2, table))
        self.target, self.offsets = torch.from_numpy(target).cuda(), torch.tensor(OFFSETS, dtype=torch.int32, device="cuda")
        self.rng = torch.tensor([1234567, 89], device="cuda")
        new = lambda *s: torch.empty(s, device="cuda", dtype=self.x.dtype)
        self.gu, self.a, self.y, self.r = new(T, 2 * f), new(T, f), new(T, h), new(T, h)
        self.dr, self.dy, self.da, self.dgu, self.dx = new(T, h), new(T, h), new(T, f), new(T, 2 * f), new(T, h)
        self.dw1, self.dw2, self.dtable = torch.empty_like(self.w1), torch.empty_like(self.w2), torch.empty_like(self.table)
        self.loss, self.losses = torch.empty(1, device="cuda"), torch.empty(T, device="cuda")
        self.scratch = torch.empty(mb.linear_ce_grad_scratch_bytes(dtype, T, h, V), device="cuda", dtype=torch.uint8)

    def run(self, quota=256):
        s, d = torch.cuda.current_stream().cuda_stream, self.dtype
        mb.op_grouped_linear_fwd(s, quota, d, T, E, h, 2 * f, self.offsets, self.x, self.w1, self.gu)
        mb.op_swiglu_fwd(s, quota, d, T, f, self.gu, self.a)
        mb.op_grouped_linear_fwd(s, quota, d, T, E, f, h, self.offsets, self.a, self.w2, self.y)
        mb.op_dropout(s, quota, d, T * h, P, SITE, self.rng, self.y, self.x, self.r)
        mb.op_linear_ce_grad(s, quota, d, T, h, V, 0.1, 0.0, self.target, self.r, self.table, self.loss, self.losses, self.dr, self.dtable, self.scratch)
        mb.op_dropout(s, quota, d, T * h, P, SITE, self.rng, self.dr, None, self.dy)
        mb.op_grouped_linear_dgrad(s, quota, d, T, E, f, h, self.offsets, self.dy, self.w2, self.da)
        mb.op_grouped_linear_wgrad(s, quota, d, T, E, f, h, self.offsets, self.a, self.dy, self.dw2)
        mb.op_swiglu_bwd(s, quota, d, T, f, self.gu, self.da, self.dgu)
        mb.op_grouped_linear_dgrad(s, quota, d, T, E, h, 2 * f, self.offsets, self.dgu, self.w1, self.dx)
        mb.op_grouped_linear_wgrad(s, quota, d, T, E, h, 2 * f, self.offsets, self.x, self.dgu, self.dw1)

    def results(self):
        torch.cuda.synchronize()
        return {k: getattr(self, k).clone() for k in ("loss", "losses", "dr", "dx", "dw1", "dw2", "dtable")}


def inputs(dtype, seed=40):
    q = lambda v: quantize(v, dtype)
    target = synth.integers(seed + 4, (T,), 0, V)
    target[::7] = -1
    return (q(synth.normal(seed, (T, h))), q(synth.normal(seed + 1, (E, h, 2 * f), 0.0, h ** -0.5)), q(synth.normal(seed + 2, (E, f, h), 0.0, f ** -0.5)),
            q(synth.normal(seed + 3, (V, h), 0.0, 2 * h ** -0.5)), target.astype(np.int32))


def reference(x, w1, w2, table, target):
    x, w1, w2, table = (torch.from_numpy(v).requires_grad_(True) for v in (x, w1, w2, table))
    part = [slice(a, b) for a, b in zip(OFFSETS, OFFSETS[1:])]
    gate, up = torch.cat([x[p] @ w1[e] for e, p in enumerate(part)]).chunk(2, dim=1)
    a = gate * torch.sigmoid(gate) * up
    y = torch.cat([a[p] @ w2[e] for e, p in enumerate(part)])
    keep, scale = O.dropout_keeps(range(T * h), P, SITE, 1234567, 89)
    r = x + y * torch.from_numpy(keep * scale).reshape(T, h)
    r.retain_grad()
    rows = np.flatnonzero(target >= 0)
    logp = torch.log_softmax(r[rows] @ table.t(), dim=1)
    each = -0.9 * logp[torch.arange(len(rows)), torch.from_numpy(target[rows]).long()] - 0.1 * logp.mean(1)
    each.mean().backward()
    losses = np.zeros(T)
    losses[rows] = each.detach().numpy()
    return dict(loss=float(each.mean().detach()), losses=losses, dr=r.grad, dx=x.grad - r.grad, dw1=w1.grad, dw2=w2.grad, dtable=table.grad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_eagerly_and_from_a_graph(dtype):
    data = inputs(dtype)
    step = Step(dtype, *data)
    step.run()
    got, ref = step.results(), reference(*data)
    for k, v in ref.items():
        assert rel_l2(from_dev(got[k]), np.asarray(v)) <= tol(dtype), k
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for turn in range(3):
        step.x.mul_(-1.0)
        step.rng[1] += 100 * turn
        graph.replay()
        torch.cuda.synchronize()
        replayed = step.results()
        step.run()
        again = step.results()
        assert all(torch.equal(replayed[k], again[k]) for k in again)


def test_two_steps_at_once():
    """On two streams, each with buffers of its own: the bits of each alone."""
    steps = [Step("bf16", *inputs("bf16", 40 + 10 * i)) for i in range(2)]
    alone = []
    for s in steps:
        s.run()
        alone.append(s.results())
    streams = [torch.cuda.Stream() for _ in steps]
    for turn in range(3):
        for s, q in zip(steps, streams):
            with torch.cuda.stream(q):
                s.run(128)
        for s, want in zip(steps, alone):
            got = s.results()
            assert all(torch.equal(got[k], want[k]) for k in got)
