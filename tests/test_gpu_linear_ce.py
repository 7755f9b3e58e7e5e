"""Softmax cross entropy behind a linear layer, with its gradients, against the definition in 64 bits.

Bounds, element by element.  u = 2^-24: a logit is a sum of h products in fp32, off by (h + 2) u sum |x w| at most (E).  The exponential and its
argument, the sums of a block, of the blocks and their joining add (64 + V / 512) 2 u to a sum relative to itself, the
logarithm and its factor 4 u |lse|.  bf16: a probability is kept in fp16 relative to the largest of its block (2^-11 of itself, or 2^-25 of that one), and
the logits' gradient rounded, by 2^-8, before the products; these are sums of V (rows) or T (table) terms in fp32 and are rounded once, by 2^-8."""
import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2605_18710_amd import binding as mb, synth
from helpers import from_dev, quantize, to_dev

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def inputs(T, h, V, ignored, dtype, seed=5):
    x = synth.normal(seed, (T, h))
    table = synth.normal(seed + 1, (V, h)) * 2.0 / np.sqrt(h)
    target = synth.integers(seed + 2, (T,), 0, V)
    sure = synth.uniform(seed + 3, (T, 1), 0.0, 3.0)
    x = x + sure * table[target]
    out = synth.uniform(seed + 4, (T,)) < ignored
    target[out] = np.where(synth.integers(seed + 5, (T,), 0, 3) == 0, -100, np.where(synth.integers(seed + 6, (T,), 0, 2) == 0, V, -1))[out]
    return quantize(x, dtype), quantize(table, dtype), target.astype(np.int32)


def bounds(x, table, target, smoothing, denom, dtype):
    """Of losses, dx and dtable."""
    T, h = x.shape
    V = len(table)
    at = np.flatnonzero((target >= 0) & (target < V))
    D = denom if denom > 0 else max(1, len(at))
    rows = x[at]
    z = rows @ table.T
    E = (h + 2) * U * (np.abs(rows) @ np.abs(table).T).max(1, initial=0.0)
    top = z.max(1, keepdims=True) if len(at) else z[:, :1]
    lse = top + np.log(np.exp(z - top).sum(1, keepdims=True))
    rel = 2 * E + (64 + V / 512) * 2 * U + 8 * U * np.abs(lse[:, 0]) + 4 * U * np.abs(z).max(1, initial=0.0)      # of a probability, and of a loss absolutely
    losses = np.zeros(T)
    losses[at] = rel + 8 * U * (np.abs(lse[:, 0]) + np.abs(z).max(1, initial=0.0))
    p = np.exp(z - lse)
    one = np.zeros(z.shape)
    one[np.arange(len(at)), target[at]] = 1.0
    dz = np.abs(p - (1 - smoothing) * one - smoothing / V) / D
    store, kept = (2.0 ** -8, 2.0 ** -11) if dtype == "bf16" else (0.0, 0.0)
    # the target's own term is formed from its fp32 logit and rounded once
    off = ((rel[:, None] + 4 * U + kept * (1 - one)) * p + kept * 2.0 ** -14 * p.max(1, initial=0.0, keepdims=True)) / D * (1 + store) + store * dz + 4 * U * (smoothing + one) / D
    last = 2.0 ** -8 if dtype == "bf16" else U
    dx, dtable = np.zeros(x.shape), None
    full = off + (V + 2) * U * (dz + off)
    dx[at] = full @ np.abs(table) * (1 + last) + last * (dz @ np.abs(table))
    off = off + (len(at) + 8) * U * (dz + off)
    dtable = off.T @ np.abs(rows) * (1 + last) + last * (dz.T @ np.abs(rows))
    return losses, dx, dtable


def call(x, table, target, smoothing, denom, dtype, grad=True, quota=256, stream=None, want=("dx", "dtable", "losses"), guard=3):
    T, h = x.shape
    V = len(table)
    X, W = to_dev(x, dtype), to_dev(table, dtype)
    y = torch.from_numpy(target).cuda()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    loss = torch.full((1,), 77.0, device="cuda")
    losses = torch.full((T + guard,), 77.0, device="cuda")
    dx, dtable = torch.full((T + guard, h), 77.0, device="cuda", dtype=dt), torch.full((V + guard, h), 77.0, device="cuda", dtype=dt)
    size = (mb.linear_ce_grad_scratch_bytes if grad else mb.linear_ce_fwd_scratch_bytes)(dtype, T, h, V)
    scratch = torch.full((size,), 0xFF, device="cuda", dtype=torch.uint8)                   # NaN wherever it is read unwritten
    torch.cuda.synchronize()
    each = losses if "losses" in want else None
    if grad:
        mb.op_linear_ce_grad(stream, quota, dtype, T, h, V, smoothing, denom, y, X, W, loss, each, dx if "dx" in want else None,
                             dtable if "dtable" in want else None, scratch)
    else:
        mb.op_linear_ce_fwd(stream, quota, dtype, T, h, V, smoothing, denom, y, X, W, loss, each, scratch)
    torch.cuda.synchronize()
    assert (losses[T:] == 77).all() and (dx[T:] == 77).all() and (dtable[V:] == 77).all()
    return dict(loss=float(loss), losses=losses[:T], dx=dx[:T], dtable=dtable[:V])


def close(got, ref, bound, what):
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    assert np.isfinite(got).all(), what
    excess = np.abs(got - ref) - bound
    assert (excess <= 0).all(), (what, float((np.abs(got - ref) / np.maximum(bound, 1e-300)).max()))


CASES = [  # T, h, V, smoothing, share ignored
    (1, 8, 1, 0.0, 0.0), (1, 64, 2, 0.1, 0.0), (3, 72, 27, 0.1, 0.0), (130, 128, 1000, 0.0, 0.5), (257, 200, 515, 0.1, 0.3), (64, 136, 4099, 0.0, 0.0),
    (520, 320, 257, 0.0, 0.9), (129, 64, 20011, 0.2, 0.1), (1500, 64, 64, 0.0, 0.2), (2100, 264, 130, 0.1, 0.0), (40, 512, 2000, 0.0, 1.0), (1030, 256, 300, 0.0, 0.02),
    # by large tiles, of 256 rows and of 128, with the contraction over the vocabulary, or the tokens, cut; fp32 rows past what a workgroup holds
    (3000, 512, 6000, 0.1, 0.3), (100, 256, 60000, 0.0, 0.1), (5000, 256, 600, 0.0, 0.1), (33, 40, 9001, 0.1, 0.2), (187, 72, 30001, 0.0, 0.0), (1000, 40, 100, 0.1, 0.3), (1500, 104, 2301, 0.1, 0.1), (600, 520, 2050, 0.0, 0.0), (1, 8, 513, 0.0, 0.0), (5, 256, 1582, 0.1, 0.0),
         (16, 1032, 2051, 0.1, 0.2), (7, 2056, 700, 0.0, 0.3), (3, 4680, 9001, 0.0, 0.0), (16, 64, 70001, 0.0, 0.0)]


@pytest.mark.parametrize("T,h,V,smoothing,ignored", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_and_gradients(T, h, V, smoothing, ignored, dtype):
    if dtype == "f32":
        h += 1                                             # rows of odd length
    x, table, target = inputs(T, h, V, ignored, dtype)
    loss, losses, dx, dtable = O.linear_ce(x, table, target, smoothing)
    bl, bx, bt = bounds(x, table, target, smoothing, 0.0, dtype)
    n = max(1, ((target >= 0) & (target < V)).sum())
    got = call(x, table, target, smoothing, 0.0, dtype)
    close(from_dev(got["losses"]), losses, bl, "losses")
    close(got["loss"], loss, bl.sum() / n + 4 * U * abs(loss), "loss")
    close(from_dev(got["dx"]), dx, bx, "dx")
    close(from_dev(got["dtable"]), dtable, bt, "dtable")
    alone = call(x, table, target, smoothing, 0.0, dtype, grad=False)
    close(from_dev(alone["losses"]), losses, bl, "losses alone")
    close(alone["loss"], loss, bl.sum() / n + 4 * U * abs(loss), "loss alone")


@pytest.mark.parametrize("T,h,V,smoothing", [(1, 8, 1, 0.0), (1, 4096, 3001, 0.0), (2, 4680, 100, 0.1), (16, 72, 17, 0.1), (16, 136, 4100, 0.0), (7, 1000, 33, 0.3), (16, 4672, 50, 0.0),
                                             (16, 4808, 50, 0.0), (5, 16384, 20, 0.0)])
def test_loss_of_a_few_tokens(T, h, V, smoothing):
    """All of them, some, one and none counting; no bits by the quota; what the rows that do not count hold."""
    for ignored in (0.0, 0.5):
        x, table, target = inputs(T, h, V, ignored, "bf16")
        if ignored:
            target[T // 2] = 0
        loss, losses, _, _ = O.linear_ce(x, table, target, smoothing)
        bl = bounds(x, table, target, smoothing, 0.0, "bf16")[0]
        x[(target < 0) | (target >= V)] = np.nan
        got = call(x, table, target, smoothing, 0.0, "bf16", grad=False)
        close(from_dev(got["losses"]), losses, bl, "losses")
        close(got["loss"], loss, bl.sum() / max(1, (losses != 0).sum()) + 4 * U * abs(loss), "loss")
        for quota in (1, 40):
            again = call(x, table, target, smoothing, 0.0, "bf16", grad=False, quota=quota)
            assert torch.equal(again["losses"], got["losses"]) and again["loss"] == got["loss"]
    none = call(x, table, np.full(T, -1, dtype=np.int32), smoothing, 0.0, "bf16", grad=False)
    assert none["loss"] == 0 and not none["losses"].any()
    fixed = call(x, table, target, smoothing, 10.0, "bf16", grad=False)
    assert abs(fixed["loss"] - losses.sum() / 10) <= bl.sum() / 10 + 4 * U * abs(loss) * T


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_denominator_and_single_gradients(dtype):
    x, table, target = inputs(70, 96, 300, 0.3, dtype)
    loss, losses, dx, dtable = O.linear_ce(x, table, target, 0.1, 1000.0)
    bl, bx, bt = bounds(x, table, target, 0.1, 1000.0, dtype)
    both = call(x, table, target, 0.1, 1000.0, dtype)
    close(both["loss"], loss, bl.sum() / 1000 + 4 * U * abs(loss), "loss")
    close(from_dev(both["dx"]), dx, bx, "dx")
    close(from_dev(both["dtable"]), dtable, bt, "dtable")
    for want in (("dx",), ("dtable", "losses")):
        one = call(x, table, target, 0.1, 1000.0, dtype, want=want)
        assert one["loss"] == both["loss"]
        for name in ("dx", "dtable", "losses"):
            assert torch.equal(one[name], both[name]) if name in want else (one[name] == 77).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ignored_rows_may_hold_anything(dtype):
    x, table, target = inputs(300, 72, 130, 0.4, dtype)
    base = call(x, table, target, 0.1, 0.0, dtype)
    out = (target < 0) | (target >= 130)
    x[out] = np.where(np.arange(out.sum())[:, None] % 2 == 0, np.nan, np.inf)
    got = call(x, table, target, 0.1, 0.0, dtype)
    for name in ("losses", "dx", "dtable"):
        assert torch.equal(got[name], base[name])
    assert (got["dx"][torch.from_numpy(out).cuda()] == 0).all() and (got["losses"][torch.from_numpy(out).cuda()] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_counts(dtype):
    x, table, target = inputs(33, 64, 50, 1.0, dtype)
    got = call(x, table, target, 0.0, 0.0, dtype)
    assert got["loss"] == 0 and not got["losses"].any() and not got["dx"].any() and not got["dtable"].any()
    none = call(x[:0], table, target[:0], 0.0, 0.0, dtype)
    assert none["loss"] == 0 and not none["dtable"].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_logits(dtype):
    """Logits of +-10^4: the largest decides; and a token whose row is NaN takes its loss with it, no other token's."""
    x, table, target = inputs(20, 64, 500, 0.0, dtype)
    x, table = quantize(x * 30, dtype), quantize(table * 30, dtype)
    loss, losses, dx, _ = O.linear_ce(x, table, target)
    bl, bx, bt = bounds(x, table, target, 0.0, 0.0, dtype)
    got = call(x, table, target, 0.0, 0.0, dtype)
    close(from_dev(got["losses"]), losses, bl, "losses")
    # a probability is off by the error of its logits times itself: beyond the first order where that is not small
    close(from_dev(got["dx"]), dx, bx * 2, "dx")
    x[7] = np.nan
    x[8, 3] = np.inf
    bad = call(x, table, target, 0.0, 0.0, dtype)
    keep = [i for i in range(20) if i not in (7, 8)]
    assert torch.equal(bad["losses"][keep], got["losses"][keep]) and torch.equal(bad["dx"][keep], got["dx"][keep])
    assert torch.isnan(bad["losses"][[7, 8]]).all() and np.isnan(bad["loss"])


def test_gradients_are_those_of_the_loss():
    """Differences of the loss along directions, fp32: the third derivative of the loss along a direction d is bounded by the cube of the
    spread of d's logits; a loss is off by less than 2^-20 of 10."""
    x, table, target = inputs(50, 48, 400, 0.2, "f32")
    got = call(x, table, target, 0.1, 0.0, "f32")
    for seed, name in ((91, "dx"), (92, "dtable")):
        base = x if name == "dx" else table
        d = synth.normal(seed, base.shape)
        move = (d @ table.T) if name == "dx" else (x @ d.T)
        step = 0.02 / np.abs(move).max()
        ends = []
        for sign in (1, -1):
            moved = quantize(base + sign * step * d, "f32")
            ends.append(call(*((moved, table) if name == "dx" else (x, moved)), target, 0.1, 0.0, "f32", grad=False)["loss"])
        slope = (ends[0] - ends[1]) / (2 * step)
        third = (2 * np.abs(move).max()) ** 3 * step ** 2 / 6
        rounding = 2 * 10 * 2.0 ** -20 / (2 * step) + U * np.abs(base).max() * np.abs(from_dev(got[name])).sum() / step
        assert abs(slope - (from_dev(got[name]) * d).sum()) <= third + rounding + 1e-5 * abs(slope)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bits_do_not_depend_on_the_quota_or_the_stream(dtype):
    x, table, target = inputs(700, 192, 3001, 0.25, dtype)
    want = call(x, table, target, 0.1, 0.0, dtype)
    mb.pool_reserve(64, 0, mb.STRIPED)
    masked = mb.pool_get(64, 0, mb.STRIPED)
    for quota, stream in ((32, None), (200, None), (8, None), (1, None), (64, masked.native), (256, torch.cuda.Stream().cuda_stream)):
        got = call(x, table, target, 0.1, 0.0, dtype, quota=quota, stream=stream)
        assert got["loss"] == want["loss"] and all(torch.equal(got[k], want[k]) for k in ("losses", "dx", "dtable"))


@pytest.mark.parametrize("T,h,V,dtype", [(5, 256, 1582, "bf16"), (300, 72, 100, "bf16"), (40, 1104, 2000, "bf16"), (1500, 104, 2301, "f32"), (3, 520, 9001, "f32"), (2000, 64, 90, "f32")])
def test_bits_of_small_workloads_do_not_depend_on_the_quota(T, h, V, dtype):
    x, table, target = inputs(T, h, V, 0.2, dtype)
    want = call(x, table, target, 0.1, 0.0, dtype)
    for quota in (1, 24, 200):
        got = call(x, table, target, 0.1, 0.0, dtype, quota=quota)
        assert got["loss"] == want["loss"] and all(torch.equal(got[k], want[k]) for k in ("losses", "dx", "dtable"))


def test_pieces_of_tokens():
    """More tokens than a piece holds: the table's gradient is summed over pieces in fp32; two of one size, one, and one of few tokens.
    dz in bf16 is off by 2^-7 relative to a probability, so the whole in the 2-norm by that at most and by 2^-8 for the last rounding."""
    T, h, V = 8300, 64, 131000
    g = torch.Generator(device="cuda").manual_seed(3)
    table = (torch.randn((V, h), generator=g, device="cuda") * 0.25).bfloat16()
    x = torch.randn((T, h), generator=g, device="cuda").bfloat16()
    target = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    for ignored in (0, 300, 8210):
        target[:ignored] = -1
        loss, losses = torch.empty(1, device="cuda"), torch.empty(T, device="cuda")
        dx, dtable = torch.empty_like(x), torch.empty_like(table)
        scratch = torch.empty(mb.linear_ce_grad_scratch_bytes("bf16", T, h, V), device="cuda", dtype=torch.uint8)
        mb.op_linear_ce_grad(torch.cuda.current_stream().cuda_stream, 256, "bf16", T, h, V, 0.0, 0.0, target, x, table, loss, losses, dx, dtable, scratch)
        rows = x[ignored:].double()
        z = rows @ table.double().t().contiguous()
        lse = torch.logsumexp(z, 1)
        at = target[ignored:].long().unsqueeze(1)
        ref = lse - z.gather(1, at).squeeze(1)
        assert (losses[ignored:].double() - ref).abs().max() < 1e-4 and abs(float(loss) - float(ref.mean())) < 1e-5
        p = torch.exp(z - lse.unsqueeze(1))
        p.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float64))
        p /= T - ignored
        for got, want in ((dx[ignored:], p @ table.double()), (dtable, p.t().contiguous() @ rows)):
            assert (got.double() - want).norm() <= (2.0 ** -7 + 2.0 ** -8) * want.norm()
        assert not dx[:ignored].any()


def test_replays_of_a_captured_call():
    T, h, V = 300, 128, 999
    x, table, target = inputs(T, h, V, 0.3, "bf16")
    X, W, y = to_dev(x, "bf16"), to_dev(table, "bf16"), torch.from_numpy(target).cuda()
    loss, losses, dx, dtable = torch.empty(1, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(X), torch.empty_like(W)
    scratch = torch.empty(mb.linear_ce_grad_scratch_bytes("bf16", T, h, V), device="cuda", dtype=torch.uint8)
    run = lambda: mb.op_linear_ce_grad(torch.cuda.current_stream().cuda_stream, 256, "bf16", T, h, V, 0.0, 0.0, y, X, W, loss, losses, dx, dtable, scratch)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for turn in range(4):
        y.copy_(torch.from_numpy(np.roll(target, 17 * turn)))
        X.mul_(1.0 if turn % 2 else -1.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (loss, losses, dx, dtable)]
        for t in (loss, losses, dx, dtable):
            t.fill_(55.0)
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (loss, losses, dx, dtable)))
