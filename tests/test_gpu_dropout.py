"""Dropout from a counter-based generator: which elements stay, bit for bit, and their values.  x / (1 - p) is one product with a factor that is
rounded once (2^-24 each), the residual a sum (2^-24), and bf16's result off by 2^-8 of itself."""
import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2605_18710_amd import binding as mb, synth
from helpers import from_dev, quantize, to_dev

pytestmark = pytest.mark.gpu
SEED, OFFSET, SITE = 0x1234567890ABCDEF, (1 << 40) + 3, 11


def state(seed=SEED, offset=OFFSET):
    return torch.from_numpy(np.array([seed, offset], dtype=np.uint64).view(np.int64)).cuda()


def call(x, r, p, dtype, off=0, inplace=None, quota=256, site=SITE, rng=None):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n = len(x)

    def place(v):
        t = torch.full((n + 64 + off,), 9.0, device="cuda", dtype=dt)
        t[32 + off:32 + off + n] = to_dev(v, dtype)
        return t

    X, R, Y = place(x), place(r if r is not None else x), place(np.zeros(n))
    out = {None: Y, "x": X, "r": R}[inplace]
    part = lambda t: t[32 + off:32 + off + n]
    torch.cuda.synchronize()
    mb.op_dropout(None, quota, dtype, n, p, site, state() if rng is None else rng, part(X), part(R) if r is not None else None, part(out))
    torch.cuda.synchronize()
    assert (out[:32 + off] == 9).all() and (out[32 + off + n:] == 9).all()
    return part(out)


@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 5003])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values(n, residual, dtype):
    x, r = quantize(synth.normal(1, (n,)), dtype), quantize(4 * synth.normal(2, (n,)), dtype) if residual else None
    for p in (0.0, 0.1, 0.5, 0.97, 1.0):
        keep, scale = O.dropout_keeps(range(n), p, SITE, SEED, OFFSET)
        kept = np.where(keep, x * scale, 0.0)
        ref = kept + r if residual else kept
        bound = 2 * 2.0 ** -24 * np.abs(kept) + (1 + 2.0 ** -20) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref) + 2.0 ** -24 * np.abs(ref)
        for off, inplace in ((0, None), (0, "x"), (1, None), (3, "x")) + (((0, "r"),) if residual else ()):
            got = from_dev(call(x, r, p, dtype, off, inplace))
            assert (np.abs(got - ref) <= bound).all(), (p, off, inplace)
            if not residual:
                assert (got[~keep] == 0).all()


def test_the_mask_goes_by_the_element_alone():
    """The same places in both types, on every quota; other places at another site, offset or seed; a seed of all ones and a counter that wraps."""
    n = 4099
    one = np.ones(n)
    base = from_dev(call(one, None, 0.3, "f32")) != 0
    assert ((from_dev(call(one, None, 0.3, "bf16")) != 0) == base).all()
    assert ((from_dev(call(one, None, 0.3, "f32", quota=1)) != 0) == base).all()
    # moving the offset by one is moving the site by one
    assert ((from_dev(call(one, None, 0.3, "f32", site=SITE - 1, rng=state(SEED, OFFSET + 1))) != 0) == base).all()
    for rng, site in ((state(SEED + 1), SITE), (state(SEED, OFFSET + 1), SITE), (state(), SITE + 1), (state((1 << 64) - 1, (1 << 64) - 1), 5)):
        got = from_dev(call(one, None, 0.3, "f32", site=site, rng=rng)) != 0
        seed, offset = (int(v) for v in rng.cpu().numpy().view(np.uint64))
        assert (got == O.dropout_keeps(range(n), 0.3, site, seed, offset)[0]).all() and (got != base).any()
    # 0.3 of 4099, six standard deviations
    assert abs((~base).sum() - 0.3 * n) < 6 * np.sqrt(n * 0.21)


def test_what_is_dropped_leaves_nothing():
    n = 1000
    x = np.where(np.arange(n) % 2, np.nan, np.inf)
    keep, _ = O.dropout_keeps(range(n), 0.5, SITE, SEED, OFFSET)
    got = from_dev(call(x, None, 0.5, "bf16"))
    assert (got[~keep] == 0).all() and not np.isfinite(got[keep]).any()
    with_r = from_dev(call(x, np.full(n, 2.0), 0.5, "f32"))
    assert (with_r[~keep] == 2).all()


def test_replays_draw_anew():
    n = 70000
    x, y, rng = torch.randn(n, device="cuda"), torch.empty(n, device="cuda"), state()
    run = lambda: mb.op_dropout(torch.cuda.current_stream().cuda_stream, 256, "f32", n, 0.4, 1, rng, x, None, y)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    seen = []
    for turn in range(4):
        rng[1] += 10
        graph.replay()
        torch.cuda.synchronize()
        seen.append(y.clone())
        run()
        torch.cuda.synchronize()
        assert torch.equal(seen[-1], y)
    assert not any(torch.equal(a, b) for i, a in enumerate(seen) for b in seen[:i])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_past_the_caches_and_past_31_bits(dtype):
    n = (1 << 31) + 11 if dtype == "bf16" else (1 << 28) + 3
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    y = torch.empty_like(x)
    mb.op_dropout(torch.cuda.current_stream().cuda_stream, 256, dtype, n, 0.2, SITE, state(), x, None, y)
    torch.cuda.synchronize()
    for at in (0, 1 << 20, n // 2, n - 100):
        keep, _ = O.dropout_keeps(range(at, at + 100), 0.2, SITE, SEED, OFFSET)
        assert ((from_dev(y[at:at + 100]) != 0) == keep).all()
