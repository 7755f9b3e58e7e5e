"""Products grouped by expert against the definition in 64 bits.  A sum of K products in fp32 is off by (K + 2) 2^-24 sum |a b| at most, and a
bf16 result by 2^-8 of itself besides."""
import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2605_18710_amd import binding as mb, synth
from helpers import from_dev, quantize, to_dev

pytestmark = pytest.mark.gpu
FORMS = ("fwd", "dgrad", "wgrad")


def operands(form, T, groups, k, n, dtype, seed=3):
    a = quantize(synth.normal(seed, (T, n if form == "dgrad" else k)), dtype)
    b = quantize(synth.normal(seed + 1, (T, n) if form == "wgrad" else (groups, k, n)), dtype)
    return a, b


def call(form, offsets, k, n, a, b, dtype, quota=256, stream=None, off=0):
    T, groups = len(a), len(offsets) - 1
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    shape = {"fwd": (T, n), "dgrad": (T, k), "wgrad": (groups, k, n)}[form]

    def place(v):                                     # `off` elements behind a 256-byte boundary, with NaN all around
        t = torch.full((v.size + 512 + off,), float("nan"), device="cuda", dtype=dt)
        t[256 + off:256 + off + v.size] = to_dev(v, dtype).reshape(-1)
        return t[256 + off:256 + off + v.size]

    A, B = place(a), place(b)
    size = int(np.prod(shape))
    out = torch.full((size + 512 + off,), 7.0, device="cuda", dtype=dt)
    C = out[256 + off:256 + off + size]
    at = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    getattr(mb, "op_grouped_linear_" + form)(stream, quota, dtype, T, groups, k, n, at, A, B, C)
    torch.cuda.synchronize()
    assert (out[:256 + off] == 7).all() and (out[256 + off + size:] == 7).all()
    return C.reshape(shape)


def check(form, offsets, k, n, dtype, T, off=0):
    groups = len(offsets) - 1
    a, b = operands(form, T, groups, k, n, dtype)
    got = call(form, offsets, k, n, a, b, dtype, off=off)
    sevens = np.full(got.shape, 7.0)
    ref = O.grouped_linear(form, offsets, a, b, sevens)
    size = O.grouped_linear(form, offsets, np.abs(a), np.abs(b), sevens * 0)
    K = {"fwd": k, "dgrad": n, "wgrad": max(np.diff(offsets), default=0)}[form]
    bound = (K + 2) * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0)
    d = np.abs(from_dev(got) - ref)
    assert np.isfinite(d).all() and (d <= bound).all(), float((d / np.maximum(bound, 1e-300)).max())


CASES = [  # offsets, k, n, T
    ([0, 1], 64, 64, 1), ([0, 3, 3, 5], 8, 16, 5), ([0, 130, 130, 131, 400], 72, 264, 400), ([0, 256, 512], 128, 256, 512), ([2, 9, 40], 200, 136, 50),
    ([0, 0, 0, 0], 64, 72, 4), ([0, 257, 300, 301, 812], 136, 520, 812), ([0, 700], 320, 96, 700), ([0] + list(range(0, 1024)), 16, 24, 1100),
    # few rows to a group: up to 16, 32, 64 at a time, and groups of many more among them
    ([0, 16, 33, 33, 40], 1032, 72, 41), ([0, 100, 100, 100, 100, 100, 100, 101], 264, 136, 101), ([0, 30, 70], 520, 200, 80), ([0, 1, 70, 100], 2000, 64, 100), ([0, 50, 130], 136, 1048, 128),
    # weight gradients of few tiles over many rows, and of many tiles
    ([0, 3000, 3000, 5100], 104, 136, 5100), ([0, 1, 1000], 72, 8, 1000), ([0, 120, 300], 1100, 1304, 300)]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offsets,k,n,T", CASES)
def test_products(form, dtype, offsets, k, n, T):
    check(form, offsets, k, n, dtype, T)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_odd_sizes_and_alignments(form, dtype):
    check(form, [0, 33, 33, 70], 33, 51, dtype, 71)
    check(form, [0, 33, 33, 70], 40, 24, dtype, 70, off=1)


# rows, columns and contraction of a product that take tiles of 64 x 64, 64 x 128, 128 x 64 and 128 x 128 in fp32, with ragged ends of each; a contraction of one piece;
# few rows over a long one
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rows,columns,depth", [(300, 1800, 100), (1500, 900, 100), (2100, 900, 100), (1500, 2300, 100), (1500, 2300, 4), (516, 2052, 516), (2108, 908, 164), (18, 404, 4168), (100, 72, 3004)])
def test_fp32_tiles(form, rows, columns, depth):
    T, k, n = {"fwd": (rows, depth, columns), "dgrad": (rows, columns, depth), "wgrad": (depth, rows, columns)}[form]
    check(form, [0, T], k, n, "f32", T)
    check(form, [1, T // 2, T // 2, T - 2], k, n, "f32", T)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rows,columns,depth", [(1500, 2300, 100), (300, 1800, 100), (18, 404, 4168)])
def test_bits_of_fp32_tiles_do_not_depend_on_the_quota(form, rows, columns, depth):
    T, k, n = {"fwd": (rows, depth, columns), "dgrad": (rows, columns, depth), "wgrad": (depth, rows, columns)}[form]
    a, b = operands(form, T, 2, k, n, "f32")
    want = call(form, [0, T // 3, T], k, n, a, b, "f32")
    for quota in (1, 40, 200):
        assert torch.equal(call(form, [0, T // 3, T], k, n, a, b, "f32", quota), want)


@pytest.mark.parametrize("form", FORMS)
def test_no_group_reads_another(form):
    """NaN in rows of no group and in one group's rows or matrix: the other groups' results have the bits that they have without."""
    k, n, offsets, T = 72, 104, [3, 60, 60, 200, 330], 340
    a, b = operands(form, T, 4, k, n, "bf16")
    base = call(form, offsets, k, n, a, b, "bf16")
    a, b = a.copy(), b.copy()
    a[:3] = a[330:] = np.nan
    a[60:200] = np.inf
    if form == "wgrad":
        b[:3] = b[330:] = b[60:200] = np.nan
    else:
        b[2] = np.nan                                  # of rows 60 .. 199
        b[1] = np.inf                                  # of no row
    got = call(form, offsets, k, n, a, b, "bf16")
    if form == "wgrad":
        assert all(torch.equal(got[g], base[g]) for g in (0, 1, 3)) and not torch.isfinite(got[2]).any()
    else:
        keep = torch.tensor([r for r in range(T) if not 60 <= r < 200])
        assert torch.equal(got[keep], base[keep]) and not torch.isfinite(got[60:200]).any()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bits_do_not_depend_on_the_quota(form, dtype):
    offsets = [0, 300, 301, 301, 1000, 1500]
    a, b = operands(form, 1500, 5, 264, 520, dtype)
    want = call(form, offsets, 264, 520, a, b, dtype)
    mb.pool_reserve(64, 0, mb.STRIPED)
    for quota, stream in ((1, None), (8, None), (200, None), (64, mb.pool_get(64, 0, mb.STRIPED).native)):
        assert torch.equal(call(form, offsets, 264, 520, a, b, dtype, quota, stream), want)


@pytest.mark.parametrize("form", FORMS)
def test_offsets_out_of_order_stay_inside(form):
    """Not a valid call, but one that the kernels' own bounds have to hold: nothing outside the output is written (call checks its surroundings)."""
    a, b = operands(form, 100, 4, 64, 72, "bf16")
    call(form, [-50, 90, 20, 5000, 2 ** 31 - 1], 64, 72, a, b, "bf16")
    call(form, [-50, 90, 20, 5000, 2 ** 31 - 1], 64, 72, a, b, "f32")


def test_replays_of_captured_calls():
    """One graph with all three forms; sizes of the groups move between replays."""
    T, groups, k, n = 500, 6, 128, 192
    a, w = operands("fwd", T, groups, k, n, "bf16")
    X, W, dY = to_dev(a, "bf16"), to_dev(w, "bf16"), to_dev(synth.normal(9, (T, n)), "bf16")
    at = torch.zeros(groups + 1, dtype=torch.int32, device="cuda")
    Y, dX, dW = torch.empty_like(dY), torch.empty_like(X), torch.empty_like(W)

    def run():
        s = torch.cuda.current_stream().cuda_stream
        mb.op_grouped_linear_fwd(s, 256, "bf16", T, groups, k, n, at, X, W, Y)
        mb.op_grouped_linear_dgrad(s, 256, "bf16", T, groups, k, n, at, dY, W, dX)
        mb.op_grouped_linear_wgrad(s, 256, "bf16", T, groups, k, n, at, X, dY, dW)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for offsets in ([0, 10, 20, 300, 300, 499, 500], [0, 0, 0, 0, 0, 0, 500], [5, 100, 200, 300, 400, 450, 460]):
        at.copy_(torch.tensor(offsets, dtype=torch.int32))
        outs = []
        for go in (graph.replay, run):
            for t in (Y, dX, dW):
                t.fill_(3.0)
            go()
            torch.cuda.synchronize()
            outs.append([t.clone() for t in (Y, dX, dW)])
        assert all(torch.equal(p, q) for p, q in zip(*outs))
