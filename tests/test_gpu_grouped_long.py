"""fp32 products of a long contraction: what rounding leaves is that of short chains.  A sum of n products of normal values, kept in a chain of c at a time whose sums are added in turn: the partial
sums of a chain of c are of size sqrt(i), each rounded by up to u = 2^-24 of itself, so the chain is off by u c / sqrt(2) at most in the root mean square if the roundings are independent, all n / c of
them by u sqrt(n c / 2), and the additions of their sums by u n / sqrt(2 c); relative to the result, sqrt(n): u (sqrt(c / 2) + sqrt(n / (2 c))).  A rounding's own root mean square is below u / sqrt(3) and
a matrix instruction rounds a few products together, so single chains of n measure at about 0.2 u sqrt(n); c is 2048 at most."""
import math

import pytest
import torch

from paper_2605_18710_amd import binding as mb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def limit(n, c=2048):
    return U * (math.sqrt(c / 2) + math.sqrt(n / (2 * c)))


def rms(t):
    return float(t.double().square().mean().sqrt())


# rows, columns: tiles of 32 x 32, 64 x 64, 64 x 128, 128 x 64, 128 x 128; the loops of rows that are not whole pieces
@pytest.mark.parametrize("k,n", [(64, 96), (640, 1000), (1032, 1728), (1728, 1032), (2048, 2048), (33, 51), (2049, 2047)])
def test_weight_gradient_over_many_rows(k, n):
    T = 500_000
    g = torch.Generator(device="cuda").manual_seed(k + n)
    X, dY = (torch.randn((T, w), generator=g, device="cuda") for w in (k, n))
    at = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    dW = torch.empty((1, k, n), device="cuda")
    mb.op_grouped_linear_wgrad(torch.cuda.current_stream().cuda_stream, 256, "f32", T, 1, k, n, at, X, dY, dW)
    some = torch.cat([torch.arange(32), torch.arange(n - 32, n)]).unique().cuda()
    ref = torch.zeros((k, len(some)), device="cuda", dtype=torch.float64)
    for a in range(0, T, 50_000):
        ref += X[a:a + 50_000].double().t().contiguous() @ dY[a:a + 50_000, some].double()
    off = rms(dW[0][:, some].double() - ref) / math.sqrt(T)
    print("off by %.3g of the result, %.2f of the limit" % (off, off / limit(T)))
    assert off <= limit(T)


@pytest.mark.parametrize("form", ["fwd", "dgrad"])
@pytest.mark.parametrize("T,columns,odd", [(40, 64, 0), (700, 1000, 0), (2100, 1028, 0), (2048, 2048, 0), (70, 51, 1), (1500, 1203, 1)])
def test_products_over_many_columns(form, T, columns, odd):
    K = 200_000 + odd
    k, n = (K, columns) if form == "fwd" else (columns, K)
    g = torch.Generator(device="cuda").manual_seed(T)
    A = torch.randn((T, K), generator=g, device="cuda")
    W = torch.randn((1, k, n), generator=g, device="cuda")
    at = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    C = torch.empty((T, columns), device="cuda")
    getattr(mb, "op_grouped_linear_" + form)(torch.cuda.current_stream().cuda_stream, 256, "f32", T, 1, k, n, at, A, W, C)
    rows = torch.cat([torch.arange(20), torch.arange(T - 20, T)]).unique().cuda()
    a, w = A[rows].double(), W[0].double()
    ref = a @ (w if form == "fwd" else w.t().contiguous())
    off = rms(C[rows].double() - ref) / math.sqrt(K)
    print("off by %.3g of the result, %.2f of the limit" % (off, off / limit(K)))
    assert off <= limit(K)


@pytest.mark.parametrize("form", ["fwd", "dgrad", "wgrad"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_no_whole_pieces(form, dtype):
    """Enough of them for tiles of 64 x 64.  Element by element: (K + 2) u sum |a b|, and bf16's last rounding."""
    T, k, n, ends = 2600, 1023, 1025, [3, 700, 700, 2001, 2597]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(6)
    make = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dt)
    A = make(T, n if form == "dgrad" else k)
    B = make(T, n) if form == "wgrad" else make(4, k, n)
    at = torch.tensor(ends, dtype=torch.int32, device="cuda")
    C = torch.full({"fwd": (T, n), "dgrad": (T, k), "wgrad": (4, k, n)}[form], 7.0, device="cuda", dtype=dt)
    getattr(mb, "op_grouped_linear_" + form)(torch.cuda.current_stream().cuda_stream, 256, dtype, T, 4, k, n, at, A, B, C)
    for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
        a = A[lo:hi].double()
        if form == "wgrad":
            left, right, got = a.t().contiguous(), B[lo:hi].double(), C[e]
        else:
            w = B[e].double()
            left, right, got = a, w if form == "fwd" else w.t().contiguous(), C[lo:hi]
        ref = left @ right
        bound = (left.shape[1] + 2) * U * (left.abs() @ right.abs()) + (2.0 ** -8 * ref.abs() if dtype == "bf16" else 0.0)
        assert ((got.double() - ref).abs() <= bound).all()
    if form != "wgrad":
        assert (C[:3] == 7).all() and (C[2597:] == 7).all()


@pytest.mark.parametrize("dtype,k,n", [("bf16", 64, 72), ("bf16", 2048, 1024), ("f32", 64, 72), ("f32", 33, 51), ("f32", 2048, 2048)])
def test_weight_gradient_of_no_rows(dtype, k, n):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    at = torch.zeros(4, dtype=torch.int32, device="cuda")
    none = torch.empty((0, k), device="cuda", dtype=dt), torch.empty((0, n), device="cuda", dtype=dt)
    dW = torch.full((3, k, n), 7.0, device="cuda", dtype=dt)
    mb.op_grouped_linear_wgrad(torch.cuda.current_stream().cuda_stream, 256, dtype, 0, 3, k, n, at, *none, dW)
    assert not dW.any()
