"""The operators of a language module's training step on arrays whose offsets pass 32 bits, against 64 bits at sampled rows.  Tolerances: bf16's last rounding, 2^-8
of a value, and what the sums in fp32 leave (K 2^-24 of the terms' sizes, taken as their root mean square times sqrt(K) times 8)."""
import pytest
import torch

from paper_2605_18710_amd import binding as mb

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def close(got, ref, noise):
    """Element by element: 2^-8 of the value and `noise`."""
    assert torch.isfinite(got).all()
    assert ((got.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + noise).all()


def test_grouped_rows_past_4_gib():
    T, k, n, ends = 1_100_000, 2048, 256, [0, 5, 700_001, 1_099_990]
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randn((T, k), generator=g, device="cuda", dtype=torch.bfloat16)
    dY = torch.randn((T, n), generator=g, device="cuda", dtype=torch.bfloat16)
    W = torch.randn((3, k, n), generator=g, device="cuda", dtype=torch.bfloat16)
    at = torch.tensor(ends, dtype=torch.int32, device="cuda")
    Y = torch.full((T, n), 5.0, device="cuda", dtype=torch.bfloat16)
    mb.op_grouped_linear_fwd(stream(), 256, "bf16", T, 3, k, n, at, X, W, Y)
    rows = [0, 4, 5, 6, 350_000, 524_288, 700_000, 700_001, 1_048_575, 1_048_576, 1_099_989]
    group = [sum(r >= e for e in ends[1:3]) for r in rows]
    noise = 8 * 2.0 ** -24 * k
    for r, e in zip(rows, group):
        close(Y[r], X[r].double() @ W[e].double(), noise)
    assert (Y[ends[-1]:] == 5).all()
    del Y
    dX = torch.full((T, k), 5.0, device="cuda", dtype=torch.bfloat16)
    mb.op_grouped_linear_dgrad(stream(), 256, "bf16", T, 3, k, n, at, dY, W, dX)
    for r, e in zip(rows, group):
        close(dX[r], W[e].double() @ dY[r].double(), noise)
    assert (dX[ends[-1]:] == 5).all()
    del dX
    dW = torch.empty_like(W)
    mb.op_grouped_linear_wgrad(stream(), 256, "bf16", T, 3, k, n, at, X, dY, dW)
    for e in range(3):
        ref = torch.zeros((k, n), device="cuda", dtype=torch.float64)
        for a in range(ends[e], ends[e + 1], 50_000):
            b = min(a + 50_000, ends[e + 1])
            ref += X[a:b].double().t().contiguous() @ dY[a:b].double()
        close(dW[e], ref, 8 * 2.0 ** -24 * (ends[e + 1] - ends[e]))


def test_cross_entropy_past_4_gib_of_logits():
    T, h, V = 32_768, 8192, 65_000
    g = torch.Generator(device="cuda").manual_seed(2)
    X = torch.randn((T, h), generator=g, device="cuda", dtype=torch.bfloat16)
    table = torch.randn((V, h), generator=g, device="cuda", dtype=torch.bfloat16) * (2.0 * h ** -0.5)
    target = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    target[1::97] = -1
    loss, losses = torch.empty(1, device="cuda"), torch.empty(T, device="cuda")
    dX, dtable = torch.empty_like(X), torch.empty_like(table)
    size = mb.linear_ce_grad_scratch_bytes("bf16", T, h, V)
    assert size > 1 << 32
    scratch = torch.empty(size, device="cuda", dtype=torch.uint8)
    mb.op_linear_ce_grad(stream(), 256, "bf16", T, h, V, 0.0, 0.0, target, X, table, loss, losses, dX, dtable, scratch)
    counts = target >= 0
    D = int(counts.sum())
    assert not losses[~counts].any() and not dX[~counts].any()
    assert abs(float(loss) - float(losses.double().sum()) / D) < 1e-5
    t64 = table.double()
    at_target = (X.double() * t64[target.clamp(min=0).long()]).sum(1)
    lse = losses.double() + at_target                          # of the tokens that count
    rows = torch.tensor([0, 2, 3, 255, 256, 16_384, 32_000, 32_766, 32_767], device="cuda")
    rows = rows[counts[rows]]
    z = X[rows].double() @ t64.t().contiguous()
    assert (torch.logsumexp(z, 1) - lse[rows]).abs().max() < 2e-5
    p = torch.exp(z - lse[rows].unsqueeze(1))
    p[torch.arange(len(rows)), target[rows].long()] -= 1.0
    # dz is off by 2^-8 of itself, probabilities by 2^-11 of themselves
    off = (2.0 ** -8 + 2.0 ** -11 + 2e-5) * p.abs()
    close(dX[rows], p @ t64 / D, off @ t64.abs() / D)
    words = torch.tensor([0, 1, 63, 64, 32_767, 64_998, 64_999], device="cuda")
    q = torch.exp(X.double() @ t64[words].t().contiguous() - lse.unsqueeze(1))
    q[target.unsqueeze(1) == words.to(torch.int32)] -= 1.0
    q[~counts] = 0
    close(dtable[words], q.t().contiguous() @ X.double() / D, (2.0 ** -8 + 2.0 ** -11 + 2e-5) * (q.abs().t().contiguous() @ X.double().abs()) / D)
