"""Cross entropy of more tokens than a piece holds: later pieces add to the table's gradient, the last one that has tokens finishes it, pieces behind it have none.  References in 64 bits on
the GPU, a stretch of tokens at a time; bounds element by element, from the roundings that test_gpu_linear_ce.py lists."""
import pytest
import torch

from paper_2605_18710_amd import binding as mb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
V = 131000


def reference(x, table, target, smoothing, dtype):
    """Of the tokens that count: losses, dx, and dtable, with their bounds."""
    W = table.double()
    wa = W.abs()
    D, h = len(target), x.shape[1]
    losses, bl, dx, bx = [], [], [], []
    dtable, bt, size = (torch.zeros_like(W) for _ in range(3))
    store, kept = (2.0 ** -8, 2.0 ** -11) if dtype == "bf16" else (0.0, 0.0)
    last = 2.0 ** -8 if dtype == "bf16" else U
    for a in range(0, D, 1000):
        r, y = x[a:a + 1000].double(), target[a:a + 1000].long().unsqueeze(1)
        z = r @ W.t().contiguous()
        E = (h + 2) * U * (r.abs() @ wa.t().contiguous()).amax(1, keepdim=True)
        lse, top, most = torch.logsumexp(z, 1, keepdim=True), z.amax(1, keepdim=True), z.abs().amax(1, keepdim=True)
        rel = 2 * E + (64 + V / 512) * 2 * U + 8 * U * lse.abs() + 4 * U * most
        losses.append((lse - (1 - smoothing) * z.gather(1, y) - smoothing * z.mean(1, keepdim=True)).squeeze(1))
        bl.append((rel + 8 * U * (lse.abs() + most)).squeeze(1))
        p = torch.exp(z - lse)
        floor = kept * 2.0 ** -14 * torch.exp(top - lse)
        del z
        dz = p - smoothing / V
        dz.scatter_add_(1, y, torch.full_like(lse, smoothing - 1.0))
        off = ((rel + 4 * U + kept) * p + floor) * (1 + store) + store * dz.abs() + 4 * U * smoothing
        off.scatter_add_(1, y, torch.full_like(lse, 4 * U))
        del p
        dx.append(dz @ W / D)
        full = off + (V + 2) * U * (dz.abs() + off)
        bx.append((full @ wa * (1 + last) + last * (dz.abs() @ wa)) / D)
        del full
        off += (D + 8) * U * (dz.abs() + off)
        dtable += dz.t().contiguous() @ r / D
        bt += off.t().contiguous() @ r.abs() / D
        size += dz.abs().t().contiguous() @ r.abs() / D
    return torch.cat(losses), torch.cat(bl), torch.cat(dx), torch.cat(bx), dtable, bt * (1 + last) + last * size


def close(got, ref, bound, what):
    assert torch.isfinite(got).all(), what
    d = (got.double() - ref).abs()
    assert (d <= bound).all(), (what, float((d / bound.clamp(min=1e-300)).max()))


# T * (V rounded up to 64) is past what one piece holds: 2^30 + 2 V h (bf16), 2^29 (fp32); three pieces each.  Tokens that count: all three pieces; two of them, or one; a few; none
@pytest.mark.parametrize("dtype,T,h,counted", [("bf16", 17000, 64, (17000, 9000, 5000, 30, 0)), ("f32", 9300, 36, (9300, 4000, 7, 0)), ("f32", 9300, 35, (9300, 3400))])
def test_pieces(dtype, T, h, counted):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    assert T * 131008 > ((1 << 30) + 2 * V * h if dtype == "bf16" else 1 << 29)
    size = mb.linear_ce_grad_scratch_bytes(dtype, T, h, V)
    assert size < T * 131008 * (2 if dtype == "bf16" else 4)                     # less than one piece of all tokens takes
    g = torch.Generator(device="cuda").manual_seed(3)
    table = (torch.randn((V, h), generator=g, device="cuda") * 0.25).to(dt)
    x = torch.randn((T, h), generator=g, device="cuda").to(dt)
    every = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    order = torch.randperm(T, generator=g, device="cuda")
    scratch = torch.full((size,), 0xFF, device="cuda", dtype=torch.uint8)
    forward = torch.full((mb.linear_ce_fwd_scratch_bytes(dtype, T, h, V),), 0xFF, device="cuda", dtype=torch.uint8)
    stream = torch.cuda.current_stream().cuda_stream
    for n in counted:
        smoothing = 0.1 if n == counted[0] else 0.0
        out = order[n:]
        at = torch.sort(order[:n]).values
        target = every.clone()
        target[out] = -100
        X = x.clone()
        X[out] = float("nan")
        loss, losses = torch.full((1,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
        dx, dtable = torch.full_like(X, 7.0), torch.full_like(table, 7.0)
        mb.op_linear_ce_grad(stream, 256, dtype, T, h, V, smoothing, 0.0, target, X, table, loss, losses, dx, dtable, scratch)
        assert not losses[out].any() and not dx[out].any()
        if n == 0:
            assert float(loss) == 0 and not dtable.any()
            continue
        want, bl, wx, bx, wt, bt = reference(x[at], table, every[at], smoothing, dtype)
        close(losses[at], want, bl, (n, "losses"))
        close(loss.double(), want.mean(), bl.mean() + 4 * U * want.mean().abs(), (n, "loss"))
        close(dx[at], wx, bx, (n, "dx"))
        close(dtable, wt, bt, (n, "dtable"))
        del wt, bt
        alone, each = torch.full((1,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
        mb.op_linear_ce_fwd(stream, 256, dtype, T, h, V, smoothing, 0.0, target, X, table, alone, each, forward)
        close(each[at], want, bl, (n, "losses alone"))
        close(alone.double(), want.mean(), bl.mean() + 4 * U * want.mean().abs(), (n, "loss alone"))
        # one gradient at a time has the bits of both together
        one = torch.full_like(X, 7.0)
        mb.op_linear_ce_grad(stream, 40, dtype, T, h, V, smoothing, 0.0, target, X, table, loss, None, one, None, scratch)
        assert torch.equal(one, dx)
        one = torch.full_like(table, 7.0)
        mb.op_linear_ce_grad(stream, 40, dtype, T, h, V, smoothing, 0.0, target, X, table, loss, None, None, one, scratch)
        assert torch.equal(one, dtable)
