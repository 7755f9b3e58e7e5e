"""The operators around a layer's products on arrays whose offsets pass 32 bits: rows and blocks at the end against the plain definitions in
64 bits (the bounds are those of the small tests)."""
import numpy as np
import pytest
import torch

from oracle import operators as P
from helpers import from_dev
from test_gpu_pack8 import act_ref
from test_gpu_qk_rope import U, last, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_18710_amd import binding
    binding.lib()
    return binding


def filled(n, seed):
    """n bf16 numbers on the GPU: a long period of normal numbers."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    piece = torch.randn((1 << 22) + 32 * 7, generator=g, device="cuda").bfloat16()
    return piece.repeat((n + piece.numel() - 1) // piece.numel())[:n].contiguous()


def test_rows_behind_four_gigabytes(mb):
    T, H, Hkv, d = 9000001, 2, 1, 64
    w = (H + 2 * Hkv) * d
    assert T * w * 2 > 1 << 32
    x, dy = filled(T * w, 1).view(T, w), filled(T * w, 2).view(T, w)
    pos = torch.stack((torch.arange(T, device="cuda"), torch.arange(T, device="cuda") % 1000)).to(torch.int32).contiguous()
    table = torch.empty(mb.rope_axes_table_bytes(d), dtype=torch.uint8, device="cuda")
    mb.op_rope_axes_table(None, 256, d, (16, 16), "own", 100.0, table)
    axis, freq = P.pair_table(d, (16, 16), "own", 100.0)
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    scratch = torch.empty(mb.qk_norm_rope_bwd_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    grads = [torch.empty_like(gain) for _ in range(2)]
    head = (T, H, Hkv, d, 1e-5, "halves", 2, pos, table)
    for rows in (slice(0, 40), slice(T - 40, T)):
        mb.op_qk_norm_rope_fwd(None, 256, "bf16", "rmsnorm", *head, x, gain, None, gain, None, y)
        torch.cuda.synchronize()
        xs = from_dev(x[rows]).reshape(40, H + 2 * Hkv, d)
        n, xhat, rstd = P.head_norm(xs[:, :3], "rmsnorm", 1e-5, 1.0)
        ref = P.rotate(n, pos[:, rows].cpu().numpy(), axis, freq, "halves")
        got = from_dev(y[rows]).reshape(40, 4, d)
        # the oracle's own angles, up to 10^7, are exact to 2^-29
        within(got[:, :3], ref, last("bf16", ref) + 64 * U * (np.abs(n).max(2, keepdims=True) + 1), "y")
        assert np.array_equal(got[:, 3], xs[:, 3])
        mb.op_qk_norm_rope_bwd(None, 256, "bf16", "rmsnorm", *head, x, gain, gain, dy, y, grads[0], None, grads[1], None, scratch)
        torch.cuda.synchronize()
        ds = from_dev(dy[rows]).reshape(40, 4, d)
        g = P.rotate(ds[:, :3], pos[:, rows].cpu().numpy(), axis, freq, "halves", -1)
        dx = P.head_norm_bwd(g, xhat, rstd, "rmsnorm", 1.0)[0]
        size = rstd * 2 * np.abs(ds[:, :3]).max(2, keepdims=True) * (2 + np.abs(xhat).max(2, keepdims=True))
        got = from_dev(y[rows]).reshape(40, 4, d)
        within(got[:, :3], dx, last("bf16", dx) + 64 * U * size, "dx")
        assert np.array_equal(got[:, 3], ds[:, 3])
    assert all(torch.isfinite(v.float()).all() for v in grads)


def test_packed_behind_four_gigabytes(mb):
    n = (1 << 32) + 32 * 1000 + 17
    x = filled(n, 3)
    q, scale = torch.empty(n, dtype=torch.int8, device="cuda"), torch.empty(mb.pack8_scale_bytes(n), dtype=torch.uint8, device="cuda")
    mb.op_pack8(None, 256, "bf16", n, x, q, scale)
    torch.cuda.synchronize()
    for first in (0, n // 32 * 32 - 32 * 1000):
        part = slice(first, min(n, first + 32 * 1000 + 17))
        q_ref, byte_ref = P.pack8(from_dev(x[part]))
        assert np.array_equal(q[part].cpu().numpy(), q_ref)
        assert np.array_equal(scale[first // 32:first // 32 + byte_ref.size].cpu().numpy()[:1000], byte_ref[:1000])
    back = x
    back.zero_()
    mb.op_unpack8(None, 256, "bf16", n, q, scale, back)
    torch.cuda.synchronize()
    part = slice(n // 32 * 32 - 32 * 1000, n)
    assert np.array_equal(from_dev(back[part]), P.unpack8(q[part].cpu().numpy(), scale[part.start // 32:].cpu().numpy()))


@pytest.mark.parametrize("f", [32768, 32744])
def test_activation_behind_four_gigabytes(mb, f):
    T = 66000
    assert T * 2 * f > 1 << 32
    z, da = filled(T * 2 * f, 4).view(T, 2 * f), filled(T * f, 5).view(T, f)
    a, again, dz = torch.empty_like(da), torch.empty_like(da), torch.empty_like(z)
    q, scale = torch.empty(T * 2 * f, dtype=torch.int8, device="cuda"), torch.empty(mb.pack8_scale_bytes(T * 2 * f), dtype=torch.uint8, device="cuda")
    mb.op_act_fwd_pack8(None, 256, "bf16", "swiglu", T, f, z, a, q, scale)
    mb.op_act_bwd_pack8(None, 256, "bf16", "swiglu", T, f, q, scale, da, dz, again)
    torch.cuda.synchronize()
    for rows in (slice(0, 4), slice(T - 4, T)):            # four rows are whole blocks
        zs, ds = from_dev(z[rows]), from_dev(da[rows])
        kept = P.unpack8(*P.pack8(zs)).reshape(zs.shape)
        a_ref, _, a_tol, _ = act_ref("swiglu", zs, ds)
        again_ref, dz_ref, again_tol, dz_tol = act_ref("swiglu", kept, ds)
        within(from_dev(a[rows]), a_ref, last("bf16", a_ref) + a_tol, "a")
        within(from_dev(again[rows]), again_ref, last("bf16", again_ref) + again_tol, "again")
        within(from_dev(dz[rows]), dz_ref, last("bf16", dz_ref) + dz_tol, "dz")


def test_gains_gradients_over_five_million_tokens(mb):
    """Sums over all tokens in 32 bits, against 64, of gradients that lie on the normalised rows: the sums grow with the tokens, so that a partition, or a wave's
    share of one (1 of 4096), that were missing would be 2e-3 or 2e-4 of them.  A wave adds up 1221 tokens, all heads at once; then come 3 joins of heads, 8 waves
    and slices of 64 partitions: below 1400 additions in a row, of terms off by 40 u, 1440 u in all (9e-5)."""
    T, H, Hkv, d = 5000001, 2, 1, 64
    w = (H + 2 * Hkv) * d
    assert T * w * 4 > 1 << 32
    x = filled(T * w, 6).view(T, w).float()
    pos = torch.stack((torch.arange(T, device="cuda") % 4096, torch.arange(T, device="cuda") % 1000)).to(torch.int32).contiguous()
    table = torch.empty(mb.rope_axes_table_bytes(d), dtype=torch.uint8, device="cuda")
    mb.op_rope_axes_table(None, 256, d, (16, 16), "own", 100.0, table)
    axis, freq = (torch.from_numpy(v).cuda() for v in P.pair_table(d, (16, 16), "own", 100.0))
    one = torch.ones(d, device="cuda")
    head = (T, H, Hkv, d, 1e-5, "halves", 2, pos, table)
    y, grads = torch.empty_like(x), [torch.empty_like(one) for _ in range(4)]
    mb.op_qk_norm_rope_fwd(None, 256, "f32", "layernorm", *head, x, one, one, one, one, y)          # turned: xhat + 1
    scratch = torch.empty(mb.qk_norm_rope_bwd_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    mb.op_qk_norm_rope_bwd(None, 256, "f32", "layernorm", *head, x, one, one, y, torch.empty_like(x), grads[0], grads[2], grads[1], grads[3], scratch)
    sums = torch.zeros((4, 2, d), dtype=torch.float64, device="cuda")              # [gain q, gain k, shift q, shift k][sum, sum of sizes]
    for first in range(0, T, 1 << 20):
        rows = slice(first, min(T, first + (1 << 20)))
        xs, ds = (v[rows].view(-1, H + 2 * Hkv, d)[:, :H + Hkv].double() for v in (x, y))
        angle = (pos[:, rows].double()[axis].t() * freq)[:, None]
        p, q = ds.chunk(2, 2)
        g = torch.cat((p * torch.cos(angle) + q * torch.sin(angle), q * torch.cos(angle) - p * torch.sin(angle)), 2)
        xhat = xs - xs.mean(2, keepdim=True)
        xhat = xhat * torch.rsqrt((xhat * xhat).mean(2, keepdim=True) + 1e-5)
        for i, term in enumerate(((g * xhat)[:, :H], (g * xhat)[:, H:], g[:, :H], g[:, H:])):
            sums[i, 0] += term.sum((0, 1))
            sums[i, 1] += term.abs().sum((0, 1))
    for i, got in enumerate(grads):
        heads = Hkv if i % 2 else H
        # what a missing share is measured against: mean xhat^2 + xhat or xhat + 1 of a column's 131079 different numbers, off by sqrt(3 / 131079) = 0.005, six of these
        assert float((sums[i, 0] / (T * heads) - 1).abs().max()) < 0.03
        over = (got.double() - sums[i, 0]).abs() - 1440 * U * sums[i, 1]
        assert float(over.max()) <= 0, (i, float(over.max()))
