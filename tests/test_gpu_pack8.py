"""GPU parity of the activation checkpoints in 8 bits: the packed bytes and what they stand for, bit for bit, against the plain
definition; the activations' and the weight gradient's backward passes from them against 64 bits.

Bounds, u = 2^-24; a bf16 result is off by 2^-8 of its size besides.  GELU: the distribution is off by 4 u (erf by 1.5e-7 = 2.5 u, halved, and roundings), so the
result by at most 8 u |z|, its derivative by 8 u (1 + |z|).  A logistic function is off by 6 u (exponential 2 u, its correction 1 u, sum 1 u, reciprocal
2 u).  Tanh form: with its argument's 4 u, at most 0.28 of them in the result, 12 u |z|; its derivative meets z^3, at most 8.7 before the function is 1: 128 u (1 + |z|).
SwiGLU: two more products, 16 u of the result's size (and 1e-36 where exp overflows); the gate's derivative is s (1 + gate e s), where e s is off by
13 u and the rest by 9 u: 24 u of the sum of both terms' sizes.  Weight gradient: T additions and products, T u of the sum of magnitudes."""
import math

import numpy as np
import pytest
import torch

from oracle import operators as P
from paper_2605_18710_amd import synth
from helpers import from_dev, quantize, to_dev
from test_gpu_qk_rope import Framed, bits, last, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_18710_amd import binding
    binding.lib()
    return binding


class Bytes:
    """n bytes `shift` behind a 16-byte boundary with a frame that must stay."""

    def __init__(self, n, shift=0):
        self.flat = torch.full((n + 128,), 77, dtype=torch.uint8, device="cuda")
        self.at = slice(64 + shift, 64 + shift + n)
        self.t = self.flat[self.at]

    def framed(self):
        f = self.flat.clone()
        f[self.at] = 77
        return bool((f == 77).all())

    def host(self, kind):
        return self.t.cpu().numpy().view(kind).copy()


def values(dtype, n, seed=7000):
    """Wide in size, with ties, zeros, blocks of tiny numbers, of the type's largest, and of NaN and infinities."""
    x = synth.normal(seed, (n,)) * np.exp(np.repeat(synth.normal(seed + 1, (n // 32 + 1,), 0.0, 8.0), 32)[:n])
    x[::7] = np.round(x[::7] * 2) / 2
    for b, v in ((3, 0.0), (5, 1e-39), (6, 1e-45), (7, 127.5), (8, 255.0), (9, 3.3e38), (10, 2.0 ** -120)):
        x[32 * b:32 * b + 32] *= 0
        x[32 * b:32 * b + 32] += v * np.linspace(-1, 1, 32)[:max(0, min(32, n - 32 * b))]
    for i, v in ((32 * 12 + 3, np.nan), (32 * 13, np.inf), (32 * 14 + 31, -np.inf)):
        if i < n:
            x[i] = v
    with np.errstate(over="ignore"):
        return quantize(x, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 1000, 4096, 8 * 1031, 65536 + 17])
@pytest.mark.parametrize("shift", [0, 1])
def test_pack_and_unpack(mb, dtype, n, shift):
    x = values(dtype, n) if n else np.zeros(0)
    q_ref, byte_ref = P.pack8(x)
    back_ref = P.unpack8(q_ref, byte_ref)
    for quota in (256, 24):
        x_ = Framed(x, dtype, shift)
        q, scale = Bytes(n, shift), Bytes(mb.pack8_scale_bytes(n), shift)
        mb.op_pack8(None, quota, dtype, n, x_.at_, q.t if n else q.flat, scale.t if n else scale.flat)
        torch.cuda.synchronize()
        assert q.framed() and scale.framed() and x_.framed()
        assert np.array_equal(scale.host(np.uint8), byte_ref)
        assert np.array_equal(q.host(np.int8), q_ref)
        for to in ("bf16", "f32"):
            back = Framed(None, to, shift, (n,))
            mb.op_unpack8(None, quota, to, n, q.t if n else q.flat, scale.t if n else scale.flat, back.at_)
            torch.cuda.synchronize()
            assert back.framed()
            assert np.array_equal(from_dev(back.t), back_ref, equal_nan=True)          # exact in either type


def act_ref(act, z, da):
    """a, dz, and the sizes that their bounds count."""
    if act == "swiglu":
        f = z.shape[1] // 2
        gate, up = z[:, :f], z[:, f:]
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-gate))
        a = gate * s * up
        dz = np.concatenate([da * up * s * (1 + gate * (1 - s)), da * gate * s], axis=1)
        size = np.concatenate([np.abs(da * up) * s * (1 + np.abs(gate) * (1 - s)), np.abs(da * gate) * s], axis=1)
        return a, dz, 16 * U * np.abs(a) + 1e-36 * (1 + np.abs(gate * up)), 24 * U * size + 1e-36 * (1 + np.abs(np.concatenate([up * da * gate, da * gate], axis=1)))
    if act == "gelu":
        p = 0.5 * np.vectorize(math.erfc)(-z * math.sqrt(0.5)) if z.size else z
        return z * p, da * (p + z * np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)), 8 * U * np.abs(z), 8 * U * (1 + np.abs(z)) * np.abs(da)
    c = math.sqrt(2 / math.pi)
    t = np.tanh(c * (z + 0.044715 * z ** 3))
    dz = da * (0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z))
    return 0.5 * z * (1 + t), dz, 12 * U * np.abs(z), 128 * U * (1 + np.abs(z)) * np.abs(da)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "swiglu"])
@pytest.mark.parametrize("T,f", [(1, 1), (1, 32), (3, 40), (5, 64), (17, 24), (2, 1000), (7, 33), (0, 64), (65, 1056)])
def test_activation(mb, dtype, act, T, f):
    width = 2 * f if act == "swiglu" else f
    z = quantize(synth.normal(7100, (T, width), 0.0, 2.0) * np.exp(synth.normal(7101, (width,))), dtype)
    if T > 2:
        z[1] = 0.0
        z[2, : width // 2] = quantize(synth.normal(7102, (width // 2,), 0.0, 60.0), dtype)
    da = quantize(synth.normal(7103, (T, f)), dtype)
    q_ref, byte_ref = P.pack8(z)
    kept = P.unpack8(q_ref, byte_ref).reshape(z.shape)
    a_ref, _, a_tol, _ = act_ref(act, z, da)
    again_ref, dz_ref, again_tol, dz_tol = act_ref(act, kept, da)
    n = T * width
    outs = []
    for quota, shift in ((256, 0), (24, 0), (256, 1)):
        z_, da_ = Framed(z, dtype, shift), Framed(da, dtype, shift)
        a, again, dz = Framed(None, dtype, shift, (T, f)), Framed(None, dtype, shift, (T, f)), Framed(None, dtype, shift, (T, width))
        alone = Framed(None, dtype, shift, (T, width))
        q, scale = Bytes(n, shift), Bytes(mb.pack8_scale_bytes(n), shift)
        pq, ps = (q.t, scale.t) if n else (q.flat, scale.flat)
        at = lambda framed: framed.at_
        mb.op_act_fwd_pack8(None, quota, dtype, act, T, f, at(z_), at(a), pq, ps)
        mb.op_act_bwd_pack8(None, quota, dtype, act, T, f, pq, ps, at(da_), at(dz), at(again))
        mb.op_act_bwd_pack8(None, quota, dtype, act, T, f, pq, ps, at(da_), at(alone))
        torch.cuda.synchronize()
        if act != "swiglu":
            mb.op_act_bwd_pack8(None, quota, dtype, act, T, f, pq, ps, at(da_), at(da_))      # over the gradient that it reads
            torch.cuda.synchronize()
            assert np.array_equal(bits(da_.t), bits(dz.t))
        assert all(b.framed() for b in (z_, da_, a, again, dz, alone, q, scale))
        assert np.array_equal(q.host(np.int8), q_ref) and np.array_equal(scale.host(np.uint8), byte_ref)
        assert np.array_equal(bits(alone.t), bits(dz.t))
        if n:
            within(from_dev(a.t), a_ref, last(dtype, a_ref) + a_tol, ("a", shift))
            within(from_dev(again.t), again_ref, last(dtype, again_ref) + again_tol, ("again", shift))
            within(from_dev(dz.t), dz_ref, last(dtype, dz_ref) + dz_tol, ("dz", shift))
        outs.append([bits(a.t), bits(again.t), bits(dz.t)])
    assert all(np.array_equal(x, y) for x, y in zip(outs[0], outs[1]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "swiglu"])
def test_activation_far_out(mb, act, dtype):
    """Sizes from 20 to 10^30, where an exponential overflows and z^3 does: the limits, and zeros where the result is one."""
    sizes = (20.0, 85.0, 89.0, 120.0, 130.0, 200.0, 1e4, 1e15, 1e18, 1e30)
    T, f = 2 * len(sizes), 64
    row = np.linspace(0.6, 1.0, f)
    gate = quantize(np.concatenate([[m * row, -m * row] for m in sizes]), dtype)
    up = quantize(synth.normal(7900, (T, f)) + 3.0, dtype)
    z = np.concatenate([gate, up], axis=1) if act == "swiglu" else gate
    da = quantize(synth.normal(7901, (T, f)) + 2.0, dtype)
    kept = P.unpack8(*P.pack8(z)).reshape(z.shape)
    z_, da_ = to_dev(z, dtype), to_dev(da, dtype)
    a, again, dz = torch.empty_like(da_), torch.empty_like(da_), torch.empty_like(z_)
    q, scale = torch.empty(z.size, dtype=torch.int8, device="cuda"), torch.empty(z.size // 32, dtype=torch.uint8, device="cuda")
    mb.op_act_fwd_pack8(None, 256, dtype, act, T, f, z_, a, q, scale)
    mb.op_act_bwd_pack8(None, 256, dtype, act, T, f, q, scale, da_, dz, again)
    for got, ref, tol in ((a, act_ref(act, z, da)[0], act_ref(act, z, da)[2]), (again, act_ref(act, kept, da)[0], act_ref(act, kept, da)[2]),
                          (dz, act_ref(act, kept, da)[1], act_ref(act, kept, da)[3])):
        got = from_dev(got)
        if act != "swiglu":          # the bounds grow with |z|, and so do the results on the one side alone
            tol = np.minimum(tol, 32 * U * (np.abs(ref) + 300))
        within(got, ref, last(dtype, ref) + tol, act)
        assert (np.abs(got[np.abs(ref) < 1e-45]) < 1e-36).all()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "swiglu"])
def test_activation_of_a_block_with_nan(mb, act):
    """The forward result of what is finite stays; the block comes back as NaN, in the gradient and in the activation formed again."""
    T, f = 4, 64
    width = 2 * f if act == "swiglu" else f
    z = quantize(synth.normal(7200, (T, width)), "bf16")
    z[2, 40] = np.inf
    z_, da = to_dev(z, "bf16"), torch.ones((T, f), dtype=torch.bfloat16, device="cuda")
    a, again, dz = torch.empty_like(da), torch.empty_like(da), torch.empty_like(z_)
    q, scale = torch.empty(T * width, dtype=torch.int8, device="cuda"), torch.empty(T * width // 32, dtype=torch.uint8, device="cuda")
    mb.op_act_fwd_pack8(None, 256, "bf16", act, T, f, z_, a, q, scale)
    mb.op_act_bwd_pack8(None, 256, "bf16", act, T, f, q, scale, da, dz, again)
    bad = np.isnan(from_dev(again))
    assert bad[2, 32:64].all() and bad.sum() == 32
    bad = np.isnan(from_dev(dz))
    assert bad[2, 32:64].all() and bad.sum() == (64 if act == "swiglu" else 32)
    fine = np.isfinite(from_dev(a))
    fine[2, 40] = True
    assert fine.all()


@pytest.mark.parametrize("dtype,T,k,n,db", [("bf16", 1, 8, 8, True), ("bf16", 37, 64, 72, True), ("bf16", 300, 136, 256, False), ("bf16", 1500, 320, 264, True),
                                            ("bf16", 5, 33, 7, True), ("bf16", 513, 256, 512, True), ("f32", 1, 1, 1, True), ("f32", 70, 20, 12, True),
                                            ("f32", 257, 128, 64, False), ("bf16", 64, 128, 128, True), ("bf16", 2100, 512, 512, False), ("bf16", 200, 1040, 1048, True),
                                            ("bf16", 5000, 256, 512, True)])
def test_weight_gradient(mb, dtype, T, k, n, db):
    x = quantize(synth.normal(7300, (T, k)) * np.exp(synth.normal(7301, (k,))), dtype)
    if T > 4:
        x[T - 3:] = 0.0
    dy = quantize(synth.normal(7302, (T, n)), dtype)
    q, byte = P.pack8(x)
    kept = P.unpack8(q, byte).reshape(T, k)
    outs = []
    for quota in (256, 24):
        q_, s_ = Bytes(T * k), Bytes(byte.size)
        q_.t.copy_(torch.from_numpy(q.view(np.uint8))); s_.t.copy_(torch.from_numpy(byte))
        dw, bias = Framed(None, dtype, 0, (k, n)), Framed(None, dtype, 0, (n,))
        scratch = Bytes(mb.linear_wgrad_pack8_scratch_bytes(dtype, T, k, n))
        if db and n % (8 if dtype == "bf16" else 4):         # column sums of such rows are refused, before anything is launched
            with pytest.raises(mb.MosaicError) as e:
                mb.op_linear_wgrad_pack8(None, quota, dtype, T, k, n, q_.t, s_.t, to_dev(dy, dtype), dw.t, bias.t, scratch.t)
            assert e.value.status == mb.EUNSUPPORTED
            torch.cuda.synchronize()
            assert (dw.t == 7.0).all() and (bias.t == 7.0).all()
            db = False
        mb.op_linear_wgrad_pack8(None, quota, dtype, T, k, n, q_.t, s_.t, to_dev(dy, dtype), dw.t, bias.t if db else None, scratch.t)
        torch.cuda.synchronize()
        assert dw.framed() and bias.framed() and scratch.framed() and q_.framed() and s_.framed()
        outs.append((bits(dw.t), bits(bias.t)))
    assert all(np.array_equal(a, b) for a, b in zip(outs[0], outs[1]))
    ref = kept.T @ dy
    within(from_dev(dw.t), ref, last(dtype, ref) + (T + 8) * U * (np.abs(kept).T @ np.abs(dy)), "dw")
    if db:
        within(from_dev(bias.t), dy.sum(0), last(dtype, dy.sum(0)) + (T + 8) * U * np.abs(dy).sum(0), "db")
    else:
        assert (bias.t == 7.0).all()


@pytest.mark.parametrize("T", [100, 4500])
def test_weight_gradient_of_extreme_blocks(mb, T):
    """Blocks of the largest and of the smallest numbers, and one with a NaN, which stays in its columns; in one launch and in several."""
    k, n = 160, 64
    x = quantize(synth.normal(7800, (T, k)), "bf16")
    x[:, 32:64] = quantize(np.clip(x[:, 32:64], -3, 3) * 1.1e38, "bf16")
    x[:, 64:96] = quantize(x[:, 64:96] * 2.0 ** -121, "bf16")            # steps of 2^-127
    x[T // 2, 100] = np.inf
    dy = quantize(synth.normal(7801, (T, n)), "bf16")
    q, byte = P.pack8(x)
    assert byte.max() == 255 and (byte == 248).any() and (byte < 2).any()      # 248: the largest step of bf16 numbers
    kept = P.unpack8(q, byte).reshape(T, k)
    scaled = [(slice(0, 32), 1.0), (slice(32, 64), 2.0 ** -40), (slice(64, 96), 2.0 ** 120), (slice(128, 160), 1.0)]
    for cols, by in scaled:
        dy_ = dy if by == 1.0 else quantize(dy * by, "bf16")
        dw = torch.empty((k, n), dtype=torch.bfloat16, device="cuda")
        scratch = torch.empty(mb.linear_wgrad_pack8_scratch_bytes("bf16", T, k, n), dtype=torch.uint8, device="cuda")
        mb.op_linear_wgrad_pack8(None, 256, "bf16", T, k, n, torch.from_numpy(q).cuda(), torch.from_numpy(byte).cuda(), to_dev(dy_, "bf16"), dw, None, scratch)
        got = from_dev(dw)
        assert np.isnan(got[96:128]).all()
        ref = kept[:, cols].T @ dy_
        within(got[cols], ref, last("bf16", ref) + (T + 8) * U * (np.abs(kept[:, cols]).T @ np.abs(dy_)), (cols, by))


def test_captured_and_replayed(mb):
    T, k, n, f = 200, 64, 72, 96
    x, dy = to_dev(quantize(synth.normal(7400, (T, k)), "bf16"), "bf16"), to_dev(quantize(synth.normal(7401, (T, n)), "bf16"), "bf16")
    z, da = to_dev(quantize(synth.normal(7402, (T, 2 * f)), "bf16"), "bf16"), to_dev(quantize(synth.normal(7403, (T, f)), "bf16"), "bf16")
    byte = lambda size: torch.empty(size, dtype=torch.uint8, device="cuda")
    xq, xs, zq, zs = byte(T * k), byte(T * k // 32), byte(T * 2 * f), byte(T * 2 * f // 32)
    out = dict(a=torch.empty_like(da), dz=torch.empty_like(z), again=torch.empty_like(da), dw=torch.empty((k, n), dtype=torch.bfloat16, device="cuda"),
               db=torch.empty(n, dtype=torch.bfloat16, device="cuda"))
    scratch = byte(mb.linear_wgrad_pack8_scratch_bytes("bf16", T, k, n))

    def step(stream):
        mb.op_act_fwd_pack8(stream, 256, "bf16", "swiglu", T, f, z, out["a"], zq, zs)
        mb.op_pack8(stream, 256, "bf16", T * k, x, xq, xs)
        mb.op_act_bwd_pack8(stream, 256, "bf16", "swiglu", T, f, zq, zs, da, out["dz"], out["again"])
        mb.op_linear_wgrad_pack8(stream, 256, "bf16", T, k, n, xq, xs, dy, out["dw"], out["db"], scratch)

    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step(s.cuda_stream)
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            step(torch.cuda.current_stream().cuda_stream)
    for turn in range(3):
        for t, seed in ((x, 0), (z, 1), (dy, 2)):
            t.copy_(to_dev(quantize(synth.normal(7500 + 3 * turn + seed, tuple(t.shape)), "bf16"), "bf16"))
        torch.cuda.synchronize()
        step(None)
        torch.cuda.synchronize()
        want = {name: bits(t) for name, t in out.items()}
        for t in (*out.values(), xq, xs, zq, zs):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in out.items():
            assert np.array_equal(want[name], bits(t)), name


def test_swiglu_from_8_bits_rounds_like_the_plain_form(mb):
    """Gates from 2 to 17 times up numbers of 7 bits, where results often lie within a few u of a tie between two bf16 numbers, so that the last bits of s = 1 / (1 + e)
    decide them (5.9375 times a power of two is 1.6 u from one): those of the plain form in 32 bits, bit for bit.  e, off by 5 u of its size here, gives
    d = fl(1 + e) = 1 + 2 u k but for gates whose e / 2u lies that near to a half; the approximate reciprocal, one bit off at most, is after a step of Newton's
    2^-46 from 1 / d, and its nearest number is that of 1 / d but for gates where 1 / d lies that near to a tie.  Both are left out."""
    gates = np.concatenate([np.arange(2.0, 7.95, 0.0625), np.arange(8.0, 15.9, 0.125), np.arange(16.0, 17.1, 0.25)])
    from_half = lambda v: np.abs(v - np.floor(v) - 0.5)
    ratio = np.exp(-gates) / (2 * U)
    d = np.float32(1) + np.exp(-gates).astype(np.float32)
    s = np.float32(1) / d
    gates, s = (v[(from_half(ratio) > 5 * U * ratio + 1e-6) & (from_half(1 / d.astype(np.float64) / U) > 1e-3)] for v in (gates, s))
    assert len(gates) > 130 and 5.9375 in gates
    T, f = len(gates), 1024
    up = np.clip(np.round(synth.normal(8200, (T, f), 0.0, 60.0)), -127, 127)
    up[:, ::32] = 127.0
    up[:, 1:8] = 2.0 ** np.arange(7)
    z = np.concatenate([np.repeat(gates[:, None], f, 1), up], axis=1)
    q_ref, byte_ref = P.pack8(z)
    assert np.array_equal(P.unpack8(q_ref, byte_ref).reshape(z.shape), z)             # nothing is lost in 8 bits
    want = quantize((gates.astype(np.float32) * s)[:, None] * up.astype(np.float32), "bf16")
    z_, da = to_dev(z, "bf16"), torch.ones((T, f), dtype=torch.bfloat16, device="cuda")
    a, again, dz = torch.empty_like(da), torch.empty_like(da), torch.empty_like(z_)
    q, scale = torch.empty(z.size, dtype=torch.int8, device="cuda"), torch.empty(z.size // 32, dtype=torch.uint8, device="cuda")
    mb.op_act_fwd_pack8(None, 256, "bf16", "swiglu", T, f, z_, a, q, scale)
    mb.op_act_bwd_pack8(None, 256, "bf16", "swiglu", T, f, q, scale, da, dz, again)
    for got in (a, again):
        off = from_dev(got) != want
        assert not off.any(), (int(off.sum()), gates[off.any(1)])


@pytest.mark.parametrize("T,k,n", [(37, 48, 64), (101, 48, 72), (101, 16, 520), (37, 80, 64), (101, 112, 200), (201, 1040, 1048), (4501, 48, 64)])
def test_weight_gradient_of_a_last_block_with_nan(mb, T, k, n):
    """T * k ends within a block: the NaN of that block stays in its columns, the last sixteen, in one launch (one group of waves or two, few or many
    tiles) and, with many tokens and few tiles, in several."""
    assert T * k % 32 == 16
    x, dy = quantize(synth.normal(8300, (T, k)), "bf16"), quantize(synth.normal(8301, (T, n)), "bf16")
    x[T - 1, k - 5] = np.inf
    q, byte = P.pack8(x)
    assert byte[-1] == 255 and (byte[:-1] < 255).all()
    kept = P.unpack8(q, byte).reshape(T, k)
    dw, db = torch.empty((k, n), dtype=torch.bfloat16, device="cuda"), torch.empty(n, dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(mb.linear_wgrad_pack8_scratch_bytes("bf16", T, k, n), dtype=torch.uint8, device="cuda")
    mb.op_linear_wgrad_pack8(None, 256, "bf16", T, k, n, torch.from_numpy(q).cuda(), torch.from_numpy(byte).cuda(), to_dev(dy, "bf16"), dw, db, scratch)
    got = from_dev(dw)
    assert np.isnan(got[k - 16:]).all()
    ref = kept[:, :k - 16].T @ dy
    within(got[:k - 16], ref, last("bf16", ref) + (T + 8) * U * (np.abs(kept[:, :k - 16]).T @ np.abs(dy)), "dw")
    within(from_dev(db), dy.sum(0), last("bf16", dy.sum(0)) + (T + 8) * U * np.abs(dy).sum(0), "db")


def test_tanh_gelu_derivative_f32(mb):
    """The derivative s + z w p of the tanh form in fp32 keeps its digits where s is near 1; s = 1 / (1 + e), e = exp(-v), p = s (1 - s), v = c (z + 0.044715 z^3), w = v'.

    Bound in u: v 7 |v| (five operations and two constants); e 7 |v| + 2 of its size, s (1 - s)(7 |v| + 2) + 2, p 7 |v| + 8 at most, w 5, the products 2: the second
    term 7 |v| + 15 of its size; the sum and the product with da 2 of both sizes.  (With 1 - s as a difference p would be off by up to 1.5 of 1, which w z takes up to 30 times.)"""
    T, f = 64, 1024
    z = quantize(synth.normal(8400, (T, f), 0.0, 1.0) * np.exp(np.linspace(-4.0, 2.5, T))[:, None], "f32")
    da = quantize(synth.normal(8401, (T, f)), "f32")
    q, byte = P.pack8(z)
    z = P.unpack8(q, byte).reshape(T, f)
    c = math.sqrt(2 / math.pi) * 2
    v, w = c * (z + 0.044715 * z ** 3), c * (1 + 3 * 0.044715 * z * z)
    with np.errstate(over="ignore"):
        s, rest = 1 / (1 + np.exp(-v)), 1 / (1 + np.exp(v))
    second = z * w * s * rest
    bound = U * np.abs(da) * (s * (rest * (7 * np.abs(v) + 2) + 2) + np.abs(second) * (7 * np.abs(v) + 15) + 2 * (s + np.abs(second))) + 1e-36
    dz = torch.empty((T, f), device="cuda")
    mb.op_act_bwd_pack8(None, 256, "f32", "gelu_tanh", T, f, torch.from_numpy(q).cuda(), torch.from_numpy(byte).cuda(), to_dev(da, "f32"), dz)
    within(from_dev(dz), da * (s + second), bound, "dz")
    shifted, any_dz = Bytes(T * f, 1), torch.empty((T, f), device="cuda")                # element by element
    shifted.t.copy_(torch.from_numpy(q.view(np.uint8)))
    mb.op_act_bwd_pack8(None, 256, "f32", "gelu_tanh", T, f, shifted.t, torch.from_numpy(byte).cuda(), to_dev(da, "f32"), any_dz)
    within(from_dev(any_dz), da * (s + second), bound, "dz, element by element")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shifts", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 0, 4), (1, 1, 1)])
@pytest.mark.parametrize("T,k,n,db", [(70, 48, 72, True), (37, 64, 64, False), (513, 40, 88, True)])
def test_weight_gradient_off_boundaries(mb, dtype, shifts, T, k, n, db):
    """Numbers, exponent bytes, dY and the outputs off 16-byte boundaries by some elements."""
    x, dy = quantize(synth.normal(8500, (T, k)), dtype), quantize(synth.normal(8501, (T, n)), dtype)
    q, byte = P.pack8(x)
    kept = P.unpack8(q, byte).reshape(T, k)
    q_, s_ = Bytes(T * k, shifts[0]), Bytes(byte.size, 3 * shifts[0])
    q_.t.copy_(torch.from_numpy(q.view(np.uint8))); s_.t.copy_(torch.from_numpy(byte))
    dy_, dw, bias = Framed(dy, dtype, shifts[1]), Framed(None, dtype, shifts[2], (k, n)), Framed(None, dtype, shifts[2], (n,))
    scratch = Bytes(mb.linear_wgrad_pack8_scratch_bytes(dtype, T, k, n))
    mb.op_linear_wgrad_pack8(None, 256, dtype, T, k, n, q_.t, s_.t, dy_.t, dw.t, bias.t if db else None, scratch.t)
    torch.cuda.synchronize()
    assert all(b.framed() for b in (q_, s_, dy_, dw, bias, scratch))
    ref = kept.T @ dy
    within(from_dev(dw.t), ref, last(dtype, ref) + (T + 8) * U * (np.abs(kept).T @ np.abs(dy)), "dw")
    if db:
        within(from_dev(bias.t), dy.sum(0), last(dtype, dy.sum(0)) + (T + 8) * U * np.abs(dy).sum(0), "db")
    else:
        assert (bias.t == 7.0).all()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh"])
def test_gelu_past_the_caches(mb, act):
    """More than 256 MB read and written, a size that is no multiple of a block: every element, against 64 bits on the GPU; with and without the activation again."""
    T, f = 8213, 6603
    n = T * f
    assert 5 * n > 256 << 20 and n % 32
    g = torch.Generator(device="cuda").manual_seed(92)
    z, da = (torch.randn((T, f), generator=g, device="cuda") * 2).bfloat16(), torch.randn((T, f), generator=g, device="cuda").bfloat16()
    a, again, dz, alone = (torch.empty_like(da) for _ in range(4))
    q, scale = torch.empty(n, dtype=torch.int8, device="cuda"), torch.empty(mb.pack8_scale_bytes(n), dtype=torch.uint8, device="cuda")
    mb.op_act_fwd_pack8(None, 256, "bf16", act, T, f, z, a, q, scale)
    mb.op_act_bwd_pack8(None, 256, "bf16", act, T, f, q, scale, da, dz, again)
    mb.op_act_bwd_pack8(None, 256, "bf16", act, T, f, q, scale, da, alone)
    assert torch.equal(alone, dz)
    q_, scale_ = torch.empty_like(q), torch.empty_like(scale)
    mb.op_pack8(None, 256, "bf16", n, z, q_, scale_)
    assert torch.equal(q, q_) and torch.equal(scale, scale_)
    for part in (slice(0, 3200), slice(n // 32 * 32 - 3200, n)):
        q_ref, byte_ref = P.pack8(from_dev(z.view(-1)[part]))
        assert np.array_equal(q[part].cpu().numpy(), q_ref) and np.array_equal(scale[part.start // 32:][:byte_ref.size].cpu().numpy(), byte_ref)
    kept = (q.double() * torch.exp2(scale.double() - 127).repeat_interleave(32)[:n]).view(T, f)

    def ref(z):
        if act == "gelu":
            p = 0.5 * torch.erfc(-z * math.sqrt(0.5))
            return z * p, p + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi), 8, 8
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z), 12, 128

    for got, at, size in ((a, z.double(), None), (again, kept, None), (dz, kept, da.double())):
        value, slope, by_value, by_slope = ref(at)
        want = value if size is None else size * slope
        bound = want.abs() * 2.0 ** -8 + (by_value * U * at.abs() if size is None else by_slope * U * (1 + at.abs()) * size.abs())
        assert float(((got.double() - want).abs() - bound).max()) <= 0
