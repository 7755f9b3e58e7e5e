"""GPU parity of the rotary positions with several axes and of the query/key norms with the rotation, forward and backward, against
the plain definitions in 64 bits; bits across quotas; rows in place, off 16-byte boundaries, and what lies around them.

Bounds, u = 2^-24 (half a step of fp32).  The relative error of a normalised element is at most 10 u for the mean, 8 u for rstd (a tree of
additions, a square root, a quotient), 4 u for the gain and the shift; sine and cosine are off by 7 u (a rounded angle of at
most half a turn, two units of the function); the rotation adds 3 u to each of two terms: below 32 u of
twice the head's largest normalised magnitude M.  Backward: 40 u of S = rstd * max|w| * (2 + max|xhat|), taken as 64.  A gain's gradient is a sum of at
most 300 additions in a row here, its terms off by 40 u: 512 u of the sum of magnitudes.  A bf16 result is off by 2^-8 of its size besides."""
import numpy as np
import pytest
import torch

from oracle import operators as P
from paper_2605_18710_amd import synth
from helpers import from_dev, quantize, to_dev

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_18710_amd import binding
    binding.lib()
    return binding


def bits(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy().copy()


def last(dtype, ref):
    return np.abs(ref) * (2.0 ** -8 if dtype == "bf16" else 0.0)


def within(got, ref, bound, what):
    over = np.abs(got - ref) - bound
    assert np.isfinite(got).all() and (over <= 0).all(), (what, float(over.max()), np.unravel_index(over.argmax(), over.shape))


class Framed:
    """A tensor of `shape` whose first element lies `shift` elements behind a 16-byte boundary, with a frame that must stay."""

    def __init__(self, value, dtype, shift=0, shape=None):
        td = torch.bfloat16 if dtype == "bf16" else torch.float32
        shape = np.shape(value) if shape is None else shape
        n = int(np.prod(shape))
        self.flat = torch.full((n + 128,), 7.0, dtype=td, device="cuda")
        self.at = slice(64 + shift, 64 + shift + n)
        self.t = self.flat[self.at].view(shape)
        if value is not None:
            self.t.copy_(to_dev(value, dtype))

    @property
    def at_(self):
        """What a call gets: an address for no elements too."""
        return self.t if self.t.numel() else self.flat

    def framed(self):
        f = self.flat.clone()
        f[self.at] = 7.0
        return bool((f == 7.0).all())


class Case:
    def __init__(self, mb, dtype, norm, T, H, Hkv, d, sections, order, pairing, seed=5000, far=0):
        self.__dict__.update(dtype=dtype, norm=norm, T=T, H=H, Hkv=Hkv, d=d, sections=sections, order=order, pairing=pairing)
        w = (H + 2 * Hkv) * d
        self.x = quantize(synth.normal(seed, (T, w), 0.3, 1.7), dtype)
        if T > 2:
            self.x[T // 2] = 0.0                                     # a padded token
        self.dy = quantize(synth.normal(seed + 1, (T, w)), dtype)
        self.gains = [quantize(1 + synth.normal(seed + 2 + i, (d,), 0.0, 0.3), dtype) for i in range(2)]
        self.shifts = [quantize(synth.normal(seed + 4 + i, (d,), 0.0, 0.3), dtype) for i in range(2)]
        self.pos = synth.integers(seed + 6, (max(1, len(sections)), T), -5, 300) + np.int32(far)
        self.axis, self.freq = P.pair_table(d, sections, order, 10000.0)
        self.pos_ = torch.from_numpy(self.pos.astype(np.int32)).cuda().contiguous() if T else torch.zeros(8, dtype=torch.int32, device="cuda")
        self.table_ = torch.empty(max(16, mb.rope_axes_table_bytes(d)), dtype=torch.uint8, device="cuda")
        mb.op_rope_axes_table(None, 256, d, sections, order, 10000.0, self.table_)

    def parts(self, a):
        a = np.asarray(a).reshape(self.T, self.H + 2 * self.Hkv, self.d)
        return a[:, :self.H], a[:, self.H:self.H + self.Hkv], a[:, self.H + self.Hkv:]

    def rotate(self, x, direction=1):
        return P.rotate(x, self.pos, self.axis, self.freq, self.pairing, direction)


LAYOUTS = [
    # T, H, Hkv, d, sections, order, pairing
    (1, 1, 1, 2, (1,), "split", "adjacent"),
    (1, 16, 4, 128, (24, 20, 20), "split", "halves"),
    (7, 4, 2, 64, (8, 12, 12), "own", "adjacent"),
    (33, 3, 1, 40, (7, 6, 7), "dealt", "halves"),
    (5, 6, 6, 72, (18, 18), "own", "halves"),
    (9, 5, 5, 80, (16, 12, 12), "dealt", "adjacent"),
    (3, 8, 2, 96, (20, 0, 20), "dealt", "halves"),
    (4, 2, 1, 256, (128,), "split", "halves"),
    (6, 2, 2, 250, (60, 65), "split", "adjacent"),
    (11, 9, 3, 32, (4, 4, 4, 4), "dealt", "adjacent"),
    (3, 7, 7, 6, (1, 1), "own", "halves"),
    (130, 20, 4, 64, (32,), "split", "halves"),
    (5, 1, 1, 16, (3,), "split", "adjacent"),
    (2, 40, 8, 128, (16, 24, 24), "own", "adjacent"),
    (0, 4, 2, 64, (8, 12, 12), "own", "adjacent"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("shift", [0, 1])
def test_rotation(mb, dtype, layout, shift):
    c = Case(mb, dtype, "none", *layout)
    T, H, Hkv, d = layout[:4]
    for direction in (1, -1):
        q, k, v = c.parts(c.x)
        ref = np.concatenate([c.rotate(q, direction), c.rotate(k, direction), v], axis=1).reshape(c.x.shape)
        outs = []
        for quota in (256, 24):
            x, y = Framed(c.x, dtype, shift), Framed(None, dtype, shift, c.x.shape)
            mb.op_rope_axes(None, quota, dtype, T, H, Hkv, d, c.pairing, direction, len(c.sections), c.pos_, c.table_, x.at_, y.at_)
            mb.op_rope_axes(None, quota, dtype, T, H, Hkv, d, c.pairing, direction, len(c.sections), c.pos_, c.table_, x.at_, x.at_)      # in place
            torch.cuda.synchronize()
            assert x.framed() and y.framed()
            assert np.array_equal(bits(x.t), bits(y.t))
            outs.append(bits(y.t))
        assert np.array_equal(outs[0], outs[1])
        if T:
            got = from_dev(y.t)
            size = np.abs(c.x).reshape(T, -1, d).max(2, keepdims=True).repeat(d, 2).reshape(T, -1)
            within(got, ref, last(dtype, ref) + 32 * U * 2 * size, "y")
            assert np.array_equal(c.parts(got)[2], v)
            moved = [i for i in range(d // 2) if c.axis[i] < 0]
            cols = [j for i in moved for j in ((i, i + d // 2) if c.pairing == "halves" else (2 * i, 2 * i + 1))]
            assert np.array_equal(c.parts(got)[0][..., cols], q[..., cols])


def norm_fwd(mb, c, x, y, quota, rotate=True, stream=None):
    layer = c.norm == "layernorm"
    g, s = [to_dev(v, c.dtype) for v in c.gains], [to_dev(v, c.dtype) for v in c.shifts]
    mb.op_qk_norm_rope_fwd(stream, quota, c.dtype, c.norm, c.T, c.H, c.Hkv, c.d, 1e-5, c.pairing, len(c.sections) if rotate else 0, c.pos_ if rotate else None,
                           c.table_ if rotate else None, x, g[0], s[0] if layer else None, g[1], s[1] if layer else None, y)
    return g, s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", ["rmsnorm", "layernorm"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_norm_forward(mb, dtype, norm, layout):
    c = Case(mb, dtype, norm, *layout)
    T, H, Hkv, d = layout[:4]
    for rotate in (True, False):
        q, k, v = c.parts(c.x)
        n = [P.head_norm(p, norm, 1e-5, g, s)[0] for p, g, s in zip((q, k), c.gains, c.shifts)]
        ref = np.concatenate([c.rotate(p) if rotate else p for p in n] + [v], axis=1).reshape(c.x.shape)
        size = np.concatenate([np.broadcast_to(np.abs(p).max(2, keepdims=True) + np.abs(s).max() + np.abs(g).max(), p.shape) for p, g, s in zip(n, c.gains, c.shifts)]
                              + [0 * v], axis=1).reshape(T, -1) if T else 0
        outs = []
        for quota, shift in ((256, 0), (24, 0), (256, 1)):
            x, y = Framed(c.x, dtype, shift), Framed(None, dtype, shift, c.x.shape)
            norm_fwd(mb, c, x.at_, y.at_, quota, rotate)
            norm_fwd(mb, c, x.at_, x.at_, quota, rotate)
            torch.cuda.synchronize()
            assert x.framed() and y.framed() and np.array_equal(bits(x.t), bits(y.t))
            if T:
                within(from_dev(y.t), ref, last(dtype, ref) + 32 * U * 2 * size, ("y", rotate, shift))
            outs.append(bits(y.t))
        assert np.array_equal(outs[0], outs[1])


def norm_bwd(mb, c, x, dy, dx, quota, scratch, rotate=True, stream=None):
    layer = c.norm == "layernorm"
    g = [to_dev(v, c.dtype) for v in c.gains]
    out = [Framed(None, c.dtype, 0, (c.d,)) for _ in range(4)]
    mb.op_qk_norm_rope_bwd(stream, quota, c.dtype, c.norm, c.T, c.H, c.Hkv, c.d, 1e-5, c.pairing, len(c.sections) if rotate else 0, c.pos_ if rotate else None,
                           c.table_ if rotate else None, x, g[0], g[1], dy, dx, out[0].t, out[2].t if layer else None, out[1].t,
                           out[3].t if layer else None, scratch)
    return g, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", ["rmsnorm", "layernorm"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_norm_backward(mb, dtype, norm, layout):
    c = Case(mb, dtype, norm, *layout)
    T, H, Hkv, d = layout[:4]
    scratch = torch.full((mb.qk_norm_rope_bwd_scratch_bytes(d) // 4,), float("nan"), device="cuda")      # nothing in it has to be zero
    for rotate in (True, False):
        refs, sizes, sums, mags = [], [], [], []
        for x, dy, gain, shift in zip(c.parts(c.x), c.parts(c.dy), c.gains, c.shifts):
            _, xhat, rstd = P.head_norm(x, norm, 1e-5, gain, shift)
            g = c.rotate(dy, -1) if rotate else dy
            dx, dgain, dshift = P.head_norm_bwd(g, xhat, rstd, norm, gain)
            refs.append(dx)
            if T:
                peak = np.abs(dy).max(2, keepdims=True) * 2 * np.abs(gain).max()
                sizes.append(np.broadcast_to(rstd * peak * (2 + np.abs(xhat).max(2, keepdims=True)), dx.shape))
            sums.append((dgain, dshift))
            mags.append((np.abs(g * xhat).sum((0, 1)) + 1e-30, np.abs(g).sum((0, 1)) + 1e-30, np.abs(dy).max(initial=0) * T * 2 * max(H, Hkv)))
        ref = np.concatenate(refs + [c.parts(c.dy)[2]], axis=1).reshape(c.x.shape)
        size = np.concatenate(sizes + [0 * c.parts(c.dy)[2]], axis=1).reshape(T, -1) if T else 0
        outs = []
        for quota, shift in ((256, 0), (24, 0), (256, 1)):
            x, dy, dx = Framed(c.x, dtype, shift), Framed(c.dy, dtype, shift), Framed(None, dtype, shift, c.x.shape)
            _, grads = norm_bwd(mb, c, x.at_, dy.at_, dx.at_, quota, scratch, rotate)
            norm_bwd(mb, c, x.at_, dy.at_, dy.at_, quota, scratch, rotate)
            torch.cuda.synchronize()
            assert x.framed() and dy.framed() and dx.framed() and all(g.framed() for g in grads)
            assert np.array_equal(bits(dx.t), bits(dy.t))
            if T:
                within(from_dev(dx.t), ref, last(dtype, ref) + 64 * U * size, ("dx", rotate, shift))
            for part in (0, 1):
                (dgain, dshift), (mg, ms, _) = sums[part], mags[part]
                within(from_dev(grads[part].t), dgain, last(dtype, dgain) + 512 * U * (mg + ms), ("dgain", part, rotate, shift))
                if norm == "layernorm":
                    within(from_dev(grads[2 + part].t), dshift, last(dtype, dshift) + 512 * U * 2 * ms, ("dshift", part, rotate, shift))
                else:
                    assert (grads[2 + part].t == 7.0).all()
            outs.append([bits(dx.t)] + [bits(g.t) for g in grads])
        assert all(np.array_equal(a, b) for a, b in zip(outs[0], outs[1]))


@pytest.mark.parametrize("far", [1000000, 2 ** 31 - 400, -2 ** 31 + 10])
def test_far_positions_keep_their_digits(mb, far):
    c = Case(mb, "f32", "none", 6, 2, 1, 64, (16, 16), "own", "halves", far=far)
    y = torch.empty((6, 4 * 64), device="cuda")
    mb.op_rope_axes(None, 256, "f32", 6, 2, 1, 64, "halves", 1, 2, c.pos_, c.table_, to_dev(c.x, "f32"), y)
    q, k, v = c.parts(c.x)
    ref = np.concatenate([c.rotate(q), c.rotate(k), v], axis=1).reshape(6, -1)
    # the oracle's own angle, up to 2^31 radians in 64 bits, is off by 2^-22
    within(from_dev(y), ref, (32 * U + 2.0 ** -21) * 2 * np.abs(c.x).max(), "y")


def test_table_made_for_more_axes(mb):
    """A pair whose axis the call does not have stays; nothing behind the positions is read."""
    c = Case(mb, "f32", "none", 4, 2, 2, 32, (5, 5, 6), "split", "adjacent")
    y = torch.empty((4, 6 * 32), device="cuda")
    mb.op_rope_axes(None, 256, "f32", 4, 2, 2, 32, "adjacent", 1, 1, c.pos_[:1].contiguous(), c.table_, to_dev(c.x, "f32"), y)
    got = from_dev(y).reshape(4, 6, 32)
    assert np.array_equal(got[..., 10:], c.x.reshape(4, 6, 32)[..., 10:]) and not np.array_equal(got[:, 0, :10], c.x.reshape(4, 6, 32)[:, 0, :10])


def test_nan_stays_in_its_head(mb):
    """A NaN or an infinity makes its own head NaN and nothing else; v takes anything."""
    c = Case(mb, "bf16", "rmsnorm", 3, 4, 2, 64, (16, 16), "own", "halves")
    x = c.x.reshape(3, 8, 64)
    x[1, 2, 5], x[2, 5, 0], x[0, 7, 1] = np.nan, np.inf, np.nan
    y = torch.empty((3, 8 * 64), dtype=torch.bfloat16, device="cuda")
    norm_fwd(mb, c, to_dev(c.x, "bf16"), y, 256)
    bad = np.isnan(from_dev(y)).reshape(3, 8, 64)
    assert bad[1, 2].all() and bad[2, 5].any() and bad[0, 7, 1] and bad[0, 7].sum() == 1
    bad[1, 2] = bad[2, 5] = bad[0, 7] = False
    assert not bad.any()


def test_partitions_of_many_tokens(mb):
    """More tokens than partitions: the gains' sums over 5000 tokens, and their bits on few CUs."""
    c = Case(mb, "bf16", "layernorm", 5000, 2, 1, 32, (8, 8), "dealt", "halves")
    scratch = torch.empty(mb.qk_norm_rope_bwd_scratch_bytes(32), dtype=torch.uint8, device="cuda")
    x, dy = to_dev(c.x, "bf16"), to_dev(c.dy, "bf16")
    outs = []
    for quota in (256, 8, 96):
        dx = torch.empty_like(x)
        _, grads = norm_bwd(mb, c, x, dy, dx, quota, scratch)
        torch.cuda.synchronize()
        outs.append([bits(dx)] + [bits(g.t) for g in grads])
    for o in outs[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(outs[0], o))
    for part in (0, 1):
        _, xhat, rstd = P.head_norm(c.parts(c.x)[part], "layernorm", 1e-5, c.gains[part], c.shifts[part])
        g = c.rotate(c.parts(c.dy)[part], -1)
        within(from_dev(grads[part].t), (g * xhat).sum((0, 1)), last("bf16", (g * xhat).sum((0, 1))) + 512 * U * (np.abs(g * xhat) + np.abs(g)).sum((0, 1)), "dgain")
        within(from_dev(grads[2 + part].t), g.sum((0, 1)), last("bf16", g.sum((0, 1))) + 1024 * U * np.abs(g).sum((0, 1)), "dshift")


def test_captured_and_replayed(mb):
    c = Case(mb, "bf16", "rmsnorm", 300, 4, 2, 64, (10, 11, 11), "dealt", "halves")
    x, dy = to_dev(c.x, "bf16"), to_dev(c.dy, "bf16")
    scratch = torch.empty(mb.qk_norm_rope_bwd_scratch_bytes(64), dtype=torch.uint8, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    g = [to_dev(v, "bf16") for v in c.gains]
    dg = [torch.empty_like(v) for v in g]
    head = (c.T, c.H, c.Hkv, c.d, 1e-5, c.pairing, 3, c.pos_, c.table_)

    def both(stream):
        mb.op_qk_norm_rope_fwd(stream, 256, "bf16", "rmsnorm", *head, x, g[0], None, g[1], None, y)
        mb.op_qk_norm_rope_bwd(stream, 256, "bf16", "rmsnorm", *head, x, g[0], g[1], dy, dx, dg[0], None, dg[1], None, scratch)

    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        both(s.cuda_stream)
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            both(torch.cuda.current_stream().cuda_stream)
    for step in range(3):
        x.copy_(to_dev(quantize(synth.normal(6000 + step, c.x.shape), "bf16"), "bf16"))
        torch.cuda.synchronize()
        both(None)
        torch.cuda.synchronize()
        want = [bits(t) for t in (y, dx, *dg)]
        for t in (y, dx, *dg):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(a, bits(t)) for a, t in zip(want, (y, dx, *dg)))


def same_kinds(got, ref, bound, what):
    """NaNs and infinities where the formulas have them, with their signs, and the other numbers within the bound."""
    assert np.array_equal(np.isnan(got), np.isnan(ref)), (what, np.argwhere(np.isnan(got) != np.isnan(ref))[:4])
    assert np.array_equal(np.where(np.isinf(got), got, 0), np.where(np.isinf(ref), ref, 0)), what
    fine = np.isfinite(ref)
    within(got[fine], ref[fine], np.broadcast_to(bound, ref.shape)[fine], what)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", ["none", "rmsnorm", "layernorm"])
@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
@pytest.mark.parametrize("shift", [0, 1])
def test_nan_and_infinity_go_by_the_formulas(mb, dtype, norm, pairing, shift):
    """In turned pairs and in ones that stay, of queries, keys and v; what does not meet them is as without them.  Under RMS norm an infinity makes its pair NaN
    and the rest of its head 0; under LayerNorm its head NaN; in the backward pass either makes its head NaN, and a gain's gradient NaN where it met one."""
    c = Case(mb, dtype, norm, 6, 4, 2, 64, (11, 12), "split", pairing)            # pairs 23 to 31 stay
    turned, stays = (5, 26) if pairing == "halves" else (10, 52)
    c.pos[:, 3] = 0                                                               # cosine 1 and sine 0
    c.pos_.copy_(torch.from_numpy(c.pos.astype(np.int32)))
    x = c.x.reshape(6, 8, 64)
    for at, v in (((0, 1, turned), np.nan), ((1, 2, turned), np.inf), ((2, 4, turned + 1), -np.inf), ((2, 0, stays), np.inf), ((3, 5, turned), np.inf),
                  ((4, 3, stays), np.nan), ((4, 7, 9), np.inf), ((5, 6, 8), np.nan)):
        x[at] = v
    x_, y = Framed(c.x, dtype, shift), Framed(None, dtype, shift, c.x.shape)
    q, k, v = c.parts(c.x)
    with np.errstate(invalid="ignore", over="ignore"):
        if norm == "none":
            mb.op_rope_axes(None, 256, dtype, 6, 4, 2, 64, pairing, 1, 2, c.pos_, c.table_, x_.t, y.t)
            n = [q, k]
        else:
            norm_fwd(mb, c, x_.t, y.t, 256)
            n = [P.head_norm(p, norm, 1e-5, g, s)[0] for p, g, s in zip((q, k), c.gains, c.shifts)]
        ref = np.concatenate([c.rotate(p) for p in n] + [v], axis=1)
        top = max(np.abs(p[np.isfinite(p)]).max() for p in n) + 4
        got = from_dev(y.t).reshape(ref.shape)
        same_kinds(got, ref, last(dtype, ref) + 64 * U * top, "y")
        if norm == "rmsnorm":
            other = [i for i in range(64) if i not in ((5, 37) if pairing == "halves" else (10, 11))]
            assert np.isnan(got[1, 2]).sum() == 2 and (got[1, 2, other] == 0).all()
        elif norm == "layernorm":
            assert np.isnan(got[1, 2]).all() and np.isnan(got[3, 5]).all()
        if norm == "none":
            return
        c.dy.reshape(6, 8, 64)[0, 0, turned] = np.nan
        dy_, dx = Framed(c.dy, dtype, shift), Framed(None, dtype, shift, c.x.shape)
        scratch = torch.empty(mb.qk_norm_rope_bwd_scratch_bytes(64), dtype=torch.uint8, device="cuda")
        _, grads = norm_bwd(mb, c, x_.t, dy_.t, dx.t, 256, scratch)
        refs = []
        for part, (p, d, gain, sh) in enumerate(zip((q, k), c.parts(c.dy), c.gains, c.shifts)):
            _, xhat, rstd = P.head_norm(p, norm, 1e-5, gain, sh)
            g = c.rotate(d, -1)
            dx_ref, dgain, dshift = P.head_norm_bwd(g, xhat, rstd, norm, gain)
            refs.append(dx_ref)
            assert np.array_equal(np.isnan(from_dev(grads[part].t)), np.isnan(dgain))
            if norm == "layernorm":
                assert np.array_equal(np.isnan(from_dev(grads[2 + part].t)), np.isnan(dshift))
        ref = np.concatenate(refs + [c.parts(c.dy)[2]], axis=1)
        got = from_dev(dx.t).reshape(ref.shape)
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and not np.isinf(got).any()
        assert np.isnan(got[1, 2]).all() and np.isnan(got[0, 1]).all() and np.isfinite(got[1, 3]).all()


def rows_on_gpu(mb, dtype, norm, T, H, Hkv, d, pairing, seed):
    """Rows, gradients and gains on the GPU, and y, dx and the gains' gradients in 64 bits from the definitions."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    n = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(td)
    x, dy, w = n(T, (H + 2 * Hkv) * d), n(T, (H + 2 * Hkv) * d), H + Hkv
    gains, shifts = [n(d) for _ in range(2)], [n(d) for _ in range(2)]
    pos = torch.randint(-5, 300, (2, T), generator=g, device="cuda", dtype=torch.int32)
    sections = (d // 4, d // 4)
    axis, freq = P.pair_table(d, sections, "dealt", 1e4)
    table = torch.empty(mb.rope_axes_table_bytes(d), dtype=torch.uint8, device="cuda")
    mb.op_rope_axes_table(None, 256, d, sections, "dealt", 1e4, table)
    angle = (pos.double()[torch.from_numpy(axis).cuda()].t() * torch.from_numpy(freq).cuda())[:, None]
    cos, sin = torch.cos(angle), torch.sin(angle)
    cut = (lambda a: a.chunk(2, 2)) if pairing == "halves" else (lambda a: (a[..., 0::2], a[..., 1::2]))

    def turned(a, sign):
        p, q = cut(a)
        parts = (p * cos - sign * q * sin, sign * p * sin + q * cos)
        return torch.cat(parts, 2) if pairing == "halves" else torch.stack(parts, 3).flatten(2)

    per_head = lambda pair: torch.cat((pair[0].double().expand(H, d), pair[1].double().expand(Hkv, d)))
    gain, shift = per_head(gains), per_head(shifts)
    layer = norm == "layernorm"
    xs, ds = x.view(T, -1, d)[:, :w].double(), dy.view(T, -1, d)[:, :w].double()
    centred = xs - xs.mean(2, keepdim=True) if layer else xs
    rstd = torch.rsqrt((centred * centred).mean(2, keepdim=True) + 1e-5)
    xhat = centred * rstd
    y = turned(xhat * gain + shift if layer else xhat * gain, 1)
    up = turned(ds, -1)
    m = up * gain
    dx = rstd * (m - (m.mean(2, keepdim=True) if layer else 0) - xhat * (m * xhat).mean(2, keepdim=True))
    peak = 2 * ds.abs().amax(2, keepdim=True) * gain.abs().max()
    part = lambda a: (a[:, :H].sum((0, 1)), a[:, H:].sum((0, 1)))
    return dict(x=x, dy=dy, gains=gains, shifts=shifts, pos=pos, table=table, y=y, dx=dx, y_size=2 * (xhat.abs().amax(2, keepdim=True) * gain.abs().max() + shift.abs().max()),
                dx_size=rstd * peak * (2 + xhat.abs().amax(2, keepdim=True)), dgain=part(up * xhat), dshift=part(up), dgain_size=part((up * xhat).abs() + up.abs()),
                dshift_size=part(2 * up.abs()))


def near(got, ref, bound, what):
    over = (got.double() - ref).abs() - bound
    assert bool(torch.isfinite(got).all()) and float(over.max()) <= 0, (what, float(over.max()))


@pytest.mark.parametrize("dtype,norm,T,H,Hkv,d,pairing", [
    ("bf16", "rmsnorm", 33000, 12, 4, 128, "halves"), ("bf16", "layernorm", 33000, 12, 4, 128, "adjacent"), ("f32", "layernorm", 33000, 12, 4, 64, "halves"),
    ("f32", "rmsnorm", 33000, 6, 2, 128, "adjacent"), ("bf16", "rmsnorm", 17000, 12, 4, 256, "adjacent")])
def test_rows_past_the_caches(mb, dtype, norm, T, H, Hkv, d, pairing):
    """More than 256 MB read and written, in rows whose halves of a head are whole lines, also in place; every element, and the gains' sums over more than 8192 tokens
    (about 200 additions one after the other: waves of 9 tokens of 12 heads, 8 waves, slices of 64 partitions)."""
    es = 2 if dtype == "bf16" else 4
    assert 2 * T * (H + Hkv) * d * es > 256 << 20 and d // 2 * es % 128 == 0
    r = rows_on_gpu(mb, dtype, norm, T, H, Hkv, d, pairing, 91)
    layer, w, rel = norm == "layernorm", H + Hkv, 2.0 ** -8 if dtype == "bf16" else 0.0
    head = (T, H, Hkv, d, 1e-5, pairing, 2, r["pos"], r["table"])
    gq, gk, bq, bk = r["gains"][0], r["gains"][1], r["shifts"][0] if layer else None, r["shifts"][1] if layer else None
    y = torch.empty_like(r["x"])
    mb.op_qk_norm_rope_fwd(None, 256, dtype, norm, *head, r["x"], gq, bq, gk, bk, y)
    rows = lambda t: t.view(T, -1, d)
    near(rows(y)[:, :w], r["y"], r["y"].abs() * rel + 32 * U * r["y_size"], "y")
    assert torch.equal(rows(y)[:, w:], rows(r["x"])[:, w:])
    here = r["x"].clone()
    mb.op_qk_norm_rope_fwd(None, 256, dtype, norm, *head, here, gq, bq, gk, bk, here)
    assert torch.equal(here, y)
    outs = []
    for quota, into in ((256, torch.empty_like(y)), (64, torch.empty_like(y)), (256, r["dy"].clone())):
        grads = [torch.empty_like(gq) for _ in range(4)]
        scratch = torch.empty(mb.qk_norm_rope_bwd_scratch_bytes(d), dtype=torch.uint8, device="cuda")
        up = into if len(outs) == 2 else r["dy"]
        mb.op_qk_norm_rope_bwd(None, quota, dtype, norm, *head, r["x"], gq, gk, up, into, grads[0], grads[2] if layer else None, grads[1], grads[3] if layer else None, scratch)
        outs.append([into] + grads[:4 if layer else 2])
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(outs[0], o))
    near(rows(outs[0][0])[:, :w], r["dx"], r["dx"].abs() * rel + 64 * U * r["dx_size"], "dx")
    assert torch.equal(rows(outs[0][0])[:, w:], rows(r["dy"])[:, w:])
    for part in (0, 1):
        near(outs[0][1 + part], r["dgain"][part], r["dgain"][part].abs() * rel + 512 * U * r["dgain_size"][part], ("dgain", part))
        if layer:
            near(outs[0][3 + part], r["dshift"][part], r["dshift"][part].abs() * rel + 512 * U * r["dshift_size"][part], ("dshift", part))


@pytest.mark.parametrize("T,H,Hkv,d,shift", [(2100, 3, 1, 6, 0), (2600, 2, 1, 250, 0), (8300, 2, 1, 64, 1), (8300, 2, 1, 64, 0)])
@pytest.mark.parametrize("norm", ["rmsnorm", "layernorm"])
def test_partitions_of_more_tokens(mb, norm, T, H, Hkv, d, shift):
    """Element by element, partitions of more than four tokens; in vectors, more than 8192 tokens; outputs off 16-byte boundaries."""
    c = Case(mb, "bf16", norm, T, H, Hkv, d, (d // 4, d // 4), "dealt", "halves")
    scratch = torch.full((mb.qk_norm_rope_bwd_scratch_bytes(d) // 4,), float("nan"), device="cuda")
    outs, layer = [], norm == "layernorm"
    for quota in (256, 24):
        x, dy, dx = Framed(c.x, "bf16", shift), Framed(c.dy, "bf16", shift), Framed(None, "bf16", shift, c.x.shape)
        grads, gains = [Framed(None, "bf16", 1, (d,)) for _ in range(4)], [to_dev(v, "bf16") for v in c.gains]
        mb.op_qk_norm_rope_bwd(None, quota, "bf16", norm, T, H, Hkv, d, 1e-5, "halves", 2, c.pos_, c.table_, x.t, gains[0], gains[1], dy.t, dx.t, grads[0].t,
                               grads[2].t if layer else None, grads[1].t, grads[3].t if layer else None, scratch)
        torch.cuda.synchronize()
        assert x.framed() and dy.framed() and dx.framed() and all(g.framed() for g in grads)
        outs.append([bits(dx.t)] + [bits(g.t) for g in grads])
    assert all(np.array_equal(a, b) for a, b in zip(*outs))
    for part in (0, 1):
        _, xhat, rstd = P.head_norm(c.parts(c.x)[part], norm, 1e-5, c.gains[part], c.shifts[part])
        g = c.rotate(c.parts(c.dy)[part], -1)
        dx_ref, dgain, dshift = P.head_norm_bwd(g, xhat, rstd, norm, c.gains[part])
        size = rstd * 2 * np.abs(c.gains[part]).max() * np.abs(c.parts(c.dy)[part]).max(2, keepdims=True) * (2 + np.abs(xhat).max(2, keepdims=True))
        within(c.parts(from_dev(dx.t))[part], dx_ref, last("bf16", dx_ref) + 64 * U * size, "dx")
        within(from_dev(grads[part].t), dgain, last("bf16", dgain) + 512 * U * (np.abs(g * xhat) + np.abs(g)).sum((0, 1)), "dgain")
        if layer:
            within(from_dev(grads[2 + part].t), dshift, last("bf16", dshift) + 1024 * U * np.abs(g).sum((0, 1)), "dshift")
