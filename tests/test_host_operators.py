"""Refusals of the operators around a layer's products: found before the device is asked for, so they are the same
here and on a GPU.  Addresses stand for device memory and are never read."""
import pytest

from paper_2605_18710_amd import binding as mb

A, B, C, D, E, F = (0x10000000 * i for i in range(1, 7))


def status(call, *args, **kw):
    with pytest.raises(mb.MosaicError) as e:
        call(*args, **kw)
    return e.value.status


def table(d=64, sections=(16, 16), order="own", base=1e4, at=A):
    return status(mb.op_rope_axes_table, None, 256, d, sections, order, base, at)


def test_table_of_axes():
    assert table(d=0) == table(d=63) == table(d=-2) == mb.EINVAL
    assert table(d=258) == mb.EUNSUPPORTED
    assert table(sections=()) == table(sections=(1,) * 5) == table(sections=(-1, 4)) == table(sections=(16, 17)) == mb.EINVAL
    assert table(base=0.0) == table(base=-1.0) == table(base=float("nan")) == table(base=float("inf")) == mb.EINVAL
    assert table(at=None) == table(at=A + 8) == mb.EINVAL
    assert mb.rope_axes_table_bytes(64) == 32 * 16 and mb.rope_axes_table_bytes(0) == mb.rope_axes_table_bytes(-4) == 0


def rope(dtype="bf16", T=4, H=4, Hkv=2, d=64, pairing="halves", direction=1, axes=2, pos=A, tab=B, x=C, y=D):
    return status(mb.op_rope_axes, None, 256, dtype, T, H, Hkv, d, pairing, direction, axes, pos, tab, x, y)


def fwd(norm="rmsnorm", T=4, H=4, Hkv=2, d=64, eps=1e-6, axes=2, pos=A, tab=B, x=C, y=D, gq=E, bq=None, gk=F, bk=None):
    return status(mb.op_qk_norm_rope_fwd, None, 256, "bf16", norm, T, H, Hkv, d, eps, "halves", axes, pos, tab, x, gq, bq, gk, bk, y)


def bwd(norm="rmsnorm", T=4, H=4, Hkv=2, d=64, eps=1e-6, axes=2, pos=A, tab=B, x=C, dy=D, dx=D, dgq=E, dbq=None, dgk=E + 512, dbk=None, scratch=F):
    return status(mb.op_qk_norm_rope_bwd, None, 256, "bf16", norm, T, H, Hkv, d, eps, "halves", axes, pos, tab, x, A + 64, A + 256, dy, dx, dgq, dbq, dgk, dbk, scratch)


def test_heads():
    for call in (rope, fwd, bwd):
        assert call(T=-1) == call(H=0) == call(Hkv=0) == call(H=5) == call(d=0) == call(d=33) == mb.EINVAL
        assert call(d=258) == mb.EUNSUPPORTED
        assert call(H=1 << 24, Hkv=1 << 24, d=256) == mb.EUNSUPPORTED
        assert call(T=1 << 61) == mb.EINVAL
        assert call(axes=0) == call(axes=5) == call(pos=None) == call(tab=B + 4) == mb.EINVAL
        assert call(x=None) == mb.EINVAL
    assert rope(direction=0) == rope(tab=None) == rope(y=None) == mb.EINVAL
    assert fwd(norm="none") == bwd(norm="none") == mb.EINVAL
    assert fwd(eps=0.0) == fwd(eps=float("nan")) == bwd(eps=-1.0) == mb.EINVAL
    assert fwd(norm="layernorm") == bwd(norm="layernorm") == mb.EINVAL            # no shifts
    assert fwd(gq=None) == fwd(gk=None) == fwd(y=None) == bwd(dgq=None) == bwd(dgk=None) == bwd(dx=None) == mb.EINVAL
    assert bwd(scratch=None) == bwd(scratch=F + 8) == mb.EINVAL


def test_rows_that_overlap():
    row = 8 * 64 * 2
    for step in (16, row, -16):
        assert rope(y=C + step) == fwd(y=C + step) == bwd(dx=D + step) == bwd(dx=C + step) == mb.EINVAL
    assert bwd(dx=C) == mb.EINVAL                                                # the rows before the norm are read


def test_packed():
    pack = lambda n=64, x=A, q=B, scale=C: status(mb.op_pack8, None, 256, "f32", n, x, q, scale)
    unpack = lambda n=64, x=A, q=B, scale=C: status(mb.op_unpack8, None, 256, "f32", n, q, scale, x)
    for call in (pack, unpack):
        assert call(n=-1) == call(x=None) == call(q=None) == call(scale=None) == call(q=A + 255) == call(scale=A + 1) == call(n=1 << 60) == mb.EINVAL
    assert pack(scale=B + 63) == mb.EINVAL
    assert [mb.pack8_scale_bytes(n) for n in (-1, 0, 1, 32, 33)] == [0, 0, 1, 1, 2]


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "swiglu"])
def test_packed_activation(act):
    size = 4 * 64 * 4 * (2 if act == "swiglu" else 1)          # bytes of z, dz
    fwd = lambda T=4, f=64, z=A, a=B, q=C, scale=D: status(mb.op_act_fwd_pack8, None, 256, "f32", act, T, f, z, a, q, scale)
    bwd = lambda T=4, f=64, q=A, scale=B, da=C, dz=D, a=E: status(mb.op_act_bwd_pack8, None, 256, "f32", act, T, f, q, scale, da, dz, a)
    for call in (fwd, bwd):
        assert call(T=-1) == call(f=-8) == call(T=1 << 40, f=1 << 40) == call(q=None) == call(scale=None) == mb.EINVAL
    assert fwd(z=None) == fwd(a=None) == fwd(a=A) == fwd(a=A + size - 4) == fwd(q=A + 4) == fwd(scale=C + 1) == fwd(q=B) == mb.EINVAL
    assert bwd(da=None) == bwd(dz=None) == bwd(dz=C + 4) == bwd(a=C) == bwd(a=D + size - 4) == bwd(dz=A) == bwd(a=B) == mb.EINVAL
    if act == "swiglu":
        assert bwd(dz=C) == mb.EINVAL


def test_packed_weight_gradient():
    call = lambda T=4, k=8, n=8, q=A, scale=B, dy=C, dw=D, scratch=E: status(mb.op_linear_wgrad_pack8, None, 256, "bf16", T, k, n, q, scale, dy, dw, None, scratch)
    assert call(T=-1) == call(k=0) == call(n=-1) == call(q=None) == call(scale=None) == call(dy=None) == call(dw=None) == call(scratch=None) == mb.EINVAL
    assert call(scratch=E + 4) == call(T=1 << 57, k=1 << 10) == mb.EINVAL
    assert call(T=0) == mb.EUNSUPPORTED
    assert status(mb.op_linear_wgrad_pack8, None, 256, "f32", 4, 8, 6, A, B, C, D, F, E) == mb.EUNSUPPORTED      # db of 6 columns
    assert mb.linear_wgrad_pack8_scratch_bytes("bf16", 0, 8, 8) == 0
    assert mb.linear_wgrad_pack8_scratch_bytes("f32", 100, 8, 8) >= mb.linear_wgrad_pack8_scratch_bytes("bf16", 100, 8, 8) >= 1600


def test_unknown_numbers():
    l = mb.lib()
    assert l.mosaic_op_pack8(None, 256, 7, 64, A, B, C) == mb.EINVAL
    assert l.mosaic_op_act_fwd_pack8(None, 256, 1, 3, 4, 64, A, B, C, D) == mb.EINVAL
    assert l.mosaic_op_act_bwd_pack8(None, 256, 1, -1, 4, 64, A, B, C, D, E) == mb.EINVAL
    assert l.mosaic_op_rope_axes(None, 256, 5, 4, 4, 2, 64, 0, 1, 1, A, B, C, D) == mb.EINVAL
    assert l.mosaic_op_rope_axes(None, 256, 1, 4, 4, 2, 64, 2, 1, 1, A, B, C, D) == mb.EINVAL
    sections = (mb.C.c_int32 * 1)(8)
    assert l.mosaic_op_rope_axes_table(None, 256, 64, 1, sections, 3, 10.0, A) == mb.EINVAL
    assert l.mosaic_op_rope_axes_table(None, 256, 64, 1, None, 0, 10.0, A) == mb.EINVAL


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_weight_gradient_with_buffers_that_overlap(dtype):
    T, k, n, es = 40, 16, 24, 4 if dtype == "f32" else 2
    size = mb.linear_wgrad_pack8_scratch_bytes(dtype, T, k, n)
    G = 0x70000000
    call = lambda q=A, scale=B, dy=C, dw=D, db=E, scratch=F: status(mb.op_linear_wgrad_pack8, None, 256, dtype, T, k, n, q, scale, dy, dw, db, scratch)
    inputs = ((A, T * k), (B, T * k // 32), (C, T * n * es))
    for first, length in inputs:
        for other in (first, first + length - 1):
            assert call(dw=other) == call(db=other) == mb.EINVAL
        assert call(scratch=first) == call(dw=first - k * n * es + 1) == call(db=first - n * es + 1) == mb.EINVAL
        assert call(scratch=first - (size - 1) // 16 * 16) == call(scratch=first + (length - 1) // 16 * 16) == mb.EINVAL
    assert call(db=D) == call(db=D + k * n * es - 1) == call(db=D - n * es + 1) == call(scratch=D) == call(scratch=E) == call(db=F + size - 1) == call(dw=F + size - 1) == mb.EINVAL
    assert status(mb.op_linear_wgrad_pack8, None, 256, dtype, T, k, n, A, B, C, C, None, G) == mb.EINVAL             # without db too


def test_packed_weight_gradient_of_sizes_past_31_bits():
    """Refused before the input is unpacked: nothing is launched for a call that fails."""
    for T, k, n in ((1 << 31, 8, 8), (8, 1 << 31, 8), (8, 8, 1 << 31)):
        assert status(mb.op_linear_wgrad_pack8, None, 256, "bf16", T, k, n, 1 << 40, 1 << 42, 1 << 44, 1 << 46, None, 1 << 48) == mb.EUNSUPPORTED


@pytest.mark.parametrize("norm", ["rmsnorm", "layernorm"])
def test_gradients_of_head_norms_that_overlap(norm):
    """The four gradients, the rows' gradient and scratch memory each lie apart: the sums are written while others are read."""
    d, row, es = 64, 8 * 64, 2
    size = mb.qk_norm_rope_bwd_scratch_bytes(d)
    layer = norm == "layernorm"
    apart = dict(dgq=E, dgk=E + 512, **(dict(dbq=E + 1024, dbk=E + 1536) if layer else {}))
    call = lambda **kw: bwd(norm=norm, **{**apart, **kw})
    for one in apart:
        for other in apart:
            if other != one:
                assert call(**{one: apart[other]}) == call(**{one: apart[other] + d * es - 2}) == mb.EINVAL
        assert call(**{one: D}) == call(**{one: D + 4 * row * es - 2}) == call(**{one: F}) == call(**{one: F + size - 2}) == mb.EINVAL
    for buffer in (C, D):
        assert call(scratch=buffer) == call(scratch=buffer + 4 * row * es - 16) == call(scratch=buffer - size + 16) == mb.EINVAL
    assert call(scratch=A + 64, dx=D) == call(scratch=A + 256) == mb.EINVAL                     # the gains
