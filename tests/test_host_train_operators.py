"""Refusals of the operators of a language module's training step: found before the device is asked for, so they are the same here and
on a GPU.  Addresses stand for device memory and are never read."""
import pytest

from paper_2605_18710_amd import binding as mb
from test_host_wait_states import listings, looking_back, matrix_too_close, vector_registers  # noqa: F401

A, B, C, D, E, F, G, H = (0x100000000 * i for i in range(1, 9))


def status(call, *args, **kw):
    with pytest.raises(mb.MosaicError) as e:
        call(*args, **kw)
    return e.value.status


def ce_fwd(dtype="bf16", T=4, h=64, V=100, smoothing=0.0, denom=0.0, targets=A, X=B, table=C, loss=D, losses=E, scratch=F):
    return status(mb.op_linear_ce_fwd, None, 256, dtype, T, h, V, smoothing, denom, targets, X, table, loss, losses, scratch)


def ce_grad(dtype="bf16", T=4, h=64, V=100, smoothing=0.0, denom=0.0, targets=A, X=B, table=C, loss=D, losses=E, scratch=F, dX=G, dtable=H):
    return status(mb.op_linear_ce_grad, None, 256, dtype, T, h, V, smoothing, denom, targets, X, table, loss, losses, dX, dtable, scratch)


@pytest.mark.parametrize("call", [ce_fwd, ce_grad])
def test_cross_entropy(call):
    nan, inf = float("nan"), float("inf")
    assert call(T=-1) == call(h=0) == call(V=0) == call(V=-5) == mb.EINVAL
    assert call(smoothing=-0.1) == call(smoothing=1.0) == call(smoothing=nan) == call(denom=-1.0) == call(denom=inf) == call(denom=nan) == mb.EINVAL
    assert call(targets=None) == call(X=None) == call(table=None) == call(loss=None) == call(scratch=None) == call(scratch=F + 128) == mb.EINVAL
    assert call(h=60) == call(X=B + 8) == call(table=C + 2) == mb.EUNSUPPORTED
    assert call(V=(1 << 22) + 1) == call(h=1 << 21) == call(h=8192, V=1 << 18) == call(T=1 << 31) == mb.EUNSUPPORTED
    assert call(dtype="f32", h=8192, V=1 << 17) == mb.EUNSUPPORTED
    for out in ("loss", "losses", "scratch"):
        for at in (A, B, C):
            assert call(**{out: at}) == mb.EINVAL
    assert call(losses=D) == call(loss=F + 4) == call(losses=F + 1024) == mb.EINVAL


def test_cross_entropy_gradients():
    assert ce_grad(dX=None, dtable=None) == mb.EINVAL
    assert ce_grad(dX=G + 8) == ce_grad(dtable=H + 4) == mb.EUNSUPPORTED
    for out in ("dX", "dtable"):
        for at in (A, B, C, F):
            assert ce_grad(**{out: at}) == mb.EINVAL
    assert ce_grad(dtable=G) == ce_grad(loss=G) == mb.EINVAL


def test_cross_entropy_scratch():
    """It grows with the tokens up to a piece of them, and holds no logits where the loss alone is asked for."""
    grad, fwd = mb.linear_ce_grad_scratch_bytes, mb.linear_ce_fwd_scratch_bytes
    for call in (grad, fwd):
        assert call("bf16", -1, 64, 100) == call("bf16", 4, 0, 100) == call("f32", 4, 64, 0) == 0
        assert call("bf16", 0, 64, 100) > 0 and call("f32", 1, 1, 1) > 0
    assert fwd("bf16", 8192, 4096, 32000) < 8192 * (4096 * 2 + 500 * 12 + 64) + (1 << 20)
    logits = 2 * 8192 * 32000
    pieces = 2048 * 65536 * 4                  # fp32 tiles of dX, where its contraction is cut
    assert logits < grad("bf16", 8192, 4096, 32000) < logits + pieces + 8192 * (4096 * 2 + 500 * 12 + 64) + (1 << 20)
    # 64 times the tokens: the logits of a piece, and the table's gradient in fp32
    assert grad("bf16", 64 * 8192, 4096, 32000) < (2 << 30) + 4 * 4096 * 32000 + pieces + 64 * 8192 * (4096 * 2 + 16) + 33554 * 500 * 12 + (1 << 24)


def grouped(form, dtype="bf16", T=4, groups=2, k=64, n=64, offsets=A, a=B, b=C, out=D):
    return status(getattr(mb, "op_grouped_linear_" + form), None, 256, dtype, T, groups, k, n, offsets, a, b, out)


@pytest.mark.parametrize("form", ["fwd", "dgrad", "wgrad"])
def test_grouped(form):
    assert grouped(form, T=-1) == grouped(form, groups=-1) == grouped(form, k=0) == grouped(form, n=-8) == mb.EINVAL
    assert grouped(form, groups=1025) == grouped(form, T=1 << 31) == grouped(form, k=1 << 29) == grouped(form, k=1 << 21, n=1 << 21) == mb.EUNSUPPORTED
    for name in ("offsets", "a", "b", "out"):
        assert grouped(form, **{name: None}) == mb.EINVAL
    assert grouped(form, out=A) == grouped(form, out=B) == grouped(form, out=C + 64) == grouped(form, out=B + 4 * 64 * 2 - 2) == mb.EINVAL


def test_dropout():
    call = lambda dtype="bf16", n=64, p=0.5, rng=A, x=B, R=C, y=D: status(mb.op_dropout, None, 256, dtype, n, p, 3, rng, x, R, y)
    assert call(n=-1) == call(n=1 << 60) == call(p=-0.01) == call(p=1.01) == call(p=float("nan")) == mb.EINVAL
    assert call(rng=None) == call(rng=A + 4) == call(x=None) == call(y=None) == mb.EINVAL
    assert call(y=B + 2) == call(y=C - 2) == call(y=A) == call(y=A + 8) == mb.EINVAL


def test_matrix_instructions_of_the_four_wave_kernel_keep_their_distance(listings):  # noqa: F811
    """The kernel writes its matrix instructions as strings, of whose latency the compiler knows nothing, and moves the accumulators where it has registers
    to move them to: not with tiles of 160 rows and more; lower tiles use the instruction itself."""
    seen = []
    for name, ins in listings:
        if "gemm_bf16_w4_kernel" in name:
            seen.append(int(name.split("w4_kernelILb")[1].split("Li")[2].split("E")[0]))      # rows of a tile / 32
            if seen[-1] > 4:
                assert not [x for x in ins if x[1] == "v_accvgpr_mov_b32"] and not matrix_too_close(ins), name
    assert set(seen) == {4, 5, 6, 7, 8}


def test_sums_wait_for_the_matrix_instructions(listings):  # noqa: F811
    """v_mfma_f32_16x16x4_f32 wants 10 wait states before anything else reads its result, v_mfma_f32_32x32x2_f32 18, v_mfma_f32_16x16x32_bf16 (here: in the
    kernels of few rows) 8.  The compiler does not see to it where the reader begins a block that can be reached around the loop of matrix instructions as well."""
    seen, bad = 0, []
    for name, ins in listings:
        waits = ((10, "v_mfma_f32_16x16x4_f32"), (18, "v_mfma_f32_32x32x2_f32"), (8, "v_mfma_f32_16x16x32_bf16"))[:3 if "few" in name else 2]
        if not any(x[1].startswith(tuple(which for _, which in waits)) for x in ins):
            continue
        seen += 1
        found = looking_back(ins)
        for i, (at, op, operands, _) in enumerate(ins):
            if op.startswith("v_mfma") or not op.startswith(("v_", "ds_write", "global_store", "buffer_store", "scratch_store")):
                continue
            uses = vector_registers(operands)
            for states, which in waits:
                if found(i, states, lambda x: x[1].startswith(which) and vector_registers(x[2].split(", ")[0]) & uses):  # noqa: B023
                    bad.append("%s: %x %s %s" % (name[:90], at, op, operands))
    assert seen > 20 and not bad, (len(bad), bad[:5])
