"""Cross entropy over a vocabulary of which rows are masked: column 0 of X is 1, and the table holds the mask's value there for rows that no token may take (padding of the
vocabulary, forbidden words) and 0 for the others, whose logits lie far below zero or not.  A masked row's probability is 0 in 64 bits as in 32, so the results are those of
the table without these rows, and its own gradient is 0.  (An infinite entry of the table times a gradient of 0 is NaN: in column 0 of dX, and only there.)"""
import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2605_18710_amd import synth
from helpers import from_dev, quantize
from test_gpu_linear_ce import U, bounds, call, close

pytestmark = pytest.mark.gpu
MASKS = [-np.inf]


def masked_inputs(T, h, V, level, value, dtype, seed=11):
    """Allowed logits lie around `level`.  Masked: whole blocks of 16, 64 and 4096 columns, the first ones and the last, and some rows here and there."""
    x = synth.normal(seed, (T, h))
    table = synth.normal(seed + 1, (V, h)) / np.sqrt(h)
    v = np.arange(V)
    masked = (v // 64 % 3 == 0) | (v // 16 % 7 == 2) | (v % 11 == 5) | (v // 4096 % 3 == 0) & (V > 8192) | (v >= V - 20)
    if V > 8192:
        masked |= v >= V // 4096 * 4096
    x[:, 0] = x[:, 1] = 1.0
    table[:, 0], table[:, 1] = 0.0, level
    table[masked, 0] = value
    allowed = np.flatnonzero(~masked)
    target = allowed[synth.integers(seed + 2, (T,), 0, len(allowed))]
    target[T // 2:T // 2 + T // 5] = -1
    return quantize(x, dtype), quantize(table, dtype), target.astype(np.int32), allowed


# up to 16 tokens (blocks of 16 columns; gradients by few_tile); blocks joined by the gradient's own launch (V up to 4096) and ahead of it; large tiles of 128 and 256 rows; fp32 rows held
# by a wave, a workgroup, and in blocks of 4096 columns
SHAPES = [(7, 64, 1000), (16, 200, 5000), (40, 72, 300), (300, 136, 3000), (100, 256, 30000), (1500, 512, 6000), (20, 64, 13001)]


@pytest.mark.parametrize("value", MASKS)
@pytest.mark.parametrize("level", [-110.0, 3.0])
@pytest.mark.parametrize("T,h,V", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_rows_of_the_table(T, h, V, level, value, dtype):
    x, table, target, allowed = masked_inputs(T, h, V, level, value, dtype)
    place = np.full(V, -1)
    place[allowed] = np.arange(len(allowed))
    small = np.where(target >= 0, place[target], -1)
    loss, losses, dx, dtable = O.linear_ce(x, table[allowed], small)
    bl, bx, bt = bounds(x, table[allowed], small, 0.0, 0.0, dtype)
    n = (small >= 0).sum()
    got = call(x, table, target, 0.0, 0.0, dtype)
    close(from_dev(got["losses"]), losses, bl, "losses")
    close(got["loss"], loss, bl.sum() / n + 4 * U * abs(loss), "loss")
    close(from_dev(got["dx"])[:, 1:], dx[:, 1:], bx[:, 1:], "dx")
    close(from_dev(got["dtable"])[allowed], dtable, bt, "dtable")
    rest = np.delete(from_dev(got["dtable"]), allowed, axis=0)
    assert not rest.any()
    alone = call(x, table, target, 0.0, 0.0, dtype, grad=False)
    close(from_dev(alone["losses"]), losses, bl, "losses alone")
    close(alone["loss"], loss, bl.sum() / n + 4 * U * abs(loss), "loss alone")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(5, 3000), (40, 3000), (40, 6001), (40, 9001)])
def test_every_row_masked_by_infinity(T, V, dtype):
    """No distribution is left: NaN, as the definition gives, for that token and no other."""
    x, table, target, allowed = masked_inputs(T, 64, V, -110.0, -np.inf, dtype)
    base = call(x, table, target, 0.0, 0.0, dtype)
    x[3, 1] = np.inf                                        # times -110: -inf in every column
    target[3] = allowed[0]
    bad = call(x, table, target, 0.0, 10.0, dtype)
    keep = [t for t in range(T) if t != 3]
    assert torch.isnan(bad["losses"][3]) and torch.isfinite(bad["losses"][keep]).all() and torch.equal(bad["losses"][keep], base["losses"][keep])
