"""Cross entropy in fp32 on rows of whole 16-byte pieces (tiles, copies and joins of four values at a time), where the vocabulary is a multiple of four and where it is not; bounds
element by element as for rows of odd length."""
import numpy as np
import pytest

from oracle import operators as O
from helpers import from_dev
from test_gpu_linear_ce import CASES, U, bounds, call, close, inputs

pytestmark = pytest.mark.gpu

# tiles of 16 x 16 whose last row of dz ends inside a piece; contractions that are cut, over the vocabulary and over the tokens; rows past what a workgroup holds
MORE = [(300, 72, 130, 0.1, 0.4), (300, 72, 131, 0.0, 0.0), (18, 404, 4169, 0.0, 0.1), (2600, 36, 203, 0.1, 0.0), (3, 520, 9001, 0.1, 0.0), (388, 752, 8203, 0.0, 0.1), (64, 100, 12290, 0.1, 0.2),
        (1100, 132, 8195, 0.0, 0.3), (5, 928, 33331, 0.1, 0.0)]


@pytest.mark.parametrize("T,h,V,smoothing,ignored", CASES + MORE)
def test_loss_and_gradients_of_whole_pieces(T, h, V, smoothing, ignored):
    assert h % 4 == 0
    x, table, target = inputs(T, h, V, ignored, "f32")
    loss, losses, dx, dtable = O.linear_ce(x, table, target, smoothing)
    bl, bx, bt = bounds(x, table, target, smoothing, 0.0, "f32")
    n = max(1, ((target >= 0) & (target < V)).sum())
    got = call(x, table, target, smoothing, 0.0, "f32")
    close(from_dev(got["losses"]), losses, bl, "losses")
    close(got["loss"], loss, bl.sum() / n + 4 * U * abs(loss), "loss")
    close(from_dev(got["dx"]), dx, bx, "dx")
    close(from_dev(got["dtable"]), dtable, bt, "dtable")
    alone = call(x, table, target, smoothing, 0.0, "f32", grad=False)
    close(from_dev(alone["losses"]), losses, bl, "losses alone")
    assert alone["loss"] == got["loss"]


def test_last_row_of_the_input_gradient():
    """V of 4 i + 1, 2, 3: the last values of the last counted row of dz lie in a piece that ends past the row.  Their rows of the table are a thousand times the others, so a lost one shows."""
    for T, h, V in ((300, 72, 129), (300, 72, 130), (300, 72, 131), (17, 400, 1021), (33, 64, 257)):
        x, table, target = inputs(T, h, V, 0.0, "f32")
        x *= 2.0 ** -14
        table[-3:] *= 1024.0
        target[-1] = V - 1
        _, _, dx, _ = O.linear_ce(x, table, target)
        bx = bounds(x, table, target, 0.0, 0.0, "f32")[1]
        assert bx[-1].max() < 0.3 * np.median(np.abs(table[-3:])) / V / T          # what one of them is worth
        close(from_dev(call(x, table, target, 0.0, 0.0, "f32")["dx"]), dx, bx, (T, h, V))
