"""Pins of the plain definitions of cross entropy behind a linear layer, grouped products and dropout in oracle/operators.py."""
import numpy as np
import pytest

from oracle import operators as P


def test_philox_known_answers():
    """The test vectors that its authors publish with it (kat_vectors: philox4x32, 10 rounds)."""
    ones = 0xFFFFFFFF
    assert P.philox4x32((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert P.philox4x32((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert P.philox4x32((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_keeps_what_its_bits_say():
    # the first block of counter 0 under key 0: two elements to a word, the low half first
    keeps, scale = P.dropout_keeps(range(8), 0x6000 / 65536, 0, 0, 0)
    halves = [0xE8D5, 0x6627, 0xC58D, 0xE169, 0xAC4C, 0xBC57, 0xDBD8, 0x9B00]
    assert list(keeps) == [h >= 0x6000 for h in halves]
    assert scale == 65536 / (65536 - 0x6000)
    keeps, scale = P.dropout_keeps(range(100), 0.0, 1, 2, 3)
    assert keeps.all() and scale == 1.0
    keeps, scale = P.dropout_keeps(range(100), 1.0, 1, 2, 3)
    assert not keeps.any() and scale == 0.0
    # offset and site are one number
    assert np.array_equal(P.dropout_keeps(range(99), 0.5, 3, 7, 2)[0], P.dropout_keeps(range(99), 0.5, 5, 7, 0)[0])
    # 40000 elements: off the expected share by five standard deviations at most
    p = 0.1
    assert abs(P.dropout_keeps(range(40000), p, 0, 5, 0)[0].mean() - (1 - p)) < 5 * np.sqrt(p * (1 - p) / 40000)


@pytest.mark.parametrize("smoothing,denom", [(0.0, 0.0), (0.2, 0.0), (0.1, 7.0)])
def test_cross_entropy_gradients_against_differences(smoothing, denom):
    rng = np.random.default_rng(3)
    x, table, targets = rng.normal(size=(6, 5)), rng.normal(size=(7, 5)), np.array([0, -1, 6, 3, 7, 3])
    loss, losses, dx, dtable = P.linear_ce(x, table, targets, smoothing, denom)
    assert losses[1] == losses[4] == 0 and not dx[1].any() and not dx[4].any()
    assert np.isclose(loss, losses.sum() / (denom or 4))
    # written out for one token
    z = table @ x[2]
    lse = np.log(np.exp(z).sum())
    assert np.isclose(losses[2], lse - (1 - smoothing) * z[6] - smoothing * z.mean())
    step = 1e-6                                  # central differences: off by about step^2, and 1e-16 / step
    for at, grad in ((x, dx), (table, dtable)):
        for i in np.ndindex(at.shape):
            keep = at[i]
            at[i] = keep + step
            up = P.linear_ce(x, table, targets, smoothing, denom)[0]
            at[i] = keep - step
            down = P.linear_ce(x, table, targets, smoothing, denom)[0]
            at[i] = keep
            assert abs((up - down) / (2 * step) - grad[i]) < 1e-8


def test_cross_entropy_of_nothing():
    loss, losses, dx, dtable = P.linear_ce(np.ones((3, 2)), np.ones((4, 2)), np.array([-1, 4, -100]))
    assert loss == 0 and not losses.any() and not dx.any() and not dtable.any()


def test_grouped_products_are_those_of_the_slices():
    rng = np.random.default_rng(4)
    offsets, k, n = [2, 5, 5, 9], 3, 4
    x, dy, w = rng.normal(size=(11, k)), rng.normal(size=(11, n)), rng.normal(size=(3, k, n))
    y = P.grouped_linear("fwd", offsets, x, w, np.full((11, n), 8.0))
    assert np.allclose(y[2:5], x[2:5] @ w[0]) and np.allclose(y[5:9], x[5:9] @ w[2])
    assert (y[:2] == 8).all() and (y[9:] == 8).all()
    dx = P.grouped_linear("dgrad", offsets, dy, w, np.full((11, k), 8.0))
    dw = P.grouped_linear("wgrad", offsets, x, dy, np.full((3, k, n), 8.0))
    assert not dw[1].any()
    # <dy, y> is linear in x and in w: both gradients give it back
    inside = (dy[2:9] * y[2:9]).sum()
    assert np.isclose((dx[2:9] * x[2:9]).sum(), inside) and np.isclose((dw * w).sum(), inside)
