"""Pins of the plain definitions in oracle/operators.py: written-out cases, invariants and finite differences."""
import numpy as np
import pytest

from oracle import operators as P


def test_pairs_are_dealt_to_axes():
    axis, freq = P.pair_table(16, (2, 3, 2), "split", 100.0)
    assert list(axis) == [0, 0, 1, 1, 1, 2, 2, -1]
    assert np.allclose(freq[:7], 100.0 ** (-np.arange(7) / 8.0))
    axis, freq = P.pair_table(16, (2, 3, 2), "own", 100.0)
    assert list(axis) == [0, 0, 1, 1, 1, 2, 2, -1]
    assert np.allclose(freq[:7], [1, 0.1, 1, 100 ** (-1 / 3), 100 ** (-2 / 3), 1, 0.1])
    axis, _ = P.pair_table(16, (4, 2, 2), "dealt", 100.0)
    assert list(axis) == [0, 1, 2, 0, 1, 2, 0, 0]
    axis, _ = P.pair_table(8, (0, 3), "dealt", 100.0)
    assert list(axis) == [1, 1, 1, -1]


@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
def test_rotation_turns_pairs_and_back(pairing):
    rng = np.random.default_rng(1)
    x, pos = rng.normal(size=(5, 3, 16)), rng.integers(-1000, 1000, size=(2, 5))
    axis, freq = P.pair_table(16, (3, 4), "own", 10.0)
    y = P.rotate(x, pos, axis, freq, pairing)
    assert np.allclose(P.rotate(y, pos, axis, freq, pairing, -1), x)
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    stays = [7, 15] if pairing == "halves" else [14, 15]
    assert np.array_equal(y[..., stays], x[..., stays])
    a, b = (0, 8) if pairing == "halves" else (0, 1)
    angle = pos[0][:, None] * 1.0
    assert np.allclose(y[..., a] + 1j * y[..., b], (x[..., a] + 1j * x[..., b]) * np.exp(1j * angle))


@pytest.mark.parametrize("norm", ["rmsnorm", "layernorm"])
def test_head_norm_gradients_against_differences(norm):
    rng = np.random.default_rng(2)
    x, gain, shift = rng.normal(0.3, 1, size=(2, 3, 8)), rng.normal(1, 0.2, 8), rng.normal(size=8)
    up = rng.normal(size=x.shape)
    value = lambda x, gain, shift: (P.head_norm(x, norm, 1e-3, gain, shift)[0] * up).sum()
    _, xhat, rstd = P.head_norm(x, norm, 1e-3, gain, shift)
    grads = P.head_norm_bwd(up, xhat, rstd, norm, gain)
    for which, (at, grad) in enumerate(zip((x, gain, shift), grads)):
        if which == 2 and norm == "rmsnorm":
            continue
        for i in np.ndindex(at.shape):
            step = np.zeros_like(at); step[i] = 1e-6
            args = [x, gain, shift], [x, gain, shift]
            args[0][which], args[1][which] = at + step, at - step
            assert abs((value(*args[0]) - value(*args[1])) / 2e-6 - grad[i]) < 1e-7


def test_packing_written_out():
    x = np.zeros(70)
    x[:4] = [127.5, -127.5, 63.5, 0.5]       # e = 0: 127.5 is the largest that it holds, ties go to even
    x[32:35] = [255.0, 2.0, 3.0]             # e = 1
    x[64:66] = [1e-45, 0.0]                  # below the smallest step
    q, byte = P.pack8(x)
    assert list(byte) == [127, 128, 0]
    assert list(q[:4]) == [127, -127, 64, 0] and list(q[32:35]) == [127, 1, 2] and not q[64:].any()
    q, byte = P.pack8(np.array([np.nan, 1.0] + [0.0] * 30 + [np.inf, 2.0]))
    assert list(byte) == [255, 255] and np.isnan(P.unpack8(q, byte)).all()


def test_packing_is_off_by_half_a_step_at_most():
    rng = np.random.default_rng(3)
    x = rng.normal(size=1000) * np.exp(rng.normal(0, 20, size=1000))
    q, byte = P.pack8(x)
    step = np.repeat(2.0 ** (byte.astype(float) - 127), 32)[:1000]
    assert (np.abs(P.unpack8(q, byte) - x) <= step / 2).all()
    again = P.pack8(P.unpack8(q, byte))
    assert np.array_equal(P.unpack8(*again), P.unpack8(q, byte))
