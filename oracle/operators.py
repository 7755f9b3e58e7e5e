"""Plain definitions, in 64 bits, of the operators around a layer's products: rotary positions with several axes, the
norm of every query and key head with that rotation, and activations kept in 8 bits."""
import math

import numpy as np


def pair_table(d, sections, order, base):
    """(axis, frequency) of each pair of a head; axis -1: the pair stays."""
    axis, freq = np.full(d // 2, -1), np.zeros(d // 2)
    if order == "dealt":
        left, a = list(sections), 0
        for i in range(sum(sections)):
            while left[a] == 0:
                a = (a + 1) % len(left)
            axis[i], freq[i] = a, base ** (-2.0 * i / d)
            left[a] -= 1
            a = (a + 1) % len(left)
        return axis, freq
    i = 0
    for a, s in enumerate(sections):
        for j in range(s):
            axis[i], freq[i] = a, base ** (-j / s) if order == "own" else base ** (-2.0 * i / d)
            i += 1
    return axis, freq


def rotate(x, pos, axis, freq, pairing, direction=1):
    """x [T, heads, d]; pos [axes, T]."""
    d = x.shape[2]
    angle = np.where(axis < 0, 0.0, direction * np.asarray(pos, dtype=np.float64)[np.maximum(axis, 0)].T * freq)[:, None, :]
    first, second = (slice(0, d // 2), slice(d // 2, d)) if pairing == "halves" else (slice(0, d, 2), slice(1, d, 2))
    y = np.empty_like(x)
    y[..., first] = x[..., first] * np.cos(angle) - x[..., second] * np.sin(angle)
    y[..., second] = x[..., first] * np.sin(angle) + x[..., second] * np.cos(angle)
    return y


def head_norm(x, norm, eps, gain, shift=None):
    """(result, xhat, rstd) of a norm over the last axis."""
    mean = x.mean(-1, keepdims=True) if norm == "layernorm" else 0.0
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    xhat = (x - mean) * rstd
    return xhat * gain + (shift if norm == "layernorm" else 0.0), xhat, rstd


def head_norm_bwd(g, xhat, rstd, norm, gain):
    """(dx, dgain, dshift) from the gradient g of the norm's result [T, heads, d]."""
    w = g * gain
    centre = w.mean(-1, keepdims=True) if norm == "layernorm" else 0.0
    dx = rstd * (w - centre - xhat * (w * xhat).mean(-1, keepdims=True))
    return dx, (g * xhat).sum((0, 1)), g.sum((0, 1))


def pack8(x):
    """(q int8, byte uint8) of the flat elements in blocks of 32."""
    x = np.asarray(x, dtype=np.float64).reshape(-1)
    blocks = np.concatenate([x, np.zeros(-x.size % 32)]).reshape(-1, 32)
    q, byte = np.zeros(blocks.shape, dtype=np.int8), np.zeros(len(blocks), dtype=np.uint8)
    for b, row in enumerate(blocks):
        top = np.abs(row).max()
        if not math.isfinite(top):
            byte[b] = 255
            continue
        e = -127
        while top > 127.5 * 2.0 ** e:
            e += 1
        byte[b] = e + 127
        q[b] = np.clip(np.rint(row * 2.0 ** -e), -127, 127)
    return q.reshape(-1)[:x.size], byte


def unpack8(q, byte):
    step = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return q.astype(np.float64) * np.repeat(step, 32)[:q.size]
