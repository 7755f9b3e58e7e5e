"""Plain definitions, in 64 bits, of the operators around a layer's products: rotary positions with several axes, the
norm of every query and key head with that rotation, activations kept in 8 bits, softmax cross entropy behind a linear
layer, products grouped by expert, and dropout."""
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


def linear_ce(x, table, targets, smoothing=0.0, denom=0.0):
    """(loss, losses [T], dx, dtable) of softmax cross entropy behind z = x table^T; a target outside the table: the token does not count."""
    T, V = len(x), len(table)
    counts = (targets >= 0) & (targets < V)
    at = np.flatnonzero(counts)
    D = denom if denom > 0 else max(1, len(at))
    losses, dx, dtable = np.zeros(T), np.zeros(x.shape), np.zeros(table.shape)
    rows = x[at]
    z = rows @ table.T
    top = z.max(1, keepdims=True) if len(at) else z[:, :1]
    lse = top + np.log(np.exp(z - top).sum(1, keepdims=True))
    one = np.zeros(z.shape)
    one[np.arange(len(at)), targets[at]] = 1.0
    q = (1.0 - smoothing) * one + smoothing / V
    losses[at] = lse[:, 0] - (z * q).sum(1)
    dz = (np.exp(z - lse) - q) / D
    dx[at] = dz @ table
    return losses.sum() / D, losses, dx, dz.T @ rows


def grouped_linear(form, offsets, a, b, out):
    """Rows offsets[g] .. offsets[g + 1] - 1 with matrix g; `out` [T, n], [T, k] or [groups, k, n] keeps its rows of no group."""
    out = out.copy()
    for g in range(len(offsets) - 1):
        r = slice(offsets[g], offsets[g + 1])
        if form == "fwd":
            out[r] = a[r] @ b[g]
        elif form == "dgrad":
            out[r] = a[r] @ b[g].T
        else:
            out[g] = a[r].T @ b[r]
    return out


def philox4x32(counter, key):
    """Ten rounds of Philox4x32 (Salmon, Moraes, Dror and Shaw, 2011) on Python's whole numbers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_keeps(elements, p, site, seed, offset):
    """Whether each of the elements (whole numbers) is kept."""
    drop, turn = int(np.rint(np.float32(p) * np.float32(65536))), (offset + site) % (1 << 64)
    out, words = [], {}
    for i in elements:
        b = int(i) // 8
        if b not in words:
            words[b] = philox4x32((b & 0xFFFFFFFF, b >> 32, turn & 0xFFFFFFFF, turn >> 32), (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF))
        out.append((words[b][int(i) % 8 // 2] >> (16 * (int(i) % 2))) & 0xFFFF >= drop)
    return np.array(out, dtype=bool), 1.0 / (1.0 - drop / 65536) if drop < 65536 else 0.0
