"""Plain float64 definitions of the dense operators (numpy): layer norm, MX matrices, orthogonalised updates.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MX_TAG = 0x4D583443


def layernorm(x, gamma, beta, eps):
    """(y, mean, rstd) of rows."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        mean = x.mean(1)
        rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
        return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def layernorm_backward(x, dy, mean, rstd, gamma):
    """(dx, dgamma, dbeta) for given statistics."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1)[:, None] - h * (g * h).mean(1)[:, None])
    return dx, (dy * h).sum(0), dy.sum(0)


def philox16(rows, columns, seed):
    """16-bit rounding numbers [rows, columns] of an MX matrix; columns a multiple of 8."""
    shape = (rows, columns // 8)
    low = np.uint64(0xFFFFFFFF)
    c = [np.broadcast_to(np.arange(shape[1], dtype=np.uint64), shape).copy(), np.broadcast_to(np.arange(rows, dtype=np.uint64)[:, None], shape).copy(),
         np.zeros(shape, np.uint64), np.full(shape, MX_TAG, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    halves = [(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in c for s in (0, 16)]
    return np.stack(halves, -1).reshape(rows, columns).astype(np.int64)


def mx4_quantize(x, seed=None):
    """(codes, scales) as the library lays them out, to nearest or (seed) stochastically."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    full = np.zeros((rows, -(-cols // 128) * 128))
    full[:, :cols] = x
    block = full.reshape(rows, -1, 32)
    with np.errstate(invalid="ignore"):
        most = np.abs(block).max(2)
        bad = ~np.isfinite(block).all(2)
        fraction, exponent = np.frexp(np.where(bad, 1.0, most))              # most = fraction 2^exponent, 1/2 <= fraction < 1
    e = exponent - 1 - 2 if seed is None else exponent - 1 - 2 + (fraction > 0.75)
    e = np.where(most == 0, -127, np.maximum(e, -127))
    y = np.abs(np.where(bad[:, :, None], 0.0, block)) * np.exp2(-e.astype(np.float64))[:, :, None]
    if seed is None:
        distance = np.abs(y[..., None] - VALUES)
        best = distance.min(-1, keepdims=True)
        near = distance == best                                               # one, or two at a tie: the even code
        code = np.where(near.sum(-1) > 1, np.where(np.argmax(near, -1) % 2 == 0, np.argmax(near, -1), np.argmax(near, -1) + 1), np.argmax(near, -1))
    else:
        below = np.minimum(np.searchsorted(VALUES, y, side="right") - 1, 7)
        above = np.minimum(below + 1, 7)
        gap = VALUES[above] - VALUES[below]
        share = np.where(gap > 0, (y - VALUES[below]) / np.where(gap > 0, gap, 1.0), 0.0)
        r = philox16(rows, full.shape[1], seed).reshape(y.shape)
        code = np.where(np.floor(share * 65536) + r >= 65536, above, below)
        code = np.where((e[:, :, None] == 126) & (code == 6), 5, code)         # 4 * 2^126 is no fp32 number
    code = np.where(bad[:, :, None], 0, code | (np.signbit(block).astype(np.int64) << 3)).reshape(rows, -1)
    codes = (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)
    byte = np.where(bad, 255, e + 127).astype(np.uint8)
    return codes, np.ascontiguousarray(byte.reshape(rows, -1, 4).transpose(1, 0, 2))


def mx4_values(codes, scales, cols):
    rows = codes.shape[0]
    code = np.stack([codes & 15, codes >> 4], -1).reshape(rows, -1)
    value = np.where(code >= 8, -VALUES[code % 8], VALUES[code % 8])
    byte = scales.transpose(1, 0, 2).reshape(rows, -1)
    scale = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return (value.reshape(rows, -1, 32) * scale[:, :, None]).reshape(rows, -1)[:, :cols]


def orthogonalize(g, steps, eps, dtype=np.float64):
    """One matrix; dtype: of the arithmetic."""
    g = np.asarray(g, dtype=np.float64)
    flip = g.shape[0] > g.shape[1]
    x = ((g.T if flip else g) / (np.sqrt((g * g).sum()) + eps)).astype(dtype)
    for a, b, c in steps:
        a, b, c = (dtype(v) for v in (a, b, c))
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.T if flip else x
