"""Plain float64 definitions of what a node classifier has besides its layers (numpy): embedding, dropout, matrices in 8 bits, log probabilities.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

DROP_TAG = 0x44524F50


def embedding(table, ids, scale):
    table, ids = np.asarray(table, dtype=np.float64), np.asarray(ids)
    out = np.zeros((ids.size, table.shape[1]))
    there = (ids >= 0) & (ids < table.shape[0])
    out[there] = table[ids[there]] * scale
    return out


def embedding_gradient(dy, ids, n_entries, scale):
    dy, ids = np.asarray(dy, dtype=np.float64), np.asarray(ids)
    out = np.zeros((n_entries, dy.shape[1]))
    there = (ids >= 0) & (ids < n_entries)
    np.add.at(out, ids[there], dy[there])
    return out * scale


def sort_ids(ids, n_entries):
    """(sorted, order) with ids outside the table last, as n_entries."""
    ids = np.asarray(ids).astype(np.int64)
    key = np.where((ids >= 0) & (ids < n_entries), ids, n_entries)
    order = np.argsort(key, kind="stable")
    return key[order], order


def drop_numbers(rows, columns, seed, first_row=0):
    """16-bit numbers [rows, columns], columns a multiple of 8."""
    shape = (rows, columns // 8)
    low = np.uint64(0xFFFFFFFF)
    row = np.broadcast_to((np.arange(rows, dtype=np.uint64) + np.uint64(first_row))[:, None], shape)
    c = [np.broadcast_to(np.arange(shape[1], dtype=np.uint64), shape).copy(), row & low, row >> np.uint64(32), np.full(shape, DROP_TAG, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    halves = [(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in c for s in (0, 16)]
    return np.stack(halves, -1).reshape(rows, columns).astype(np.int64)


def dropped(rows, dim, p, seed, first_row=0):
    """(which elements stay, what they are multiplied by)."""
    t = int(np.floor(p * 65536 + 0.5))
    keep = drop_numbers(rows, -(-dim // 8) * 8, seed % 2 ** 64, first_row)[:, :dim] >= t
    return keep, 65536 / (65536 - t) if t < 65536 else 0.0


# the values of the 256 codes of e4m3
_CODE = np.arange(256)
F8_VALUES = np.where(_CODE // 8 % 16 == 0, _CODE % 8 / 8 * 2.0 ** -6, (1 + _CODE % 8 / 8) * 2.0 ** (_CODE // 8 % 16 - 7.0)) * np.where(_CODE >= 128, -1.0, 1.0)
F8_VALUES[[0x7F, 0xFF]] = np.nan


def f8_quantize(x, tiles=False):
    """(codes, scales) as the library lays them out."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    high = 128 if tiles else 1
    full = np.zeros((-(-rows // high) * high, -(-cols // 128) * 128))
    full[:rows, :cols] = x
    block = full.reshape(-1, high, full.shape[1] // 128, 128)
    bad = ~np.isfinite(block).all((1, 3), keepdims=True)
    block = np.where(bad, 0.0, block)
    most = np.abs(block).max((1, 3), keepdims=True)
    e = np.full(most.shape, -127)
    for power in range(-127, 121):                                           # the smallest that holds
        e = np.where(most > 448.0 * 2.0 ** (power - 1), np.maximum(e, power), e)
    y = np.abs(block) / 2.0 ** e.astype(np.float64)
    positive = F8_VALUES[:127]
    above = np.clip(np.searchsorted(positive, y, side="left"), 0, 126)       # the first value that is not below
    below = np.maximum(above - 1, 0)
    up, down = positive[above] - y, y - positive[below]
    code = np.where(up < down, above, np.where(down < up, below, np.where(above % 2 == 0, above, below)))
    code = np.where(positive[above] == y, above, code)
    code = np.where((e == 120) & (code == 0x78), 0x77, code)                 # 256 * 2^120 is no fp32 number
    code = np.where(bad, 0, code | np.signbit(block).astype(np.int64) << 7)
    byte = np.where(bad, 255, e + 127)
    byte = np.broadcast_to(byte, (byte.shape[0], high, byte.shape[2], 1)).reshape(full.shape[0], -1)[:rows]
    scales = np.zeros((full.shape[1] // 128, -(-rows // 16) * 16), np.uint8)
    scales[:, :rows] = byte.T
    return code.reshape(full.shape)[:rows].astype(np.uint8), scales


def f8_values(codes, scales, cols):
    rows = codes.shape[0]
    byte = scales[:, :rows].T.astype(np.float64)
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte - 127))
    return (F8_VALUES[codes].reshape(rows, -1, 128) * scale[:, :, None]).reshape(rows, -1)[:, :cols]


def log_probabilities(x):
    """(logp, max, rest, entropy) of rows that are not -inf throughout and hold no NaN or +inf."""
    x = np.asarray(x, dtype=np.float64)
    u = x - x.max(1, keepdims=True)
    one = np.zeros(u.shape, bool)
    one[np.arange(len(u)), u.argmax(1)] = True
    rest = np.log1p(np.where(one, 0.0, np.exp(u)).sum(1))
    logp = u - rest[:, None]
    p = np.exp(logp)
    return logp, x.max(1), rest, -np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0).sum(1)


def largest(x, n):
    """The classes of each row's n largest: NaN first, then by value, equal ones by class."""
    x = np.asarray(x, dtype=np.float64) + 0.0
    key = np.where(np.isnan(x), np.inf, x)
    classes = np.broadcast_to(np.arange(x.shape[1]), x.shape)
    return np.lexsort((classes, -key, ~np.isnan(x)), axis=1)[:, :n]


def logprob_gradient(x, targets, top, rest, entropy, dlogp, dentropy, scale):
    """top, rest, entropy: of each row, as the forward pass gave them; dlogp, dentropy: of each row."""
    x = np.asarray(x, dtype=np.float64)
    logp = (x - top[:, None]) - rest[:, None]
    p = np.exp(logp)
    given = (targets >= 0) & (targets < x.shape[1])
    at = np.zeros(x.shape)
    at[np.nonzero(given)[0], targets[given]] = 1.0
    d = np.where(given, dlogp, 0.0)[:, None] * (at - p)
    d = d - dentropy[:, None] * np.where(p > 0, p * (np.where(p > 0, logp, 0.0) + entropy[:, None]), 0.0)
    return scale * d
