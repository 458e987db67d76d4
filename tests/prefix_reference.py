"""Plain 64-bit implementations of the paged cache in the element type and of shared prefixes, from their definitions in include/dma.h: numpy, no torch, no GPU."""
import numpy as np

import cache4_reference as ref4


def rotate(x, pos, inv_freq, interleaved=False, scale=1.0):
    """x [rows, heads, d], pos [rows] integers, inv_freq [rot / 2] fp32."""
    x = np.array(x, np.float64)
    half = len(inv_freq)
    a = np.asarray(pos, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    u, v = x[..., first].copy(), x[..., second].copy()
    x[..., first], x[..., second] = scale * (u * np.cos(a) - v * np.sin(a)), scale * (u * np.sin(a) + v * np.cos(a))
    return x


def visible_slots(table, n, page, pages):
    """Slots of a sequence's first n keys that lie in the pool, by position."""
    j = np.arange(max(n, 0))
    p = np.asarray(table)[j // page].astype(np.int64)
    return (p * page + j % page)[(p >= 0) & (p < pages)]


def best(delta, w):
    """Indices of the w largest, largest first, ties to the lower index."""
    return np.argsort(-np.asarray(delta, np.float64), kind="stable")[:w]


def order(delta, table, n, w, page):
    """delta [pages, Hq, page] -> slots [Hq, min(w, visible)]."""
    at = visible_slots(table, n, page, delta.shape[0])
    return np.stack([at[best(delta[at // page, h, at % page], w)] for h in range(delta.shape[1])]) if len(at) else np.zeros((delta.shape[1], 0), np.int64)


def decode_row(q, kv, delta, slots, w, scale):
    """One row over the keys in `slots` (its context in order): what cache4_reference.decode returns."""
    page = kv.shape[2]
    keys = kv[slots // page, :, slots % page].astype(np.float64)                 # [n, Hkv, 2, d]
    return ref4.decode(np.asarray(q, np.float64), keys[:, :, 0], keys[:, :, 1], delta[slots // page, :, slots % page].T, w, scale)
