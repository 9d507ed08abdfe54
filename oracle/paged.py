"""Paged, quantised caches in fp64 numpy: what the stored rows stand for, and attention over them.

TEST INFRASTRUCTURE ONLY, like oracle.py.  Nothing here knows how the library lays a pool out: a sequence's stored
rows are the values they stand for.
"""
import numpy as np

TILE, D = 64, 128


def round_to(x, dtype):
    """The nearest number of the element type, ties to even, as fp64."""
    x32 = np.asarray(x, np.float64).astype(np.float32)
    if dtype == "f32":
        return x32.astype(np.float64)
    u = x32.view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32).astype(np.float64)


def _f32(x):
    return np.asarray(x, np.float64).astype(np.float32).astype(np.float64)


def codes(x, bits, dtype):
    """Codes, scales and minima of groups along the last axis."""
    top = 2 ** bits - 1
    m = x.min(-1, keepdims=True)
    s = round_to(_f32(_f32(x.max(-1, keepdims=True) - m) / top), dtype)
    safe = np.where(s > 0, s, 1.0)
    c = np.minimum(np.rint(_f32(_f32(x - m) / safe)), top)
    return np.where(s > 0, c, 0.0), s, m


def stored(k, v, bits, dtype):
    """What the rows k [n, T], v [n, 128] of a unit stand for once stored from a tile's first row on (fp64, not rounded)."""
    if bits == 0 or len(k) == 0:
        return k.astype(np.float64), v.astype(np.float64)
    ko, vo = np.empty(k.shape), np.empty(v.shape)
    for r in range(0, len(k), TILE):
        c, s, m = codes(k[r:r + TILE].T, bits, dtype)
        ko[r:r + TILE] = (m + c * s).T
    c, s, m = codes(v.reshape(-1, 2, 64), bits, dtype)
    vo[:] = (m + c * s).reshape(-1, D)
    return ko, vo


def attend(q, idx, k, v, k_tail, v_tail):
    """q [G, 128], kept rows k [n, T], v [n, 128], tails [t, 128] -> [G, 128]; without any row zeros."""
    z = np.concatenate([q[:, idx] @ k.T, q @ k_tail.T], axis=1) / np.sqrt(float(D))
    if z.shape[1] == 0:
        return np.zeros((len(q), D))
    p = np.exp(z - z.max(1, keepdims=True))
    return p @ np.concatenate([v, v_tail]) / p.sum(1, keepdims=True)
