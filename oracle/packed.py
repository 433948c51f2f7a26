"""Oracle: the packed cache (8 bits a value, one scale for each block of 64 tokens and head) and
the drawing of tokens.

Test infrastructure only (see the package docstring). The paper holds its cache in 16 bits and
decodes greedily; these are the definitions of the operators that extend both.
"""

import numpy as np

BLOCK = 64


def key_place(t, j, d):
    """Byte of a block of keys that holds column j of token t."""
    return (t // 32 * (d // 32) + j // 32) * 1024 + j % 32 // 16 * 512 + t % 32 * 16 + j % 16


def value_place(t, j, d):
    """Byte of a block of values that holds column j of token t."""
    return (t // 32 * (d // 32) + j // 32) * 1024 + t // 4 % 2 * 512 + j % 32 * 16 + t % 32 // 8 * 4 + t % 4


def pack_rows(x):
    """One sequence's rows [n, hkv, d] (float values) in blocks: integers [blocks, hkv, 64, d] and float32 scales
    [blocks, hkv]."""
    x = np.asarray(x, np.float64)
    n, hkv, d = x.shape
    blocks = (n + BLOCK - 1) // BLOCK
    full = np.zeros((blocks * BLOCK, hkv, d))
    full[:n] = x
    full = full.reshape(blocks, BLOCK, hkv, d).transpose(0, 2, 1, 3)
    top = np.abs(full).max(axis=(2, 3), keepdims=True)
    c = np.rint(127.0 * full / np.where(top > 0, top, 1.0))
    scale = np.float32(top[:, :, 0, 0]) / np.float32(127)
    return c.astype(np.int64), scale


def to_bytes(c, values):
    """Integers [blocks, hkv, 64, d] in the blocks' byte order: int8 [blocks, hkv, 64 * d]."""
    blocks, hkv, _, d = c.shape
    out = np.zeros((blocks, hkv, BLOCK * d), np.int8)
    place = value_place if values else key_place
    for t in range(BLOCK):
        out[:, :, place(t, np.arange(d), d)] = c[:, :, t]
    return out


def from_bytes(b, values):
    """The other way: int8 [blocks, hkv, 64 * d] as integers [blocks, hkv, 64, d]."""
    d = b.shape[-1] // BLOCK
    place = value_place if values else key_place
    return np.stack([b[:, :, place(t, np.arange(d), d)] for t in range(BLOCK)], axis=2).astype(np.int64)


def packed_rows(b, scale, values):
    """A sequence's blocks as rows [64 * blocks, hkv, d] in float64."""
    x = from_bytes(b, values) * np.asarray(scale, np.float64)[:, :, None, None]
    return x.transpose(0, 2, 1, 3).reshape(-1, b.shape[1], b.shape[2] // BLOCK)


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: (token, log probability, kept), or None where no token can be drawn."""
    x = np.asarray(x, np.float64)
    if not 0 <= temperature < np.inf or np.isnan(top_p) or np.isnan(min_p) or np.isnan(u):
        return None
    if np.isnan(x).any() or (x == np.inf).any() or not np.isfinite(x).any():
        return None
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[np.isfinite(x[order])]
    if temperature == 0:
        return int(order[0]), 0.0, 1
    t = np.float64(np.float32(temperature))
    order = order[x[order[0]] - x[order] <= 64 * t]
    if top_k > 0:
        order = order[:top_k]
    w = np.exp((x[order] - x[order[0]]) / t)
    if top_p < 1:
        before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
        order = order[:max(1, int((before < np.float64(np.float32(top_p)) * w.sum()).sum()))]
    if min_p > 0:
        order = order[:max(1, int((w[:len(order)] >= np.float64(np.float32(min_p))).sum()))]
    w = w[:len(order)]
    j = min(int((np.cumsum(w) <= max(0.0, np.float64(np.float32(u))) * w.sum()).sum()), len(w) - 1)
    return int(order[j]), float(np.log(w[j] / w.sum())), len(w)
