"""Oracle: rotary positions and the cache rows of new tokens, attention over
prompts, and tree attention over a shared prefix.

Test infrastructure only (see the package docstring). The paper runs these inside
its target model and does not describe them; they are the definitions of a
transformer's attention layer. Values arrive as float arrays, already widened.
"""

import numpy as np

from .tree import ancestors


def rope_append(q, k, v, pos, inv_freq, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, mscale=1.0):
    """Queries and keys of rows at positions pos, normalised per head and rotated.

    q [rows, hq, d], k and v [rows, hkv, d], pos [rows], inv_freq [rot / 2]. Returns
    (q, k, v) in float64: what the attention reads and the cache takes.
    """
    inv_freq = np.asarray(inv_freq, np.float64)
    half = len(inv_freq)
    out = []
    for x, w in ((q, q_weight), (k, k_weight)):
        x = np.array(x, np.float64)
        if w is not None:
            x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(w, np.float64)
        y = x.copy()
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            t = np.asarray(pos, np.float64)[:, None] * inv_freq[i]
            y[..., a] = mscale * (x[..., a] * np.cos(t) - x[..., b] * np.sin(t))
            y[..., b] = mscale * (x[..., a] * np.sin(t) + x[..., b] * np.cos(t))
        out.append(y)
    return out[0], out[1], np.array(v, np.float64)


def tree_positions(parent, n_nodes, first):
    """Position of every node: `first` plus its depth."""
    return first + np.array(ancestors(parent, n_nodes)[1], np.int64).reshape(-1)


def attend(q, k, v, scale):
    """One query row [d] over keys and values [n, d]: (output, log-sum-exp, sum of p |v|)."""
    s = scale * (k @ q)
    m = np.max(s)
    p = np.exp(s - m)
    return p @ v / p.sum(), m + np.log(p.sum()), p @ np.abs(v) / p.sum()


def prompt_attention(q, k, v, row_off, n_rows, kv_off, ctx_len, scale):
    """Causal attention of packed new tokens.

    q [rows, hq, d]; k, v [cache_rows, hkv, d]. Returns (o, lse, mass): o [rows, hq, d],
    lse [rows, hq] and mass = sum_j p_j |v_j|, the size of what o sums (error bounds
    scale with it), all float64; rows of no sequence are zero.
    """
    rows, hq, d = q.shape
    hkv = k.shape[1]
    o, lse, mass = np.zeros((rows, hq, d)), np.zeros((rows, hq)), np.zeros((rows, hq, d))
    for r0, n, off, ctx in zip(row_off, n_rows, kv_off, ctx_len):
        for i in range(int(n)):
            seen = slice(int(off), int(off) + int(ctx) + i + 1)
            for h in range(hq):
                g = h // (hq // hkv)
                o[r0 + i, h], lse[r0 + i, h], mass[r0 + i, h] = attend(
                    q[r0 + i, h].astype(np.float64), k[seen, g].astype(np.float64),
                    v[seen, g].astype(np.float64), scale)
    return o, lse, mass


def prefix_attention(q, k, v, prefix_off, prefix_len, kv_off, ctx_len, n_nodes, parent, scale):
    """Tree attention over a shared prefix, a sequence's own context and its tree.

    q [batch, n_max, hq, d]; returns (o, lse, mass) as prompt_attention, zero for
    nodes that do not exist.
    """
    batch, n_max, hq, d = q.shape
    hkv = k.shape[1]
    o, lse, mass = np.zeros(q.shape), np.zeros((batch, n_max, hq)), np.zeros(q.shape)
    shared = np.arange(prefix_off, prefix_off + prefix_len)
    for b in range(batch):
        L, off = int(ctx_len[b]), int(kv_off[b])
        anc, _ = ancestors(parent[b], int(n_nodes[b]))
        for n in range(int(n_nodes[b])):
            seen = np.concatenate([shared, np.arange(off, off + L), off + L + np.array(anc[n])]).astype(np.int64)
            for h in range(hq):
                g = h // (hq // hkv)
                o[b, n, h], lse[b, n, h], mass[b, n, h] = attend(
                    q[b, n, h].astype(np.float64), k[seen, g].astype(np.float64),
                    v[seen, g].astype(np.float64), scale)
    return o, lse, mass
