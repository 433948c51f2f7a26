"""Shared by the tests of the attention over a packed context: inputs on the GPU, the 64-bit
reference and its error bound.

The bound (u = 2^-24; h = half a step of the output's type): a score sums d products of exact
factors and is scaled twice, off by e = (d + 6) u scale sum |q k|; a probability by 2 e relative to the
row's sum and 4 u for the exponential; for bf16, probability times scale is rounded once more, 2^-8 of
the numerator alone; sums over n keys add (n + 16) u; with mass = sum p |v|:
    |err o|   <= (2^-8 [bf16] + 2 e + (n + 16) u) (mass + |o|) (1 + 2^-7) + h |o|
    |err lse| <= e + (n + 16) u + 4 u |lse|.
"""

import numpy as np
import torch

import oracle
import paper_2608_00531_amd as pc
from prompt_util import DTYPES, HALF, U, ints, normal, random_parents, wide


class Case:
    """Sequences with packed tokens, open rows and new rows: trees (padded), or packed or padded causal rows."""

    def __init__(self, dtype, rows, packed, ctx, hq, hkv, d, form="tree", seed=0, parents=None, n_max=None, std=1.5, scale=None):
        t = self.t = DTYPES[dtype]
        rng = np.random.default_rng(seed)
        batch = len(rows)
        self.dtype, self.rows, self.packed, self.ctx, self.hq, self.hkv, self.d = dtype, rows, packed, ctx, hq, hkv, d
        self.scale = scale or d ** -0.5
        self.n_max = n_max or max(rows)
        self.parents = parents or [random_parents(rng, n) for n in rows] if form == "tree" else None
        self.blk_off, self.kv_off, blk, at = [0] * batch, [0] * batch, 1, 2
        for b in rng.permutation(batch):
            self.blk_off[b], self.kv_off[b] = blk, at
            blk += (packed[b] + 63) // 64 + 1
            at += ctx[b] + rows[b] + 1
        self.blocks, self.cache_rows = blk, at
        self.row_off = None
        if form == "packed":
            self.row_off, r = [], 1
            for n in rows:
                self.row_off.append(r)
                r += n
            self.shape = (r + 2,)
            self.first = self.row_off
        else:
            self.shape = (batch, self.n_max)
            self.first = [b * self.n_max for b in range(batch)]
        self.total = int(np.prod(self.shape))
        self.q = normal(seed + 1, *self.shape, hq, d, dtype=t, std=std)
        self.k, self.v = (normal(seed + 2 + i, at, hkv, d, dtype=t) for i in range(2))
        # Bytes and scales that no packing need have made: whatever lies past a sequence's tokens is arbitrary.
        self.pk, self.pv = (torch.from_numpy(rng.integers(-127, 128, (blk, hkv, 64 * d)).astype(np.int8)) for _ in range(2))
        self.ks, self.vs = (torch.from_numpy((rng.uniform(0.2, 2.0, (blk, hkv)) / 73).astype(np.float32)) for _ in range(2))

    def call(self, out=None, **kw):
        dev = lambda v, t=torch.int32: None if v is None else ints(v, t)  # noqa: E731
        parent = None if self.parents is None else ints([p + [-9] * (self.n_max - len(p)) for p in self.parents])
        self.args = dict(q=self.q.cuda(), pk=self.pk.cuda(), pv=self.pv.cuda(), k_scale=self.ks.cuda(), v_scale=self.vs.cuda(),
                         blk_off=dev(self.blk_off, torch.int64), packed_len=dev(self.packed), k=self.k.cuda(), v=self.v.cuda(),
                         kv_off=dev(self.kv_off, torch.int64), ctx_len=dev(self.ctx), n_rows=dev(self.rows),
                         host_packed_len=self.packed, host_ctx_len=self.ctx, host_n_rows=self.rows, scale=self.scale,
                         parent=parent, row_off=dev(self.row_off, torch.int64), out=out)
        self.args.update(kw)
        return pc.cure_packed_attn(**self.args)

    def keys(self, b):
        """Sequence b's keys and values in 64 bits: packed tokens, open rows, new rows."""
        span = slice(self.blk_off[b], self.blk_off[b] + (self.packed[b] + 63) // 64)
        rows = slice(self.kv_off[b], self.kv_off[b] + self.ctx[b] + self.rows[b])
        old = [oracle.packed_rows(x[span].numpy(), s[span].numpy(), values)[:self.packed[b]] if self.packed[b] else
               np.zeros((0, self.hkv, self.d)) for x, s, values in ((self.pk, self.ks, False), (self.pv, self.vs, True))]
        return [np.concatenate((o, wide(x[rows]))) for o, x in zip(old, (self.k, self.v))]

    def seen(self, b):
        """[rows, keys]: what each new row sees."""
        n, old = self.rows[b], self.packed[b] + self.ctx[b]
        s = np.zeros((n, old + n), bool)
        s[:, :old] = True
        for m in range(n):
            if self.parents is None:
                s[m, old:old + m + 1] = True
            else:
                j = m
                while j >= 0:
                    s[m, old + j] = True
                    j = self.parents[b][j]
        return s

    def check(self, got, every=1, heads=None):
        """o, lse, status of a call: every `every`-th row of each sequence, of some heads, within the bounds."""
        o, lse, status = got
        assert status.tolist() == [0] * len(self.rows)
        half = HALF[o.dtype]
        p = 2.0 ** -8 if self.dtype == "bf16" else 0.0
        o = wide(o).reshape(self.total, self.hq, self.d)
        lse = None if lse is None else wide(lse).reshape(self.total, self.hq)
        q = wide(self.q).reshape(self.total, self.hq, self.d)
        group = self.hq // self.hkv
        for b, n in enumerate(self.rows):
            if n == 0:
                continue
            keys, values = self.keys(b)
            seen = self.seen(b)
            at = np.unique(np.concatenate((np.arange(0, n, every), [n - 1])))
            for h in heads or range(self.hq):
                kh, vh = keys[:, h // group], values[:, h // group]
                x = q[self.first[b] + at, h]
                e = (self.d + 6) * U * self.scale * np.max(np.where(seen[at], np.abs(x) @ np.abs(kh).T, 0.0), axis=1, keepdims=True)
                s = np.where(seen[at], self.scale * (x @ kh.T), -np.inf)
                top = s.max(axis=1, keepdims=True)
                w = np.exp(s - top)
                total = w.sum(axis=1, keepdims=True)
                ref, mass, ref_lse = w @ vh / total, w @ np.abs(vh) / total, top + np.log(total)
                count = seen[at].sum(axis=1, keepdims=True)
                tol = (p + 2 * e + (count + 16) * U) * (mass + np.abs(ref)) * (1 + 2.0 ** -7)
                tol = tol + half * (np.abs(ref) + tol)
                err = np.abs(o[self.first[b] + at, h] - ref)
                assert np.all(err <= tol), (b, h, float(np.max(err - tol)), float(np.max(err)))
                if lse is not None:
                    err = np.abs(lse[self.first[b] + at, h] - ref_lse[:, 0])
                    assert np.all(err <= (e + (count + 16) * U + 4 * U * np.abs(ref_lse))[:, 0]), (b, h, float(np.max(err)))
