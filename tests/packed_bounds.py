"""Tighter bounds for the attention over a packed context than those of packed_util.py, with what the header
says of its roundings.

For bf16, P of packed tokens is rounded to fp16, whose 11 bits leave half a step of 2^(e - 11) to a number of 2^e or
more: 2^-11 of it, or half a step of the subnormals, 2^-25, which is 2^-32 of the row's largest P (a reference leaves the largest
that it has met at 2^7 or more, and those of waves and splits are none above the row's). P of open rows is two bf16
numbers: the first leaves at most 2^(e - 8), the second of that 2^(e - 9 - 8): 2^-17. Query values are fp16 times a power of two, off
by 2^-39 of the row's largest. With mass = sum p |v| of the packed and the open part and peak the largest p s:
    |err o| <= 2^-11 packed + 2^-17 open + 2^-32 127 count peak [bf16] + (2 e + (n + 16) u) (mass + |o|), that (1 + 2^-7), + h |o|
    e = (d + 6) u scale sum |q k| + 2^-39 [bf16] scale max |q| sum |k|
and lse as there. Rows may be of any magnitude: a type's smallest step is added.
"""

import numpy as np

from packed_util import Case
from prompt_util import HALF, U, wide

STEP = {"torch.bfloat16": 2.0 ** -133, "torch.float32": 2.0 ** -149}


class Bounded(Case):
    def check(self, got, every=1, heads=None):
        o, lse, status = got
        assert status.tolist() == [0] * len(self.rows)
        half, step = HALF[o.dtype], STEP[str(o.dtype)]
        o, lse = wide(o).reshape(self.total, self.hq, self.d), wide(lse).reshape(self.total, self.hq)
        q = wide(self.q).reshape(self.total, self.hq, self.d)
        group = self.hq // self.hkv
        bf16 = self.dtype == "bf16"
        for b, n in enumerate(self.rows):
            if n == 0:
                continue
            keys, values = self.keys(b)
            seen = self.seen(b)
            old = self.packed[b]
            scales = np.repeat(self.vs[self.blk_off[b]:self.blk_off[b] + (old + 63) // 64].numpy().astype(np.float64), 64, axis=0)[:old]
            at = np.unique(np.concatenate((np.arange(0, n, every), [n - 1])))
            for h in heads or range(self.hq):
                kh, vh = keys[:, h // group], values[:, h // group]
                x = q[self.first[b] + at, h]
                e = (self.d + 6) * U * self.scale * np.max(np.where(seen[at], np.abs(x) @ np.abs(kh).T, 0.0), axis=1, keepdims=True)
                if bf16:
                    e = e + 2.0 ** -39 * self.scale * np.abs(x).max(axis=1, keepdims=True) * np.abs(kh).sum(axis=1).max()
                s = np.where(seen[at], self.scale * (x @ kh.T), -np.inf)
                top = s.max(axis=1, keepdims=True)
                w = np.exp(s - top)
                total = w.sum(axis=1, keepdims=True)
                p = w / total
                ref, ref_lse = p @ vh, top + np.log(total)
                packed, opened = p[:, :old] @ np.abs(vh[:old]), p[:, old:] @ np.abs(vh[old:])
                count = seen[at].sum(axis=1, keepdims=True)
                tol = (2 * e + (count + 16) * U) * (packed + opened + np.abs(ref))
                if bf16:
                    peak = np.max(np.concatenate((p[:, :old] * scales[:, h // group], p[:, old:]), axis=1), axis=1, keepdims=True)
                    tol = tol + 2.0 ** -11 * packed + 2.0 ** -17 * opened + 2.0 ** -32 * 127 * old * peak
                tol = tol * (1 + 2.0 ** -7)
                tol = tol + half * (np.abs(ref) + tol) + step
                err = np.abs(o[self.first[b] + at, h] - ref)
                assert np.all(err <= tol), (b, h, float(np.max(err / tol)), float(np.max(err)))
                err = np.abs(lse[self.first[b] + at, h] - ref_lse[:, 0])
                tol = (e + (count + 16) * U + 4 * U * np.abs(ref_lse))[:, 0]
                assert np.all(err <= tol), (b, h, float(np.max(err / tol)), float(np.max(err)))
