"""The bounds of packed_bounds.py on the CPU: attention whose probabilities are rounded as the header says keeps
them, and one that rounds packed tokens' to bf16, or leaves out open rows' second part, does not."""

import numpy as np
import pytest
import torch

from packed_bounds import Bounded
from prompt_util import wide


def attend(c, packed, opened):
    """The definition, with P (times the value's scale, the largest of a row 2^7 to 2^8) rounded by `packed` and `opened`."""
    q = wide(c.q).reshape(c.total, c.hq, c.d)
    o, lse = torch.zeros(c.total, c.hq, c.d), torch.zeros(c.total, c.hq)
    group = c.hq // c.hkv
    for b, n in enumerate(c.rows):
        keys, values = c.keys(b)
        seen, old = c.seen(b), c.packed[b]
        for h in range(c.hq):
            s_v = c.vs[c.blk_off[b]:c.blk_off[b] + (old + 63) // 64, h // group].double().numpy()
            s_v = np.concatenate((np.repeat(s_v, 64)[:old], np.ones(len(keys) - old)))
            for r in range(n):
                at = c.first[b] + r
                s = np.where(seen[r], c.scale * (keys[:, h // group] @ q[at, h]), -np.inf)
                w = np.exp(s - s.max())
                p = w * s_v * 2.0 ** (7 - np.floor(np.log2((w * s_v).max())))
                p = np.concatenate((packed(torch.from_numpy(p[:old])).numpy(), opened(torch.from_numpy(p[old:])).numpy()))
                norm = w.sum() * 2.0 ** (7 - np.floor(np.log2((w * s_v).max())))
                o[at, h] = torch.from_numpy((p / s_v) @ values[:, h // group] / norm).float()
                lse[at, h] = s.max() + np.log(w.sum())
    return o.reshape(*c.shape, c.hq, c.d), lse.reshape(*c.shape, c.hq), torch.zeros(len(c.rows), dtype=torch.int32)


def half(p):
    return p.half().double()


def bf16(p):
    return p.bfloat16().double()


def two_bf16(p):
    return bf16(p) + bf16(p - bf16(p))


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("packed,ctx", [([300, 90], 0), ([0, 0], 40), ([200, 64], 20)])
def test_bounds(packed, ctx, seed):
    c = Bounded("bf16", [5, 2], packed, [ctx, ctx], 8, 2, 64, seed=seed)
    c.check(attend(c, half, two_bf16))
    coarse = (bf16, two_bf16) if packed[0] else (half, bf16)
    with pytest.raises(AssertionError):
        c.check(attend(c, *coarse))
