"""Workspace of cure_prefix_attn where one long own context would give every row of the batch its splits: parts by
each sequence's own. Sizes on the CPU; results on the GPU, with the device's sizes as the host's and others."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2608_00531_amd as pc
from prompt_util import DTYPES, ints
from test_prompt_abi import L  # noqa: F401

GB = 1 << 30


def size(prefix, ctx, nodes, n_max, hq=32, hkv=8, d=128):
    arrays = [np.array(x, np.int32) for x in (ctx, nodes)]
    c, n = (a.ctypes.data_as(ctypes.c_void_p) for a in arrays)
    return pc.lib().cure_prefix_attn_workspace_size(len(ctx), hq, hkv, d, n_max, prefix, c, n, 0)


@pytest.mark.parametrize("batch,nodes,own", [(256, 48, 131072), (256, 48, 1 << 20), (1024, 16, 1 << 20), (64, 256, 131072)])
def test_one_long_context_does_not_size_every_row(L, batch, nodes, own):  # noqa: F811
    """Two slots for every row, or three, and some hundred for one sequence's."""
    each = batch * nodes * 32 * 129 * 4
    assert size(200, [own] + [100] * (batch - 1), [nodes] * batch, nodes) <= max(GB, 3 * each + nodes * 32 * 256 * 129 * 4) + 65536


class Case:
    """Queries of zero and one-hot values: element t % d of the output, times the number of keys that a node sees, is
    how many of them have that remainder. Every tree is a chain."""

    def __init__(self, dtype, prefix, ctx, nodes, n_max, hq=32, hkv=1, d=64):
        t = DTYPES[dtype]
        self.prefix, self.ctx, self.nodes, self.n_max, self.d = prefix, ctx, nodes, n_max, d
        self.kv_off = (prefix + np.concatenate([[0], np.cumsum([c + n for c, n in zip(ctx, nodes)])])).tolist()
        at = self.kv_off.pop()
        self.v = torch.zeros(at, hkv, d, dtype=t, device="cuda")
        self.v[torch.arange(at, device="cuda"), :, torch.arange(at, device="cuda") % d] = 1
        self.k = torch.zeros_like(self.v)
        self.q = torch.zeros(len(ctx), n_max, hq, d, dtype=t, device="cuda")
        self.parent = ints([[m - 1 for m in range(n_max)]] * len(ctx))

    def run(self, host_ctx, host_nodes):
        out = torch.full(self.q.shape, 9.0, dtype=torch.float32, device="cuda")
        o, lse, status = pc.cure_prefix_attn(self.q, self.k, self.v, 0, self.prefix, ints(self.kv_off, torch.int64), ints(self.ctx),
                                             ints(self.nodes), self.parent, host_ctx, host_nodes, 1.0,
                                             out_dtype=torch.float32, out=out)
        assert not status.any()
        return o, lse

    def check(self, o, lse):
        """Whole numbers are exact in a part; its division, the join's weights (exponentials of differences of
        logarithms of up to 11, each off by 3 * 2^-24 of itself) and the last division stay below 64 * 2^-24."""
        shared = self.v[:self.prefix, 0].double().sum(0)
        for b, (n, at, c) in enumerate(zip(self.nodes, self.kv_off, self.ctx)):
            assert bool((o[b, n:] == 9.0).all())
            if n == 0:
                continue
            want = shared + torch.cumsum(self.v[at:at + c + n, 0].double(), 0)[c:]
            keys = self.prefix + torch.arange(c + 1, c + n + 1, dtype=torch.float64, device="cuda")
            got = o[b, :n].double() * keys[:, None, None]
            assert bool(((got - want[:, None]).abs() <= 64 * 2.0 ** -24 * (want[:, None] + 1)).all()), b
            assert float((lse[b, :n].double() - keys.log()[:, None]).abs().max()) <= 64 * 2.0 ** -24, b


HOST = ([30000] + [17 * b for b in range(62)] + [9000], [5] + [b % 4 for b in range(62)] + [256])


def even_bytes(parts):
    return 64 * 256 * 32 * parts * 65 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [100, 3000, 8000])
def test_placed_parts(dtype, prefix):
    assert GB < even_bytes(9) and size(prefix, *HOST, 256, hkv=1, d=64) < even_bytes(9)   # 10 slots and more in each row otherwise
    c = Case(dtype, prefix, *HOST, 256)
    first = c.run(*HOST)
    c.check(*first)
    again = c.run(*HOST)
    for b, n in enumerate(c.nodes):
        assert torch.equal(first[0][b, :n], again[0][b, :n]) and torch.equal(first[1][b, :n], again[1][b, :n])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx,nodes", [([9000] + [40] * 62 + [30000], [256] + [3] * 62 + [5]), ([2000] * 64, [3] * 64),
                                       ([3000] * 3 + [0] * 61, [256] * 64), ([0] * 64, [0] * 63 + [1])])
def test_placed_parts_with_other_sizes_than_the_hosts(dtype, ctx, nodes):
    """Sequences whose parts do not fit have one split of their own rows, whichever come first."""
    c = Case(dtype, 100, ctx, nodes, 256)
    c.check(*c.run(*HOST))


@pytest.mark.gpu
def test_placed_parts_in_a_captured_call():
    """Replayed on other sizes, with eager work between the replays."""
    c = Case("bf16", 100, *HOST, 256)
    nodes, ctx = ints(c.nodes), ints(c.ctx)
    out = torch.full(c.q.shape, 9.0, dtype=torch.float32, device="cuda")
    kv_off = ints(c.kv_off, torch.int64)
    call = lambda o: pc.cure_prefix_attn(c.q, c.k, c.v, 0, 100, kv_off, ctx, nodes, c.parent, *HOST, 1.0,  # noqa: E731
                                         out_dtype=torch.float32, out=o)
    call(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lse = call(out)[1]
    for c.ctx, c.nodes in (HOST, ([7] * 64, [5] * 1 + [b % 4 for b in range(62)] + [256]), (HOST[0], [0] * 63 + [1]), HOST):
        c.ctx = [min(x, y) for x, y in zip(c.ctx, HOST[0])]
        nodes.copy_(ints(c.nodes))
        ctx.copy_(ints(c.ctx))
        out.fill_(9.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.check(out, lse)
        assert torch.equal(call(torch.full_like(out, 9.0))[0], out)
