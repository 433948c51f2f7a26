"""Workspace of cure_prompt_attn where one long context would give every row of the batch its splits: parts by
each sequence's own. Sizes on the CPU; results on the GPU, with the device's sizes as the host's and others."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2608_00531_amd as pc
from prompt_util import DTYPES, ints
from test_prompt_abi import L  # noqa: F401

MB = 1 << 20


def size(n, ctx, kv_split=0, hq=32, hkv=8, d=128):
    arrays = [np.array(x, np.int32) for x in (n, ctx)]
    a, c = (x.ctypes.data_as(ctypes.c_void_p) for x in arrays)
    return pc.lib().cure_prompt_attn_workspace_size(len(n), sum(n), hq, hkv, d, a, c, kv_split)


@pytest.mark.parametrize("n,ctx,most", [
    ([2048] * 16 + [1], [0] * 16 + [131071], 1200 * MB),  # 32 at most for one row, one or two for 32768
    ([8192] * 4 + [1], [0] * 4 + [1 << 20], 1200 * MB),
    ([2048] * 8 + [1] * 4, [0] * 8 + [131071] * 4, 600 * MB),
    ([256] * 64 + [1], [0] * 64 + [131071], 1200 * MB)])
def test_one_long_context_does_not_size_every_row(L, n, ctx, most):  # noqa: F811
    assert size(n, ctx) <= most


def test_small_workspaces_have_room_for_every_split_of_every_row(L):  # noqa: F811
    """Replays with other sizes than the host's copies keep their splits."""
    assert size([40, 7, 1], [600, 30, 0], kv_split=4, hq=4, hkv=2, d=64) >= 48 * 4 * 4 * 65 * 4
    assert size([64, 1], [700, 1500], kv_split=4, hq=8, hkv=2) >= 65 * 8 * 4 * 129 * 4


class Case:
    """Equal scores and one-hot values: element t % d of a row's output, times the number of keys that it
    sees, is how many of those have that remainder."""

    def __init__(self, dtype, n, ctx, d=64, hq=32, hkv=1, rows=0):
        t = DTYPES[dtype]
        self.n, self.ctx, self.d = n, ctx, d
        self.row_off = np.concatenate([[0], np.cumsum([x + 1 for x in n])])[:-1].tolist()   # a row of nobody's between
        self.kv_off = np.concatenate([[0], np.cumsum([a + b for a, b in zip(n, ctx)])]).tolist()
        at = self.kv_off.pop()
        self.v = torch.zeros(at, hkv, d, dtype=t, device="cuda")
        self.v[torch.arange(at, device="cuda"), :, torch.arange(at, device="cuda") % d] = 1
        self.k = torch.zeros_like(self.v)
        self.q = torch.zeros(max(rows, sum(n) + len(n)), hq, d, dtype=t, device="cuda")

    def run(self, host_n, host_ctx, kv_split):
        out = torch.full(self.q.shape, 9.0, dtype=torch.float32, device="cuda")
        return pc.cure_prompt_attn(self.q, self.k, self.v, ints(self.row_off, torch.int64), ints(self.n),
                                   ints(self.kv_off, torch.int64), ints(self.ctx), host_n, host_ctx, 1.0, kv_split=kv_split,
                                   out_dtype=torch.float32, out=out)

    def check(self, o, lse):
        """Whole numbers are exact in a part; its division, the join's weights (exponentials of differences of
        logarithms of up to 11, each off by 3 * 2^-24 of itself) and the last division stay below 64 * 2^-24."""
        left = torch.ones(len(o), dtype=torch.bool, device="cuda")
        for r, n, at, c in zip(self.row_off, self.n, self.kv_off, self.ctx):
            left[r:r + n] = False
            if n == 0:
                continue
            want = torch.cumsum(self.v[at:at + c + n, 0].double(), 0)[c:]
            keys = torch.arange(c + 1, c + n + 1, dtype=torch.float64, device="cuda")
            got = o[r:r + n].double() * keys[:, None, None]
            assert bool(((got - want[:, None]).abs() <= 64 * 2.0 ** -24 * (want[:, None] + 1)).all()), (n, c)
            assert float((lse[r:r + n].double() - keys.log()[:, None]).abs().max()) <= 64 * 2.0 ** -24, (n, c)
        assert bool((o[left] == 9.0).all())


LARGE = [([2100, 1], [0, 30000], 64), ([1300, 0, 3, 900, 1], [100, 7, 20000, 0, 31], 64), ([5500, 33, 1], [900, 0, 9000], 24),
         ([40] * 70 + [1] * 1200, [17 * i for i in range(70)] + [i * 5 for i in range(1200)], 48)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,ctx,kv_split", LARGE)
def test_placed_parts(dtype, n, ctx, kv_split):
    even = sum(n) * 32 * kv_split * 65 * 4
    assert even > 1024 * MB and size(n, ctx, kv_split, hkv=1, d=64) < even
    c = Case(dtype, n, ctx)
    c.check(*c.run(n, ctx, kv_split))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx", [[0, 30000, 40], [30000, 0, 2000], [9000, 9000, 9000], [0, 0, 0]])
@pytest.mark.parametrize("n", [[2100, 1, 5], [3, 1, 2100], [2100, 2100, 2100], [0, 0, 1]])
def test_placed_parts_with_other_sizes_than_the_hosts(dtype, n, ctx):
    """Sequences whose parts do not fit are written whole, whichever come first."""
    c = Case(dtype, n, ctx, rows=2200)
    c.check(*c.run([2100, 1, 5], [0, 30000, 40], 64))


@pytest.mark.gpu
def test_placed_parts_in_a_captured_call():
    """Replayed on other sizes, with eager work between the replays."""
    c = Case("bf16", [2100, 1, 5], [0, 30000, 40])
    n, ctx = ints(c.n), ints(c.ctx)
    args = (c.q, c.k, c.v, ints(c.row_off, torch.int64), n, ints(c.kv_off, torch.int64), ctx, c.n, c.ctx, 1.0)
    out = torch.full(c.q.shape, 9.0, dtype=torch.float32, device="cuda")
    call = lambda o: pc.cure_prompt_attn(*args, kv_split=64, out_dtype=torch.float32, out=o)  # noqa: E731
    call(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lse = call(out)[1]
    for rows, lens in (([2100, 1, 5], [0, 30000, 40]), ([3, 1, 5], [2097, 29, 0]), ([2100, 0, 5], [0, 0, 40]), ([2100, 1, 5], [0, 30000, 40])):
        n.copy_(ints(rows))
        ctx.copy_(ints(lens))
        out.fill_(9.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.n, c.ctx = rows, lens
        c.check(out, lse)
        fresh = call(torch.full_like(out, 9.0))[0]
        assert torch.equal(fresh, out)
