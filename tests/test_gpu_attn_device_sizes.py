"""cure_prompt_attn and cure_prefix_attn where the device's sizes cannot be: such a sequence's rows are
left as they were, and the others get the bits that they get without it."""

import pytest
import torch

import paper_2608_00531_amd as pc
from prompt_util import DTYPES, ints, normal

pytestmark = pytest.mark.gpu

HQ, HKV, D = 4, 2, 64


def inputs(dtype, rows, cache):
    t = DTYPES[dtype]
    return normal(1, rows, HQ, D, dtype=t).cuda(), *(normal(s, cache, HKV, D, dtype=t).cuda() for s in (2, 3))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_split", [0, 1, 3])
@pytest.mark.parametrize("bad", [dict(row_off=-1), dict(row_off=-2 ** 40), dict(row_off=92), dict(row_off=2 ** 40), dict(ctx=-1),
                                 dict(ctx=-40), dict(ctx=-2 ** 31), dict(ctx=2 ** 31 - 1)])
def test_prompt_rows_outside_and_contexts_that_cannot_be(dtype, kv_split, bad):
    rows, n, ctx, row_off, kv_off = 100, [9, 9, 33], [500, 400, 300], [0, 20, 40], [0, 600, 1100]
    q, k, v = inputs(dtype, rows, 1500)
    fill = 9.0

    def call(row_off, ctx):
        out = torch.full_like(q, fill)
        _, lse = pc.cure_prompt_attn(q, k, v, ints(row_off, torch.int64), ints(n), ints(kv_off, torch.int64), ints(ctx), n,
                                     [500, 400, 300], 0.125, kv_split=kv_split, out=out)
        torch.cuda.synchronize()
        return out, lse
    want, want_lse = call(row_off, ctx)
    got, lse = call([row_off[0], bad.get("row_off", 20), row_off[2]], [ctx[0], bad.get("ctx", 400), ctx[2]])
    live = torch.cat([torch.arange(0, 9), torch.arange(40, 73)]).cuda()
    other = torch.ones(rows, dtype=torch.bool, device="cuda")
    other[live] = False
    assert torch.equal(got[live], want[live]) and torch.equal(lse[live], want_lse[live])
    assert bool((got[other] == fill).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx", [-1, -6, -300, -2 ** 31, 2 ** 31 - 1])
def test_prefix_contexts_that_cannot_be(dtype, ctx):
    """-6 leaves six nodes no rows at all."""
    nodes, kv_off, n_max = [5, 6, 7], [200, 600, 1000], 8
    q, k, v = inputs(dtype, 3 * n_max, 1500)
    q = q.view(3, n_max, HQ, D)
    parent = ints([[m - 1 for m in range(n_max)]] * 3)
    fill = 9.0

    def call(c):
        out = torch.full_like(q, fill)
        _, lse, status = pc.cure_prefix_attn(q, k, v, 0, 150, ints(kv_off, torch.int64), ints(c), ints(nodes), parent,
                                             [300, 300, 300], nodes, 0.125, out=out)
        return out, lse, status.tolist()
    want, want_lse, status = call([300, 300, 300])
    assert status == [0, 0, 0]
    got, lse, status = call([300, ctx, 300])
    assert status == [0, pc.CURE_ERR_BAD_TREE, 0]
    for b, n in ((0, 5), (2, 7)):
        assert torch.equal(got[b, :n], want[b, :n]) and torch.equal(lse[b, :n], want_lse[b, :n])
    assert bool((got[1] == fill).all())
