"""cure_prefix_attn where a row's parts meet: each key counted once at every split's edge, malformed trees in
contexts of several splits, and sizes around what the launch decides by."""

import math

import pytest
import torch

import paper_2608_00531_amd as pc
from prompt_util import DTYPES, ints
from test_gpu_prefix_attn import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv_split", [0, 1, 3, 8])
@pytest.mark.parametrize("prefixes,own", [([1, 31, 32, 33, 64], [0, 1, 30, 31, 32]), ([127, 128, 129, 255], [33, 96, 127, 128]),
                                          ([256, 257, 300, 513], [250, 255, 256, 257]), ([700, 1025], [511, 513, 1030, 1700])])
def test_every_key_counts_once(dtype, d, kv_split, prefixes, own):
    """Queries of zero and one-hot values: element t % d of the output, times the number of keys that a node sees, is
    how many of them there are with that remainder. A path of three nodes beside a root of its own.

    Whole numbers below 2^24 (and their bf16 probabilities, 1) are exact in a part; its division, the join's weights
    (exponentials of differences of logarithms of up to 8, each off by 3 * 2^-24 of itself) and the last division
    stay below 64 * 2^-24 of what is counted."""
    t = DTYPES[dtype]
    parents = [-1, 0, 1, -1]
    paths = [[0], [0, 1], [0, 1, 2], [3]]
    for prefix in prefixes:
        for ctx in own:
            batch, n = 3, 4
            lens = [ctx, max(ctx - 1, 0), ctx + 1]
            kv_off, at = [], prefix
            for c in lens:
                kv_off.append(at)
                at += c + n
            v = torch.zeros(at, 2, d, dtype=t)
            v[torch.arange(at), :, torch.arange(at) % d] = 1
            q, k = torch.zeros(batch, n, 4, d, dtype=t, device="cuda"), torch.zeros(at, 2, d, dtype=t, device="cuda")
            o, lse, st = pc.cure_prefix_attn(q, k, v.cuda(), 0, prefix, ints(kv_off, torch.int64), ints(lens), ints([n] * batch),
                                             ints([parents] * batch), lens, [n] * batch, 1.0, out_dtype=torch.float32,
                                             kv_split=kv_split)
            assert st.tolist() == [0] * batch
            one = v[:, 0].double()
            for b in range(batch):
                rows = one[kv_off[b] + lens[b]:kv_off[b] + lens[b] + n]
                base = one[:prefix].sum(0) + one[kv_off[b]:kv_off[b] + lens[b]].sum(0)
                for i, path in enumerate(paths):
                    want, keys = base + rows[path].sum(0), prefix + lens[b] + len(path)
                    got = o[b, i].cpu().double() * keys
                    assert bool(((got - want).abs() <= 64 * 2.0 ** -24 * (want + 1)).all()), (prefix, lens[b], i)
                    assert float((lse[b, i].cpu().double() - math.log(keys)).abs().max()) <= 64 * 2.0 ** -24, (prefix, lens[b], i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (8, 1, 128), (4, 2, 64)])
@pytest.mark.parametrize("nodes,ctx", [([6, 6, 6], [5, 5, 5]), ([150, 150, 150], [1500, 1500, 40]), ([40, 7, 64], [90, 2000, 33])])
@pytest.mark.parametrize("bad", [4, 2 ** 31 - 1, -2, -2 ** 31])
def test_a_malformed_tree_leaves_the_others(dtype, hq, hkv, d, nodes, ctx, bad):
    """A parent that comes later, is none, or is the node itself; trees of one and of several tiles, one and several splits
    of their own rows."""
    c = Case(dtype, 100, nodes, ctx, hq, hkv, d, seed=7)
    want, want_lse, st = c.run()
    assert st.tolist() == [0, 0, 0]
    for at, parent in ((2, bad), (nodes[1] - 1, nodes[1] - 1)):
        good = c.parents[1][at]
        c.parents[1][at] = parent
        o, lse, st = c.run()
        c.parents[1][at] = good
        assert st.tolist() == [0, pc.CURE_ERR_BAD_TREE, 0]
        for b in (0, 2):
            n = nodes[b]
            assert torch.equal(o[b, :n], want[b, :n]) and torch.equal(lse[b, :n], want_lse[b, :n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,hq", [([31, 1], 1), ([32, 1], 1), ([33, 31], 1), ([8, 8], 4), ([16, 17], 8), ([127], 1), ([128, 129], 1)])
@pytest.mark.parametrize("ctx", [255, 256, 700])
def test_tiles_and_splits_at_their_edges(dtype, nodes, hq, ctx):
    """Rows around a tile of 32 (fp32) and of 128 (bf16), own contexts around the first that is split."""
    c = Case(dtype, 129, nodes, [ctx - n for n in nodes], hq, 1, 64, seed=9)
    o, lse, st = c.run()
    assert st.tolist() == [0] * len(nodes)
    c.check(o, lse, only=lambda n: [0, n // 2, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_short_prefixes_and_long_own_contexts_repeat_their_bits(dtype):
    c = Case(dtype, 200, [48, 33, 1], [5000, 1900, 4096], 8, 2, 128, seed=3)
    o, lse, _ = c.run()
    c.check(o, lse, only=lambda n: [0, n // 2, n - 1])
    for _ in range(3):
        again, again_lse, _ = c.run()
        for b, n in enumerate(c.nodes):
            assert torch.equal(o[b, :n], again[b, :n]) and torch.equal(lse[b, :n], again_lse[b, :n])
