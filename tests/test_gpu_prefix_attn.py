"""cure_prefix_attn against the 64-bit definition, within the bounds derived in prompt_util.py."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_00531_amd as pc
from prompt_util import DTYPES, check_rows, ints, normal, random_parents, wide

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, dtype, prefix, nodes, ctx, hq, hkv, d, n_max=None, seed=0, std=1.5):
        t = DTYPES[dtype]
        rng = np.random.default_rng(seed)
        self.dtype, self.prefix, self.nodes, self.ctx, self.scale = dtype, prefix, nodes, ctx, d ** -0.5
        self.batch, self.n_max = len(nodes), n_max or max(nodes)
        self.prefix_off = 4
        self.kv_off, at = [], self.prefix_off + prefix + 2
        for n, c in zip(nodes, ctx):
            self.kv_off.append(at)
            at += n + c + 1
        self.parents = [random_parents(rng, n) for n in nodes]
        self.q = normal(seed, self.batch, self.n_max, hq, d, dtype=t, std=std)
        self.k, self.v = normal(seed + 1, at, hkv, d, dtype=t), normal(seed + 2, at, hkv, d, dtype=t)

    def parent(self):
        return ints([p + [-1] * (self.n_max - len(p)) for p in self.parents])

    def run(self, **kw):
        r = pc.cure_prefix_attn(self.q.cuda(), self.k.cuda(), self.v.cuda(), self.prefix_off, self.prefix,
                                ints(self.kv_off, torch.int64), ints(self.ctx), ints(self.nodes), self.parent(),
                                self.ctx, self.nodes, self.scale, **kw)
        torch.cuda.synchronize()
        return r

    def check(self, o, lse, only=None):
        q, k, v = wide(self.q), wide(self.k), wide(self.v)
        seen, rows = {}, []
        for b, n in enumerate(self.nodes):
            anc, _ = oracle.ancestors(self.parents[b], n)
            for i in range(n) if only is None else [i for i in only(n) if 0 <= i < n]:
                rows.append((b, i))
                seen[b, i] = np.concatenate([self.prefix_off + np.arange(self.prefix), self.kv_off[b] + np.arange(self.ctx[b]),
                                             self.kv_off[b] + self.ctx[b] + np.array(anc[i])]).astype(np.int64)
        ref = [np.zeros(q.shape), np.zeros(q.shape[:3]), np.zeros(q.shape)]
        hq, hkv = q.shape[2], k.shape[1]
        for r in rows:
            for h in range(hq):
                g = h // (hq // hkv)
                for dst, x in zip(ref, oracle.attend(q[r][h], k[seen[r], g], v[seen[r], g], self.scale)):
                    dst[r][h] = x
        # Two parts and their join: each rounds its own probabilities, so the sum's bound is theirs;
        # the join's weights add their log-sum-exps' errors, which check_rows' terms hold twice over.
        check_rows(o, lse, ref, rows, seen, q, k, self.scale, self.dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (5, 1)])
@pytest.mark.parametrize("prefix,nodes,ctx", [
    (1, [1], [0]), (31, [3, 1], [0, 5]), (33, [17, 0, 40], [2, 100, 0]), (300, [1] * 9, [0] * 9), (513, [64, 33], [70, 1])])
def test_sizes(dtype, d, hq, hkv, prefix, nodes, ctx):
    c = Case(dtype, prefix, nodes, ctx, hq, hkv, d)
    o, lse, st = c.run()
    assert st.tolist() == [0] * len(nodes)
    c.check(o, lse)


@pytest.mark.parametrize("dtype,out", [("bf16", torch.float32), ("f32", torch.bfloat16)])
@pytest.mark.parametrize("kv_split", [0, 1, 5])
def test_splits_and_output_types(dtype, out, kv_split):
    c = Case(dtype, 1000, [20, 7, 31], [300, 0, 64], 4, 1, 128)
    o, lse, _ = c.run(kv_split=kv_split, out_dtype=out)
    assert o.dtype == out
    c.check(o, lse, only=lambda n: [0, n // 2, n - 1])


@pytest.mark.parametrize("d", [64, 128])
def test_fp32_tiles_that_fill_the_chip(d):
    """Launches whose tiles of 128 rows number 256 and more and are full take a kernel of their own."""
    c = Case("f32", 150, [40] * 8, [0, 5, 33, 64, 90, 1, 31, 32], 64, 16, d)
    o, lse, st = c.run()
    assert st.tolist() == [0] * 8
    c.check(o, lse, only=lambda n: [0, 17, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,hq,hkv", [([256, 200], 2, 1), ([256], 5, 5), ([129, 3, 128], 33, 1)])
def test_large_trees(dtype, nodes, hq, hkv):
    """Trees of several tiles and of four words of ancestor bits."""
    c = Case(dtype, 65, nodes, [37, 0, 300][:len(nodes)], hq, hkv, 64)
    o, lse, st = c.run()
    assert st.tolist() == [0] * len(nodes)
    c.check(o, lse, only=lambda n: [0, 63, 64, n // 2, 127, 128, 199, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_own_contexts_longer_than_the_prefix(dtype):
    c = Case(dtype, 40, [9, 17], [3000, 1500], 8, 2, 128)
    for kv_split in (0, 1, 2):
        o, lse, _ = c.run(kv_split=kv_split)
        c.check(o, lse, only=lambda n: [0, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nodes_off_a_path_may_be_anything(dtype):
    """Keys and values of nodes that a node does not descend from: NaN and infinities there leave it its bits."""
    c = Case(dtype, 50, [20, 12], [33, 0], 4, 2, 64, seed=5)
    want, want_lse, _ = c.run()
    anc, _ = oracle.ancestors(c.parents[0], 20)
    bad = 11                                               # a node of sequence 0
    at = c.kv_off[0] + c.ctx[0] + bad
    c.k[at], c.v[at, :, ::2], c.v[at, :, 1::2] = float("nan"), float("inf"), float("nan")
    o, lse, _ = c.run()
    for n in range(20):
        if bad in anc[n]:
            assert torch.isnan(o[0, n]).all()
        else:
            assert torch.equal(o[0, n], want[0, n]) and torch.equal(lse[0, n], want_lse[0, n]), n
    assert torch.equal(o[1, :12], want[1, :12])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", [-60.0, -300.0])
def test_low_scores_behind_hidden_nodes(dtype, low):
    """A row whose first visible token is not among its first 32, with scores whose exponentials are
    none: a tree of roots, each of which sees itself and a prefix of lower scores yet."""
    c = Case(dtype, 40, [90, 64], [0, 0], 4, 2, 64)
    c.parents = [[-1] * 90, [-1] * 64]
    side = torch.full((64,), 64 ** -0.5)
    rise = normal(9, c.k.shape[0], 1, 1)
    c.q = (side * 8 * torch.ones(c.q.shape[:3]).unsqueeze(-1)).to(c.q.dtype)
    c.k = ((low - 5 + rise) * side).expand(c.k.shape).to(c.k.dtype).contiguous()
    for off, n in zip(c.kv_off, c.nodes):
        c.k[off:off + n] += (5 * side).to(c.k.dtype)
    o, lse, _ = c.run()
    c.check(o, lse)


def test_many_sequences():
    """More sequences than lanes of a wave, some of them without nodes."""
    c = Case("bf16", 200, [b % 4 for b in range(131)], [b % 7 for b in range(131)], 2, 1, 64)
    o, lse, st = c.run()
    assert st.tolist() == [0] * 131
    c.check(o, lse)


def test_no_prefix_is_the_tree_attention():
    c = Case("bf16", 0, [12, 30], [200, 33], 8, 2, 128)
    o, lse, st = c.run()
    want, want_lse, _ = pc.cure_tree_attn(c.q.cuda(), c.k.cuda(), c.v.cuda(), ints(c.kv_off, torch.int64), ints(c.ctx),
                                          ints(c.nodes), c.parent(), c.ctx, c.nodes, c.scale)
    for b, n in enumerate(c.nodes):
        assert torch.equal(o[b, :n], want[b, :n]) and torch.equal(lse[b, :n], want_lse[b, :n])


def test_nodes_that_do_not_exist_are_left():
    c = Case("f32", 70, [5, 0, 9], [3, 4, 0], 4, 2, 64, n_max=11)
    out = torch.full(c.q.shape, 9.0, device="cuda")
    o, lse, _ = c.run(out=out, with_lse=False)
    assert o.data_ptr() == out.data_ptr() and lse is None
    c.check(o, None)
    for b, n in enumerate(c.nodes):
        assert bool((o[b, n:] == 9.0).all())


def test_no_nodes_at_all():
    c = Case("bf16", 70, [0, 0], [3, 4], 4, 2, 64, n_max=2)
    out = torch.full(c.q.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    _, _, st = c.run(out=out)
    assert st.tolist() == [0, 0] and bool((out == 9.0).all())


def test_a_malformed_tree_is_reported():
    c = Case("bf16", 100, [6, 6, 6], [5, 5, 5], 4, 2, 64)
    want, _, _ = c.run()
    c.parents[1][2] = 4
    o, _, st = c.run()
    assert st.tolist() == [0, pc.CURE_ERR_BAD_TREE, 0]
    assert torch.equal(o[0], want[0]) and torch.equal(o[2], want[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_rows_around_the_prefix_may_be_anything(dtype):
    c = Case(dtype, 77, [9, 3], [10, 0], 4, 2, 64)
    want, want_lse, _ = c.run()
    inside = np.zeros(len(c.k), bool)
    inside[c.prefix_off:c.prefix_off + c.prefix] = True
    for off, n, l in zip(c.kv_off, c.nodes, c.ctx):
        inside[off:off + n + l] = True
    for x in (c.k, c.v):
        x[~inside] = float("nan")
    o, lse, _ = c.run()
    for b, n in enumerate(c.nodes):
        assert torch.equal(o[b, :n], want[b, :n]) and torch.equal(lse[b, :n], want_lse[b, :n])


def test_captured_calls_replay_on_other_trees():
    c = Case("bf16", 500, [20, 20, 20], [100, 40, 0], 8, 2, 128)
    q, k, v, kv_off = c.q.cuda(), c.k.cuda(), c.v.cuda(), ints(c.kv_off, torch.int64)
    nodes, parent, ctx = ints(c.nodes), c.parent(), ints(c.ctx)
    out = torch.zeros_like(q)
    call = lambda o: pc.cure_prefix_attn(q, k, v, c.prefix_off, c.prefix, kv_off, ctx, nodes, parent, c.ctx, c.nodes,  # noqa: E731
                                         c.scale, with_lse=False, out=o)
    call(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out)
    rng = np.random.default_rng(1)
    for new in ([20, 20, 20], [3, 20, 1], [0, 11, 0], [20, 0, 19]):
        c.nodes = new
        c.parents = [random_parents(rng, n) for n in new]
        nodes.copy_(ints(new))
        parent.copy_(c.parent())
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        fresh = call(torch.zeros_like(q))[0]
        torch.cuda.synchronize()
        assert torch.equal(out, fresh), new
        c.check(out, None, only=lambda n: [0, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_split", [0, 1, 5])
def test_sizes_other_than_the_hosts_copies(dtype, kv_split):
    """A captured call is replayed on contexts that grew or shrank and on other trees: the plan is the host's, the sizes
    are the device's."""
    c = Case(dtype, 700, [20, 31, 3], [900, 40, 0], 4, 2, 64, n_max=40)
    for ctx, nodes in (([5, 700, 64], [1, 40, 17]), ([0, 0, 0], [40, 40, 40])):
        other = Case(dtype, 700, nodes, ctx, 4, 2, 64, n_max=40)
        q, k, v = other.q.cuda(), other.k.cuda(), other.v.cuda()
        o, lse, st = pc.cure_prefix_attn(q, k, v, other.prefix_off, 700, ints(other.kv_off, torch.int64), ints(ctx), ints(nodes),
                                         other.parent(), c.ctx, c.nodes, other.scale, kv_split=kv_split)
        assert st.tolist() == [0, 0, 0]
        other.check(o, lse, only=lambda n: [0, n // 2, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_streams_at_once(dtype):
    """Calls under way together on two streams, each with scratch of its own."""
    cases = [Case(dtype, 900, [30, 12], [64, 300], 8, 2, 128, seed=s) for s in (1, 2)]
    args = [(c.q.cuda(), c.k.cuda(), c.v.cuda(), c.prefix_off, c.prefix, ints(c.kv_off, torch.int64), ints(c.ctx), ints(c.nodes),
             c.parent(), c.ctx, c.nodes, c.scale) for c in cases]
    want = [pc.cure_prefix_attn(*a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(10):
        for i, (st, a) in enumerate(zip(streams, args)):
            with torch.cuda.stream(st):
                got[i].append(pc.cure_prefix_attn(*a))
    torch.cuda.synchronize()
    for c, w, runs in zip(cases, want, got):
        for r in runs:
            for b, n in enumerate(c.nodes):
                assert torch.equal(r[0][b, :n], w[0][b, :n]) and torch.equal(r[1][b, :n], w[1][b, :n])
