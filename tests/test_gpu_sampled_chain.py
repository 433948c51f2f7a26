"""The packed cache and sampling together, as a serving loop uses them: prompts appended and packed in whole
blocks, candidate trees appended behind the rows that are still open, attended over packed and open
context, the target's token drawn for every node, the walk over the drawn tokens, the winning path
committed, and blocks packed as they fill."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_00531_amd as pc
from packed_util import Case
from prompt_util import DTYPES, HALF, ints, normal, random_parents, wide
from test_gpu_serving_chain import D, HKV, HQ, Loop

pytestmark = pytest.mark.gpu

VOCAB = 4000
BLOCK = pc.CURE_PACK_TOKENS
SETTINGS = [(0.7, 50, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0)]
U = 2.0 ** -24


class Packed(Loop):
    """A loop whose context is packed in whole blocks; the rows behind them are open."""

    def __init__(self, dtype, prompts):
        super().__init__(dtype, prompts, 0)
        blocks = [(n + 200) // BLOCK + 1 for n in prompts]
        self.blk_off = [sum(blocks[:b]) + 1 for b in range(self.batch)]
        total = sum(blocks) + 2
        self.pk, self.pv = (torch.full((total, HKV, BLOCK * D), 77, dtype=torch.int8, device="cuda") for _ in range(2))
        self.ks, self.vs = (torch.full((total, HKV), float("nan"), device="cuda") for _ in range(2))
        self.off, self.packed, self.ctx = list(self.kv_off), [0] * self.batch, [0] * self.batch
        self.head = normal(9, HQ * D, VOCAB, std=0.3).cuda()

    def pack(self):
        n = [c // BLOCK * BLOCK for c in self.ctx]
        st = pc.cure_kv_pack(self.k, self.v, ints(self.off, torch.int64), ints(n), self.pk, self.pv, self.ks, self.vs,
                             ints(self.blk_off, torch.int64), ints(self.packed), n_max=max(n))
        assert st.tolist() == [0] * self.batch
        for b, x in enumerate(n):
            self.off[b] += x
            self.packed[b] += x
            self.ctx[b] -= x

    def attend(self, q, nodes, parent, **kw):
        return pc.cure_packed_attn(q, self.pk, self.pv, self.ks, self.vs, ints(self.blk_off, torch.int64), ints(self.packed), self.k,
                                   self.v, ints(self.off, torch.int64), ints(self.ctx), ints(nodes), self.packed, self.ctx, nodes,
                                   D ** -0.5, parent=parent, **kw)

    def logits(self, o, tree, parents):
        """Of the target: a token's logits, with the node's children among the likely ones."""
        x = (o.float().flatten(2) @ self.head)
        for b, p in enumerate(parents):
            for i, up in enumerate(p):
                if up >= 0:
                    x[b, up, tree[b][i]] += 12.0
        return x.to(self.t)


def case_of(s, dtype, q, nodes, parents):
    """What the attention's check needs to know of a step."""
    c = Case.__new__(Case)
    c.dtype, c.rows, c.packed, c.ctx, c.hq, c.hkv, c.d, c.scale = dtype, nodes, s.packed, s.ctx, HQ, HKV, D, D ** -0.5
    c.parents, c.blk_off, c.kv_off = parents, s.blk_off, s.off
    c.n_max = q.shape[1]
    c.total, c.first = len(nodes) * c.n_max, [b * c.n_max for b in range(len(nodes))]
    c.q, c.k, c.v, c.pk, c.pv, c.ks, c.vs = (x.cpu() for x in (q, s.k, s.v, s.pk, s.pv, s.ks, s.vs))
    return c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_trees_draws_and_blocks(dtype):
    rng = np.random.default_rng(5)
    prompts = [150, 1, 64]
    s = Packed(dtype, prompts)
    token = lambda: int(rng.integers(1, VOCAB))  # noqa: E731
    lists = [[token() for _ in range(n)] for n in prompts]
    s.append(lists, s.off, s.ctx, [0] * 3)
    s.tokens, s.ctx = [list(x) for x in lists], list(prompts)
    s.pack()
    assert s.packed == [128, 0, 64] and s.ctx == [22, 1, 0]
    packs = 0
    for step in range(14):
        nodes = [int(rng.integers(1, 40)) for _ in range(3)]
        n_max = max(nodes)
        parents = [random_parents(rng, n) for n in nodes]
        tree = [[token() for _ in range(n)] for n in nodes]
        parent = ints([p + [-1] * (n_max - len(p)) for p in parents])
        q = s.append(tree, s.off, s.ctx, s.packed, parent=parent)
        got = s.attend(q, nodes, parent)
        if step % 4 == 0:
            torch.cuda.synchronize()
            case_of(s, dtype, q, nodes, parents).check(got)
        x = s.logits(got[0], tree, parents)
        u = torch.rand((3, n_max), generator=torch.Generator().manual_seed(step))
        t, k, p, m = (list(v) for v in zip(*SETTINGS))
        f = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
        drawn = pc.cure_sample(x, u.cuda(), f(t), ints(k), f(p), f(m), n_rows=ints(nodes))
        if step % 4 == 0:
            for b in range(3):
                for r in range(n_max):
                    ref = oracle.sample(wide(x[b, r]), float(u[b, r]), *SETTINGS[b]) if r < nodes[b] else (pc.CURE_NO_TOKEN, -np.inf, 0)
                    assert (int(drawn["token"][b, r]), int(drawn["kept"][b, r])) == (ref[0], ref[2]), (step, b, r)
                    assert ref[1] == float(drawn["logprob"][b, r]) or abs(float(drawn["logprob"][b, r]) - ref[1]) <= U * (abs(ref[1]) + 1)
        toks = ints([y + [0] * (n_max - len(y)) for y in tree])
        acc = pc.cure_accept(parent, toks, drawn["token"], ints([y[0] for y in tree]), ints(nodes), 16)
        com = pc.cure_commit(s.k, s.v, ints(s.off, torch.int64), ints(s.ctx), ints(nodes), acc["path"], acc["acc_len"], toks,
                             acc["bonus"], 16)
        for b in range(3):
            n = int(acc["acc_len"][b])
            assert n >= 1                                  # the root was what the last step drew
            s.tokens[b] += com["emit"][b, :n].tolist()
            assert int(com["new_ctx_len"][b]) == s.ctx[b] + n and len(s.tokens[b]) == s.packed[b] + s.ctx[b] + n
            s.ctx[b] += n
        if max(s.ctx) >= BLOCK:
            s.pack()
            packs += 1
    assert packs >= 1
    # What is packed is what a prompt of the accepted tokens would have written, within half a step of its
    # block and head and the row's own rounding; what is open is it, bit for bit.
    for b in range(3):
        k, v = s.cache_of(s.tokens[b], 0)
        n = s.packed[b]
        rows = slice(s.off[b], s.off[b] + s.ctx[b])
        assert torch.equal(s.k[rows], k[n:]) and torch.equal(s.v[rows], v[n:]), b
        back = [torch.zeros(n + 1, HKV, D, dtype=s.t, device="cuda") for _ in range(2)]
        st = pc.cure_kv_unpack(s.pk, s.pv, s.ks, s.vs, ints([s.blk_off[b]], torch.int64), ints([0]), *back, ints([0], torch.int64), ints([n]))
        assert st.tolist() == [0]
        for got, want, scale in zip(back, (k, v), (s.ks, s.vs)):
            step = wide(scale[s.blk_off[b]:s.blk_off[b] + n // BLOCK]).repeat(BLOCK, axis=0)[:, :, None]
            got, want = wide(got[:n]), wide(want[:n])
            assert np.all(np.abs(got - want) <= (step / 2 + HALF[DTYPES[dtype]] * np.abs(got)) * (1 + 2.0 ** -20)), b


def test_a_captured_step():
    """Attention, draws and the walk in one graph, replayed on new rows and numbers, with eager work between."""
    rng = np.random.default_rng(8)
    s = Packed("bf16", [300, 70])
    lists = [[int(rng.integers(1, VOCAB)) for _ in range(n)] for n in (300, 70)]
    s.append(lists, s.off, s.ctx, [0] * 2)
    s.ctx = [300, 70]
    s.pack()
    nodes, n_max = [24, 9], 24
    parents = [random_parents(rng, n) for n in nodes]
    parent = ints([p + [-1] * (n_max - len(p)) for p in parents])
    trees = [[[int(rng.integers(1, VOCAB)) for _ in range(n)] for n in nodes] for _ in range(4)]
    toks, u = ints([[0] * n_max] * 2), torch.zeros(2, n_max, device="cuda")
    q = torch.zeros(2, n_max, HQ, D, dtype=s.t, device="cuda")
    count, root = ints(nodes), ints([0] * 2)
    args = (s.pk, s.pv, s.ks, s.vs, ints(s.blk_off, torch.int64), ints(s.packed), s.k, s.v, ints(s.off, torch.int64), ints(s.ctx), count,
            list(s.packed), list(s.ctx), nodes, D ** -0.5)
    head = s.head.to(s.t)

    def step():
        o, _, status = pc.cure_packed_attn(q, *args, parent=parent, kv_split=3)
        x = (o.flatten(2).view(2 * n_max, HQ * D) @ head).view(2, n_max, VOCAB)
        drawn = pc.cure_sample(x, u, n_rows=count)
        return [o, status, drawn["token"], drawn["logprob"], pc.cure_accept(parent, toks, drawn["token"], root, count, 16)["path"]]

    def load(i):
        q.copy_(s.append(trees[i], s.off, s.ctx, s.packed, parent=parent))
        u.copy_(torch.rand((2, n_max), generator=torch.Generator().manual_seed(i)))
        toks.copy_(ints([y + [0] * (n_max - len(y)) for y in trees[i]]))
        root.copy_(toks[:, 0])

    load(0)
    for _ in range(2):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in (1, 2, 3, 1):
        load(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        want = step()
        torch.cuda.synchronize()
        names = ("o", "status", "token", "logprob", "path")
        for name, x, y in zip(names, got, want):           # a padded row's output is nobody's
            same = [bool(torch.equal(x[b, :n], y[b, :n]) if x.dim() > 1 else x[b] == y[b]) for b, n in enumerate(nodes)]
            assert all(same), (i, name, same)
