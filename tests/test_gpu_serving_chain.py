"""The operators together, as a serving loop uses them: prompts into the cache and through the prompt
attention, candidate trees appended, verified with and without a shared prefix, the winning path
committed, and the next step on the new context."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_00531_amd as pc
from prompt_util import DTYPES, check_rows, ints, normal, random_parents, wide

pytestmark = pytest.mark.gpu

HQ, HKV, D = 8, 2, 64


class Loop:
    """One attention layer over a batch; a token's vector stands for its hidden state."""

    def __init__(self, dtype, prompts, prefix):
        t = DTYPES[dtype]
        self.t, self.prefix, self.batch = t, prefix, len(prompts)
        self.states = normal(0, 4000, (HQ + 2 * HKV) * D, dtype=t).view(4000, HQ + 2 * HKV, D).cuda()
        self.freq, self.mscale = pc.cure_rope_frequencies(D, 10000.0, "ramp", factor=4.0, orig_len=256)
        self.freq = self.freq.cuda()
        self.qw, self.kw = ((normal(i, D, std=0.1) + 1).to(t).cuda() for i in (1, 2))
        rows = prefix + sum(n + 200 for n in prompts)
        self.k, self.v = (torch.full((rows, HKV, D), float("nan"), dtype=t, device="cuda") for _ in range(2))
        self.kv_off = [prefix + sum(n + 200 for n in prompts[:b]) for b in range(self.batch)]
        self.tokens = [[] for _ in prompts]                # of each sequence's own context
        self.prefix_tokens = []

    def append(self, tokens, off, ctx, first, **kw):
        """tokens: a list per sequence; packed rows, or with `parent` padded ones."""
        n = [len(x) for x in tokens]
        flat = [x for row in tokens for x in row]
        if "parent" in kw:
            n_max = kw["parent"].shape[1]
            flat = [x for row in tokens for x in row + [0] * (n_max - len(row))]
        both = self.states[torch.tensor(flat, device="cuda")]
        if "parent" in kw:
            both = both.view(len(n), n_max, HQ + 2 * HKV, D)
        else:
            kw["row_off"] = ints([sum(n[:b]) for b in range(len(n))], torch.int64)
        q, k, v = both.split([HQ, HKV, HKV], dim=-2)
        q, st = pc.cure_rope_append(q, k, v, self.k, self.v, ints(off, torch.int64), ints(ctx), ints(n), self.freq,
                                    pos_off=ints(first), q_weight=self.qw, k_weight=self.kw, mscale=self.mscale, **kw)
        assert st.tolist() == [0] * len(n)
        return q

    def prompt(self, tokens, off, ctx, first):
        q = self.append(tokens, off, ctx, first)
        n = [len(x) for x in tokens]
        return pc.cure_prompt_attn(q, self.k, self.v, ints([sum(n[:b]) for b in range(len(n))], torch.int64), ints(n),
                                   ints(off, torch.int64), ints(ctx), n, ctx, D ** -0.5), q

    def cache_of(self, tokens, first):
        """The cache rows of tokens at positions from `first` on, written by a fresh call."""
        k, v = torch.zeros(len(tokens), HKV, D, dtype=self.t, device="cuda"), torch.zeros(len(tokens), HKV, D, dtype=self.t, device="cuda")
        both = self.states[torch.tensor(tokens, device="cuda")]
        pc.cure_rope_append(None, both[:, HQ:HQ + HKV], both[:, HQ + HKV:], k, v, ints([0], torch.int64), ints([0]),
                            ints([len(tokens)]), self.freq, row_off=ints([0], torch.int64), pos_off=ints([first]),
                            k_weight=self.kw, mscale=self.mscale)
        return k, v


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [0, 150])
def test_prompts_trees_and_commits(dtype, prefix):
    rng = np.random.default_rng(prefix)
    prompts = [37, 1, 90]
    s = Loop(dtype, prompts, prefix)
    token = lambda: int(rng.integers(1, 4000))  # noqa: E731
    if prefix:
        s.prefix_tokens = [token() for _ in range(prefix)]
        s.prompt([s.prefix_tokens], [0], [0], [0])
    # The prompts, in two chunks each; a prompt's own attention sees its own tokens only here.
    lists = [[token() for _ in range(n)] for n in prompts]
    for part in (0, 1):
        chunk = [x[:len(x) // 2] if part == 0 else x[len(x) // 2:] for x in lists]
        ctx = [0 if part == 0 else len(x) // 2 for x in lists]
        (o, lse), q = s.prompt(chunk, s.kv_off, ctx, [prefix] * 3)
        torch.cuda.synchronize()
        n = [len(x) for x in chunk]
        ref = oracle.prompt_attention(wide(q), wide(s.k), wide(s.v), [sum(n[:b]) for b in range(3)], n, s.kv_off, ctx, D ** -0.5)
        rows = [(sum(n[:b]) + i,) for b in range(3) for i in range(n[b])]
        seen = {(sum(n[:b]) + i,): np.arange(s.kv_off[b], s.kv_off[b] + ctx[b] + i + 1) for b in range(3) for i in range(n[b])}
        check_rows(o, lse, ref, rows, seen, wide(q), wide(s.k), D ** -0.5, dtype == "bf16")
    s.tokens = [list(x) for x in lists]
    for step in range(3):
        nodes = [int(rng.integers(1, 30)) for _ in range(3)]
        n_max = max(nodes)
        parents = [random_parents(rng, n) for n in nodes]
        tree = [[token() for _ in range(n)] for n in nodes]
        parent = ints([p + [-1] * (n_max - len(p)) for p in parents])
        ctx = [len(x) for x in s.tokens]
        q = s.append(tree, s.kv_off, ctx, [prefix] * 3, parent=parent)
        args = (ints(s.kv_off, torch.int64), ints(ctx), ints(nodes), parent, ctx, nodes, D ** -0.5)
        if prefix:
            o, lse, st = pc.cure_prefix_attn(q, s.k, s.v, 0, prefix, *args)
        else:
            o, lse, st = pc.cure_tree_attn(q, s.k, s.v, *args)
        assert st.tolist() == [0] * 3
        ref = oracle.prefix_attention(wide(q), wide(s.k), wide(s.v), 0, prefix, s.kv_off, ctx, nodes, parents, D ** -0.5)
        seen = {}
        for b in range(3):
            anc, _ = oracle.ancestors(parents[b], nodes[b])
            for i in range(nodes[b]):
                seen[b, i] = np.concatenate([np.arange(prefix), s.kv_off[b] + np.arange(ctx[b]),
                                             s.kv_off[b] + ctx[b] + np.array(anc[i])]).astype(np.int64)
        check_rows(o, lse, ref, list(seen), seen, wide(q), wide(s.k), D ** -0.5, dtype == "bf16")
        # The target accepts a path to a random node of each tree: its argmax before a node is the
        # node's token on the path and no token elsewhere.
        tgt, root = [[0] * n_max for _ in nodes], [0] * 3
        for b in range(3):
            path = oracle.ancestors(parents[b], nodes[b])[0][int(rng.integers(0, nodes[b]))]
            root[b] = tree[b][path[0]]
            for a, c in zip(path, path[1:]):
                tgt[b][a] = tree[b][c]
        toks = ints([x + [0] * (n_max - len(x)) for x in tree])
        acc = pc.cure_accept(parent, toks, ints(tgt), ints(root), ints(nodes), 16)
        com = pc.cure_commit(s.k, s.v, ints(s.kv_off, torch.int64), ints(ctx), ints(nodes), acc["path"], acc["acc_len"], toks,
                             acc["bonus"], 16)
        for b in range(3):
            s.tokens[b] += com["emit"][b, :int(acc["acc_len"][b])].tolist()
            assert len(s.tokens[b]) == int(com["new_ctx_len"][b]) > ctx[b]
    # Every committed row is what a prompt of the accepted tokens would have written, bit for bit:
    # a node was rotated by the position that its path gave it.
    for b in range(3):
        k, v = s.cache_of(s.tokens[b], prefix)
        r = slice(s.kv_off[b], s.kv_off[b] + len(s.tokens[b]))
        assert torch.equal(s.k[r], k) and torch.equal(s.v[r], v), b
