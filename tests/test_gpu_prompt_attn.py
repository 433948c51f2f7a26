"""cure_prompt_attn against the 64-bit definition, within the bounds derived in prompt_util.py."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_00531_amd as pc
from prompt_util import DTYPES, check_rows, ints, normal, wide

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, dtype, rows, ctx, hq, hkv, d, scale=None, seed=0, std=1.5, gap=3):
        t = DTYPES[dtype]
        self.rows, self.ctx, self.dtype = rows, ctx, dtype
        self.scale = scale if scale is not None else d ** -0.5
        self.row_off, at = [], 2
        for n in rows:
            self.row_off.append(at)
            at += n + 1                                   # a row of nobody's between sequences
        self.total = at
        self.kv_off, at = [0] * len(rows), gap
        for b in reversed(range(len(rows))):              # cache regions in another order
            self.kv_off[b] = at
            at += rows[b] + ctx[b] + gap
        self.q = normal(seed, self.total, hq, d, dtype=t, std=std)
        self.k, self.v = normal(seed + 1, at, hkv, d, dtype=t), normal(seed + 2, at, hkv, d, dtype=t)

    def run(self, kv_split=0, out_dtype=None, with_lse=True, out=None):
        o, lse = pc.cure_prompt_attn(self.q.cuda(), self.k.cuda(), self.v.cuda(), ints(self.row_off, torch.int64),
                                     ints(self.rows), ints(self.kv_off, torch.int64), ints(self.ctx), self.rows,
                                     self.ctx, self.scale, out_dtype=out_dtype, kv_split=kv_split, with_lse=with_lse,
                                     out=out)
        torch.cuda.synchronize()
        return o, lse

    def check(self, o, lse, only=None):
        """Every row, or `only` some tokens of each sequence."""
        q, k, v = wide(self.q), wide(self.k), wide(self.v)
        seen, rows = {}, []
        for b, n in enumerate(self.rows):
            for i in range(n) if only is None else [i for i in only(n) if 0 <= i < n]:
                r = (self.row_off[b] + i,)
                rows.append(r)
                seen[r] = np.arange(self.kv_off[b], self.kv_off[b] + self.ctx[b] + i + 1)
        ref = [np.zeros(self.q.shape), np.zeros(self.q.shape[:2]), np.zeros(self.q.shape)]
        hq, hkv = q.shape[1], k.shape[1]
        for r in rows:
            for h in range(hq):
                g = h // (hq // hkv)
                for dst, x in zip(ref, oracle.attend(q[r][h], k[seen[r], g], v[seen[r], g], self.scale)):
                    dst[r][h] = x
        check_rows(o, lse, ref, rows, seen, q, k, self.scale, self.dtype == "bf16")


LENGTHS = [([1], [0]), ([1, 1, 1], [0, 31, 32]), ([31, 32, 33], [0, 1, 64]), ([127, 2], [0, 255]), ([129], [0]),
           ([0, 5, 0], [7, 300, 0]), ([65], [191])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (5, 1)])
@pytest.mark.parametrize("rows,ctx", LENGTHS)
def test_lengths_and_heads(dtype, d, hq, hkv, rows, ctx):
    c = Case(dtype, rows, ctx, hq, hkv, d)
    c.check(*c.run())


@pytest.mark.parametrize("dtype,out", [("bf16", torch.float32), ("f32", torch.bfloat16)])
@pytest.mark.parametrize("kv_split", [0, 1, 3, 7])
def test_splits_and_output_types(dtype, out, kv_split):
    c = Case(dtype, [3, 40, 1], [700, 900, 64], 6, 2, 128)
    o, lse = c.run(kv_split=kv_split, out_dtype=out)
    assert o.dtype == out
    c.check(o, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 3, 8, 33])
def test_long_prompts(dtype, group):
    """Several tiles and many steps: the first, last and some middle tokens."""
    c = Case(dtype, [1111, 300], [0, 513], group, 1, 128)
    c.check(*c.run(), only=lambda n: [0, 1, 31, 32, n // 3, n // 2, n - 33, n - 2, n - 1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,ctx,hq,hkv", [([1111], [70], 32, 8), ([130, 100], [0, 33], 128, 128)])
def test_fp32_tiles_that_fill_the_chip(d, rows, ctx, hq, hkv):
    """Launches whose tiles of 128 rows number 256 and more and are full take a kernel of their own."""
    assert sum(-(-n * hq // hkv // 128) for n in rows) * hkv >= 256
    c = Case("f32", rows, ctx, hq, hkv, d)
    c.check(*c.run(), only=lambda n: [0, 31, n // 2, n - 1])
    c.check(*c.run(kv_split=2), only=lambda n: [0, n - 2])


@pytest.mark.parametrize("dtype,rows,ctx,kv_split", [("bf16", [70, 9], [400, 0], 1), ("bf16", [70, 9], [400, 0], 3),
                                                     ("f32", [70, 9], [400, 0], 1), ("f32", [70, 9], [400, 0], 3)])
def test_the_output_may_be_the_queries(dtype, rows, ctx, kv_split):
    c = Case(dtype, rows, ctx, 4, 2, 64)
    want, want_lse = c.run(kv_split=kv_split)
    q = c.q.cuda()
    o, lse = pc.cure_prompt_attn(q, c.k.cuda(), c.v.cuda(), ints(c.row_off, torch.int64), ints(c.rows), ints(c.kv_off, torch.int64),
                                 ints(c.ctx), c.rows, c.ctx, c.scale, kv_split=kv_split, out=q)
    live = torch.cat([torch.arange(r, r + n) for r, n in zip(c.row_off, c.rows)]).cuda()
    assert torch.equal(q[live], want[live]) and torch.equal(lse[live], want_lse[live])


def test_one_token_over_a_long_context():
    c = Case("bf16", [1, 1, 1], [9000, 0, 4097], 8, 2, 128)
    c.check(*c.run())
    c.check(*c.run(kv_split=40))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,ctx,kv_split,hkv", [([70, 9], [0, 40], 1, 2), ([70, 9], [400, 300], 3, 2), ([1, 1], [33, 5], 1, 2),
                                                   ([120, 100], [0, 64], 1, 128)])
def test_values_a_row_does_not_see_may_be_anything(dtype, rows, ctx, kv_split, hkv):
    """Keys and values outside the sequences, and those of later tokens, hold NaN and infinities: rows
    before them keep their bits, rows that see them have none that is finite."""
    clean = Case(dtype, rows, ctx, 2 * hkv, hkv, 64, seed=3)
    want, want_lse = clean.run(kv_split=kv_split)
    dirty = Case(dtype, rows, ctx, 2 * hkv, hkv, 64, seed=3)
    inside = np.zeros(len(dirty.k), bool)
    for off, n, c in zip(dirty.kv_off, rows, ctx):
        inside[off:off + n + c] = True
    bad = torch.tensor([float("nan"), float("inf"), float("-inf")])
    for x in (dirty.k, dirty.v):
        x[~inside] = bad[torch.arange(int((~inside).sum())) % 3].to(x.dtype)[:, None, None]
    from_tok = rows[0] - 5                                # sequence 0: tokens from here on
    if from_tok > 0:
        at = dirty.kv_off[0] + ctx[0] + from_tok
        dirty.v[at, 0, 7], dirty.v[at + 2, 1, 60], dirty.v[at + 3, 0, 0] = float("nan"), float("inf"), float("-inf")
        dirty.k[at + 1] = float("nan")
    got, got_lse = dirty.run(kv_split=kv_split)
    for b, n in enumerate(rows):
        last = n if b or from_tok <= 0 else from_tok
        r = slice(clean.row_off[b], clean.row_off[b] + last)
        assert torch.equal(got[r], want[r]) and torch.equal(got_lse[r], want_lse[r]), b
    if from_tok > 0:
        r = clean.row_off[0] + from_tok
        assert not torch.isfinite(got[r, :2, 7]).any()    # the first row that sees the NaN: heads of kv-head 0
        assert torch.equal(got[r, 2:], want[r, 2:]) and torch.equal(got[r, :2, 8:], want[r, :2, 8:])
        assert torch.isnan(got[r + 1:r + 5]).all()        # a NaN key reaches the whole row


def test_infinite_values_are_seen():
    c = Case("bf16", [40], [0], 2, 1, 64, seed=4)
    c.v[30, 0, 5] = float("inf")
    o, _ = c.run()
    r, token = c.row_off[0], 30 - c.kv_off[0]
    assert torch.isfinite(o[r:r + token]).all() and (o[r + token:r + 40, :, 5] == float("inf")).all()
    o[r + token:r + 40, :, 5] = 0
    assert torch.isfinite(o[r:r + 40]).all()


def test_rows_of_nobody_are_left():
    c = Case("bf16", [33, 0, 4], [1, 2, 3], 4, 2, 128)
    out = torch.full(c.q.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    o, lse = c.run(out=out, with_lse=False)
    assert o.data_ptr() == out.data_ptr() and lse is None
    c.check(o, None)
    used = np.zeros(c.total, bool)
    for r, n in zip(c.row_off, c.rows):
        used[r:r + n] = True
    assert bool((o[torch.from_numpy(~used)] == 9.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_climbing_scores(dtype):
    """Row maxima that keep rising through the keys, by far more than a softmax step, and fall again."""
    c = Case(dtype, [140], [300], 4, 1, 64, scale=1.0, std=0.5)
    ramp = torch.cat((torch.linspace(0, 30, 300), torch.linspace(30, -30, len(c.k) - 300)))
    c.k[:, 0, 0] = ramp.to(c.k.dtype)
    c.q[:, :, 0] = 2.0
    c.check(*c.run())
    c.q[:, :, 0] = -2.0
    c.check(*c.run(kv_split=2))


def test_equal_scores_average_the_values():
    """Queries of zero: the mean of the values seen, exactly what the sums of 1s give."""
    c = Case("f32", [50], [0], 2, 1, 64, std=0.0)
    o, lse = c.run()
    n = torch.arange(1, 51, dtype=torch.float64)
    mean = wide(c.v[c.kv_off[0]:c.kv_off[0] + 50, 0]).cumsum(0) / n.numpy()[:, None]
    got = wide(o[c.row_off[0]:c.row_off[0] + 50])
    assert np.max(np.abs(got - mean[:, None])) <= 60 * 2.0 ** -24 * 4
    assert np.max(np.abs(wide(lse[c.row_off[0]:c.row_off[0] + 50, 0]) - np.log(n.numpy()))) <= 1e-6


def test_other_streams_and_repeats_agree():
    c = Case("bf16", [5, 90], [800, 0], 8, 2, 128)
    want, want_lse = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            o, lse = c.run()
            assert torch.equal(o[c.row_off[0]:c.row_off[0] + 5], want[c.row_off[0]:c.row_off[0] + 5])
            assert torch.equal(lse[c.row_off[1]:c.row_off[1] + 90], want_lse[c.row_off[1]:c.row_off[1] + 90])


def test_captured_calls_replay_on_shorter_prompts():
    """Two calls captured into graphs of their own, replayed on two streams at once: each has its own
    scratch. The device's sizes may fall below the host copies."""
    c = Case("bf16", [64, 1], [700, 1500], 8, 2, 128)
    row_off, kv_off = ints(c.row_off, torch.int64), ints(c.kv_off, torch.int64)
    q, k, v = c.q.cuda(), c.k.cuda(), c.v.cuda()
    sizes, host = [(ints(c.rows), ints(c.ctx)) for _ in range(2)], (c.rows, c.ctx)
    outs = [torch.zeros_like(q) for _ in range(2)]

    def call(i, out):
        return pc.cure_prompt_attn(q, k, v, row_off, sizes[i][0], kv_off, sizes[i][1], *host, c.scale,
                                   kv_split=4, with_lse=False, out=out)[0]
    graphs = []
    for i in range(2):
        call(i, outs[i])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i, outs[i])
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rows, ctx in (([64, 1], [700, 1500]), ([10, 1], [3, 999]), ([0, 1], [0, 0]), ([33, 0], [640, 2])):
        for i, (n, l) in enumerate(sizes):
            n.copy_(ints(rows))
            l.copy_(ints(ctx if i == 0 else [x // 2 for x in ctx]))
            outs[i].zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            same = torch.equal(outs[i], call(i, torch.zeros_like(q)))
            assert same, (rows, i)
            c.rows, c.ctx = rows, ctx if i == 0 else [x // 2 for x in ctx]
            c.check(outs[i], None)


def test_cache_rows_past_4_gb():
    """A sequence whose rows lie beyond what 32-bit byte offsets reach."""
    rows, hkv, d = 2 ** 22 + 5000, 8, 128                 # 8.6 GB of keys
    k = torch.zeros(rows, hkv, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    n, ctx = 70, 400
    off = rows - n - ctx
    tail = [normal(i, n + ctx, hkv, d, dtype=torch.bfloat16) for i in (1, 2)]
    k[off:], v[off:] = tail[0].cuda(), tail[1].cuda()
    q = normal(3, n, 8, d, dtype=torch.bfloat16).cuda()
    args = (ints([0], torch.int64), ints([n]))
    o, _ = pc.cure_prompt_attn(q, k, v, *args, ints([off], torch.int64), ints([ctx]), [n], [ctx], 0.1)
    near, _ = pc.cure_prompt_attn(q, tail[0].cuda(), tail[1].cuda(), *args, ints([0], torch.int64), ints([ctx]), [n],
                                  [ctx], 0.1)
    assert torch.equal(o, near) and bool(near.any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,group,kv_split,hkv", [(1, 1, 1, 1), (33, 1, 1, 1), (7, 5, 1, 1), (1, 1, 2, 1), (100, 1, 1, 256)])
def test_every_key_counts_once(dtype, d, n, group, kv_split, hkv):
    """Equal scores and one-hot values: element t % d of the output, times the number of keys, is how many
    of the visible tokens t counted. Every number of steps around several turns of the tile rings."""
    t = DTYPES[dtype]
    for total in list(range(n, n + 70, 3)) + list(range(n + 90, n + 460, 29)):
        ctx = total - n
        v = torch.zeros(total, hkv, d, dtype=t)
        v[torch.arange(total), :, torch.arange(total) % d] = 1
        q, k = torch.zeros(n, group * hkv, d, dtype=t, device="cuda"), torch.zeros(total, hkv, d, dtype=t, device="cuda")
        zero = ints([0], torch.int64)
        o, lse = pc.cure_prompt_attn(q, k, v.cuda(), zero, ints([n]), zero, ints([ctx]), [n], [ctx], 1.0,
                                     out_dtype=torch.float32, kv_split=kv_split)
        seen = torch.cumsum(v[:, 0].double(), 0)[ctx:]
        keys = torch.arange(ctx + 1, total + 1, dtype=torch.float64)
        got = o.cpu().double() * keys[:, None, None]
        # 1 / n, the sum and the products of ones are exact up to a few fp32 roundings.
        assert float((got - seen[:, None]).abs().max()) <= 8 * 2.0 ** -24 * total, total
        assert float((lse.cpu().double() - keys.log()[:, None]).abs().max()) <= 2e-6, total


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_split", [0, 1, 4])
def test_contexts_other_than_the_hosts_copies(dtype, kv_split):
    c = Case(dtype, [40, 7, 1], [600, 30, 0], 4, 2, 64)
    for ctx, rows in (([10, 900, 33], [40, 40, 1]), ([0, 0, 1500], [38, 0, 1])):
        other = Case(dtype, rows, ctx, 4, 2, 64)
        o, lse = pc.cure_prompt_attn(other.q.cuda(), other.k.cuda(), other.v.cuda(), ints(other.row_off, torch.int64), ints(rows),
                                     ints(other.kv_off, torch.int64), ints(ctx), c.rows, c.ctx, other.scale, kv_split=kv_split)
        other.check(o, lse, only=lambda n: [0, n // 2, n - 1])
