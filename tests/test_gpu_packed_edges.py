"""Packed context: every length around a step's, a block's and a ring's end, against every number of rows that
changes how rows are shared out; far offsets; calls at once on two streams."""

import numpy as np
import pytest
import torch

import paper_2608_00531_amd as pc
from packed_util import Case
from prompt_util import ints, random_parents
from test_packed_plan import LENGTHS, MANY, shape

pytestmark = pytest.mark.gpu



@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [64, 68, 128, 132, 252, 256, 260])
@pytest.mark.parametrize("form", ["tree", "packed"])
def test_lengths(d, rows, form):
    """Rows of a kv-head: few, one tile of 128 or of 256, and several; the last waves have none, or some of theirs."""
    n, batch = rows // 4, len(LENGTHS)
    rng = np.random.default_rng(rows)
    parents = [random_parents(rng, n) for _ in LENGTHS] if form == "tree" else None
    for split, ctx in ((1, [0] * batch), (0, [(7 * i) % 45 for i in range(batch)]), (3, [33] * batch)):
        c = Case("bf16", [n] * batch, LENGTHS, ctx, 4, 1, d, form=form, seed=split, parents=parents)
        c.check(c.call(kv_split=split), every=9)


@pytest.mark.parametrize("nodes", [40, 64, 100])
def test_far_offsets_of_many_rows(nodes):
    """As for few rows: blocks and cache rows more than 2^31 elements into their buffers."""
    hkv, d = 8, 128
    blocks, rows = (1 << 31) // (hkv * 64 * d) + 40, (1 << 31) // (hkv * d) + 400
    c = Case("bf16", [nodes], [150], [20], 4 * hkv, hkv, d)
    pk, pv = (torch.zeros(blocks, hkv, 64 * d, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(blocks, hkv, device="cuda") for _ in range(2))
    k, v = (torch.zeros(rows, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    b0, r0 = blocks - c.blocks, rows - c.cache_rows
    for big, x in ((pk, c.pk), (pv, c.pv), (ks, c.ks), (vs, c.vs)):
        big[b0:] = x.cuda()
    for big, x in ((k, c.k), (v, c.v)):
        big[r0:] = x.cuda()
    c.check(c.call(pk=pk, pv=pv, k_scale=ks, v_scale=vs, k=k, v=v, blk_off=ints([b0 + c.blk_off[0]], torch.int64),
                   kv_off=ints([r0 + c.kv_off[0]], torch.int64)), every=5)


def test_scales_and_masks_of_many_rows():
    """Blocks whose scales lie far apart, a block of zeros, and infinities and NaN in rows and scales that nobody sees."""
    c = Case("bf16", [33, 40], [300, 64], [30, 0], 8, 2, 128)
    c.ks[:, 0] *= 2.0 ** -10
    c.vs[::2] *= 2.0 ** 20
    c.vs[1::2] *= 2.0 ** -40
    first = c.blk_off[0]
    c.vs[first + 1, 1], c.pv[first + 1, 1] = 0.0, 0
    c.ks[first + 2, 0], c.pk[first + 2, 0] = 0.0, 0
    used = {c.blk_off[b] + i for b in range(2) for i in range((c.packed[b] + 63) // 64)}
    rows = {c.kv_off[b] + i for b in range(2) for i in range(c.ctx[b] + c.rows[b])}
    for i in range(c.blocks):
        if i not in used:
            c.ks[i], c.vs[i] = float("nan"), float("inf")
    for i in range(c.cache_rows):
        if i not in rows:
            c.k[i], c.v[i] = float("nan"), float("inf")
    c.check(c.call())


def test_two_streams_at_once():
    """Calls of one shape on two streams, each with a workspace of its own, give what they give alone."""
    cases = [Case("bf16", [n, 3], [900, 4000], [10, 0], 8, 2, 128, seed=n) for n in (2, 20, 50)]
    alone = [c.call() for c in cases]
    torch.cuda.synchronize()
    args = [dict(c.args) for c in cases]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        for i, a in enumerate(args):
            for s in streams:
                with torch.cuda.stream(s):
                    got.append((i, pc.cure_packed_attn(**a)))
    torch.cuda.synchronize()
    for i, (o, lse, status) in got:
        for b, n in enumerate(cases[i].rows):
            assert torch.equal(o[b, :n], alone[i][0][b, :n]) and torch.equal(lse[b, :n], alone[i][1][b, :n]), i
        assert status.tolist() == [0, 0]


@pytest.mark.parametrize("heads", [1, 128])
def test_many_small_probabilities_beside_a_large_one(heads):
    """A million tokens of one score, each of 2^-21 of the first one's weight: together they are a third of the
    row, and their roundings to 16 bits would all be alike. In 64 bits by hand; the bound is 2^-8 of the whole
    for the probabilities, as of the other tests, and half a step of the output."""
    n, d = 1 << 20, 64
    bits = 21 - np.log2(1.0625)
    pk = torch.ones(n // 64, 1, 64 * d, dtype=torch.int8, device="cuda")
    pv = torch.full_like(pk, 100)
    at = torch.arange(d)
    pk[0, 0, (at // 32 * 1024 + at % 32 // 16 * 512 + at % 16).cuda()] = 25      # token 0's keys
    pv[0, 0, (at // 32 * 1024 + at % 32 * 16).cuda()] = 0                        # and values
    ks = torch.full((n // 64, 1), float(np.float32(bits * np.log(2) / (24 * 8))), device="cuda")
    vs = torch.full((n // 64, 1), 0.01, device="cuda")
    q = torch.ones(1, 1, heads, d, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros(2, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    zero = ints([0], torch.int64)
    k[0] = -300.0                                                                # the new token's own row: no weight
    o, lse, _ = pc.cure_packed_attn(q, pk, pv, ks, vs, zero, ints([n]), k, v, zero, ints([0]), ints([1]), [n], [0], [1], 0.125,
                                    kv_split=1)
    one = float(ks[0, 0]) * 8.0                                                  # a token's score
    w = (n - 1) * np.exp(-24 * one)
    want, want_lse = w * 100 * float(vs[0, 0]) / (1 + w), 25 * one + np.log1p(w)
    assert np.all(np.abs(o.double().cpu().numpy() - want) <= (2.0 ** -8 + 2.0 ** -8) * want)
    assert np.all(np.abs(lse.double().cpu().numpy() - want_lse) <= ((d + 6) * 25 * one + n + 16) * 2.0 ** -24)


@pytest.mark.parametrize("planned", [1, 16, 40])
@pytest.mark.parametrize("split", [0, 1, 3])
def test_more_rows_than_planned(planned, split):
    """Trees on the device with more nodes, up to n_max, than the host's sizes say."""
    c = Case("bf16", [40, 33, 5], [640, 128, 64], [60, 0, 5], 8, 2, 128)
    c.check(c.call(host_n_rows=[planned] * 3, kv_split=split), every=3)


@pytest.mark.parametrize("rows,d,tree,waves", MANY)
def test_lengths_of_many_rows(rows, d, tree, waves):
    """The shapes at which the form of many rows is launched; every twelfth row of every eleventh head."""
    at = shape(rows, d, tree)
    parents = [random_parents(np.random.default_rng(rows), n) for n in at["rows"]] if tree else None
    c = Case("bf16", at["rows"], at["packed"], at["ctx"], at["hq"], at["hkv"], d, form="tree" if tree else "padded", parents=parents, seed=d)
    whole = c.call()
    c.check(whole, every=12, heads=range(0, at["hq"], 11))
    # Splits are a tile's own affair: the same rows in two parts are within the bounds too.
    c.check(c.call(kv_split=2), every=12, heads=range(5, at["hq"], 23))


def test_far_offsets_and_masks_of_many_rows():
    """Blocks and rows more than 2^31 elements into their buffers, with infinities and NaN wherever nobody looks."""
    hkv, d = 64, 128
    at = shape(68, d, True)
    parents = [random_parents(np.random.default_rng(3), n) for n in at["rows"]]
    c = Case("bf16", at["rows"], at["packed"], at["ctx"], at["hq"], hkv, d, parents=parents)
    c.vs[::2] *= 2.0 ** 20
    c.vs[1::2] *= 2.0 ** -40
    used = {c.blk_off[b] + i for b in range(len(c.rows)) for i in range((c.packed[b] + 63) // 64)}
    rows = {c.kv_off[b] + i for b in range(len(c.rows)) for i in range(c.ctx[b] + c.rows[b])}
    for i in set(range(c.blocks)) - used:
        c.ks[i], c.vs[i] = float("nan"), float("inf")
    for i in set(range(c.cache_rows)) - rows:
        c.k[i], c.v[i] = float("nan"), float("inf")
    blocks, far = (1 << 31) // (hkv * 64 * d) + c.blocks + 8, (1 << 31) // (hkv * d) + c.cache_rows + 8
    pk, pv = (torch.zeros(blocks, hkv, 64 * d, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(blocks, hkv, device="cuda") for _ in range(2))
    k, v = (torch.zeros(far, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    b0, r0 = blocks - c.blocks, far - c.cache_rows
    for big, x in ((pk, c.pk), (pv, c.pv), (ks, c.ks), (vs, c.vs)):
        big[b0:] = x.cuda()
    for big, x in ((k, c.k), (v, c.v)):
        big[r0:] = x.cuda()
    c.check(c.call(pk=pk, pv=pv, k_scale=ks, v_scale=vs, k=k, v=v, blk_off=ints([b0 + x for x in c.blk_off], torch.int64),
                   kv_off=ints([r0 + x for x in c.kv_off], torch.int64)), every=8, heads=range(0, at["hq"], 13))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_packed_yet(dtype):
    """A packed cache of no blocks: the first steps of a sequence. Calls that would need blocks say so."""
    c = Case(dtype, [7, 3], [0, 0], [40, 0], 8, 2, 64)
    none = dict(pk=c.pk[:0].cuda(), pv=c.pv[:0].cuda(), k_scale=c.ks[:0].cuda(), v_scale=c.vs[:0].cuda(), blk_off=ints([0, 0], torch.int64))
    c.check(c.call(**none))
    assert c.call(**{**none, "packed_len": ints([0, 1])})[2].tolist() == [0, pc.CURE_ERR_BAD_TREE]
    a = c.args
    st = pc.cure_kv_pack(a["k"], a["v"], ints([0, 0], torch.int64), ints([0, 5]), none["pk"], none["pv"], none["k_scale"], none["v_scale"],
                         none["blk_off"], ints([0, 0]))
    assert st.tolist() == [0, pc.CURE_ERR_BAD_TREE]
    st = pc.cure_kv_unpack(none["pk"], none["pv"], none["k_scale"], none["v_scale"], none["blk_off"], ints([0, 0]), a["k"][:0], a["v"][:0],
                           ints([0, 0], torch.int64), ints([0, 1]), n_max=4)
    assert st.tolist() == [0, pc.CURE_ERR_BAD_TREE]
