"""cure_rope_append against the 64-bit definition, within the bounds derived in prompt_util.py."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_00531_amd as pc
from prompt_util import DTYPES, HALF, U, ints, normal, random_parents, wide

pytestmark = pytest.mark.gpu


def bound(x, y, d, rot, interleaved, mscale, half):
    """x normalised values, y rotated ones: what a result may be off by."""
    pair = np.zeros_like(y)
    n = rot // 2
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        pair[..., a] = pair[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    scale = np.where(np.arange(d) < rot, mscale, 0.0)
    own = np.abs(x) * (d / 2 + 12) * U
    tol = pair * scale * (6e-7 + (d / 2 + 12) * U) + own
    return tol + half * (np.abs(y) + tol)


def run(dtype, rows, ctx, hq, hkv, d, rot, tree=False, norm=False, interleaved=False, fused=False, pos=None,
        mscale=1.0, base=10000.0, parents=None, seed=0, in_place=False):
    """One call on padded (tree) or packed rows; checks every row of q, the caches and what must stay."""
    t = DTYPES[dtype]
    batch, n_max = len(rows), max(rows)
    rng = np.random.default_rng(seed)
    total = batch * n_max if tree else sum(rows) + 3
    heads = hq + 2 * hkv
    both = normal(seed, total, heads if fused else heads, d, dtype=t, std=2.0)
    both_g = both.cuda()
    q, k, v = (x if fused else x.contiguous() for x in both_g.split([hq, hkv, hkv], dim=1))
    shape = (lambda x: x.view(batch, n_max, *x.shape[1:]) if not fused else
             x.as_strided((batch, n_max, x.shape[1], d), (n_max * heads * d, heads * d, d, 1), x.storage_offset()))
    row_off = [b * n_max for b in range(batch)]
    if not tree:
        row_off, at = [], 1
        for n in rows:
            row_off.append(at)
            at += n
    kv_off, at = [], 2
    for n, c in zip(rows, ctx):
        kv_off.append(at)
        at += n + c + 1
    caches = [normal(seed + 1 + i, at + 2, hkv, d, dtype=t) for i in range(2)]
    kc, vc = (c.cuda() for c in caches)
    qw, kw = ((normal(seed + 5 + i, d, dtype=torch.float32, std=0.2) + 1).to(t) for i in range(2)) if norm else (None, None)
    freq, _ = pc.cure_rope_frequencies(rot, base)
    parent = None
    if tree:
        parents = parents or [random_parents(rng, n) for n in rows]
        parent = ints([p + [-7] * (n_max - len(p)) for p in parents])
    out = q if in_place else normal(seed + 9, total, hq, d, dtype=t).cuda()
    keep = out.cpu().clone()
    got, status = pc.cure_rope_append(
        *(shape(x) if tree else x for x in (q, k, v)), kc, vc, ints(kv_off, torch.int64), ints(ctx), ints(rows),
        freq.cuda() if rot else None, parent=parent, row_off=None if tree else ints(row_off, torch.int64),
        pos_off=None if pos is None else ints(pos), q_weight=None if qw is None else qw.cuda(),
        k_weight=None if kw is None else kw.cuda(), interleaved=interleaved, mscale=mscale,
        n_max=n_max, out=out.view(batch, n_max, hq, d) if tree else out)
    torch.cuda.synchronize()
    assert status.tolist() == [0] * batch
    assert got.data_ptr() == out.data_ptr()
    got = wide(got).reshape(total, hq, d)
    gk, gv = kc.cpu(), vc.cpu()
    used, slots = np.zeros(total, bool), np.zeros(len(gk), bool)
    x = wide(both)
    f = freq.double().numpy()
    for b in range(batch):
        r = slice(row_off[b], row_off[b] + rows[b])
        first = ctx[b] + (0 if pos is None else pos[b])
        where = oracle.tree_positions(parents[b], rows[b], first) if tree else first + np.arange(rows[b])
        args = (x[r, :hq], x[r, hq:hq + hkv], x[r, hq + hkv:])
        kwargs = dict(q_weight=None if qw is None else wide(qw), k_weight=None if kw is None else wide(kw))
        ref_q, ref_k, _ = oracle.rope_append(*args, where, f, interleaved=interleaved, mscale=mscale, **kwargs)
        plain_q, plain_k, _ = oracle.rope_append(*args, where, f[:0], **kwargs)
        at = slice(kv_off[b] + ctx[b], kv_off[b] + ctx[b] + rows[b])
        for g, ref, plain in ((got[r], ref_q, plain_q), (wide(gk[at]), ref_k, plain_k)):
            tol = bound(plain, ref, d, rot, interleaved, mscale, HALF[t])
            assert np.all(np.abs(g - ref) <= tol), (b, float(np.max(np.abs(g - ref) - tol)))
        assert torch.equal(gv[at], both[r, hq + hkv:])
        used[r], slots[at] = True, True
    assert torch.equal(torch.from_numpy(got[~used]), wide_t(keep)[~used])       # rows of no sequence
    for g, c in ((gk, caches[0]), (gv, caches[1])):
        assert torch.equal(g[~slots], c[~slots])


def wide_t(t):
    return t.double().reshape(-1, *t.shape[-2:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,hq,hkv", [(128, 128, 32, 8), (64, 64, 4, 4), (64, 32, 3, 1), (80, 32, 5, 5),
                                          (96, 96, 12, 2), (256, 64, 2, 1), (256, 256, 1, 1), (128, 0, 8, 2), (16, 16, 7, 1)])
@pytest.mark.parametrize("interleaved,norm", [(False, False), (True, True)])
def test_packed_rows(dtype, d, rot, hq, hkv, interleaved, norm):
    run(dtype, [1, 17, 0, 5], [0, 130, 9, 1], hq, hkv, d, rot, norm=norm, interleaved=interleaved, fused=norm)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved,norm", [(False, True), (True, False)])
@pytest.mark.parametrize("rows", [[1], [12, 0, 33], [64, 65], [256, 7]])
def test_tree_rows(dtype, rows, interleaved, norm):
    run(dtype, rows, list(range(3, 3 + len(rows))), 8, 2, 128, 128, tree=True, norm=norm, interleaved=interleaved,
        fused=interleaved, pos=[11 * b for b in range(len(rows))])


def test_deepest_and_flattest_trees():
    run("bf16", [256, 256, 256], [5, 0, 7], 4, 1, 64, 64, tree=True,
        parents=[list(range(-1, 255)), [-1] * 256, [-1] + [0] * 255])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_share_workgroups(dtype):
    """From 2048 rows of batch x n_max on, a workgroup takes four; the last one of a sequence fewer."""
    run(dtype, [2051, 3, 1022], [0, 40, 7], 4, 2, 64, 64, norm=True)


@pytest.mark.parametrize("far", [131072, 10 ** 7, 2 ** 30])
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_and_amplitude(far, interleaved):
    run("f32", [9, 4], [3, 0], 2, 1, 64, 64, interleaved=interleaved, pos=[far, -far], mscale=1.25)


def test_in_place_queries():
    run("bf16", [6, 9], [4, 2], 8, 2, 128, 64, norm=True, in_place=True)


def test_keys_without_queries():
    t = torch.bfloat16
    k, v = normal(1, 5, 2, 64, dtype=t).cuda(), normal(2, 5, 2, 64, dtype=t).cuda()
    kc, vc = (torch.zeros(9, 2, 64, dtype=t, device="cuda") for _ in range(2))
    freq, _ = pc.cure_rope_frequencies(64)
    q, status = pc.cure_rope_append(None, k, v, kc, vc, ints([0], torch.int64), ints([3]), ints([5]), freq.cuda(),
                                    row_off=ints([0], torch.int64))
    assert q is None and status.tolist() == [0]
    ref = oracle.rope_append(np.zeros((5, 1, 64)), wide(k), wide(v), 3 + np.arange(5), freq.numpy())[1]
    assert np.max(np.abs(wide(kc[3:8]) - ref)) <= 2.0 ** -8 * np.max(np.abs(ref)) + 1e-5
    assert torch.equal(vc[3:8], v) and not kc[:3].any() and not kc[8:].any()


def test_queries_without_keys():
    t = torch.bfloat16
    q = normal(1, 5, 3, 64, dtype=t).cuda()
    none = torch.empty(5, 0, 64, dtype=t, device="cuda")
    freq, _ = pc.cure_rope_frequencies(64)
    got, status = pc.cure_rope_append(q, none, none, none[:0], none[:0], ints([0], torch.int64), ints([3]), ints([5]), freq.cuda(),
                                      row_off=ints([0], torch.int64))
    assert status.tolist() == [0]
    x = wide(q)
    ref = oracle.rope_append(x, np.zeros((5, 1, 64)), np.zeros((5, 1, 64)), 3 + np.arange(5), freq.double().numpy())[0]
    assert np.all(np.abs(wide(got) - ref) <= bound(x, ref, 64, 64, False, 1.0, HALF[t]))


@pytest.mark.parametrize("what", ["parent", "self", "below", "n_rows", "n_max", "ctx", "kv_off", "cache_end", "rows_end"])
def test_a_bad_sequence_is_reported_and_left_alone(what):
    t = torch.float32
    rows, ctx, kv_off, row_off = [4, 4, 3], [2, 2, 2], [0, 10, 20], [0, 4, 8]
    parents = [[-1, 0, 1, 1], [-1, 0, 1, 2], [-1, -1, 0, -9]]
    tree = what in ("parent", "self", "below")
    if what == "parent":
        parents[1][2] = 3
    if what == "self":
        parents[1][0] = 0
    if what == "below":
        parents[1][3] = -2
    if what == "n_rows":
        rows[1] = -1
    if what == "n_max":
        rows[1] = 5
    if what == "ctx":
        ctx[1] = -1
    if what == "kv_off":
        kv_off[1] = -1
    if what == "cache_end":
        kv_off[1] = 24 + 3                              # 30 cache rows: 27 + 2 + 4 reach past them
    if what == "rows_end":
        row_off[1] = 9
    shape = (3, 4) if tree else (12,)
    q, k, v = (normal(i, *shape, h, 64, dtype=t).cuda() for i, h in ((0, 4), (1, 2), (2, 2)))
    kc, vc = (normal(5 + i, 30, 2, 64, dtype=t).cuda() for i in range(2))
    before = kc.clone(), vc.clone()
    out = torch.full((*shape, 4, 64), 7.0, device="cuda")
    freq, _ = pc.cure_rope_frequencies(64)
    _, status = pc.cure_rope_append(q, k, v, kc, vc, ints(kv_off, torch.int64), ints(ctx), ints(rows), freq.cuda(),
                                    parent=ints(parents) if tree else None,
                                    row_off=None if tree else ints(row_off, torch.int64), n_max=4, out=out)
    assert status.tolist() == [0, pc.CURE_ERR_BAD_TREE, 0]
    o = out.view(12, 4, 64)
    assert bool((o[4:8] == 7.0).all()) and not bool((o[:4] == 7.0).any()) and not bool((o[8:11] == 7.0).any())
    for now, was in zip((kc, vc), before):
        assert torch.equal(now[6:22], was[6:22]) and torch.equal(now[25:], was[25:])
        assert not torch.equal(now[2:6], was[2:6]) and not torch.equal(now[22:25], was[22:25])


def test_infinities_stay_in_their_head():
    """A head's values meet no other head's: an infinite one spoils its own row and head at most."""
    t = torch.bfloat16
    q, k, v = (normal(i, 3, h, 128, dtype=t).cuda() for i, h in ((0, 4), (1, 2), (2, 2)))
    freq, _ = pc.cure_rope_frequencies(128)
    w = torch.ones(128, dtype=t, device="cuda")

    def call(q, k, v):
        kc, vc = (torch.zeros(3, 2, 128, dtype=t, device="cuda") for _ in range(2))
        o, _ = pc.cure_rope_append(q, k, v, kc, vc, ints([0], torch.int64), ints([0]), ints([3]), freq.cuda(),
                                   row_off=ints([0], torch.int64), q_weight=w, k_weight=w)
        return o, kc, vc
    clean = call(q, k, v)
    q[1, 2, 5], k[0, 1, 77], v[2, 0, 9] = float("inf"), float("nan"), float("-inf")
    dirty = call(q, k, v)
    for c, g, (r, h) in zip(clean, dirty, ((1, 2), (0, 1), (2, 0))):
        keep = torch.ones(c.shape[:2], dtype=torch.bool, device="cuda")
        keep[r, h] = False
        assert torch.equal(c[keep], g[keep])
    assert dirty[2][2, 0, 9] == float("-inf")


def test_captured_calls_replay():
    t = torch.bfloat16
    rows = ints([5, 2])
    ctx, off = ints([3, 0]), ints([0, 12], torch.int64)
    parent = ints([[-1, 0, 1, 0, 2], [-1, 0, 0, 0, 0]])
    q, k, v = (normal(i, 2, 5, h, 128, dtype=t).cuda() for i, h in ((0, 8), (1, 2), (2, 2)))
    kc, vc = (torch.zeros(20, 2, 128, dtype=t, device="cuda") for _ in range(2))
    out = torch.zeros(2, 5, 8, 128, dtype=t, device="cuda")
    freq = pc.cure_rope_frequencies(128)[0].cuda()
    call = lambda k_to, v_to, o: pc.cure_rope_append(q, k, v, k_to, v_to, off, ctx, rows, freq, parent=parent, out=o)  # noqa: E731
    call(kc, vc, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, status = call(kc, vc, out)
    for i in range(4):
        rows.copy_(ints([[5, 2], [1, 5], [0, 3], [4, 4]][i]))
        ctx.copy_(ints([[3, 0], [7, 1], [0, 0], [2, 3]][i]))
        q.normal_()
        fresh = [torch.zeros_like(x) for x in (kc, vc, out)]
        for x in (kc, vc, out):
            x.zero_()
        torch.cuda.synchronize()
        g.replay()
        call(*fresh)
        torch.cuda.synchronize()
        assert status.tolist() == [0, 0]
        for x, y in zip((kc, vc, out), fresh):
            assert torch.equal(x, y), i
