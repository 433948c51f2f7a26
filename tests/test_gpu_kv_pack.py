"""cure_kv_pack and cure_kv_unpack against the 64-bit definition.

Integers have to be the definition's: the kernel decides every rounding exactly. A scale
is one fp32 division. A row that comes back is scale * c, rounded to fp32 (2^-24) and, for bf16, once
more (2^-8): |err| <= (2^-24 + h + 2^-24 h) |scale c|.
"""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_00531_amd as pc
from prompt_util import DTYPES, HALF, U, ints, normal, wide

pytestmark = pytest.mark.gpu


class Cache:
    """Rows of several sequences in a cache of one or more layers, and a packed cache beside it."""

    def __init__(self, dtype, rows, done, hkv, d, layers=1, seed=0, gap=2):
        self.t, self.rows, self.done, self.hkv, self.d, self.layers = DTYPES[dtype], rows, done, hkv, d, layers
        self.kv_off, self.blk_off, at, blk = [], [], 1, 1
        for n, p in zip(rows, done):
            self.kv_off.append(at)
            self.blk_off.append(blk)
            at += n + gap
            blk += (p + n + 63) // 64 + 1
        self.end, self.blocks = at, blk
        lead = () if layers == 1 else (layers,)
        self.k, self.v = (normal(seed + i, *lead, at, hkv, d, dtype=self.t, std=1.5) for i in range(2))
        self.fill = 77
        self.pk, self.pv = (torch.full((*lead, blk, hkv, 64 * d), self.fill, dtype=torch.int8) for _ in range(2))
        self.ks, self.vs = (torch.full((*lead, blk, hkv), -1.0) for _ in range(2))

    def gpu(self, name):
        return getattr(self, name).cuda()


def layer(x, i, layers):
    return x if layers == 1 else x[i]


def check_pack(c, out):
    """out: (k, v, pk, pv, ks, vs) after the call, on the CPU."""
    k, v, pk, pv, ks, vs = out
    assert torch.equal(k.view(torch.uint8), c.k.view(torch.uint8)) and torch.equal(v.view(torch.uint8), c.v.view(torch.uint8))
    for i in range(c.layers):
        for x, b, s, values in ((k, pk, ks, False), (v, pv, vs, True)):
            x, b, s = wide(layer(x, i, c.layers)), layer(b, i, c.layers).numpy(), layer(s, i, c.layers).numpy()
            used = np.zeros(c.blocks, bool)
            for n, done, off, blk in zip(c.rows, c.done, c.kv_off, c.blk_off):
                ref, scale = oracle.pack_rows(x[off:off + n])
                at = slice(blk + done // 64, blk + done // 64 + len(scale))
                assert np.array_equal(b[at], oracle.to_bytes(ref, values))
                assert np.array_equal(s[at], scale)
                used[at] = True
            assert np.all(b[~used] == c.fill) and np.all(s[~used] == -1.0)


def pack(c, n_max=None):
    g = [c.gpu(n) for n in ("k", "v", "pk", "pv", "ks", "vs")]
    st = pc.cure_kv_pack(g[0], g[1], ints(c.kv_off, torch.int64), ints(c.rows), *g[2:], ints(c.blk_off, torch.int64),
                         ints(c.done), n_max=n_max)
    torch.cuda.synchronize()
    assert st.tolist() == [0] * len(c.rows)
    return [x.cpu() for x in g]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hkv", [(128, 8), (64, 3), (128, 1)])
@pytest.mark.parametrize("layers", [1, 3])
def test_pack(dtype, d, hkv, layers):
    c = Cache(dtype, [1, 64, 0, 65, 130, 63], [0, 64, 128, 0, 192, 0], hkv, d, layers)
    check_pack(c, pack(c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_zeros_and_extremes(dtype):
    """Exact halves, heads of zeros, the smallest and the largest numbers, one loud value."""
    c = Cache(dtype, [64, 64, 3, 64], [0, 0, 0, 0], 2, 64)
    o = c.kv_off
    c.k[o[0]:o[0] + 64, 0] = (torch.arange(64 * 64).view(64, 64) % 509 - 254).to(c.t)       # a = 254: x / 2
    c.v[o[0]:o[0] + 64, 0] = (torch.arange(64 * 64).view(64, 64) % 257 - 128).to(c.t)       # a = 128
    c.k[o[1]:o[1] + 64] = 0
    c.v[o[1]:o[1] + 64, 1] = -0.0
    tiny = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149
    c.k[o[2]:o[2] + 3, 0] = torch.tensor([tiny, -3 * tiny, 0.0] * 64)[:192].view(3, 64).to(c.t)
    c.v[o[2]:o[2] + 3, 0] = (torch.arange(192).view(3, 64) * 2.0 ** -118).to(c.t)
    c.k[o[3]:o[3] + 64, 1] *= 2.0 ** 120
    c.v[o[3] + 5, 0, 9] = 3.0e38
    check_pack(c, pack(c, n_max=64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hkv,layers", [(128, 8, 1), (64, 3, 2)])
def test_unpack(dtype, d, hkv, layers):
    """Any tokens of packed sequences, to rows of another cache; other rows stay."""
    c = Cache(dtype, [200, 64, 7, 129], [0] * 4, hkv, d, layers)
    _, _, pk, pv, ks, vs = pack(c)
    first, n = [37, 0, 3, 64], [163, 64, 4, 0]
    off = [5, 400, 300, 0]
    back = Cache(dtype, [500], [0], hkv, d, layers, seed=9)
    gk, gv = back.gpu("k"), back.gpu("v")
    st = pc.cure_kv_unpack(*(x.cuda() for x in (pk, pv, ks, vs)), ints(c.blk_off, torch.int64), ints(first), gk, gv,
                           ints(off, torch.int64), ints(n), n_max=163)
    torch.cuda.synchronize()
    assert st.tolist() == [0] * 4
    for i in range(layers):
        for g, b, s, was, values in ((gk, pk, ks, back.k, False), (gv, pv, vs, back.v, True)):
            g, b, s, was = (layer(x.cpu(), i, layers) for x in (g, b, s, was))
            used = np.zeros(len(g), bool)
            for f, m, o, blk, total in zip(first, n, off, c.blk_off, c.rows):
                span = slice(blk, blk + (total + 63) // 64)
                ref = oracle.packed_rows(b[span].numpy(), s[span].numpy(), values)[f:f + m]
                h = HALF[c.t] if dtype == "bf16" else 0.0
                assert np.all(np.abs(wide(g[o:o + m]) - ref) <= (U + h + U * h) * np.abs(ref))
                used[o:o + m] = True
            assert torch.equal(g[~used], was[~used])


def test_pack_again_after_unpack_keeps_the_integers():
    """fp32 rows that come from blocks pack to the same blocks: their largest value is the scale's 127."""
    c = Cache("f32", [190], [0], 2, 128, seed=4)
    k, v, pk, pv, ks, vs = (x.cuda() for x in pack(c))
    off, n, blk = ints([1], torch.int64), ints([190]), ints([1], torch.int64)
    pc.cure_kv_unpack(pk, pv, ks, vs, blk, ints([0]), k, v, off, n)
    pk2, pv2, ks2, vs2 = (torch.full_like(x, c.fill if x.dtype == torch.int8 else -1.0) for x in (pk, pv, ks, vs))
    pc.cure_kv_pack(k, v, off, n, pk2, pv2, ks2, vs2, blk, ints([0]))
    assert torch.equal(pk, pk2) and torch.equal(pv, pv2)


def test_layers_apart():
    """Layers that are slices of larger buffers."""
    c = Cache("bf16", [100, 30], [64, 0], 2, 64, layers=2)
    g = {n: c.gpu(n) for n in ("k", "v", "pk", "pv", "ks", "vs")}
    wide_ = {n: torch.stack([torch.stack([x[i], torch.zeros_like(x[i])]) for i in range(2)]) for n, x in g.items()}
    part = {n: x[:, 0] for n, x in wide_.items()}
    st = pc.cure_kv_pack(part["k"], part["v"], ints(c.kv_off, torch.int64), ints(c.rows), part["pk"], part["pv"], part["ks"],
                         part["vs"], ints(c.blk_off, torch.int64), ints(c.done))
    assert st.tolist() == [0, 0]
    check_pack(c, [part[n].cpu() for n in ("k", "v", "pk", "pv", "ks", "vs")])
    assert not any(bool(x[:, 1].any()) for x in wide_.values())


def test_sequences_that_cannot_be_are_left_alone():
    c = Cache("bf16", [10, 64, 5, 5, 5, 5, 70, 5], [0] * 8, 1, 64)
    bad_rows = [10, -1, 5, 5, 5, 5, 71, 5]
    bad_off = list(c.kv_off)
    bad_off[2], bad_off[7] = c.end - 4, -1
    bad_blk = list(c.blk_off)
    bad_blk[3], bad_blk[4] = c.blocks, -1
    done = [0, 0, 0, 0, 0, 32, 0, 0]
    g = [c.gpu(n) for n in ("k", "v", "pk", "pv", "ks", "vs")]
    st = pc.cure_kv_pack(g[0], g[1], ints(bad_off, torch.int64), ints(bad_rows), *g[2:], ints(bad_blk, torch.int64), ints(done), n_max=70)
    bad = pc.cure.CURE_ERR_BAD_TREE
    assert st.tolist() == [0] + [bad] * 7
    c.rows, c.done, c.kv_off, c.blk_off = [10], [0], c.kv_off[:1], c.blk_off[:1]
    check_pack(c, [x.cpu() for x in g])
    back = [torch.zeros(20, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    st = pc.cure_kv_unpack(*g[2:], ints([1, 1, 1, 1, c.blocks], torch.int64), ints([0, -1, 60, 0, 0]), *back,
                           ints([0, 0, 0, 15, 0], torch.int64), ints([3, 3, 11, 6, 1]), n_max=10)
    assert st.tolist() == [0, bad, bad, bad, bad]
    assert not bool(back[0][3:].any())


def test_captured():
    """A captured pack replayed on other rows and sizes."""
    c = Cache("bf16", [128, 128], [0, 64], 2, 128)
    g = [c.gpu(n) for n in ("k", "v", "pk", "pv", "ks", "vs")]
    fresh = [x.clone() for x in g]
    off, blk, done, n = ints(c.kv_off, torch.int64), ints(c.blk_off, torch.int64), ints(c.done), ints([128, 128])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        st = pc.cure_kv_pack(g[0], g[1], off, n, *g[2:], blk, done, n_max=128)
    for rows in ([128, 128], [64, 17], [0, 65]):
        for x, f in zip(g, fresh):
            x.copy_(f)
        n.copy_(ints(rows))
        graph.replay()
        torch.cuda.synchronize()
        c.rows = rows
        assert st.tolist() == [0, 0]
        check_pack(c, [x.cpu() for x in g])
