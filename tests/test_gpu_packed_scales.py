"""Attention over blocks whose value scales lie anywhere in float32, alone, beside each other and beside open
rows, in every order: a block's tokens count in the softmax by their scores alone. Bounds of packed_bounds.py."""

import math

import pytest
import torch

import paper_2608_00531_amd as pc
from packed_bounds import Bounded
from prompt_util import ints

pytestmark = pytest.mark.gpu

# Powers of two of the blocks' scales, in turn; None: a block of zeros.
PATTERNS = {
    "smallest": [-118], "below float32's normal ones": [-138], "largest": [118], "small before ordinary": [-116] * 3 + [0] * 100,
    "ordinary before small": [0] * 3 + [-116] * 100, "in turn": [-100, 100], "large before small": [60] + [-80] * 100,
    "small before large": [-80] * 5 + [100] * 100, "zeros beside large": [None, 110], "zeros first": [None, None, -120],
    "zeros": [None], "just near": [-23, 0, 37], "just apart": [-26, 0, 41],
    "small and alike": [-50, -70, -40],
}

FORMS = {
    "few": dict(dtype="bf16", rows=[5, 1], hq=8, hkv=2, d=128), "few 64": dict(dtype="bf16", rows=[7, 3], hq=4, hkv=1, d=64),
    "many": dict(dtype="bf16", rows=[40] * 4, hq=256, hkv=64, d=128), "many 64": dict(dtype="bf16", rows=[33] * 4, hq=256, hkv=64, d=64),
    "f32": dict(dtype="f32", rows=[5, 9], hq=8, hkv=2, d=128), "f32 64": dict(dtype="f32", rows=[12, 1], hq=4, hkv=1, d=64),
}


def case(form, pattern, ctx, seed=0, tokens=700):
    at = dict(FORMS[form])
    rows = at.pop("rows")
    c = Bounded(rows=rows, packed=[tokens, 130, 64, tokens][:len(rows)], ctx=[ctx] * len(rows), form="padded" if seed % 2 else "tree",
                seed=seed, **at)
    for b in range(len(rows)):
        for i in range((c.packed[b] + 63) // 64):
            power = pattern[i % len(pattern)]
            at = c.blk_off[b] + i
            if power is None:
                c.vs[at], c.pv[at] = 0.0, 0
            else:
                c.vs[at] = torch.ldexp(c.vs[at], torch.tensor(power))
    return c


@pytest.mark.parametrize("name", PATTERNS)
@pytest.mark.parametrize("form", FORMS)
def test_scales(name, form):
    many = dict(every=9, heads=range(0, 256, 37)) if form.startswith("many") else {}
    for seed, ctx, split in ((0, 0, 0), (1, 40, 1), (2, 3, 3)):
        c = case(form, PATTERNS[name], ctx, seed)
        c.check(c.call(kv_split=split, out_dtype=torch.float32), **many)
    c.check(c.call(), **many)


FAR = {"few": FORMS["few"], "f32": FORMS["f32"], "many": dict(dtype="bf16", rows=[64] * 4, hq=128, hkv=32, d=128),
       "many 64": dict(dtype="bf16", rows=[64] * 4, hq=128, hkv=32, d=64)}


@pytest.mark.parametrize("powers", [[90, -90], [-90, 90], [0] * 66 + [-100], [0] * 66 + [100]])
@pytest.mark.parametrize("form", FAR)
def test_the_far_block_decides(form, powers):
    """Blocks apart of which the small one's tokens have nearly all of the weight, or all share it evenly; some only
    behind the 64 blocks whose scales a wave of many rows loads at once."""
    many = dict(every=31, heads=range(0, 128, 51)) if form.startswith("many") else {}
    at = dict(FAR[form])
    n = len(at["rows"])
    c = Bounded(packed=[64 * (len(powers) + 1) - 5] * n, ctx=[0] * n, form="padded", **at)
    blocks = torch.tensor([c.blk_off[b] + i for b in range(n) for i in range(len(powers) + 1)])
    power = torch.tensor([powers[i % len(powers)] for _ in range(n) for i in range(len(powers) + 1)])
    c.vs[blocks] = torch.ldexp(c.vs[blocks], power[:, None])
    small = blocks[power == min(powers)]
    c.ks[:] *= 0.0
    c.check(c.call(out_dtype=torch.float32, kv_split=1), **many)
    c.ks[small] = 0.05
    c.check(c.call(out_dtype=torch.float32, kv_split=1), **many)


@pytest.mark.parametrize("form", FORMS)
def test_new_rows_of_large_values(form):
    """Open and new rows up to 2^79 beside ordinary blocks and beside ones as large."""
    many = dict(every=11, heads=range(0, 256, 43)) if form.startswith("many") else {}
    for powers in ([0], [73], [-60]):
        c = case(form, powers, 21, 1)
        c.v = (c.v.float().clamp(-3.9, 3.9) * 2.0 ** 77).to(c.t)
        c.check(c.call(out_dtype=torch.float32), **many)


@pytest.mark.parametrize("others", [0, 60, -60, -110])
@pytest.mark.parametrize("form", FORMS)
def test_scales_of_zero_with_any_bytes(form, others):
    """Where a largest value's 127th part is below float32's smallest number the scale is 0 and the bytes are not:
    keys and values are zeros, and such tokens count."""
    many = dict(every=13, heads=range(0, 256, 51)) if form.startswith("many") else {}
    c = case(form, [others], 7, 1)
    for b in range(len(c.rows)):
        c.vs[c.blk_off[b]:c.blk_off[b] + 6:2] = 0.0
        c.ks[c.blk_off[b]:c.blk_off[b] + 6:3] = 0.0
    c.check(c.call(out_dtype=torch.float32), **many)
    c.vs[:] = 0.0
    c.v[:] = 0.0
    o, lse, status = c.call(out=torch.full((*c.shape, c.hq, c.d), 3.0, dtype=c.t, device="cuda"))
    c.check((o, lse, status), **many)
    for b, n in enumerate(c.rows):
        assert not bool(o[b, :n].any())


def test_packed_values_below_a_scale():
    """fp32 rows of values up to 2^-143 pack to such blocks; beside ordinary ones they are nothing."""
    n, hkv, d = 128, 1, 64
    zero = ints([0], torch.int64)
    k, v = torch.zeros(n + 1, hkv, d, device="cuda"), torch.ones(n + 1, hkv, d, device="cuda")
    v[:64], v[n] = 2.0 ** -145, 0.0
    blocks = [torch.zeros(2, hkv, 64 * d, dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(2, hkv, device="cuda") for _ in range(2)]
    pc.cure_kv_pack(k, v, zero, ints([n]), *blocks, *scales, zero, ints([0]))
    assert scales[1][0, 0] == 0 and bool((blocks[1][0] == 127).all())
    q = torch.ones(1, 1, 1, d, device="cuda")
    one = ints([1])
    o, lse, _ = pc.cure_packed_attn(q, *blocks, *scales, zero, ints([n]), k[n:], v[n:], zero, ints([0]), one, [n], [0], [1], 0.125)
    # 64 of 129 equal weights on values of 127 (1 / 127): three roundings of 2^-24, and of sums.
    assert bool(((o - 64 / 129).abs() <= (129 + 16) * 2.0 ** -24).all()) and abs(lse.item() - math.log(129)) <= (129 + 16) * 2.0 ** -24 * 5
    v[64:] = 0.0
    pc.cure_kv_pack(k, v, zero, ints([n]), *blocks, *scales, zero, ints([0]))
    o, _, _ = pc.cure_packed_attn(q, *blocks, *scales, zero, ints([n]), k[n:], v[n:], zero, ints([0]), one, [n], [0], [1], 0.125)
    assert not bool(o.any())
