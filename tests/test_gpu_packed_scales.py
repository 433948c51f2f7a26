"""Attention over blocks whose value scales lie anywhere in float32, alone, beside each other and beside open
rows, in every order: a block's tokens count in the softmax by their scores alone. Bounds of packed_bounds.py."""

import pytest
import torch

from packed_bounds import Bounded

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
