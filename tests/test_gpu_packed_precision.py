"""What the header states of the packed attention's roundings, with fp32 outputs, whose own rounding hides
nothing: probabilities to 2^-11 over packed blocks and to 2^-17 over open rows. Bounds of packed_bounds.py, which
test_packed_bounds.py shows to tell coarser roundings apart."""

import pytest
import torch

from packed_bounds import Bounded

pytestmark = pytest.mark.gpu

FORMS = {
    "few": dict(dtype="bf16", rows=[7, 2, 1], hq=8, hkv=2, d=128), "few 64": dict(dtype="bf16", rows=[7, 2, 1], hq=8, hkv=2, d=64),
    "many": dict(dtype="bf16", rows=[40] * 4, hq=256, hkv=64, d=128), "many 64": dict(dtype="bf16", rows=[40] * 4, hq=256, hkv=64, d=64),
    "f32": dict(dtype="f32", rows=[7, 2, 1], hq=8, hkv=2, d=128), "f32 64": dict(dtype="f32", rows=[7, 2, 1], hq=8, hkv=2, d=64),
}


@pytest.mark.parametrize("packed,ctx", [([1, 2, 3, 5], 0), ([64, 700, 33, 130], 0), ([0] * 4, 0), ([0] * 4, 3), ([0] * 4, 61), ([300, 20, 64, 0], 45)])
@pytest.mark.parametrize("std", [0.5, 4.0])
@pytest.mark.parametrize("form", FORMS)
def test_roundings(form, packed, ctx, std):
    many = dict(every=7, heads=range(0, 256, 29)) if form.startswith("many") else {}
    at = FORMS[form]
    n = len(at["rows"])
    for kind, split in (("tree", 0), ("padded", 1), ("padded", 2)):
        c = Bounded(packed=packed[:n], ctx=[ctx] * n, form=kind, std=std, seed=n, **at)
        c.check(c.call(out_dtype=torch.float32, kv_split=split), **many)
