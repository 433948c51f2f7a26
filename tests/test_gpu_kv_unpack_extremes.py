"""Blocks whose largest value is near the type's: rows that come back are scale * c, rounded to fp32 (2^-24)
and for bf16 once more (2^-8). fp32's largest value alone has a scale that 127 times passes it; the float below,
2^-23 of it less, is taken: |err| <= (2^-23 + 2^-24 + 2^-47) |scale c|."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_00531_amd as pc
from prompt_util import DTYPES, HALF, U, ints, normal, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("share", [1.0, -1.0, 0.996, -0.98, 0.5])
def test_the_largest_values_come_back(dtype, d, share):
    t, n, hkv = DTYPES[dtype], 100, 2
    top = torch.tensor(torch.finfo(t).max * share, dtype=torch.float64).to(t)
    k, v = (normal(i, n, hkv, d, dtype=t, std=1e37).clamp(-1e38, 1e38) for i in range(2))
    k[::3] = v[::5] = 0
    k[3, 0, 7] = v[70, 1, 9] = top                          # a block each of one head
    blocks = [torch.zeros(2, hkv, 64 * d, dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(2, hkv, device="cuda") for _ in range(2)]
    off, rows = ints([0], torch.int64), ints([n])
    assert pc.cure_kv_pack(k.cuda(), v.cuda(), off, rows, *blocks, *scales, off, ints([0])).tolist() == [0]
    back = [torch.full((n, hkv, d), 5.0, dtype=t, device="cuda") for _ in range(2)]
    assert pc.cure_kv_unpack(*blocks, *scales, off, ints([0]), *back, off, rows).tolist() == [0]
    for x, y, b, s, values in ((k, back[0], blocks[0], scales[0], False), (v, back[1], blocks[1], scales[1], True)):
        c, scale = oracle.pack_rows(wide(x))
        assert np.array_equal(b.cpu().numpy(), oracle.to_bytes(c, values)) and np.array_equal(s.cpu().numpy(), scale)
        ref = oracle.packed_rows(b.cpu().numpy(), scale, values)[:n]
        u = U + 2.0 ** -23 if dtype == "f32" and abs(share) == 1.0 else U
        h = HALF[t] if dtype == "bf16" else 0.0
        assert np.all(np.abs(wide(y) - ref) <= (u + h + (u + h) * U) * np.abs(ref))
        assert bool((y[x.cuda() == 0] == 0).all()) and bool(y.isfinite().all())
