"""cure_prompt_attn at the sizes by which its launch is decided: rows around a tile of 32 (fp32) and 128 (bf16), keys
around the steps that the waves of a workgroup take together, and contexts around the first that is split."""

import pytest
import torch

from test_gpu_prompt_attn import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,group", [([31], 1), ([32, 33], 1), ([8, 9], 4), ([127, 128], 1), ([129], 1), ([32, 33], 4)])
@pytest.mark.parametrize("keys", [127, 128, 129, 160, 512, 513])
def test_tiles_and_steps_at_their_edges(dtype, rows, group, keys):
    c = Case(dtype, rows, [max(0, keys - n) for n in rows], 2 * group, 2, 64)
    c.check(*c.run(), only=lambda n: [0, n // 2, n - 2, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("keys,kv_split", [(255, 0), (256, 0), (511, 0), (512, 0), (513, 0), (1024, 0), (385, 3), (640, 5)])
def test_one_split_and_several(dtype, keys, kv_split):
    """Few rows, so that the plan splits as soon as it may, beside one that ends in the first split."""
    c = Case(dtype, [1, 3, 1], [keys - 1, keys - 3, 0], 4, 1, 128)
    c.check(*c.run(kv_split=kv_split))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rows,ctx,hq,hkv", [(64, [700, 1, 33], [0, 900, 400], 8, 2), (128, [300, 300], [0, 33], 32, 8), (128, [1, 1, 1], [5000, 1, 700], 8, 1)])
def test_calls_repeat_their_bits(dtype, d, rows, ctx, hq, hkv):
    c = Case(dtype, rows, ctx, hq, hkv, d)
    o, lse = c.run()
    for _ in range(3):
        again, again_lse = c.run()
        for r, n in zip(c.row_off, rows):
            assert torch.equal(o[r:r + n], again[r:r + n]) and torch.equal(lse[r:r + n], again_lse[r:r + n])
