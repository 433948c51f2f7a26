"""Device lengths past what a sequence may have, in caches that would hold them by their sizes: the sequence is
reported and neither read nor written, the others are as they were."""

import ctypes

import pytest
import torch

import paper_2608_00531_amd as pc
from packed_util import Case
from prompt_util import ints

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1 - 4096


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("packed,ctx", [(0, MOST - 2), (0, 2 ** 31 - 1), (2 ** 31 - 1, 0), (MOST, 0), (2 ** 30, 2 ** 30), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_more_tokens_than_supported(dtype, packed, ctx):
    """3 rows behind them. Through the C entry point, whose `blocks` and `cache_rows` say that all of it is there."""
    c = Case(dtype, [3, 3], [130, 64], [20, 1], 4, 2, 64, form="padded")
    o, lse, _ = c.call()
    a = c.args
    out, out_lse, status = torch.full_like(o, 7.0), torch.full_like(lse, 7.0), ints([5, 5])
    lens, ctxs = ints([130, packed]), ints([20, ctx])
    host = lambda v: (ctypes.c_int32 * 2)(*v)  # noqa: E731
    n, hp, hc = host([3, 3]), host([130, 64]), host([20, 1])
    p = lambda t: t.data_ptr()  # noqa: E731
    code = 1 if dtype == "bf16" else 0
    st = pc.lib().cure_packed_attn(p(a["q"]), p(a["pk"]), p(a["pv"]), p(a["k_scale"]), p(a["v_scale"]), 1 << 40, p(a["k"]), p(a["v"]), 1 << 40,
                                   p(out), p(out_lse), code, code, 2, 6, 3, 4, 2, 64, c.scale, None, p(a["n_rows"]), p(a["blk_off"]),
                                   p(lens), p(a["kv_off"]), p(ctxs), None, ctypes.cast(n, ctypes.c_void_p), ctypes.cast(hp, ctypes.c_void_p),
                                   ctypes.cast(hc, ctypes.c_void_p), 1, p(status), None, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == 0 and status.tolist() == [0, pc.CURE_ERR_BAD_TREE]
    assert torch.equal(out[0], o[0]) and torch.equal(out_lse[0], lse[0]) and bool((out[1] == 7.0).all()) and bool((out_lse[1] == 7.0).all())
