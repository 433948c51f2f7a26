"""Workspace of cure_prefix_attn, on the CPU: a row has a part for the prefix and parts for its own
rows, of which the estimate asks for several only while the chip lacks workgroups."""

import ctypes
import os

import numpy as np
import pytest

import paper_2608_00531_amd as pc
from paper_2608_00531_amd import build as pbuild


def slots(prefix, ctx, nodes, hq=32, hkv=8, d=128, kv_split=0):
    """Parts per row that the workspace has room for."""
    if not os.path.exists(pbuild.LIB_PATH):
        pbuild.build_library()
    arrays = [np.array(x, np.int32) for x in (ctx, nodes)]
    c, n = (a.ctypes.data_as(ctypes.c_void_p) for a in arrays)
    size = pc.lib().cure_prefix_attn_workspace_size(len(ctx), hq, hkv, d, max(nodes), prefix, c, n, kv_split)
    return size // (len(ctx) * max(nodes) * hq * (d + 1) * 4)


# 32768 own tokens behind a prefix of any length: two tiles of 48 nodes on 8 kv-heads are 256 workgroups by
# themselves for 16 sequences, and four times as many for 64. A prefix of 8192 has two splits or so.
@pytest.mark.parametrize("prefix", [1, 128, 200, 255, 257, 512, 8192])
@pytest.mark.parametrize("batch,nodes,own,most", [(16, 48, 32768, 8), (64, 48, 30000, 6), (256, 48, 4000, 4), (64, 256, 30000, 4),
                                                  (32, 48, 131072, 12)])
def test_own_rows_of_many_sequences_have_few_parts(prefix, batch, nodes, own, most):
    assert 2 <= slots(prefix, [own] * batch, [nodes] * batch) <= most + (4 if prefix > 512 else 0)


@pytest.mark.parametrize("kv_split", [1, 2, 32])
def test_the_callers_splits_of_the_prefix_leave_own_rows_alone(kv_split):
    assert kv_split < slots(8192, [32768] * 16, [48] * 16, kv_split=kv_split) <= kv_split + 7


def test_few_workgroups_still_share_long_contexts():
    """One token on 131072 of its own: 8 workgroups without splits, 256 with 32."""
    assert 33 <= slots(100, [131072], [1]) <= 129
    assert 129 <= slots(100, [131072], [1], hq=8, hkv=1) <= 257
    assert slots(100, [2 ** 30], [1], hq=8, hkv=1) <= 257


def test_short_own_contexts_have_one_part():
    """No more parts than one for each 256 keys."""
    assert slots(200, [0, 5, 250], [4, 1, 3]) == 2
    assert slots(200, [0], [1]) == 2
    assert slots(200, [260], [1]) <= 3


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("batch,n_max,hq,hkv", [(1024, 256, 512, 8), (1024, 256, 128, 32), (1024, 256, 256, 32), (1024, 256, 512, 512),
                                               (1024, 1, 131072, 1024), (2, 256, 262144, 256), (1024, 128, 1024, 1024)])
@pytest.mark.parametrize("own", [0, 1000, 100000, 1 << 20, 1 << 29])
@pytest.mark.parametrize("prefix", [200, 100000, 1 << 29])
def test_no_plan_asks_for_more_than_a_launch_holds(dtype, batch, n_max, hq, hkv, own, prefix):
    """batch * n_max * hq up to 2^27, one node each and one long context: the splits stop where the launch would pass 2^32
    threads, and the call where its workspace (of one byte here) ends."""
    assert batch * n_max * hq <= 2 ** 27
    ctx, nodes = np.zeros(batch, np.int32), np.ones(batch, np.int32)
    ctx[0] = own
    c, n = (a.ctypes.data_as(ctypes.c_void_p) for a in (ctx, nodes))
    st = pc.lib().cure_prefix_attn(4096, 4096, 4096, 4096, None, dtype, 1, batch, hq, hkv, 64, 0.1, 0, prefix, 1, 1, 1, 1, n_max,
                                   c, n, 0, None, 4096, 1, None)
    assert st == pc.CURE_ERR_WORKSPACE
