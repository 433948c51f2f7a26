"""Workspace sizes that pass 64 bits, on the CPU: the calls ask for more than there can be instead of
wrapping round to a few bytes."""

import pytest

import paper_2608_00531_amd as pc
from test_prompt_abi import L, host, prefix, prompt  # noqa: F401


@pytest.mark.parametrize("rows", [2 ** 38, 2 ** 40, 2 ** 46, 2 ** 62])
def test_prompt_workspaces_do_not_wrap(L, rows):  # noqa: F811
    """Rows, heads and splits whose product's powers of two leave nothing in 64 bits."""
    kw = dict(n=(2,), ctx=(2 ** 30,), rows=rows, hq=2 ** 18, hkv=2 ** 17, kv_split=2 ** 15)
    assert prompt(L, workspace=4096, ws_bytes=2 ** 30, **kw) == pc.CURE_ERR_WORKSPACE
    n, c = host(2), host(2 ** 30)
    assert L.cure_prompt_attn_workspace_size(1, rows, 2 ** 18, 2 ** 17, 64, n[1], c[1], 2 ** 15) >= 2 * 2 ** 18 * 2 ** 14 * 65 * 4


def test_prefix_workspaces_do_not_wrap(L):  # noqa: F811
    """1024 trees of 256 nodes (of which one each exists), 2^12 heads, 2^15 splits of the prefix: 2^53 bytes."""
    kw = dict(nodes=(1,) * 1024, ctx=(0,) * 1024, batch=1024, n_max=256, hq=2 ** 12, hkv=2 ** 11, prefix_len=2 ** 30, kv_split=2 ** 15)
    assert prefix(L, workspace=4096, ws_bytes=2 ** 52, **kw) in (pc.CURE_ERR_WORKSPACE, pc.CURE_ERR_UNSUPPORTED)
