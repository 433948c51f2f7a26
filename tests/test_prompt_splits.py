"""The caller's kv_split holds for prompts of any length: the workspace has its parts, and the result is
that of one split."""

import pytest
import torch

import paper_2608_00531_amd as pc
from prompt_util import ints, normal
from test_prompt_abi import L, host, prompt  # noqa: F401


@pytest.mark.parametrize("n", [65535, 65536, 70000, 200000])
def test_long_prompts_split_as_asked(L, n):  # noqa: F811
    a, c = host(n), host(0)
    size = lambda split: L.cure_prompt_attn_workspace_size(1, n, 1, 1, 64, a[1], c[1], split)  # noqa: E731
    assert size(1) == 0 and size(2) >= n * 2 * 65 * 4 and size(3) > size(2)
    assert prompt(L, n=(n,), ctx=(0,), rows=n, hq=1, hkv=1, kv_split=2) == pc.CURE_ERR_WORKSPACE


def test_automatic_splits_of_long_prompts(L):  # noqa: F811
    a, c = host(70000), host(0)
    assert L.cure_prompt_attn_workspace_size(1, 70000, 1, 1, 64, a[1], c[1], 0) == 0


@pytest.mark.gpu
def test_long_prompts_in_parts():
    """More tokens than one merge launch holds. Equal scores and one-hot values: element t % d of the
    output, times the number of keys, is how many of the visible tokens t counted, exactly what splits and
    their join must give; around the launches' edges and at the ends."""
    n, d = 131100, 64
    v = torch.zeros(n, 1, d, dtype=torch.bfloat16, device="cuda")
    v[torch.arange(n, device="cuda"), 0, torch.arange(n, device="cuda") % d] = 1
    q, k = torch.zeros(n, 1, d, dtype=torch.bfloat16, device="cuda"), normal(1, n, 1, d, dtype=torch.bfloat16).cuda()
    zero = ints([0], torch.int64)
    o, lse = pc.cure_prompt_attn(q, k, v, zero, ints([n]), zero, ints([0]), [n], [0], 1.0, out_dtype=torch.float32, kv_split=2)
    keys = torch.arange(1, n + 1, dtype=torch.float64, device="cuda")
    got = o[:, 0].double() * keys[:, None]
    # A part's sums are whole numbers below 2^24, exact; its division, the join's two weights (logarithms of up
    # to 12 with 2^-24 relative, their differences' exponentials) and its division are off by less than
    # 64 * 2^-24 of what is counted, which is keys / d.
    seen = torch.cumsum(v[:, 0].double(), 0)
    assert float(((got - seen).abs() - 64 * 2.0 ** -24 * (seen + 1)).max()) <= 0
    assert float((lse[:, 0].double() - keys.log()).abs().max()) <= 64 * 2.0 ** -24
