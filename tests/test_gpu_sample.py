"""cure_sample against the 64-bit definition: tokens and counts have to be its, log probabilities are
fp32 roundings of 64-bit values: |err| <= 2^-24 |x| + 2^-24 (a share near one)."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_00531_amd as pc
from prompt_util import U, ints, normal, wide

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
NONE = pc.CURE_NO_TOKEN


def check(x, u, settings, n_rows=None, got=None):
    """x [batch, rows, vocab] on the CPU, settings: a (T, k, p, m) per sequence."""
    batch, rows, _ = x.shape
    t, k, p, m = ([s[i] for s in settings] for i in range(4))
    f = lambda v: torch.tensor(v, dtype=F32, device="cuda")  # noqa: E731
    if got is None:
        got = pc.cure_sample(x.cuda(), u.cuda(), f(t), ints(k), f(p), f(m), n_rows=None if n_rows is None else ints(n_rows))
        torch.cuda.synchronize()
    got = {key: v.cpu().numpy() for key, v in got.items()}
    for b in range(batch):
        for r in range(rows):
            ref = oracle.sample(wide(x[b, r]), float(u[b, r]), *settings[b]) if n_rows is None or r < n_rows[b] else None
            if ref is None:
                assert (got["token"][b, r], got["logprob"][b, r], got["kept"][b, r]) == (NONE, -np.inf, 0), (b, r)
                continue
            assert (got["token"][b, r], got["kept"][b, r]) == (ref[0], ref[2]), (b, r, settings[b], ref)
            assert abs(got["logprob"][b, r] - ref[1]) <= U * abs(ref[1]) + U


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 0.95, 0.0), (1.3, 0, 1.0, 0.05),
            (0.8, 7, 0.5, 0.2), (2.0, 1, 1.0, 0.0), (0.05, 0, 0.99, 0.0), (1.0, 10 ** 6, 0.0, 1.0), (50.0, 0, 0.3, 0.9)]


def logits(seed, *shape, dtype=BF16, std=2.0):
    x = normal(seed, *shape, std=std)
    at = torch.randint(shape[-1], (*shape[:-1], min(30, shape[-1])), generator=torch.Generator().manual_seed(seed))
    x.scatter_(-1, at, 4 + 10 * torch.rand(at.shape, generator=torch.Generator().manual_seed(seed + 1)) ** 2)
    return x.to(dtype)


def uniform(seed, *shape):
    return torch.rand(shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [1, 2, 3, 63, 64, 65, 1000, 1025, 4097, 50257])
def test_filters(dtype, vocab):
    n = len(SETTINGS)
    check(logits(vocab, n, 3, vocab, dtype=dtype), uniform(vocab, n, 3), SETTINGS)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_large_vocabulary(dtype):
    check(logits(5, 4, 2, 262144, dtype=dtype), uniform(5, 4, 2), [SETTINGS[i] for i in (0, 1, 3, 4)])
    check(logits(6, 1, 1, 2 ** 20, dtype=dtype), uniform(6, 1, 1), [(1.0, 1000, 0.9, 0.0)])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ties(dtype):
    """Few values, each many times: ties are in index order, filters cut within them."""
    g = torch.Generator().manual_seed(2)
    x = torch.randint(-2, 3, (len(SETTINGS), 4, 3001), generator=g).to(dtype)
    check(x, uniform(3, len(SETTINGS), 4), SETTINGS)
    x = torch.full((3, 5, 2048), -1.5, dtype=dtype)             # a constant row: shares of 1 / 2048, exactly
    u = torch.tensor([0.0, 0.25, 0.5, 0.75, 2047.5 / 2048]).expand(3, 5).contiguous()
    check(x, u, [(1.0, 0, 1.0, 0.0), (0.5, 1000, 0.5, 0.0), (1.0, 0, 0.25, 1.0)])
    x = torch.tensor([0.0, -0.0, 0.0, -0.0]).to(dtype).expand(1, 8, 4).contiguous()    # both zeros are one value
    check(x, torch.arange(8).view(1, 8) / 8, [(1.0, 3, 1.0, 0.0)])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masked_entries(dtype):
    """-inf, the type's lowest value, rows that leave little or nothing, NaN and +inf."""
    low = torch.finfo(dtype).min
    x = logits(8, 8, 4, 777, dtype=dtype)
    x[0, :, 5:] = float("-inf")
    x[1, :, 5:] = low
    x[2] = float("-inf")
    x[3, 0], x[3, 1, 17], x[3, 2, 700], x[3, 3, 0] = low, float("nan"), float("inf"), float("-inf")
    x[4, :, 1:] = float("-inf")
    x[5] = x[5] * 2.0 ** 60
    x[6] = x[6] * 2.0 ** -60
    x[7] = -1e30
    for s in ((1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 3, 1.0, 0.1)):
        check(x, uniform(9, 8, 4), [s] * 8)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_settings_out_of_range(dtype):
    nan = float("nan")
    odd = [(nan, 0, 1.0, 0.0), (-1.0, 0, 1.0, 0.0), (float("inf"), 0, 1.0, 0.0), (1.0, 0, nan, 0.0), (1.0, 0, 1.0, nan),
           (1.0, -5, 2.0, -1.0), (1.0, 0, -1.0, 7.0), (1e-30, 0, 1.0, 0.0), (1e30, 3, 1.0, 0.0)]
    u = torch.tensor([0.0, 1.0, -0.5, nan, 0.999]).expand(len(odd), 5).contiguous()
    check(logits(10, len(odd), 5, 300, dtype=dtype), u, odd)


def test_numbers_at_the_ends():
    """u = 0, the largest below 1, 1 and more: the first and the last kept entry, under every filter."""
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 5.0]).expand(len(SETTINGS), 4).contiguous()
    for dtype in (BF16, F32):
        check(logits(12, len(SETTINGS), 4, 5000, dtype=dtype), u, SETTINGS)


def test_rows_left_out_strides_and_defaults():
    x = logits(14, 3, 6, 500)
    u = uniform(15, 3, 6)
    check(x, u, [(1.0, 20, 0.9, 0.0)] * 3, n_rows=[6, 0, 2])
    check(x, u, [(1.0, 20, 0.9, 0.0)] * 3, n_rows=[7, -1, 1])
    wide_ = torch.zeros(3, 6, 517, dtype=BF16, device="cuda")
    for shift in (0, 1, 3):
        part = wide_[:, :, shift:shift + 500]
        part.copy_(x)
        check(x, u, [(1.0, 0, 1.0, 0.0)] * 3, got=pc.cure_sample(part, u.cuda()))
    flat = pc.cure_sample(x.view(18, 500).cuda(), u.view(18).cuda())
    assert flat["token"].shape == (1, 18)
    check(x.view(1, 18, 500), u.view(1, 18), [(1.0, 0, 1.0, 0.0)], got=flat)


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_many_rows(rows):
    """The same rows give the same tokens however many there are beside them."""
    x = logits(20, 1, 5, 32000)
    u = uniform(21, 1, 5)
    few = pc.cure_sample(x.cuda(), u.cuda(), top_p=torch.tensor([0.9], device="cuda"))
    check(x, u, [(1.0, 0, 0.9, 0.0)], got=few)
    many = pc.cure_sample(x.repeat(1, rows, 1).cuda(), u.repeat(1, rows).cuda(), top_p=torch.tensor([0.9], device="cuda"))
    for key in few:
        assert torch.equal(many[key], few[key].repeat(1, rows))


def test_captured_and_on_two_streams():
    x, u = logits(30, 2, 3, 20000), uniform(31, 2, 3)
    gx, gu = x.cuda(), u.cuda()
    k = ints([40, 0])
    eager = pc.cure_sample(gx, gu, top_k=k)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = pc.cure_sample(gx, gu, top_k=k)
    for seed in (31, 33, 34):
        gu.copy_(uniform(seed, 2, 3))
        for _ in range(2):
            graph.replay()
            other = torch.cuda.Stream()
            other.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(other):
                beside = pc.cure_sample(gx, gu, top_k=k)
            torch.cuda.synchronize()
            for key in out:
                assert torch.equal(out[key], beside[key])
    gu.copy_(u)
    graph.replay()
    torch.cuda.synchronize()
    for key in out:
        assert torch.equal(out[key], eager[key])


def test_drawn_tokens_are_accepted_as_targets():
    """Every node's drawn token is what the acceptance walk compares with, and CURE_NO_TOKEN matches none."""
    x = torch.full((1, 3, 50), float("-inf"))
    x[0, 0, 7], x[0, 1, 9] = 0.0, 0.0                           # node 0 -> 7, node 1 -> 9, node 2 -> nothing
    got = pc.cure_sample(x.cuda(), torch.full((1, 3), 0.5, device="cuda"))
    assert got["token"].tolist() == [[7, 9, NONE]]
    i = lambda v: ints([v])  # noqa: E731
    walk = pc.cure_accept(i([-1, 0, 1]), i([5, 7, 9]), got["token"], ints([5]), ints([3]), 3)
    assert walk["acc_len"].tolist() == [3] and walk["bonus"].tolist() == [NONE]
