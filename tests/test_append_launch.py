"""The size of cure_rope_append's launch: rows beyond those that there are have no workgroups, and a launch
whose threads would pass 32 bits is refused."""

import pytest
import torch

import paper_2608_00531_amd as pc
from prompt_util import ints, normal
from test_prompt_abi import L, U, append  # noqa: F401


def test_a_launch_of_too_many_threads_is_refused(L):  # noqa: F811
    """Four rows to a workgroup of 256 threads: 2^24 workgroups have 2^32 threads."""
    for n_max in (2 ** 26 - 3, 2 ** 26, 2 ** 31 - 1):
        assert append(L, n_max=n_max, rows=2 ** 40, row_off=1) == U
        assert append(L, n_max=n_max, rows=2 ** 40) == U


@pytest.mark.gpu
@pytest.mark.parametrize("n_max", [None, 40, 41, 2 ** 26, 2 ** 31 - 1])
def test_any_bound_on_packed_rows_gives_the_same(n_max):
    """Packed rows and a bound that no sequence reaches, up to the type's largest."""
    rows, row_off, kv_off = [40, 0, 3, 17], [0, 40, 41, 45], [0, 50, 60, 70]
    q, k, v = (normal(s, 62, h, 64, dtype=torch.bfloat16).cuda() for s, h in ((1, 4), (2, 2), (3, 2)))
    freq = pc.cure_rope_frequencies(64)[0].cuda()

    def call(bound):
        kc, vc = (torch.full((90, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        out = torch.full_like(q, 9.0)
        _, status = pc.cure_rope_append(q, k, v, kc, vc, ints(kv_off, torch.int64), ints([1, 2, 3, 0]), ints(rows), freq,
                                        row_off=ints(row_off, torch.int64), n_max=bound, out=out)
        assert status.tolist() == [0] * 4
        return out, kc, vc
    for x, y in zip(call(n_max), call(40)):
        assert torch.equal(x, y)
