"""Sampling at the edges of its bins and lists: magnitudes that have no bin of their own, values held by
more entries than a list takes, rows that end inside a vector."""

import pytest
import torch

import paper_2608_00531_amd as pc
from test_gpu_sample import BF16, F32, SETTINGS, check, logits, uniform

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_magnitudes(dtype):
    """Zeros, tiny and huge values beside and instead of ordinary ones."""
    ordinary = logits(1, 1, 900, dtype=dtype)[0]
    rows = []
    for odd in ([0.0, -0.0], [2.0 ** -30, 2.0 ** -31, -2.0 ** -31, 2.0 ** -126, -2.0 ** -133, 0.0], [1016.0, 1020.0, -1020.0, -1024.0],
                [1024.0, 1032.0], [-2000.0, -65504.0, -1e30, torch.finfo(dtype).min], [3e38, 2.9e38], [2.0 ** -29, -2.0 ** -30]):
        x = ordinary.clone()
        x[torch.randperm(900, generator=torch.Generator().manual_seed(len(rows)))[:len(odd)]] = torch.tensor(odd).to(dtype)
        rows.append(x)
        rows.append(torch.tensor(odd).to(dtype).repeat(150)[:900 // len(odd) * len(odd)])
    rows.append(ordinary * 0 - 5000 + 8 * (torch.arange(900) % 7).to(dtype))      # all of it below every bin
    rows.append(ordinary * 2.0 ** -31)
    width = max(len(x) for x in rows)
    x = torch.full((len(rows), 6, width), float("-inf"), dtype=dtype)
    for i, row in enumerate(rows):
        x[i, :, :len(row)] = row
    u = torch.tensor([0.0, 0.1, 0.35, 0.6, 0.9, 1 - 2.0 ** -24]).expand(len(rows), 6).contiguous()
    for s in ((1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (20.0, 0, 1.0, 0.9)):
        check(x, u, [s] * len(rows))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("many", [1023, 1025, 2047, 2049, 5000])
def test_values_of_many_entries(dtype, many):
    """A value that `many` entries hold, the drawn one among them, with and without others above it."""
    x = torch.full((3, 5, 9001), -3.0)
    at = torch.randperm(9001, generator=torch.Generator().manual_seed(many))
    x[:, :, at[:many]] = 1.0
    x[1, :, at[many:many + 3]] = torch.tensor([2.0, 3.0, 1.5])
    x[2] = x[2].sort(descending=True).values
    u = torch.tensor([0.0, 0.2, 0.5, 0.8, 0.97]).expand(3, 5).contiguous()
    for s in ((1.0, 0, 1.0, 0.0), (1.0, many - 1, 1.0, 0.0), (0.5, 0, 0.5, 0.0), (1.0, 0, 0.9, 0.1)):
        check(x.to(dtype), u, [s] * 3)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [7, 8, 9, 4095, 4096, 4100, 16383, 16384, 16385, 16393, 20480, 32767, 32776, 36865])
def test_rows_that_end_inside_a_vector(dtype, vocab):
    """The row's last entries are its likeliest, and each counts once."""
    x = logits(3, 2, 4, vocab, dtype=dtype)
    x[0, :, -5:] = torch.tensor([9.0, 8.0, 9.0, 7.0, 9.5]).to(dtype)
    x[1, 0] = 1.0
    check(x, uniform(vocab, 2, 4), [(1.0, 0, 1.0, 0.0)] * 2)
    check(x, uniform(vocab, 2, 4), [SETTINGS[1], (1.0, vocab // 2, 0.9, 0.0)])
    # Behind the row lie values that would win.
    wide = torch.full((2, 4, vocab + 11), 60.0, dtype=dtype, device="cuda")
    wide[:, :, :vocab] = x.cuda()
    u = uniform(vocab, 2, 4)
    check(x, u, [(1.0, 0, 1.0, 0.0)] * 2, got=pc.cure_sample(wide[:, :, :vocab], u.cuda()))
