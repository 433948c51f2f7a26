"""Shared by the tests of the operators around the verify step (rotary append, prompt
attention, shared-prefix attention): inputs on the GPU, and error bounds.

Bounds, from the arithmetic (u = 2^-24, the rounding of one fp32 operation; h = half a
step of the output's type: 2^-8 bf16, 2^-24 fp32):

rotary append. A norm's factor sums d squares, (d + 4) u, halved by the root, and takes
four more operations; a rotation multiplies by cosines and sines that are off by 6e-7 (2 ulp
of the function, 1e-7 of the reduced angle) and adds, 3 u; the store rounds once:
    |err| <= (|a| + |b|) m (6e-7 + (d / 2 + 12) u) + h |y|.

attention. A score is a sum of d products, off by e = (d + 4) u scale sum |q k| with what the
scaling costs; a probability by 2 e relative to the row's sum, 4 u for the exponential and, for
bf16 inputs, 2^-8 where it is rounded (numerator and denominator alike); sums over n keys
add (n + 8) u; with mass = sum p |v|:
    |err o|   <= (2^-8 [bf16] + 2 e + (n + 16) u) (mass + |o|) (1 + 2^-7) + h |o|
    |err lse| <= 2^-8 (1 + 2^-8) [bf16] + e + (n + 16) u + 4 u |lse|.
"""

import numpy as np
import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def normal(seed, *shape, dtype=torch.float32, std=1.0):
    """A CPU tensor of the type's values."""
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype)


def wide(t):
    return t.detach().cpu().double().numpy()


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def score_error(q, k, scale):
    """e above for one row q [d] and keys [n, d]."""
    return (q.shape[0] + 4) * U * scale * np.max(np.abs(k) @ np.abs(q))


def check_rows(o, lse, ref, rows, seen, q, k, scale, bf16):
    """rows: list of index tuples of query rows; seen[row] = indexes of its keys. Every head of
    every row of o and lse within the bounds."""
    ref_o, ref_lse, mass = ref
    half = HALF[o.dtype]
    o, lse = wide(o), None if lse is None else wide(lse)
    hq, hkv = ref_o.shape[-2], k.shape[1]
    p = 2.0 ** -8 if bf16 else 0.0
    for r in rows:
        n = len(seen[r])
        for h in range(hq):
            e = score_error(q[r][h], k[seen[r], h // (hq // hkv)], scale)
            tol = (p + 2 * e + (n + 16) * U) * (mass[r][h] + np.abs(ref_o[r][h])) * (1 + 2.0 ** -7)
            tol = tol + half * (np.abs(ref_o[r][h]) + tol)
            err = np.abs(o[r][h] - ref_o[r][h])
            assert np.all(err <= tol), (r, h, float(np.max(err - tol)), float(np.max(err)))
            if lse is not None:
                t = p * (1 + 2.0 ** -8) + e + (n + 16) * U + 4 * U * abs(ref_lse[r][h])
                assert abs(lse[r][h] - ref_lse[r][h]) <= t, (r, h, lse[r][h], ref_lse[r][h])


def random_parents(rng, n):
    """A topologically ordered tree with chains, bushes and several roots."""
    return [int(rng.integers(-1, m)) if m and rng.random() < 0.4 else m - 1 for m in range(n)]
