"""Pins of the packed cache's and of sampling's oracle: hand-worked values and brute force, no GPU."""

import itertools
import math

import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("d", [64, 128])
def test_places_are_a_permutation(d):
    t, j = np.meshgrid(np.arange(64), np.arange(d), indexing="ij")
    for place in (oracle.key_place, oracle.value_place):
        assert sorted(place(t, j, d).ravel().tolist()) == list(range(64 * d))
    # By hand, d = 64: token 33 is in the second half (2 pieces of 1 KB on), column 50 in its
    # second piece, upper 16 columns, third of them.
    assert oracle.key_place(33, 50, 64) == (2 + 1) * 1024 + 512 + 1 * 16 + 2
    # Token 45 = 32 + 8 + 4 + 1: half 1, a = 1, h = 1, c = 1; column 3.
    assert oracle.value_place(45, 3, 64) == 2 * 1024 + 512 + 3 * 16 + 1 * 4 + 1


def test_pack_hand_worked():
    x = np.zeros((66, 2, 64))
    x[0, 0, :4] = [2.54, -1.27, 0.03, 0.01]              # steps of 0.02: 127, -63.5, 1.5, 0.5
    x[65, 1, 7] = -8.0
    c, scale = oracle.pack_rows(x)
    assert c.shape == (2, 2, 64, 64) and scale.dtype == np.float32
    assert c[0, 0, 0, 0] == 127 and c[0, 0, 0, 1] in (-63, -64) and scale[0, 0] == np.float32(2.54) / np.float32(127)
    assert not c[0, 1].any() and scale[0, 1] == 0 and scale[1, 0] == 0
    assert c[1, 1, 1, 7] == -127 and np.count_nonzero(c[1, 1]) == 1
    # Exact ties go to even: a = 254, so that 127 x / a = x / 2.
    x = np.zeros((1, 1, 64))
    x[0, 0, :6] = [254, 1, 3, 5, -1, -3]
    assert oracle.pack_rows(x)[0][0, 0, 0, :6].tolist() == [127, 0, 2, 2, 0, -2]


def test_bytes_and_back():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((130, 3, 64))
    c, scale = oracle.pack_rows(x)
    for values in (False, True):
        b = oracle.to_bytes(c, values)
        assert np.array_equal(oracle.from_bytes(b, values), c)
        rows = oracle.packed_rows(b, scale, values)
        step = np.repeat(scale, 64, axis=0)[:130, :, None]
        assert np.all(np.abs(rows[:130] - x) <= step * (0.5 + 1e-6)) and not rows[130:].any()


def by_definition(x, u, t, k, p, m):
    """Every prefix of the order, tried one after the other."""
    order = sorted((i for i in range(len(x)) if x[i] > -math.inf), key=lambda i: (-x[i], i))
    w = [math.exp((x[i] - x[order[0]]) / t) for i in order]
    n = len(order) if k <= 0 else min(k, len(order))
    total = math.fsum(w[:n])
    if p < 1:
        n = next(j for j in range(1, n + 1) if math.fsum(w[:j]) >= p * total or j == n)
    if m > 0:
        n = max(1, sum(v >= m for v in w[:n]))
    total = math.fsum(w[:n])
    j = next((j for j in range(n) if math.fsum(w[:j + 1]) > u * total), n - 1)
    return order[j], math.log(w[j] / total), n


def test_sample_against_the_definition():
    rng = np.random.default_rng(1)
    for t, k, p, m in itertools.product((0.5, 1.0, 2.0), (0, 1, 3, 99), (0.0, 0.3, 0.875, 1.0), (0.0, 0.1, 1.0)):
        for _ in range(5):
            x = rng.choice([-math.inf, -2.0, -0.5, 0.0, 1.0, 1.25, 3.0], size=7)
            if not np.isfinite(x).any():
                continue
            u = float(np.float32(rng.random()))
            t32, p32, m32 = (float(np.float32(v)) for v in (t, p, m))
            assert oracle.sample(x, u, t, k, p, m)[::2] == by_definition(x, u, t32, k, p32, m32)[::2]


def test_sample_hand_worked():
    x = [0.0, math.log(4.0), math.log(2.0), math.log(4.0), math.log(1.0)]    # weights 1 4 2 4 1, in order 1 3 2 0 4
    got = [oracle.sample(x, u)[0] for u in (0.0, 0.33, 0.34, 0.66, 0.67, 0.83, 0.84, 0.91, 0.92, 1.0)]
    assert got == [1, 1, 3, 3, 2, 2, 0, 0, 4, 4]
    assert oracle.sample(x, 0.5, top_k=1) == (1, 0.0, 1)
    assert oracle.sample(x, 0.99, top_p=0.5)[::2] == (3, 2)      # 4 of 12 are not enough, 8 are
    assert oracle.sample(x, 0.99, min_p=0.5)[::2] == (2, 3)
    assert oracle.sample(x, 0.99, temperature=0)[0] == 1
    assert oracle.sample([-70.0, 0.0, -64.0], 1.0)[::2] == (2, 2)  # no weight past 64 T
    assert oracle.sample([-math.inf], 0.5) is None and oracle.sample([math.nan, 0.0], 0.5) is None
    assert oracle.sample([0.0], math.nan) is None and oracle.sample([0.0], 0.5, temperature=-1.0) is None


def test_shares_are_the_probabilities():
    """Evenly spread numbers draw each token as often as its probability says."""
    x = np.array([0.3, -1.0, 2.0, 0.3, 1.1])
    p = np.exp(x) / np.exp(x).sum()
    n = 20000
    hits = np.bincount([oracle.sample(x, (i + 0.5) / n)[0] for i in range(n)], minlength=5)
    assert np.all(np.abs(hits / n - p) <= 1.0 / n)
