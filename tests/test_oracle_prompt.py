"""Pins of the prompt and rotary oracle: values worked by hand."""

import math

import numpy as np
import pytest

import oracle


def test_rotation_by_hand():
    """One head of 4 columns, position 3, frequencies pi/6 and pi/3: the pairs turn by a quarter and a half."""
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    f = [math.pi / 6, math.pi / 3]
    q, k, v = oracle.rope_append(x, x, x, [3], f)
    assert q[0, 0] == pytest.approx([-3, -2, 1, -4]) and np.array_equal(q, k) and np.array_equal(v, x)
    q, _, _ = oracle.rope_append(x, x, x, [3], f, interleaved=True, mscale=2.0)
    assert q[0, 0] == pytest.approx([-4, 2, -6, -8])
    q, _, _ = oracle.rope_append(x, x, x, [3], f[:1])
    assert q[0, 0] == pytest.approx([-2, 1, 3, 4])


def test_norm_by_hand():
    x = np.array([[[3.0, 4.0]]])                            # mean square 12.5
    q, k, _ = oracle.rope_append(x, x, x, [0], [1.0], q_weight=[1.0, 2.0], eps=0.0)
    assert q[0, 0] == pytest.approx([3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]) and k[0, 0].tolist() == [3.0, 4.0]


def test_tree_positions():
    assert oracle.tree_positions([-1, 0, 1, 0, -1], 5, 10).tolist() == [10, 11, 12, 11, 10]


def test_relative_positions():
    """Scores depend on the distance alone: rotating query and key by the same shift changes nothing."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((1, 1, 8))
    y = rng.standard_normal((1, 1, 8))
    f = [1.0, 0.1, 0.01, 0.001]
    at = lambda p, z: oracle.rope_append(z, z, z, [p], f)[0][0, 0]  # noqa: E731
    assert at(7, x) @ at(3, y) == pytest.approx(at(1004, x) @ at(1000, y))


def test_prompt_by_hand():
    """Keys of zero: every token averages the values up to its own, log-sum-exp log n; a context row first."""
    k = np.zeros((5, 1, 2))
    v = np.arange(5.0)[:, None, None] * np.ones((1, 1, 2))
    o, lse, mass = oracle.prompt_attention(np.ones((4, 2, 2)), k, v, [1], [3], [1], [1], 1.0)
    assert o[:, 0, 0].tolist() == pytest.approx([0, 1.5, 2, 2.5]) and np.array_equal(o, mass)
    assert lse[1:, 1] == pytest.approx(np.log([2, 3, 4]))


def test_prefix_by_hand_and_against_the_tree_oracle():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((1, 3, 2, 4)), rng.standard_normal((12, 1, 4)), rng.standard_normal((12, 1, 4))
    parent = [[-1, 0, 0]]
    o, lse, _ = oracle.prefix_attention(q, k, v, 0, 5, [5], [2], [3], parent, 0.5)
    # The same cache with the prefix as part of the context.
    ref, ref_lse = oracle.tree_attention(q.astype(np.float32), k.astype(np.float32), v.astype(np.float32), "f32", [0],
                                         [7], [3], parent, 2, 1, 0.5)
    assert np.max(np.abs(o - ref)) < 1e-5 and np.max(np.abs(lse - ref_lse)) < 1e-5
