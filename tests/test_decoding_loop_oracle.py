"""Pins of the plain definitions that the decoding loop's GPU tests compare against (no GPU)."""
import math

import numpy as np
import pytest

from oracle import decoding_loop as D


def test_frequencies_at_the_ends_of_each_scaling():
    f = lambda i, s, **kw: D.rope_frequency(i, 64, s, 10000.0, **kw)   # noqa: E731
    assert f(0, "plain") == 1.0 and math.isclose(f(16, "plain"), 0.01)
    assert math.isclose(f(16, "linear", factor=4.0), 0.0025)
    assert math.isclose(f(0, "base", factor=8.0), 1.0)                          # the fastest pair keeps its frequency,
    assert math.isclose(f(31, "base", factor=8.0), f(31, "plain") / 8.0)        # the slowest one is stretched by the factor
    kw = dict(factor=8.0, low=1.0, high=4.0, context=8192.0)
    assert f(0, "turns", **kw) == 1.0 and math.isclose(f(31, "turns", **kw), f(31, "plain") / 8.0)
    assert f(24, "plain") / 8 < f(24, "turns", **kw) < f(24, "plain")           # 1.3 turns: in between


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_relative_positions(interleaved):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((2, 1, 24))
    at = lambda p: D.rope(x, D.rope_angles([p[0], p[1]], 16, "plain", 100.0), 16, interleaved)   # noqa: E731
    y, z = at((5, 9)), at((1005, 1009))
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    assert np.allclose((y[0] * y[1])[..., :16].sum(), (z[0] * z[1])[..., :16].sum())
    assert np.array_equal(y[..., 16:], x[..., 16:])
    back = D.rope(y, D.rope_angles([5, 9], 16, "plain", 100.0), 16, interleaved, inverse=True)
    assert np.allclose(back, x)


def test_rank_order():
    nan, inf = math.nan, math.inf
    mass = [0.0, -0.0, 2.0, nan, inf, 2.0, -inf, 1.0]
    pos = [10, 11, 12, 13, 14, 15, 16, 99]
    # protected by being recent: slot 7; by the sink: none; then inf, 2 (lower slot first), the zeros in slot order, -inf, NaN
    assert D.ranked(mass, pos, 8, 100, 0, 1) == [7, 4, 2, 5, 0, 1, 6, 3]
    assert D.ranked(mass, pos, 4, 100, 14, 0) == [0, 1, 2, 3]


def test_append_fills_room_first_and_then_the_lightest():
    c = {"k": np.zeros((1, 1, 1, 4, 1)), "v": np.zeros((1, 1, 1, 4, 1)), "mass": np.array([[[[5.0, 1.0, 3.0, 0.0]]]]),
         "slot_pos": np.array([[[[0, 1, 2, 0]]]]), "len": np.array([3]), "next_pos": np.array([3])}
    new = np.arange(1.0, 6.0).reshape(1, 5, 1, 1)
    d = D.append(c, new, -new, 5, [[0, 2, 4, -1, 1]], 4, 0, 0)
    assert d["k"].ravel().tolist() == [0.0, 3.0, 5.0, 1.0]                       # slots 1 and 2 gave way, in the order of the slots
    assert d["slot_pos"].ravel().tolist() == [0, 4, 5, 3] and d["mass"].ravel().tolist() == [5.0, 0.0, 0.0, 0.0]
    assert d["len"][0] == 4 and d["next_pos"][0] == 6


def test_masses_sum_to_the_rows_that_see_something():
    rng = np.random.default_rng(1)
    L, S, H, cap, dim, R, G = 1, 2, 2, 9, 8, 4, 3
    k, q = rng.standard_normal((L, S, H, cap, dim)), rng.standard_normal((L, S * R, H * G, dim))
    pos = np.broadcast_to(np.arange(cap), (L, S, H, cap))
    m, p = D.attention_mass(k, np.zeros((L, S, H, cap)), pos, [9, 0], [9, 0], q, R, [[0, 2, 3], [1]], 0.3, 1.0)
    assert np.allclose(m[:, 0].sum(-1), 3 * G) and np.all(m[:, 1] == 0) and p is None
    kp = rng.standard_normal((L, H, 5, dim))
    m, p = D.attention_mass(k, np.zeros((L, S, H, cap)), pos, [9, 0], [9, 0], q, R, [[0, 2, 3], [1]], 0.3, 1.0, kp, np.zeros((L, H, 5)))
    assert np.allclose(m.sum((1, 3)) + p.sum(-1), 4 * G)
    # one key: the whole weight
    m, _ = D.attention_mass(k, np.ones((L, S, H, cap)), pos, [9, 1], [1, 1], q, R, [[1], [0]], 0.3, 0.5)
    assert np.allclose(m[0, :, :, 0], 0.5 + G) and np.allclose(m[0, 0, :, 1:], 0.5) and np.allclose(m[0, 1, :, 1:], 1.0)


def test_rules_by_hand():
    z = np.array([[2.0, -2.0, 1.0, 0.5], [2.0, -2.0, 1.0, 0.5]])
    out, counts = D.logit_rules(z, 1, 2, 2, [-1, 0], [[3, 0]], new=[[1, 1, -1, 9]], counts=np.array([[0, 0, 1, 0]]), repetition=[2.0],
                                frequency=[0.25], presence=[0.5], bias=np.array([[0.0, 0.0, 0.0, 4.0]]), bias_row=[0],
                                masks=np.array([[0b1011]], np.uint32), mask_row=[-1, 0])
    assert counts.tolist() == [[0, 2, 1, 0]]
    assert out[0].tolist() == [2.0, -4.0 - 0.5 - 0.5, 0.5 - 0.25 - 0.5, 4.5]
    assert out[1].tolist() == [1.0 - 0.25 - 0.5, -5.0, -math.inf, 4.5]           # row 1 carries token 0 itself
