"""Pins of oracle/beams.py: closed forms, invariances, brute force on small inputs."""
import itertools
import math

import numpy as np
import pytest

from oracle import beams as O
from workloads.generate import f32_to_bf16_bits


def bits(rng, *shape, scale=1.0):
    return f32_to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32)).view(np.int16)


def test_quantise():
    x = np.array([[2.0, -1.0, 0.5, 0.0, 1.0 / 127]])
    code, scale = O.quantise(x)
    assert code.tolist() == [[127, -64, 32, 0, 0]]                       # halves to the even one: 63.5 to 64, 0.5 to 0
    assert scale == np.float32(2.0) / np.float32(127)
    rng = np.random.default_rng(0)
    x = O.bf16(bits(rng, 64, 128))
    code, scale = O.quantise(x)
    # (half a scale, and up to 127 scales that are rounded to fp32: 254 * 2^-24 of that half more)
    assert np.abs(code).max() == 127 and np.all(np.abs(code * np.float64(scale) - x) <= 0.5 * scale * (1 + 254 * 2.0 ** -24))
    assert O.quantise(np.zeros((2, 2)))[1] == 0 and math.isnan(O.quantise(np.array([1.0, math.inf]))[1])


def sequence(c, l, s, h):
    return O.tokens_of(c, l, s, h)


def grown(seed, L=2, S=3, H=2, D=64, pages=24, columns=9, R=70, calls=3):
    rng = np.random.default_rng(seed)
    c, said = O.empty_cache(L, S, H, D, pages, columns), [[] for _ in range(S)]
    for _ in range(calls):
        k, v = bits(rng, L, S * R, H, D), bits(rng, L, S * R, H, D)
        rows = [list(rng.permutation(R)[:rng.integers(1, R)]) + [-1] for _ in range(S)]
        rows = [r + [-1] * (R - len(r)) for r in rows]
        c, entered = O.append(c, k, v, R, rows)
        for s in range(S):
            said[s] += [(O.bf16(k[:, s * R + r]), O.bf16(v[:, s * R + r])) for r in rows[s][:entered[s]]]
    return c, said


@pytest.mark.parametrize("seed", range(3))
def test_what_enters_is_what_is_held(seed):
    c, said = grown(seed)
    assert np.array_equal(c["refs"], np.bincount(c["table"][c["table"] >= 0], minlength=24)) and c["refs"].max() <= 1 and c["len"].max() > 64
    for s in range(3):
        assert c["len"][s] == len(said[s])
        for l, h in itertools.product(range(2), range(2)):
            where, k, v = sequence(c, l, s, h)
            assert np.array_equal(where, np.arange(len(said[s])))
            for got, i in ((k, 0), (v, 1)):
                want = np.array([x[i][l, h] for x in said[s]])
                off = np.abs(got - want)
                full = len(want) // 64 * 64
                assert np.all(off[full:] == 0) and np.all(off[:full] <= 0.5 * np.max(np.abs(want[:full]), initial=0) / 127 * (1 + 255 * 2.0 ** -24))


def test_a_stream_enters_whole_or_not_at_all():
    rng = np.random.default_rng(1)
    c = O.empty_cache(1, 3, 1, 64, 3, 2)
    new = [bits(rng, 1, 3 * 130, 1, 64) for _ in range(2)]
    c, n = O.append(c, *new, 130)
    assert n == [130, 0, 0] and c["refs"].tolist() == [1, 1, 0]           # the second finds one page of two, and so does nobody behind it
    c, n = O.append(c, *new, 130, [[0] * 64] + [[0] * 5 + [-1]] * 2)
    assert n == [0, 5, 5]                                                 # the first has no columns left
    c, n = O.append(c, *new, 130, [[0] * 60, [0] * 59, [0] * 59])
    assert n == [60, 59, 0] and c["refs"].tolist() == [1, 1, 1]


@pytest.mark.parametrize("seed", range(4))
def test_streams_that_become_others(seed):
    c, _ = grown(seed)
    rng = np.random.default_rng(100 + seed)
    source = rng.integers(-1, 4, 3)
    d = O.reorder(c, source)
    for s in range(3):
        if 0 <= source[s] < 3:
            for a, b in zip(sequence(d, 1, s, 0), sequence(c, 1, int(source[s]), 0)):
                assert np.array_equal(a, b)
        else:
            assert d["len"][s] == 0
    assert sorted(d["slot"]) == [0, 1, 2]
    e = O.reorder(d, None, window=50, sink=70)
    for s in range(3):
        where = sequence(e, 0, s, 1)[0]
        n = int(e["len"][s])
        assert {t for t in range(n) if t > n - 50 or t < 70} <= set(where.tolist()) <= set(range(n))
        gone = set(range(n)) - set(where.tolist())
        assert all(t <= n - 50 and t >= 70 // 64 * 64 + 64 for t in gone)
    small, used = O.copy(d, O.empty_cache(2, 2, 2, 64, 24, 9), [2, 0])
    assert used == np.count_nonzero(small["refs"]) and np.all(small["refs"][:used] > 0)
    for i, s in enumerate([2, 0]):
        for a, b in zip(sequence(small, 0, i, 1), sequence(d, 0, s, 1)):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("window,sink", [(0, 0), (1, 0), (40, 3), (100, 70), (9, 500)])
def test_attention_on_a_dense_mask(window, sink):
    c, _ = grown(7)
    rng = np.random.default_rng(8)
    R, H, G, D = 5, 2, 2, 64
    parent = np.array([-1, 0, 0, 2, 7] + [-1, 0, 1, 2, 3] + [-1, -1, 1, 1, 3])
    q, k, v = bits(rng, 3 * R, H * G, D), bits(rng, 3 * R, H, D), bits(rng, 3 * R, H, D)
    got, _ = O.attention(c, 1, q, k, v, parent, R, 0.125, window, sink)
    for s in range(3):
        n = int(c["len"][s])
        ups = np.zeros((R, R), bool)                                     # transitive closure by powers
        for r in range(R):
            up = parent[s * R + r]
            if 0 <= up < r:
                ups[r, up] = True
        reach = np.linalg.matrix_power(np.eye(R) + ups, R) > 0
        at = n + reach.sum(1) - 1
        for h in range(H):
            _, kk, vv = sequence(c, 1, s, h)
            kk, vv = (np.concatenate([a, O.bf16(b[s * R:(s + 1) * R, h])]) for a, b in ((kk, k), (vv, v)))
            pos = np.concatenate([np.arange(n), at])
            see = np.concatenate([np.ones((R, n), bool), reach], 1)
            if window:
                see &= (pos > at[:, None] - window) | (pos < sink)
            for g in range(G):
                x = 0.125 * O.bf16(q[s * R:(s + 1) * R, h * G + g]) @ kk.T
                e = np.exp(x - x.max()) * see
                assert np.allclose(got[s * R:(s + 1) * R, h * G + g], (e @ vv) / e.sum(1, keepdims=True), rtol=1e-9, atol=1e-9)


@pytest.mark.parametrize("power", [0.0, 0.7])
def test_selection_by_brute_force(power):
    rng = np.random.default_rng(3)
    W, V = 3, 6
    z = rng.standard_normal((2 * W, V))
    z[0, 2] = -math.inf
    score, length, done = rng.standard_normal(2 * W) - 3, np.array([4, 4, 2, 4, 4, 4]), np.array([0, 0, 1, 0, 0, 0])
    out, _ = O.beam_select(z, score, length, done, W, eos=1, pad=9, power=power)
    for g in range(2):
        every = []
        for b in range(g * W, g * W + W):
            if done[b]:
                every.append((score[b] / length[b] ** power, b, 9, score[b]))
            else:
                logp = z[b] - math.log(np.exp(z[b]).sum())
                every += [((score[b] + logp[v]) / 5 ** power, b, v, score[b] + logp[v]) for v in range(V)]
        every.sort(key=lambda x: -x[0])
        for i in range(W):
            at = g * W + i
            assert (out["source"][at], out["token"][at]) == every[i][1:3] and np.isclose(out["score"][at], every[i][3])
            assert out["length"][at] == (2 if done[every[i][1]] else 5) and out["finished"][at] == (done[every[i][1]] or every[i][2] == 1)


def test_selection_without_candidates():
    z = np.array([[0.0, 1.0], [math.nan, 0.0], [-math.inf, -math.inf], [math.inf, 0.0], [5.0, 5.0]])
    out, _ = O.beam_select(z, np.array([0.0, 0.0, 0.0, 0.0, -math.inf]), np.zeros(5), np.zeros(5), 5, pad=7)
    assert out["source"].tolist() == [0, 0, 2, 3, 4] and out["token"].tolist() == [1, 0, 7, 7, 7]
    assert np.all(out["score"][2:] == -math.inf) and out["length"].tolist() == [1, 1, 0, 0, 0]


def test_one_beam_is_greedy_and_equals_go_by_their_order():
    z = np.array([[1.0, 3.0, 3.0, 2.0]])
    assert O.beam_select(z, np.zeros(1), np.zeros(1), np.zeros(1), 1)[0]["token"].tolist() == [1]
    z = np.zeros((2, 4))
    out, _ = O.beam_select(z, np.zeros(2), np.zeros(2), np.zeros(2), 2)
    assert out["source"].tolist() == [0, 0] and out["token"].tolist() == [0, 1]
