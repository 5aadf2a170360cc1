"""Attention weights of many query vectors, at sizes that take the wide products (from 2^29 on, heads x scores x vectors of a
stream), against the definition and with the bounds of tests/test_gpu_attention_mass.py."""
import numpy as np
import pytest

import test_gpu_attention_mass as T

pytestmark = pytest.mark.gpu


def made(seed, L, S, H, G, dim, cap, P, R, length, n=None, ordered=False):
    own = (n or R) * G
    assert own >= 128 and L * H * (S * cap * own + P * S * own) * own >= 1 << 29
    return T.make(seed, L, S, H, G, dim, cap, P, R, length, ordered=ordered)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("H,G,cap,P,R,length", [
    (4, 4, 257, 0, 257, 257),                                    # all chunk
    (2, 4, 700, 0, 300, 700),
    (2, 3, 830, 0, 333, 829),                                    # vectors and keys that end inside a tile
    (1, 8, 530, 70, 129, 530),                                   # a segment in front
    (1, 1, 6000, 0, 300, 5999),
    (8, 1, 4000, 0, 130, 3990),                                  # half a tile of vectors
])
def test_a_prompt_scores_what_stands_before_it(gpu, dim, H, G, cap, P, R, length):
    T.check(gpu, made(cap + dim, 1, 1, H, G, dim, cap, P, R, [length], ordered=True), None, 0.5)


@pytest.mark.parametrize("dim", [64, 128])
def test_slots_in_any_order(gpu, dim):
    T.check(gpu, made(31, 1, 2, 2, 3, dim, 700, 0, 250, [700, 400]), None, 0.9)


def test_many_listed_rows_of_several_streams(gpu):
    """Rows that do not count, with NaN where they stand, a stream without rows, and a shared segment."""
    rng = np.random.default_rng(32)
    R, S = 70, 3
    lists = [sorted(rng.permutation(R)[:64].tolist()), sorted(rng.permutation(R)[:40].tolist()) + [-1] * 24, [-1] * 64]
    for dim in (64, 128):
        c = made(33 + dim, 4, S, 2, 4, dim, 300, 130, R, [300, 150, 20], n=64)
        listed = [s * R + r for s in range(S) for r in lists[s] if r >= 0]
        c["q"][:, [m for m in range(S * R) if m not in listed]] = 0x7FC0
        T.check(gpu, c, lists, 0.9)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("L,S,H,G,cap,P,R", [(2, 2, 2, 2, 700, 140, 150), (1, 1, 2, 4, 500, 0, 190)])
def test_rows_and_keys_that_are_not_finite(gpu, dim, L, S, H, G, cap, P, R):
    made(0, L, S, H, G, dim, cap, P, R, [cap] * S)
    T.test_rows_and_keys_that_are_not_finite(gpu, dim, L, S, H, G, cap, P, R)


def test_scores_that_grow_along_the_keys(gpu):
    for order in (1, -1):
        c = made(34, 1, 1, 1, 4, 64, 900, 0, 210, [900], ordered=True)
        ramp = np.linspace(-40.0, 40.0, 900)[::order]
        c["k"] = T.bf16(np.broadcast_to(ramp[:, None] / 8.0, (900, 64))[None, None, None])
        c["q"] = T.bf16(np.ones((1, 210, 4, 64)) * 8.0)
        T.check(gpu, c, None)


@pytest.mark.parametrize("q_std", [0.01, 40.0])
def test_sharp_and_flat_weights(gpu, q_std):
    c = made(35, 1, 1, 2, 4, 128, 600, 90, 170, [600])
    c["q"] = T.bf16(q_std * np.random.default_rng(36).standard_normal(c["q"].shape))
    T.check(gpu, c, None, 0.7)
