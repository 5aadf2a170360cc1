"""Attention weights of many query vectors, at sizes that take the wide products (by heads x scores x vectors of a stream: from 2^29
on with 128 features, from 2^32 on with 64), against the definition and with the bounds of tests/test_gpu_attention_mass.py."""
import numpy as np
import pytest

import test_gpu_attention_mass as T

pytestmark = pytest.mark.gpu


def made(seed, L, S, H, G, dim, cap, P, R, length, n=None, ordered=False):
    own = (n or R) * G
    assert own >= 128 and L * H * (S * cap * own + P * S * own) * own >= 1 << (29 if dim == 128 else 32)
    return T.make(seed, L, S, H, G, dim, cap, P, R, length, ordered=ordered)


@pytest.mark.parametrize("dim,H,G,cap,P,R,length", [
    (128, 4, 4, 257, 0, 257, 257), (64, 4, 8, 257, 0, 257, 257),         # all chunk
    (128, 2, 4, 700, 0, 300, 700), (64, 2, 8, 700, 0, 300, 700),
    (128, 2, 3, 830, 0, 333, 829), (64, 2, 8, 530, 0, 263, 529),         # vectors and keys that end inside a tile
    (128, 1, 8, 530, 70, 129, 530), (64, 2, 8, 470, 70, 257, 470),       # a segment in front
    (128, 1, 1, 6000, 0, 300, 5999), (64, 1, 8, 1100, 0, 255, 1099),
    (128, 8, 1, 4000, 0, 130, 3990),                                     # half a tile of vectors
])
def test_a_prompt_scores_what_stands_before_it(gpu, dim, H, G, cap, P, R, length):
    T.check(gpu, made(cap + dim, 1, 1, H, G, dim, cap, P, R, [length], ordered=True), None, 0.5)


@pytest.mark.parametrize("dim,G,cap,R", [(128, 3, 700, 250), (64, 8, 500, 190)])
def test_slots_in_any_order(gpu, dim, G, cap, R):
    T.check(gpu, made(31, 1, 2, 2, G, dim, cap, 0, R, [cap, cap - 250]), None, 0.9)


@pytest.mark.parametrize("dim,L,H,G", [(128, 4, 2, 4), (64, 4, 4, 8)])
def test_many_listed_rows_of_several_streams(gpu, dim, L, H, G):
    """Rows that do not count, with NaN where they stand, a stream without rows, and a shared segment."""
    rng = np.random.default_rng(32)
    R, S = 70, 3
    lists = [sorted(rng.permutation(R)[:64].tolist()), sorted(rng.permutation(R)[:40].tolist()) + [-1] * 24, [-1] * 64]
    c = made(33 + dim, L, S, H, G, dim, 300, 130, R, [300, 150, 20], n=64)
    listed = [s * R + r for s in range(S) for r in lists[s] if r >= 0]
    c["q"][:, [m for m in range(S * R) if m not in listed]] = 0x7FC0
    T.check(gpu, c, lists, 0.9)


@pytest.mark.parametrize("dim,L,S,H,G,cap,P,R", [(128, 2, 2, 2, 2, 700, 140, 150), (128, 1, 1, 2, 4, 500, 0, 190),
                                                 (64, 1, 2, 2, 8, 500, 140, 170), (64, 1, 1, 4, 8, 500, 0, 190)])
def test_rows_and_keys_that_are_not_finite(gpu, dim, L, S, H, G, cap, P, R):
    made(0, L, S, H, G, dim, cap, P, R, [cap] * S)
    T.test_rows_and_keys_that_are_not_finite(gpu, dim, L, S, H, G, cap, P, R)


@pytest.mark.parametrize("dim,G,R", [(128, 4, 210), (64, 8, 280)])
def test_scores_that_grow_along_the_keys(gpu, dim, G, R):
    for order in (1, -1):
        c = made(34, 1, 1, 1, G, dim, 900, 0, R, [900], ordered=True)
        ramp = np.linspace(-40.0, 40.0, 900)[::order]
        c["k"] = T.bf16(np.broadcast_to(ramp[:, None] / 8.0, (900, dim))[None, None, None])
        c["q"] = T.bf16(np.ones((1, R, G, dim)) * 8.0)
        T.check(gpu, c, None)


@pytest.mark.parametrize("q_std", [0.01, 40.0])
def test_sharp_and_flat_weights(gpu, q_std):
    c = made(35, 1, 1, 2, 4, 128, 600, 90, 170, [600])
    c["q"] = T.bf16(q_std * np.random.default_rng(36).standard_normal(c["q"].shape))
    T.check(gpu, c, None, 0.7)
