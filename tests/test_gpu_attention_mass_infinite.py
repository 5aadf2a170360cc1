"""Attention weights of rows and keys with infinite features, in every form of the call.  A row that meets a score of plus infinity makes
NaN of what it sees, whether other rows count or not; a key whose scores are all minus infinity receives nothing, whatever
stands in the places of rows that do not count.  Bounds as in tests/test_gpu_attention_mass.py."""
import numpy as np
import pytest

import test_gpu_attention_mass as T

pytestmark = pytest.mark.gpu

INF, MINUS_INF, ONE, NAN = 0x7F80, 0xFF80, 0x3F80, 0x7FC0


def with_ones(c):
    """Feature 0 is one in all rows and keys."""
    for name in ("q", "k", "k_prefill"):
        if c[name] is not None:
            c[name][..., 0] = ONE
    return c


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("L,S,H,G,cap,P,rows", [
    (1, 1, 2, 1, 1100, 0, [[0]]),                                 # maxima and sums by themselves
    (1, 2, 2, 4, 150, 70, [[1, -1], [-1, 0]]),
    (8, 16, 2, 2, 80, 70, [[0, 1]] + [[-1, -1]] * 15),            # one pass, then the shared segment's masses
    (1, 1, 2, 4, 90, 0, [[0]]),                                   # one pass
    (1, 1, 1, 3, 60, 50, [[0, 1]]),
])
def test_only_rows_of_infinite_scores(gpu, dim, L, S, H, G, cap, P, rows):
    c = with_ones(T.make(41 + dim, L, S, H, G, dim, cap, P, 2, [cap] * S, ordered=True))
    c["q"][:, :, :, 0] = INF
    got, got_p = T.check(gpu, c, rows, 0.9)
    n = sum(r >= 0 for r in rows[0])
    assert np.all(np.isnan(got[:, 0, :, :cap])) and n and (got_p is None or np.all(np.isnan(got_p)))
    assert all(np.all(np.isfinite(got[:, s])) for s in range(1, S))


def test_infinite_scores_in_one_of_two_waves_that_share_keys(gpu):
    """280 vectors of 64 features on 400 slots: two waves take turns with the tiles of 16 vectors."""
    for odd in (0, 1):
        c = with_ones(T.make(43, 1, 1, 1, 4, 64, 400, 0, 70, [400], ordered=True))
        c["q"][:, [r for r in range(70) if r // 4 % 2 == odd], :, 0] = INF
        got, _ = T.check(gpu, c, None, 0.9)
        assert np.all(np.isnan(got[0, 0, 0, :331]))


@pytest.mark.parametrize("dim,L,S,H,G,cap,P,R,n", [
    (64, 1, 2, 2, 4, 90, 0, 3, None), (128, 1, 2, 2, 5, 90, 0, 4, None),          # one pass
    (64, 1, 1, 1, 3, 60, 50, 3, None), (128, 1, 1, 2, 3, 60, 50, 3, None),
    (64, 1, 2, 2, 4, 150, 70, 11, None), (128, 1, 2, 2, 4, 150, 70, 11, None),    # maxima and sums by themselves
    (64, 1, 3, 2, 4, 150, 70, 11, 7), (128, 2, 1, 1, 2, 4500, 0, 4, None),
    (64, 8, 16, 2, 2, 80, 70, 6, 3), (128, 8, 16, 2, 2, 80, 70, 6, 3),            # one pass, then the shared segment's masses
    (64, 1, 1, 1, 4, 400, 0, 70, None),                                           # two waves share keys
    (64, 1, 1, 4, 8, 500, 0, 190, None), (128, 1, 1, 2, 4, 500, 0, 190, None),    # the wide products
    (128, 4, 3, 2, 4, 300, 130, 70, 64), (64, 4, 3, 4, 8, 300, 130, 70, 64),
])
def test_keys_of_minus_infinity_beside_rows_that_do_not_count(gpu, dim, L, S, H, G, cap, P, R, n):
    c = with_ones(T.make(44 + dim, L, S, H, G, dim, cap, P, R, [cap] * S, ordered=True))
    plain = {"k": c["k"].copy(), "k_prefill": None if P == 0 else c["k_prefill"].copy()}
    rows = None
    if n is not None:                                              # lists of all lengths, one of them empty
        rows = [(list(range(R))[R - n:][:k] + [-1] * n)[:n] for k in ([n, n // 2 + 1, 0, 1] * S)[:S]]
        unlisted = [s * R + r for s in range(S) for r in range(R) if r not in rows[s]]
        c["q"][:, unlisted] = NAN
    dead = [1, 17, min(33, cap - R - 1)]                           # seen by every row
    c["k"][:, :, :, dead, 0] = MINUS_INF
    if P:
        c["k_prefill"][:, :, [0, P - 1], 0] = MINUS_INF
    got, got_p = T.check(gpu, c, rows, 0.9)
    assert np.all(np.isfinite(got)) and np.array_equal(got[..., dead], np.float32(0.9) * c["mass"][..., dead])
    if P:
        assert np.all(np.isfinite(got_p)) and np.array_equal(got_p[..., [0, P - 1]], np.float32(0.9) * c["mass_prefill"][..., [0, P - 1]])
    assert not np.array_equal(plain["k"], c["k"])


@pytest.mark.parametrize("L,S,H,G,dim,cap,P,R", [
    (1, 1, 2, 4, 64, 1100, 0, 1), (1, 2, 2, 4, 128, 150, 70, 3), (1, 3, 1, 3, 64, 331, 97, 5),       # maxima and sums by themselves
    (1, 2, 2, 4, 64, 300, 0, 3), (1, 1, 2, 3, 64, 60, 50, 3),                                         # one pass
    (8, 16, 2, 2, 64, 80, 70, 3),                                                                     # and a shared segment's masses behind it
    (1, 1, 2, 4, 128, 500, 0, 190), (1, 1, 4, 8, 64, 500, 0, 190),                                    # the wide products
])
@pytest.mark.parametrize("scale", [1.0, -1.0])
def test_weights_of_large_scores_sum_to_one(gpu, L, S, H, G, dim, cap, P, R, scale):
    """Scores of some 10^7, whose step in fp32 is one: a weight's share of its row is made of the very scores that are weighed.  Bound: the
    exponentials, sums and divisions, as beside a row's weights (n^(1/2) + 16 steps)."""
    c = T.make(45 + cap, L, S, H, G, dim, cap, P, R, [cap] * S, ordered=True, q_std=1.0)
    c["q"] = T.bf16((T.bf16_bits_to_f32(c["q"]).astype(np.float64) * 2.0 ** 19).astype(np.float32))
    c["scale"], c["mass"][:] = scale, 0.0
    if P:
        c["mass_prefill"][:] = 0.0
    got, got_p = T.run(gpu, c, None, 1.0)
    total = got.astype(np.float64).sum((1, 3)) + (got_p.astype(np.float64).sum(2) if P else 0.0)      # of a layer and head
    rows = S * R * G
    assert np.all(np.abs(total - rows) <= rows * ((cap + P) ** 0.5 + 16) * 2.0 ** -23 + rows * (cap + P) ** 0.5 * 2.0 ** -23)
