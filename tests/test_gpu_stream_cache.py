"""Rows entering a bounded cache, and segments compressed to their heaviest slots, on the GPU: every output is a copy or a
whole number and matches the definition bit for bit."""
import math

import numpy as np
import pytest

from oracle import decoding_loop as D

pytestmark = pytest.mark.gpu

FIELDS = ("k", "v", "mass", "slot_pos", "len", "next_pos")


def make(seed, L, S, H, cap, dim, length, masses="random", ordered=False):
    """Cache arrays (16-bit patterns as int16); length: live slots per stream."""
    rng = np.random.default_rng(seed)
    shape = (L, S, H, cap)
    length = np.asarray(length, np.int32)
    older = rng.integers(0, 50, S).astype(np.int32)
    live = np.clip(length, 0, cap)
    pos = np.zeros(shape, np.int32)
    for s in range(S):
        for l in range(L):
            for h in range(H):
                p = np.arange(live[s]) if ordered else rng.permutation(live[s])
                pos[l, s, h, :live[s]] = p + older[s]
                pos[l, s, h, live[s]:] = rng.integers(-5, 9000, cap - live[s])           # dead slots hold anything
    mass = {"random": lambda: np.exp(1.5 * rng.standard_normal(shape)), "few": lambda: rng.integers(0, 3, shape) * 0.5, "zero": lambda: np.zeros(shape),
            "odd": lambda: rng.choice([0.0, -0.0, 1.0, -1.0, math.nan, -math.nan, math.inf, -math.inf, 1e-42, -1e-42, 3e38], shape)}[masses]().astype(np.float32)
    return {"k": rng.integers(-32768, 32768, shape + (dim,)).astype(np.int16), "v": rng.integers(-32768, 32768, shape + (dim,)).astype(np.int16),
            "mass": mass, "slot_pos": pos, "len": length, "next_pos": (older + live).astype(np.int32)}


def upload(gpu, arrays):
    lib, _, torch = gpu
    t = {n: torch.from_numpy(np.array(a)).cuda() for n, a in arrays.items()}
    return t, lib.StreamCache(*(t[n] for n in FIELDS))


def same(got, want):
    for n in FIELDS:
        a, b = got[n].cpu().numpy(), want[n]
        if a.dtype == np.float32:
            a, b = a.view(np.int32), np.asarray(b, np.float32).view(np.int32)
        assert np.array_equal(a, b), n


def check_append(gpu, seed, L, S, H, cap, dim, length, R, rows, budget, sink=0, recent=0, masses="random", calls=1):
    lib, _, torch = gpu
    c = make(seed, L, S, H, cap, dim, length, masses)
    t, cache = upload(gpu, c)
    rng = np.random.default_rng(seed + 1)
    lists = [list(range(R))] * S if rows is None else rows
    on = None if rows is None else torch.tensor(rows, dtype=torch.int32, device="cuda")
    for _ in range(calls):
        new = [rng.integers(-32768, 32768, (L, S * R, H, dim)).astype(np.int16) for _ in range(2)]
        cache.append(*(torch.from_numpy(x).cuda() for x in new), R, on, budget, sink, recent)
        torch.cuda.synchronize()
        c = D.append(c, *new, R, lists, budget, sink, recent)
        same(t, c)
        assert int(cache.tickets.abs().sum()) == 0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("masses", ["random", "few", "zero", "odd"])
def test_append_into_full_caches(gpu, dim, masses):
    check_append(gpu, 1, 2, 3, 2, 70, dim, [64, 64, 64], 9, [[0, 3, 8], [0, -1, 2], [5, 6, 9]], 64, 4, 10, masses, calls=3)


@pytest.mark.parametrize("length,budget", [([0, 1, 5], 20), ([19, 20, 18], 20), ([40, 25, 3], 20), ([40, 41, 90], 40), ([-3, 1 << 30, 40], 40)])
def test_append_with_room_without_and_beyond_the_budget(gpu, length, budget):
    """Empty caches, room for some of the rows, more live slots than the budget, lengths out of range."""
    check_append(gpu, 2, 1, 3, 3, 40, 64, length, 6, [[0, 1, 4, 5], [2, 0, 7, 1], [-1, 0, 1, 2]], budget, 2, 3, calls=2)


@pytest.mark.parametrize("R,budget,cap,length", [(1, 1, 1, 1), (1, 1, 3, 0), (17, 17, 40, 17), (64, 100, 128, 90), (300, 310, 400, 200), (1500, 2000, 2500, 1999)])
def test_append_all_rows(gpu, R, budget, cap, length):
    check_append(gpu, 3, 1, 2, 2, cap, 64, [length, min(length, 5)], R, None, budget, 1, 5, "few", calls=2)


def test_everything_protected_still_gives_way(gpu):
    check_append(gpu, 4, 1, 2, 2, 30, 64, [30, 30], 5, [[0, 1, 2, 3, 4], [0, 2, -1, -1, -1]], 30, 0, 1000, calls=2)
    check_append(gpu, 5, 1, 1, 2, 30, 64, [30], 5, None, 30, 1 << 30, 0, calls=2)


@pytest.mark.parametrize("cap", [1023, 1024, 1025, 4095, 4096, 4097, 9000])
def test_append_over_the_sizes_of_a_block(gpu, cap):
    for masses in ("random", "few"):
        check_append(gpu, cap, 1, 1, 2, cap, 64, [cap], 4, [[0, 1, 3]], cap, 3, 20, masses)


def check_compress(gpu, seed, L, S, H, cap, dim, length, budget, sink=0, recent=0, masses="random", to_cap=None):
    lib, _, torch = gpu
    c = make(seed, L, S, H, cap, dim, length, masses, ordered=True)
    d = make(seed + 1, L, S, H, to_cap or budget, dim, [0] * S)
    t, cache = upload(gpu, c)
    u, smaller = upload(gpu, d)
    kept = torch.full((L, S, H, budget), 77, dtype=torch.int32, device="cuda")
    cache.compress(smaller, kept, budget, sink, recent)
    torch.cuda.synchronize()
    want, slots = D.compress(c, d, budget, sink, recent)
    assert np.array_equal(kept.cpu().numpy(), slots)
    same(u, want)
    same(t, c)                                               # the segment itself is only read


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("masses", ["random", "few", "zero", "odd"])
def test_compress(gpu, dim, masses):
    check_compress(gpu, 6, 2, 2, 3, 203, dim, [203, 180], 67, 4, 16, masses, to_cap=80)


@pytest.mark.parametrize("length,budget", [(0, 5), (1, 1), (5, 5), (6, 5), (5, 6), (63, 64), (300, 1), (300, 299), (-2, 3), (1 << 30, 3)])
def test_compress_edges(gpu, length, budget):
    check_compress(gpu, 7, 1, 2, 2, 300, 64, [length, 7], budget)


@pytest.mark.parametrize("cap,budget", [(1024, 100), (1025, 513), (4097, 400), (16384, 900), (16385, 3000), (40000, 1111)])
def test_compress_over_the_sizes_of_a_block(gpu, cap, budget):
    for masses in ("random", "few"):
        check_compress(gpu, cap, 1, 1, 2, cap, 64, [cap], budget, 4, 64, masses)


def test_equal_masses_keep_the_lower_slots(gpu):
    lib, _, torch = gpu
    c = make(8, 1, 1, 1, 5000, 64, [5000], "zero", ordered=True)
    c["next_pos"][0] = 5000 + 5000
    t, cache = upload(gpu, c)
    u, smaller = upload(gpu, make(9, 1, 1, 1, 1234, 64, [0]))
    kept = torch.empty((1, 1, 1, 1234), dtype=torch.int32, device="cuda")
    cache.compress(smaller, kept, 1234)
    assert torch.equal(kept.view(-1), torch.arange(1234, dtype=torch.int32, device="cuda"))
