"""Accumulated attention weights on the GPU against their definition in 64 bits.

Bound: products of bf16 numbers are exact in fp32, their sum over D features is off by at most D * 2^-23 of the sum of
magnitudes (each addition by a step), the scaled score by two roundings more: d = (D + 2) * 2^-23 * scale * max sum |q||k|.  A
weight e^(s - max) / sum is off by 2 d relative (its own score and the sum's), the exponential, the sum over n keys, the
division and the sum over rows by (n^(1/2) + 16) * 2^-23 (their parts go over at most that many additions in a row).  The old
mass adds two roundings."""
import numpy as np
import pytest

from oracle import decoding_loop as D
from workloads.generate import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def bf16(a):
    return f32_to_bf16_bits(np.asarray(a, np.float32))


def make(seed, L, S, H, G, dim, cap, P, R, length, ordered=False, q_std=1.5):
    rng = np.random.default_rng(seed)
    live = np.clip(np.asarray(length), 0, cap)
    pos = np.full((L, S, H, cap), 1 << 29, np.int32)
    for s in range(S):
        for l in range(L):
            for h in range(H):
                pos[l, s, h, :live[s]] = np.arange(live[s]) if ordered else rng.permutation(live[s])
    return dict(k=bf16(rng.standard_normal((L, S, H, cap, dim))), mass=rng.random((L, S, H, cap)).astype(np.float32), slot_pos=pos,
                len=np.asarray(length, np.int32), next_pos=live.astype(np.int32), q=bf16(q_std * rng.standard_normal((L, S * R, H * G, dim))),
                k_prefill=bf16(rng.standard_normal((L, H, P, dim))) if P else None, mass_prefill=rng.random((L, H, P)).astype(np.float32) if P else None,
                R=R, scale=dim ** -0.5)


def run(gpu, c, rows, decay, workspace_fill=0xFF):
    lib, _, torch = gpu
    dev = lambda a: None if a is None else torch.from_numpy(np.array(a.view(np.int16) if a.dtype == np.uint16 else a)).cuda()   # noqa: E731
    t = {n: dev(c[n]) for n in ("k", "mass", "slot_pos", "len", "next_pos", "q", "k_prefill", "mass_prefill")}
    cache = lib.StreamCache(t["k"], torch.zeros_like(t["k"]), t["mass"], t["slot_pos"], t["len"], t["next_pos"])
    op = lib.AttentionMass(cache, t["q"].shape[2], c["R"], c["scale"], k_prefill=t["k_prefill"], mass_prefill=t["mass_prefill"], decay=decay)
    on = None if rows is None else torch.tensor(rows, dtype=torch.int32, device="cuda")
    ws = torch.full((max(256, op.workspace_bytes(0 if rows is None else on.shape[1])),), workspace_fill, dtype=torch.uint8, device="cuda")
    op.run(t["q"], on, ws)
    torch.cuda.synchronize()
    return t["mass"].cpu().numpy(), None if c["k_prefill"] is None else t["mass_prefill"].cpu().numpy()


def check(gpu, c, rows, decay=1.0):
    wide = lambda a: None if a is None else bf16_bits_to_f32(a).astype(np.float64)   # noqa: E731
    S = c["len"].shape[0]
    lists = [list(range(c["R"]))] * S if rows is None else rows
    k, q, kp = wide(c["k"]), wide(c["q"]), wide(c["k_prefill"])
    with np.errstate(invalid="ignore"):
        want, shared = D.attention_mass(k, c["mass"], c["slot_pos"], c["len"], c["next_pos"], q, c["R"], lists, float(np.float32(c["scale"])),
                                        float(np.float32(decay)), kp, c["mass_prefill"])
    got, got_p = run(gpu, c, rows, decay)
    dim, cap, P = k.shape[4], k.shape[3], 0 if kp is None else kp.shape[2]
    norm = lambda a: np.sqrt(np.nansum(np.where(np.isfinite(a), a, 0) ** 2, -1)).max() if a is not None and a.size else 0.0   # noqa: E731
    d = (dim + 2) * 2.0 ** -23 * abs(c["scale"]) * norm(q) * max(norm(k), norm(kp))
    rel = 2 * d + ((cap + P) ** 0.5 + 16) * 2.0 ** -23
    for g, w, old in ((got, want, c["mass"]), (got_p, shared, c["mass_prefill"])):
        if g is None:
            continue
        added = np.abs(w - decay * old)
        bound = added * rel + (np.abs(old) + np.abs(w)) * 2 * 2.0 ** -24 + 1e-37
        bad = ~((np.abs(g - w) <= bound) | (np.isnan(g) & np.isnan(w)))
        assert not bad.any(), (int(bad.sum()), float(np.abs(g - w)[bad].max()), np.argwhere(bad)[:3].tolist())
    again, again_p = run(gpu, c, rows, decay, 0x00)
    assert np.array_equal(got, again, equal_nan=True) and (got_p is None or np.array_equal(got_p, again_p, equal_nan=True))
    return got, got_p


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("L,S,H,G,cap,P,R,rows", [
    (1, 1, 1, 1, 1, 0, 1, [[0]]),                               # one token, itself
    (1, 1, 2, 4, 40, 70, 1, [[0]]),
    (2, 3, 2, 4, 100, 33, 6, [[0, 3, 5], [1, -1, 2], [0, 5, 9]]),
    (1, 2, 3, 8, 64, 0, 9, [[0, 1, 2, 3, 4, 5, 6, 7, 8], [4, 5, -1, 0, 0, 0, 0, 0, 0]]),   # 72 query vectors
    (1, 4, 1, 3, 31, 300, 4, None),
    (1, 2, 1, 5, 200, 129, 40, None),                           # more query vectors than a block's tiles
])
def test_against_the_definition(gpu, dim, L, S, H, G, cap, P, R, rows):
    length = [cap, max(1, cap // 2), max(1, cap - 3), min(cap, 7)][:S]
    check(gpu, make(dim + cap, L, S, H, G, dim, cap, P, R, length), rows, 0.9)


@pytest.mark.parametrize("cap,R", [(33, 33), (130, 64), (257, 257), (700, 100)])
def test_a_prompt_scores_what_stands_before_it(gpu, cap, R):
    check(gpu, make(cap, 1, 1, 2, 2, 128, cap, 0, R, [cap], ordered=True), None)
    check(gpu, make(cap, 1, 1, 1, 4, 64, cap, 50, R, [cap], ordered=True), None, 0.5)


def test_many_query_vectors_on_the_prefill_segment(gpu):
    """More than a batch of 512 over all streams."""
    rng = np.random.default_rng(3)
    rows = [[0, 2, 4, 6][:n] + [-1] * (4 - n) for n in rng.integers(0, 5, 40)]
    check(gpu, make(5, 1, 40, 1, 8, 64, 20, 140, 8, rng.integers(4, 21, 40)), rows, 0.98)


def test_rows_that_see_nothing_and_streams_without_rows(gpu):
    c = make(6, 1, 3, 2, 2, 64, 40, 0, 4, [40, 40, 0])
    c["slot_pos"][:, 0] = 1000                                   # all of stream 0 lies ahead of its rows
    got, _ = check(gpu, c, [[0, 1], [-1, 0], [0, 1]], 0.5)
    assert np.array_equal(got[:, :2], np.float32(0.5) * c["mass"][:, :2]) and np.array_equal(got[:, 2], c["mass"][:, 2])
    c["slot_pos"][:, 0, :, 7] = 0                                # but for one slot: it takes all
    got, _ = check(gpu, c, [[0, 1], [-1, 0], [0, 1]], 0.5)


def test_what_stands_in_hidden_places_does_not_matter(gpu):
    """NaN and infinities in slots behind the length, in slots ahead of the rows and in rows that are not listed."""
    c = make(7, 1, 2, 2, 4, 64, 90, 40, 5, [60, 33])
    clean, clean_p = run(gpu, c, [[0, 2], [1, -1]], 1.0)
    c["k"][:, 0, :, 60:] = 0x7FC0
    c["k"][:, 1, :, 33:] = 0x7F80
    c["mass"][:, 1, :, 40:] = np.nan
    c["q"][:, [1, 3, 4, 5, 7, 8, 9]] = 0xFFC0
    ahead = c["slot_pos"] == 59                                  # the newest slot of stream 0: hidden from its first row only
    c["k"][np.broadcast_to(ahead, c["slot_pos"].shape)] = 0
    got, got_p = check(gpu, c, [[0, 2], [1, -1]])
    assert np.array_equal(got[:, 1, :, :33], clean[:, 1, :, :33]) and np.all(np.isfinite(got[:, 0])) and np.all(np.isfinite(got_p))
    c["slot_pos"][:, 0, :, 5] = 70000                            # ahead of every row, with NaN in its key
    c["k"][:, 0, :, 5] = 0x7FC0
    got, _ = check(gpu, c, [[0, 2], [1, -1]])
    assert np.array_equal(got[:, 0, :, 5], c["mass"][:, 0, :, 5])


def test_sharp_and_flat_weights_and_lengths_out_of_range(gpu):
    for q_std in (0.01, 40.0):
        check(gpu, make(8, 1, 2, 2, 4, 64, 70, 90, 3, [70, 20], q_std=q_std), [[0, 1, 2], [2, 1, 0]])
    c = make(9, 1, 2, 1, 2, 64, 50, 10, 3, [50, 50])
    c["len"][:] = [1 << 30, -4]
    check(gpu, c, [[0, 1], [0, 1]])


def test_a_long_segment(gpu):
    """Several blocks share a query tile's keys; the last chunk is short."""
    check(gpu, make(10, 1, 1, 1, 4, 64, 9001, 4099, 2, [8999], ordered=True), [[0, 1]], 0.98)
    check(gpu, make(11, 1, 1, 1, 2, 128, 5003, 0, 48, [5003], ordered=True), None)


@pytest.mark.parametrize("dim,cap,G,rows", [
    (64, 40, 4, [0, 3, 5]), (128, 33, 2, [0, 3, 5]), (64, 513, 2, [1, 4, 5]), (128, 600, 1, [0, 5]), (64, 1200, 1, [2, 3]), (128, 1153, 2, [0]),
    (64, 40, 8, [0, 2, 3, 5]), (128, 40, 8, [0, 2, 3]), (64, 530, 6, [0, 1, 2, 3]),
])
def test_streams_in_one_pass_beside_a_prefill_segment(gpu, dim, cap, G, rows):
    """From 256 heads of streams on, their segments are held by a block each (up to 2048 slots, and 1152 with more than 16 query
    vectors), every number of slots per wave and both numbers of vector tiles; lists of all lengths, an empty stream."""
    L, S, H = (8, 8, 4) if cap < 100 else (16, 8, 2)
    n, rng = len(rows), np.random.default_rng(cap)
    lists = [(rows[:k] + [-1] * n)[:n] for k in [n, 1, n, 0, n, max(1, n - 1), n, 1]]
    length = rng.integers(max(1, cap // 2), cap + 1, S)
    length[:3] = [cap, min(cap, 5), 0]
    c = make(cap + dim, L, S, H, G, dim, cap, 70, 6, length)
    c["k"][:, 1, :, 5:] = 0x7FC0                                 # what stands behind the length
    c["q"][:, [6 * s + r for s in range(S) for r in range(6) if r not in lists[s]]] = 0xFFC0
    got, got_p = run(gpu, c, lists, 0.9)
    wide = lambda a: bf16_bits_to_f32(a).astype(np.float64)   # noqa: E731
    # every fourth layer against the definition (it takes its time)
    for l in range(0, L, 4):
        part = {k: v[l:l + 1] if k in ("k", "mass", "slot_pos", "q", "k_prefill", "mass_prefill") else v for k, v in c.items()}
        with np.errstate(invalid="ignore"):
            want, shared = D.attention_mass(wide(part["k"]), part["mass"], part["slot_pos"], c["len"], c["next_pos"], wide(part["q"]), 6, lists,
                                            float(np.float32(c["scale"])), float(np.float32(0.9)), wide(part["k_prefill"]), part["mass_prefill"])
        finite_q = np.where(np.isfinite(wide(part["q"])), wide(part["q"]), 0)
        finite_k = np.where(np.isfinite(wide(part["k"])), wide(part["k"]), 0)
        norm = lambda a: np.sqrt((a ** 2).sum(-1)).max()   # noqa: E731
        d = (dim + 2) * 2.0 ** -23 * c["scale"] * norm(finite_q) * max(norm(finite_k), norm(wide(part["k_prefill"])))
        rel = 2 * d + ((cap + 70) ** 0.5 + 16) * 2.0 ** -23
        for g, w, old in ((got[l:l + 1], want, part["mass"]), (got_p[l:l + 1], shared, part["mass_prefill"])):
            bound = np.abs(w - 0.9 * old) * rel + (np.abs(old) + np.abs(w)) * 2 * 2.0 ** -24 + 1e-37
            assert np.all(np.abs(g - w) <= bound), (l, float(np.abs(g - w).max()))


@pytest.mark.parametrize("dim", [64, 128])
def test_streams_in_one_pass_without_a_prefill_segment(gpu, dim):
    check(gpu, make(12, 2, 3, 2, 4, dim, 300, 0, 5, [300, 17, 0]), [[0, 2, 4], [1, -1, 0], [0, 1, 2]], 0.9)
    check(gpu, make(13, 1, 2, 2, 8, dim, 1000, 0, 5, [999, 64]), [[0, 2, 4], [1, -1, 0]], 0.9)
    check(gpu, make(14, 1, 1, 1, 2, dim, 2048, 0, 5, [2048]), [[0, 2, 4]])


@pytest.mark.parametrize("scale", [0.0, -0.2, 0.3])
def test_any_sign_of_the_scale(gpu, scale):
    for R, rows in ((5, [[0, 2, 4], [1, 3, -1]]), (80, None)):
        c = make(15, 1, 2, 1, 4, 64, 150, 33, R, [150, 90])
        c["scale"] = scale
        check(gpu, c, rows)


def test_many_listed_rows_of_several_streams(gpu):
    """Lists of all lengths: rows that do not count, with NaN where they stand, and a shared segment."""
    rng = np.random.default_rng(16)
    R = 70
    lists = [sorted(rng.permutation(R)[:64].tolist()), sorted(rng.permutation(R)[:40].tolist()) + [-1] * 24, [-1] * 64]
    for dim in (64, 128):
        c = make(17 + dim, 1, 3, 2, 4, dim, 300, 130, R, [300, 150, 20])
        listed = [s * R + r for s in range(3) for r in lists[s] if r >= 0]
        c["q"][:, [m for m in range(3 * R) if m not in listed]] = 0x7FC0
        check(gpu, c, lists, 0.9)


def test_scores_that_grow_along_the_keys(gpu):
    """The running maximum has to follow: every chunk's scores lie far above those before it, and the other way round."""
    for R, rows in ((3, [[0, 1, 2]]), (70, None)):
        for order in (1, -1):
            c = make(18, 1, 1, 1, 4, 64, 900, 0, R, [900], ordered=True)
            ramp = np.linspace(-40.0, 40.0, 900)[::order]
            c["k"] = bf16(np.broadcast_to(ramp[:, None] / 8.0, (900, 64))[None, None, None])
            c["q"] = bf16(np.ones((1, R, 4, 64)) * 8.0)
            check(gpu, c, rows)


@pytest.mark.parametrize("dim,cap,P,G,rows", [
    (64, 30, 17, 4, [0, 2, 3]), (64, 200, 500, 4, [1]), (128, 100, 300, 2, [0, 1, 2, 3]), (64, 300, 2000, 2, [0, 3]), (128, 1000, 1100, 4, [2]),
    (64, 100, 3900, 1, [0, 2, 3]), (64, 60, 40, 8, [0, 1, 2, 3]), (128, 300, 260, 8, [0, 1, 2]), (64, 900, 1000, 5, [0, 1, 2, 3]),
])
def test_one_stream_with_a_prompt_of_its_own_in_one_pass(gpu, dim, cap, P, G, rows):
    """128 heads of one stream: a block holds the prefill segment and the stream's own, in eight and in sixteen waves."""
    L, H = 32, 4
    c = make(cap + P, L, 1, H, G, dim, cap, P, 5, [max(1, cap - 9)])
    c["k"][:, 0, :, max(1, cap - 9):] = 0x7FC0
    got, got_p = run(gpu, c, [rows + [-1]], 0.9)
    wide = lambda a: bf16_bits_to_f32(a).astype(np.float64)   # noqa: E731
    for l in range(0, L, 13):
        part = {k: v[l:l + 1] if k in ("k", "mass", "slot_pos", "q", "k_prefill", "mass_prefill") else v for k, v in c.items()}
        with np.errstate(invalid="ignore"):
            want, shared = D.attention_mass(wide(part["k"]), part["mass"], part["slot_pos"], c["len"], c["next_pos"], wide(part["q"]), 5, [rows],
                                            float(np.float32(c["scale"])), float(np.float32(0.9)), wide(part["k_prefill"]), part["mass_prefill"])
        norm = lambda a: np.sqrt(np.where(np.isfinite(a), a * a, 0).sum(-1)).max()   # noqa: E731
        d = (dim + 2) * 2.0 ** -23 * c["scale"] * norm(wide(part["q"])) * max(norm(wide(part["k"])), norm(wide(part["k_prefill"])))
        rel = 2 * d + ((cap + P) ** 0.5 + 16) * 2.0 ** -23
        for g, w, old in ((got[l:l + 1], want, part["mass"]), (got_p[l:l + 1], shared, part["mass_prefill"])):
            assert np.all(np.abs(g - w) <= np.abs(w - 0.9 * old) * rel + (np.abs(old) + np.abs(w)) * 2 * 2.0 ** -24 + 1e-37), l


@pytest.mark.parametrize("dim,cap,G,n", [(64, 500, 2, 3), (128, 1100, 4, 4), (64, 1700, 1, 2), (64, 700, 8, 3), (128, 1100, 8, 4), (64, 2048, 5, 3)])
def test_streams_without_a_prompt_in_one_pass(gpu, dim, cap, G, n):
    L, S, H = 16, 2, 4
    c = make(cap + n, L, S, H, G, dim, cap, 0, 5, [cap, max(1, cap // 3)])
    lists = [list(range(n)) + [-1], [2, -1] + [0] * (n - 1)]
    got, _ = run(gpu, c, lists, 0.9)
    wide = lambda a: bf16_bits_to_f32(a).astype(np.float64)   # noqa: E731
    for l in (0, 15):
        part = {k: v[l:l + 1] if k in ("k", "mass", "slot_pos", "q") else v for k, v in c.items()}
        want, _ = D.attention_mass(wide(part["k"]), part["mass"], part["slot_pos"], c["len"], c["next_pos"], wide(part["q"]), 5, lists,
                                   float(np.float32(c["scale"])), float(np.float32(0.9)))
        norm = lambda a: np.sqrt((a * a).sum(-1)).max()   # noqa: E731
        rel = 2 * (dim + 2) * 2.0 ** -23 * c["scale"] * norm(wide(part["q"])) * norm(wide(part["k"])) + (cap ** 0.5 + 16) * 2.0 ** -23
        assert np.all(np.abs(got[l:l + 1] - want) <= np.abs(want - 0.9 * part["mass"]) * rel + (np.abs(part["mass"]) + np.abs(want)) * 2 * 2.0 ** -24 + 1e-37)


@pytest.mark.parametrize("dim", [64, 128])
def test_hidden_chunks_of_many_rows(gpu, dim):
    """A prompt that is all chunk: half of all scores are hidden.  A row with NaN spoils what it sees, and nothing ahead of it."""
    R = 330
    c = make(19, 1, 1, 2, 3, dim, R, 0, R, [R], ordered=True)
    check(gpu, c, None, 0.9)
    c["q"][:, 100] = 0x7FC0
    got, _ = check(gpu, c, None, 0.9)
    assert np.all(np.isnan(got[:, 0, :, :101])) and np.all(np.isfinite(got[:, 0, :, 101:]))
    shuffled = make(20, 1, 2, 1, 3, dim, 700, 0, 150, [700, 400])
    check(gpu, shuffled, None, 0.9)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("L,S,H,G,cap,P,R", [
    (1, 2, 2, 4, 90, 0, 7),                                      # the keys in one block: one pass
    (1, 1, 1, 3, 60, 50, 5),
    (1, 2, 2, 4, 150, 70, 12),                                   # maxima and sums by themselves
    (2, 1, 1, 2, 4500, 0, 4),
    (1, 2, 1, 2, 200, 140, 150),                                 # the wide products
    (8, 16, 2, 2, 80, 70, 6),                                    # one pass after a shared segment's maxima
])
def test_rows_and_keys_that_are_not_finite(gpu, dim, L, S, H, G, cap, P, R):
    """The definition's answer, element for element: a NaN row spoils the slots that it sees; a NaN key what its rows see; scores that are
    all minus infinity count for nothing, plus infinity makes NaN."""
    def fresh():
        return make(21, L, S, H, G, dim, cap, P, R, [cap, cap - 2, *[cap - s % 3 for s in range(S)]][:S], ordered=True)
    c = fresh()
    c["q"][:, R // 2] = 0x7FC0                                   # stream 0, a row in the middle
    got, got_p = check(gpu, c, None, 0.9)
    assert np.all(np.isnan(got[:, 0, :, :cap - R + R // 2 + 1])) and np.all(np.isfinite(got[:, 0, :, cap - R + R // 2 + 1:]))
    assert np.all(np.isfinite(got[:, 1:][~np.isnan(c["mass"][:, 1:])])) and (got_p is None or np.all(np.isnan(got_p)))
    c = fresh()
    c["k"][:, 0, :, cap - 2] = 0x7FC0                            # what only the two newest rows of stream 0 see
    got, _ = check(gpu, c, None, 0.9)
    assert np.all(np.isnan(got[:, 0]))
    c["slot_pos"][:, 0, :, cap - 2] = cap + 5                    # nobody does
    got, _ = check(gpu, c, None, 0.9)
    assert np.all(np.isfinite(got[:, 0]))
    if P:
        c["k_prefill"][:, :, P // 2] = 0x7FC0                    # of a shared segment: a slot for which no row is there
        c["q"][:] = 0x7FC0
        got, got_p = check(gpu, c, [[-1] * R] * S, 0.9)
        assert np.array_equal(got_p, np.float32(0.9) * c["mass_prefill"])
    for sign in (0xFF80, 0x7F80):
        c = fresh()
        c["k"][..., 0] = 0x3F80
        if P:
            c["k_prefill"][..., 0] = 0x3F80
        c["q"][:, R - 1, :, 0] = sign                            # the newest row of stream 0: all scores infinite
        got, _ = check(gpu, c, None, 0.9)
        assert np.all(np.isfinite(got[:, 0]) if sign == 0xFF80 else np.isnan(got[:, 0]))
