"""Attention over the paged cache on the GPU against float64, to bounds counted from roundings.

Scores: a query vector's numbers are cut at 2^-22 of its largest, which moves a score by at most scale * max |q| * sum |k| * 2^-22; products of bf16
(tail, rows) and the conversions, scales and exponents around them are fp32: D + 16 roundings of 2^-24 of sum |q k| * scale.  Each moves a
weighted mean by twice itself.  Weights: on pages cut at 2^-24 of the page's largest, 64 of them, twice; in the tail three bf16 numbers
(2^-27, with the sum's own roundings 2^-21).  Sums: a rounding of 2^-23 per item and merge.

Outputs in bf16 are the same, rounded once.  bound() leaves them more (query vectors cut at 2^-15 of their largest number, weights at 2^-16 of the page's
largest, tails 2^-16); the tests of uneven query vectors and small weights hold them to the bound of fp32 and that rounding."""
import math

import numpy as np
import pytest

from oracle import beams as O
from test_gpu_page_cache import bits, make, upload
from workloads.generate import f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def bound(size, q, scale, D, items, want, fp32):
    vmax, s1, k1 = size[..., 0], size[..., 1], size[..., 2]
    qmax = np.abs(q).max(-1)
    q_cut, p_cut, tail = (2.0 ** -22, 2.0 ** -24, 2.0 ** -21) if fp32 else (2.0 ** -15, 2.0 ** -16, 2.0 ** -16)
    far = 2 * (abs(scale) * k1 * qmax * q_cut + (D + 16) * 2.0 ** -24 * s1) + tail + 128 * p_cut + (items + 32) * 2.0 ** -23
    return (vmax * far)[..., None] + (0 if fp32 else np.abs(want) * 2.0 ** -8)


def run(gpu, c, layer, q, k_new, v_new, parent, R, scale, window=0, sink=0, fp32=True, stream=None):
    lib, _, torch = gpu
    _, cache = upload(gpu, c)
    on = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (q, k_new, v_new, np.asarray(parent, np.int32))]
    op = lib.PageAttention(cache, layer, q.shape[1], R, scale, on[1], on[2], on[3], window, sink)
    out = torch.empty(q.shape, dtype=torch.float32 if fp32 else torch.bfloat16).cuda()
    ws = torch.full((op.workspace_bytes(),), 0xFF, dtype=torch.uint8).cuda()             # (nothing in it counts)
    op.run(on[0], out, lib.Y_FP32 if fp32 else lib.Y_BF16, ws)
    torch.cuda.synchronize()
    first = out.double().cpu().numpy()
    op.run(on[0], out, lib.Y_FP32 if fp32 else lib.Y_BF16, ws)
    torch.cuda.synchronize()
    assert np.array_equal(first, out.double().cpu().numpy(), equal_nan=True)             # the same from call to call
    return first, op


def check(gpu, seed, lengths, R, H, G, D, window=0, sink=0, fp32=True, L=1, columns=None, share=None, q_scale=1.5, tree=True, scale=None):
    rng = np.random.default_rng(seed)
    S, need = len(lengths), sum(n // 64 for n in lengths)
    columns = columns or max(lengths) // 64 + 1
    c = make(seed, L, S, H, D, need + 3, columns, lengths)
    if share:
        c = O.reorder(c, share)
    scale = D ** -0.5 if scale is None else scale
    q, k, v = bits(rng, S * R, H * G, D, scale=q_scale), bits(rng, S * R, H, D), bits(rng, S * R, H, D)
    parent = np.array([[rng.integers(-1, max(r, 1)) if r and tree else r - 1 for r in range(R)] for _ in range(S)]).reshape(-1)
    layer = int(rng.integers(0, L))
    got, op = run(gpu, c, layer, q, k, v, parent, R, scale, window, sink, fp32)
    want, size = O.attention(c, layer, q, k, v, parent, R, float(np.float32(scale)), window, sink)
    assert np.all(np.isfinite(got))
    items = max(lengths) // 64 + 5
    assert np.all(np.abs(got - want) <= bound(size, O.bf16(q), scale, D, items, want, fp32))
    return op.plan()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("length", [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 1000])
def test_one_token(gpu, D, length):
    check(gpu, length, [length], 1, 2, 3, D)


@pytest.mark.parametrize("R,G", [(1, 1), (1, 8), (2, 8), (3, 5), (5, 3), (16, 1), (17, 1), (30, 4), (33, 1), (64, 8), (64, 1)])
def test_rows_and_heads(gpu, R, G):
    check(gpu, R * 10 + G, [100, 321, 64], R, 2, G, 64, fp32=R % 2 == 1)


@pytest.mark.parametrize("window,sink", [(1, 0), (2, 1), (33, 0), (64, 64), (65, 5), (100, 70), (300, 200), (10000, 3), (7, 10000)])
@pytest.mark.parametrize("R", [1, 40])
def test_windows(gpu, window, sink, R):
    check(gpu, window + sink + R, [700, 64, 130, 5, 0, 449], R, 2, 4, 64, window, sink)
    check(gpu, window + sink + R + 1, [333, 200], R, 1, 2, 128, window, sink, tree=False)


def test_layers_and_shared_pages(gpu):
    check(gpu, 1, [400, 200, 64, 70], 3, 3, 2, 64, L=4, share=[0, 0, 0, 1])


@pytest.mark.parametrize("D", [64, 128])
def test_many_pages(gpu, D):
    plan = check(gpu, 2, [6000, 10], 1, 2, 4, D)
    assert plan["splits"] > 1
    check(gpu, 3, [9000], 20, 1, 4, D, fp32=False)


def test_a_table_far_longer_than_the_stream(gpu):
    plan = check(gpu, 4, [70, 3, 0], 2, 2, 4, 64, columns=3000)
    assert plan["splits"] > 1


@pytest.mark.parametrize("columns", [8, 20, 64, 500])
@pytest.mark.parametrize("R,G", [(1, 1), (1, 4), (1, 5), (2, 4), (5, 3), (9, 2)])
def test_short_streams_in_long_tables(gpu, columns, R, G):
    check(gpu, columns + R, [70, 0, 63, 64, 300, 1, 129, 500, 33, 2], R, 2, G, 64, columns=columns, fp32=R % 2 == 1)
    check(gpu, columns + R + 1, [100, 511, 5], R, 1, G, 128, columns=columns, window=70, sink=5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,R", [(1, 1), (4, 1), (2, 2)])
@pytest.mark.parametrize("longest", [28, 29, 30, 31, 32, 40])
def test_bundles_of_short_and_long_streams(gpu, D, G, R, longest):
    """Around the number of pages from which streams of a bundle are taken together; some share what they have, some have nothing."""
    lengths = [64 * longest + 5, 64, 0, 64 * longest - 1, 1000, 64 * longest, 3, 70, 64 * longest + 63, 10, 100]
    check(gpu, longest + G, lengths, R, 1, G, D, columns=60, fp32=G == 1)
    check(gpu, longest + G + 50, lengths, R, 1, G, D, columns=60, share=[0, 0, 0, 3, 3, 5, 0, 7, 8, 0, 8])
    check(gpu, longest + G + 90, lengths, R, 1, G, D, columns=60, share=[0, 0, 0, 3, 3, 5, 0, 7, 8, 0, 8], window=1500, sink=130)


@pytest.mark.parametrize("length", [90, 2300])
def test_more_bundles_than_fill_the_card(gpu, length):
    n = 300 if length == 90 else 216
    plan = check(gpu, 60 + length, [length] + [70, 3, 0, 64] * 100 if length == 90 else [length, 64] * (n // 2), 1, 8, 1, 64, columns=50, fp32=False)
    assert plan["splits"] == 1


@pytest.mark.parametrize("S,G", [(1, 4), (9, 1), (6, 4)])
def test_replays_while_the_streams_grow_and_shrink(gpu, S, G):
    """One graph and one workspace, from streams that go alone to ones that share blocks, and back."""
    lib, _, torch = gpu
    H, D, R, most = 2, 64, 2, 64 * 45 + 7
    rng = np.random.default_rng(70 + S)
    c = make(70, 1, S, H, D, S * 45 + 3, 50, [most] * S)
    q, k, v = bits(rng, S * R, H * G, D), bits(rng, S * R, H, D), bits(rng, S * R, H, D)
    parent = [-1, 0] * S
    t, cache = upload(gpu, c)
    on = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (q, k, v, np.asarray(parent, np.int32))]
    op = lib.PageAttention(cache, 0, H * G, R, D ** -0.5, on[1], on[2], on[3])
    assert op.plan()["splits"] > 1
    out, eager = (torch.zeros(q.shape, dtype=torch.float32).cuda() for _ in range(2))
    ws, other = (torch.full((op.workspace_bytes(),), 0xFF, dtype=torch.uint8).cuda() for _ in range(2))
    op.run(on[0], out, lib.Y_FP32, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.run(on[0], out, lib.Y_FP32, ws)
    for n in (0, 5, 64 * 20, 64 * 28, 64 * 29 + 63, 64 * 31, most, 64 * 33, 70, most, 1):
        lengths = [n] + [max(0, n - 64 * i) for i in range(1, S)]
        cache.len.copy_(torch.tensor(lengths, dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        op.run(on[0], eager, lib.Y_FP32, other)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), n
        c["len"][:] = lengths
        want, size = O.attention(c, 0, q, k, v, parent, R, float(np.float32(D ** -0.5)), 0, 0)
        got = out.double().cpu().numpy()
        assert np.all(np.abs(got - want) <= bound(size, O.bf16(q), D ** -0.5, D, n // 64 + 5, want, True)), n


@pytest.mark.parametrize("q_scale", [1e-30, 1e-3, 40.0])
def test_sharp_and_flat(gpu, q_scale):
    check(gpu, 5, [500, 130], 3, 2, 2, 64, q_scale=q_scale)


def test_scales_of_either_sign(gpu):
    check(gpu, 6, [300], 2, 1, 2, 64, scale=-0.2)
    check(gpu, 7, [300], 2, 1, 2, 64, scale=0.0)


def test_means_of_equal_values(gpu):
    """All keys alike: every weight is the same, and a mean of equal numbers is that number."""
    lib, _, torch = gpu
    c = make(8, 1, 1, 1, 64, 5, 5, [200])
    c["k"][:], c["v"][:], c["v_scale"][:] = 3, 64, 0.03125
    c["k_scale"][:] = 0.5
    c["k_tail"][:], c["v_tail"][:] = 0x3FC0, 0x4000                                      # 1.5 and 2
    q = np.full((1, 4, 64), 0x3F80, np.int16)
    new = [np.full((1, 1, 64), x, np.int16) for x in (0x3FC0, 0x4000)]
    got, _ = run(gpu, c, 0, q, *new, [-1], 1, 0.125)
    assert np.all(np.abs(got - 2.0) <= 2.0 * 4 * 2.0 ** -23)                             # page, tail, merge and quotient


def test_what_a_row_does_not_see_does_not_touch_it(gpu):
    """Infinities and NaN behind the window, on other branches, behind the tail's end, in pages that only others hold."""
    rng = np.random.default_rng(9)
    R, H, G, D = 6, 2, 2, 64
    c = make(9, 1, 2, H, D, 12, 5, [300, 200])
    parent = [-1, 0, 1, 0, 3, 3, -1, 0, 0, 0, 0, 0]
    q, k, v = bits(rng, 2 * R, H * G, D), bits(rng, 2 * R, H, D), bits(rng, 2 * R, H, D)
    # the first 2 pages and the tail's rest are poison, and so are rows 1 (seen by 2) and 5 of stream 0
    for s in range(2):
        for i in range(2):
            p = c["table"][c["slot"][s], i]
            c["k_scale"][:, p], c["v_scale"][:, p] = math.nan, math.nan
            c["k"][:, p], c["v"][:, p] = 0, 0
        c["k_tail"][:, c["slot"][s], :, c["len"][s] % 64:], c["v_tail"][:, c["slot"][s], :, c["len"][s] % 64:] = 0x7FC0, 0x7F80
    k[1], v[5, 0, 3], v[1, 1, 7] = 0x7FC0, 0x7F80, 0x7FC0
    window, sink = 60, 0
    got, _ = run(gpu, c, 0, q, k, v, parent, R, 0.125, window, sink)
    want, size = O.attention(c, 0, q, k, v, parent, R, 0.125, window, sink)
    clean = np.array([r not in (1, 2, 5) for r in range(2 * R)])
    assert np.all(np.isfinite(want[clean])) and np.all(np.isfinite(got[clean]))
    assert np.all(np.abs(got[clean] - want[clean]) <= bound(size, O.bf16(q), 0.125, D, 9, want, True)[clean])
    assert np.all(np.isnan(got[1])) and np.all(np.isnan(got[2]))                         # NaN among the scores
    odd = np.zeros(D, bool)
    odd[3] = True
    assert np.all(got[5, :G][:, odd] == math.inf) and np.all(np.isfinite(got[5, :G][:, ~odd])) and np.all(np.isfinite(got[5, G:]))
    # seen from a wider window all is NaN, in every feature
    got, _ = run(gpu, c, 0, q, k, v, parent, R, 0.125, 400)
    assert np.all(np.isnan(got))


def test_values_of_nan_alone(gpu):
    """A page whose keys are numbers and whose values are not: NaN for those that see one of its tokens, in every feature."""
    rng = np.random.default_rng(10)
    c = make(10, 1, 1, 1, 64, 6, 5, [200])
    c["v_scale"][:, c["table"][c["slot"][0], 0]] = math.nan
    q, k, v = bits(rng, 3, 1, 64), bits(rng, 3, 1, 64), bits(rng, 3, 1, 64)
    for window, sink, bad in ((0, 0, [0, 1, 2]), (138, 0, [0]), (137, 0, []), (10, 1, [0, 1, 2])):
        got, _ = run(gpu, c, 0, q, k, v, [-1, 0, 1], 3, 0.125, window, sink)             # rows at 200, 201, 202: the page is 0 .. 63
        assert [r for r in range(3) if np.any(np.isnan(got[r]))] == bad
        assert all(np.all(np.isnan(got[r])) for r in bad)


@pytest.mark.parametrize("odd", [0x7FC0, 0x7F80, 0xFF80])
def test_query_vectors_that_are_not_finite(gpu, odd):
    rng = np.random.default_rng(11)
    c = make(11, 1, 1, 2, 64, 6, 5, [200])
    q, k, v = bits(rng, 4, 4, 64), bits(rng, 4, 2, 64), bits(rng, 4, 2, 64)
    q.view(np.uint16)[1, 2, 17] = odd
    want, size = O.attention(c, 0, q, k, v, [-1, 0, 1, 2], 4, 0.125)
    got, _ = run(gpu, c, 0, q, k, v, [-1, 0, 1, 2], 4, 0.125)
    assert np.all(np.isnan(got[1, 2]))
    got[1, 2] = want[1, 2] = 0
    q[1, 2] = 0
    assert np.all(np.abs(got - want) <= bound(np.nan_to_num(size), O.bf16(q), 0.125, 64, 9, want, True))


def test_pages_that_are_not_there(gpu):
    rng = np.random.default_rng(12)
    c = make(12, 1, 2, 2, 64, 20, 8, [450, 300])
    c["table"][c["slot"][0], 2], c["table"][c["slot"][0], 5], c["table"][c["slot"][1], :] = -1, 20, -1
    q, k, v = bits(rng, 4, 4, 64), bits(rng, 4, 2, 64), bits(rng, 4, 2, 64)
    want, size = O.attention(c, 0, q, k, v, [-1, 0] * 2, 2, 0.125, 420, 3)
    got, _ = run(gpu, c, 0, q, k, v, [-1, 0] * 2, 2, 0.125, 420, 3)
    assert np.all(np.abs(got - want) <= bound(size, O.bf16(q), 0.125, 64, 12, want, True))


def test_lengths_outside_the_table(gpu):
    """They count as the nearer end."""
    rng = np.random.default_rng(13)
    c = make(13, 1, 2, 1, 64, 20, 4, [4 * 64 + 63, 0])
    q, k, v = bits(rng, 2, 1, 64), bits(rng, 2, 1, 64), bits(rng, 2, 1, 64)
    want, _ = run(gpu, c, 0, q, k, v, [-1, -1], 1, 0.125)
    c["len"][:] = [1 << 30, -5]
    got, _ = run(gpu, c, 0, q, k, v, [-1, -1], 1, 0.125)
    assert np.array_equal(got, want)


def test_offsets_past_32_bits(gpu):
    lib, _, torch = gpu
    pages, H, D = 36000, 16, 64
    rng = np.random.default_rng(14)
    cache = lib.PageCache.empty(1, 1, H, D, pages, 4)
    cache.refs[:-3] = 1
    k, v = (bits(rng, 1, 200, H, D) for _ in range(2))
    cache.append(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), 200)
    assert cache.table.tolist() == [[pages - 3, pages - 2, pages - 1, -1]]
    c, _ = O.append(O.empty_cache(1, 1, H, D, 3, 4), k, v, 200)
    q, kn, vn = bits(rng, 1, H, D), bits(rng, 1, H, D), bits(rng, 1, H, D)
    on = [torch.from_numpy(x).cuda() for x in (q, kn, vn)]
    op = lib.PageAttention(cache, 0, H, 1, 0.125, on[1], on[2], torch.tensor([-1], dtype=torch.int32).cuda())
    out, ws = torch.empty((1, H, D)).cuda(), torch.empty(op.workspace_bytes(), dtype=torch.uint8).cuda()
    op.run(on[0], out, lib.Y_FP32, ws)
    want, size = O.attention(c, 0, q, kn, vn, [-1], 1, 0.125)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound(size, O.bf16(q), 0.125, D, 9, want, True))


def test_what_is_appended_is_seen_alike(gpu):
    """Rows of a step, then the same tokens in the tail: as long as no page fills, the next row sees the same numbers."""
    lib, _, torch = gpu
    rng = np.random.default_rng(15)
    H, G, D, R = 2, 4, 64, 7
    c = make(15, 1, 1, H, D, 8, 5, [130])
    q, k, v = bits(rng, R, H * G, D), bits(rng, R, H, D), bits(rng, R, H, D)
    tree, _ = run(gpu, c, 0, q, k, v, np.arange(-1, R - 1), R, 0.125)
    for r in range(1, R):
        d, _ = O.append(c, k[None], v[None], R, [list(range(r)) + [-1] * (R - r)])
        one, _ = run(gpu, d, 0, q[r:r + 1], k[r:r + 1], v[r:r + 1], [-1], 1, 0.125)
        # both are within their bounds of one number
        want, size = O.attention(d, 0, q[r:r + 1], k[r:r + 1], v[r:r + 1], [-1], 1, 0.125)
        assert np.all(np.abs(one[0] - tree[r]) <= 2 * bound(size, O.bf16(q[r:r + 1]), 0.125, D, 9, want, True)[0])


def test_pages_of_zeros(gpu):
    """Scale 0: all scores alike, and what the window hides stays hidden; values of zero."""
    rng = np.random.default_rng(16)
    c = make(16, 1, 1, 2, 64, 6, 5, [200])
    pages = c["table"][c["slot"][0], :3]
    for n in ("k", "v"):
        c[n][:, pages[1]], c[n + "_scale"][:, pages[1]] = 0, 0
    q, k, v = bits(rng, 2, 4, 64), bits(rng, 2, 2, 64), bits(rng, 2, 2, 64)
    for window, sink in ((0, 0), (100, 0), (90, 70)):
        want, size = O.attention(c, 0, q, k, v, [-1, 0], 2, 0.125, window, sink)
        got, _ = run(gpu, c, 0, q, k, v, [-1, 0], 2, 0.125, window, sink)
        assert np.all(np.abs(got - want) <= bound(size, O.bf16(q), 0.125, 64, 9, want, True))


@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("R,G", [(1, 1), (1, 2), (1, 4), (2, 4), (3, 1), (5, 3), (1, 5)])
def test_streams_that_share_some_of_their_pages(gpu, R, G, fp32):
    """Bundles of streams: the same pages at the same places, others, none, and other lengths; windows of several starts."""
    rng = np.random.default_rng(17 + R * G)
    S, H, D = 19, 2, 64
    c = make(17, 1, S, H, D, 200, 12, [int(x) for x in rng.integers(0, 700, S)])
    c = O.reorder(c, [0, 0, 0, 3, 3, 5, 6, 6, 6, 6, 6, 0, 12, 13, 14, 12, 12, 12, 18])
    k, v = bits(rng, 1, S * 70, H, D), bits(rng, 1, S * 70, H, D)                       # then they go on by themselves
    c, _ = O.append(c, k, v, 70, [(list(range(rng.integers(0, 71))) + [-1] * 70)[:70] for _ in range(S)])
    c["table"][c["slot"][7], 1] = -1
    q, kn, vn = bits(rng, S * R, H * G, D, scale=1.5), bits(rng, S * R, H, D), bits(rng, S * R, H, D)
    parent = np.array([[rng.integers(-1, max(r, 1)) if r else -1 for r in range(R)] for _ in range(S)]).reshape(-1)
    for window, sink in ((0, 0), (150, 70)):
        want, size = O.attention(c, 0, q, kn, vn, parent, R, 0.125, window, sink)
        got, _ = run(gpu, c, 0, q, kn, vn, parent, R, 0.125, window, sink, fp32)
        assert np.all(np.abs(got - want) <= bound(size, O.bf16(q), 0.125, D, 17, want, fp32))


def test_a_page_of_nan_that_only_one_of_a_bundle_holds(gpu):
    rng = np.random.default_rng(18)
    S, H, D = 8, 1, 64
    c = make(18, 1, S, H, D, 40, 5, [200] * S)
    c = O.reorder(c, [0, 0, 0, 3, 4, 5, 6, 7])
    bad = c["table"][c["slot"][4], 1]
    c["k_scale"][:, bad], c["v_scale"][:, c["table"][c["slot"][6], 0]] = np.nan, np.nan
    q, kn, vn = bits(rng, S, 2, D), bits(rng, S, 1, D), bits(rng, S, 1, D)
    kn[1], vn[2], vn[7] = 0x7FC0, 0x7F80, 0x7FC0
    want, size = O.attention(c, 0, q, kn, vn, [-1] * S, 1, 0.125)
    got, _ = run(gpu, c, 0, q, kn, vn, [-1] * S, 1, 0.125)
    for s in range(S):
        if s in (1, 4, 6, 7):
            assert np.all(np.isnan(got[s]))
        elif s == 2:
            assert np.all(got[s] == np.inf)
        else:
            assert np.all(np.abs(got[s] - want[s]) <= bound(size, O.bf16(q), 0.125, D, 9, want, True)[s])


@pytest.mark.parametrize("D", [64, 128])
def test_large_values_and_rising_maxima(gpu, D):
    """Every page heavier than the one before, by up to 2^20, and values of 1e33: sums relative to an older maximum must not pass the largest
    number."""
    rng = np.random.default_rng(19)
    c = make(19, 1, 1, 1, D, 30, 25, [24 * 64 + 9])
    c["k"][:] = 0
    for i in range(24):
        c["k"][:, c["table"][c["slot"][0], i], :, :, 0] = 4 * i + rng.integers(0, 4, (1, 1, 64))
    c["k_scale"][:], c["v_scale"][:] = 1.0, 1e33 / 127
    c["k_tail"][:] = 0
    q, kn = np.zeros((3, 2, D), np.int16), np.zeros((3, 1, D), np.int16)
    vn = bits(rng, 3, 1, D)
    for scale in (0.02, 0.2, 1.0, 3.5):
        q[..., 0] = 0x3F80                                                                # 1
        want, size = O.attention(c, 0, q, kn, vn, [-1, 0, 1], 3, float(np.float32(scale)))
        for fp32 in (True, False):
            got, _ = run(gpu, c, 0, q, kn, vn, [-1, 0, 1], 3, scale, fp32=fp32)
            assert np.all(np.abs(got - want) <= bound(size, O.bf16(q), scale, D, 30, want, fp32))


def check_bf16(gpu, c, q, k_new, v_new, parent, R, scale):
    got, _ = run(gpu, c, 0, q, k_new, v_new, parent, R, scale, fp32=False)
    want, size = O.attention(c, 0, q, k_new, v_new, parent, R, float(np.float32(scale)))
    exact = bound(size, O.bf16(q), scale, q.shape[2], int(c["len"].max()) // 64 + 5, want, True)
    assert np.all(np.abs(got - want) <= exact + np.abs(want) * 2.0 ** -8)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("times", [30.0, 100.0])
@pytest.mark.parametrize("length,R", [(1000, 1), (4096, 3), (63, 2)])
def test_bf16_outputs_of_uneven_query_vectors(gpu, D, times, length, R):
    """One feature is many times the others, where the keys have little: the other features' part of the scores is as exact as elsewhere."""
    rng = np.random.default_rng(80)
    c = make(80, 1, 2, 2, D, 2 * (length // 64) + 1, 70, [length, length])
    c["k"][..., 5] = rng.integers(-2, 3, c["k"].shape[:-1])
    little = lambda *shape: bits(rng, *shape, scale=0.02)   # noqa: E731
    c["k_tail"][..., 5] = little(*c["k_tail"].shape[:-1])
    q, k, v = O.bf16(bits(rng, 2 * R, 6, D)), bits(rng, 2 * R, 2, D), bits(rng, 2 * R, 2, D)
    q[..., 5] = times * np.sign(q[..., 5])
    k[..., 5] = little(2 * R, 2)
    check_bf16(gpu, c, f32_to_bf16_bits(q.astype(np.float32)).view(np.int16), k, v, [-1, 0, 1][:R] * 2, R, D ** -0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("top", [24.0, 96.0, 384.0])
@pytest.mark.parametrize("length", [64, 1024])
def test_bf16_outputs_of_query_vectors_with_one_large_number(gpu, D, top, length):
    """Half of the keys look at one small number of the query vector, half at another, and all have the same score: their values cancel.  The first
    number has 8 significant bits, the last of which is 2^-15 of the largest one's power of two."""
    last = 2.0 ** (math.floor(math.log2(top)) - 15)
    c = make(82, 1, 1, 1, D, 20, 20, [length])
    half = np.random.default_rng(82).permuted(np.tile(np.arange(64) % 2, (20, 1)), axis=1)       # [page][token]
    c["k"][:], c["v"][:] = 0, np.where(half, 127, -127)[None, :, None, None, :]
    c["k"][0, :, 0, :, 9], c["k"][0, :, 0, :, D - 2] = np.where(half, 124, 0), np.where(half, 0, 93)
    c["k_scale"][:], c["v_scale"][:] = 4 / (0.125 * 124 * 129 * last), 1 / 127
    q, k, v = (np.zeros((1, n, D)) for n in (3, 1, 1))
    q[..., 0], q[..., 9], q[..., D - 2] = top, 129 * last, 172 * last                            # 124 * 129 = 93 * 172
    of = lambda x: f32_to_bf16_bits(x.astype(np.float32)).view(np.int16)   # noqa: E731
    check_bf16(gpu, c, of(q), of(k), of(v), [-1], 1, 0.125)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("less", [10.0, 11.1, 11.8])
def test_bf16_outputs_of_many_small_weights(gpu, D, less):
    """In every page one key with the value 0, and 63 whose weights are e^-less of its: what they bring is all that there is."""
    c = make(81, 1, 1, 1, D, 5, 4, [64 * 4])
    c["k"][:], c["k"][:, :, :, 17, 0], c["v"][:], c["v"][..., 17] = 0, 127, np.abs(c["v"]), 0
    c["k_scale"][:], c["v_scale"][:] = less / (127 * 0.125), 1.0
    q, k, v = (np.zeros((1, n, D)) for n in (2, 1, 1))
    q[..., 0], k[..., 0] = 1.0, -8.0 * less              # (the row itself weighs e^-less of that)
    of = lambda x: f32_to_bf16_bits(x.astype(np.float32)).view(np.int16)   # noqa: E731
    check_bf16(gpu, c, of(q), of(k), of(v), [-1], 1, 0.125)
