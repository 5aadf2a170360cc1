"""The paged cache of 8 bits on the GPU: rows that enter, streams that become others, copies.  Codes, scales, pages and lengths match the
definition bit for bit (127 x / m is a quotient of numbers of 15 and 8 bits: no rounding to fp32 carries it over a half)."""
import numpy as np
import pytest

from oracle import beams as O
from workloads.generate import f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def bits(rng, *shape, scale=1.0):
    return f32_to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32)).view(np.int16)


def upload(gpu, c):
    lib, _, torch = gpu
    t = {n: torch.from_numpy(a.copy()).cuda() for n, a in c.items()}
    return t, lib.PageCache(*(t[n] for n in O.FIELDS))


def same(t, want):
    for n in O.FIELDS:
        a, b = t[n].cpu().numpy(), want[n]
        if a.dtype == np.float32:
            assert np.array_equal(np.isnan(a), np.isnan(b)), n
            a, b = (np.where(np.isnan(x), np.float32(0), x).view(np.int32) for x in (a, b))
        assert np.array_equal(a, b), n


def make(seed, L, S, H, D, pages, columns, lengths, used=()):
    """Streams that hold random pages, in any slots; `used`: pages that somebody else holds."""
    rng = np.random.default_rng(seed)
    c = O.empty_cache(L, S, H, D, pages, columns)
    for n in ("k", "v"):
        c[n][:] = rng.integers(-127, 128, c[n].shape)
        c[n + "_scale"][:] = rng.uniform(0.01, 0.03, c[n + "_scale"].shape)
        c[n + "_tail"][:] = bits(rng, *c[n + "_tail"].shape)
    c["slot"][:], c["len"][:] = rng.permutation(S), lengths
    free = [p for p in rng.permutation(pages) if p not in set(used)]
    for s in range(S):
        for i in range(lengths[s] // 64):
            c["table"][c["slot"][s], i] = free.pop()
    c["refs"][:] = np.bincount(c["table"][c["table"] >= 0], minlength=pages)
    c["refs"][list(used)] = 1
    return c


def check_append(gpu, c, R, rows, seed=0, calls=1, values=None):
    lib, _, torch = gpu
    t, cache = upload(gpu, c)
    rng = np.random.default_rng(seed)
    L, S, H, D = c["k_tail"].shape[0], len(c["len"]), c["k_tail"].shape[2], c["k_tail"].shape[4]
    entered = torch.full((S,), -7, dtype=torch.int32).cuda()
    on = None if rows is None else torch.tensor(rows, dtype=torch.int32).cuda()
    for _ in range(calls):
        k, v = (bits(rng, L, S * R, H, D) if values is None else values(rng, (L, S * R, H, D)) for _ in range(2))
        cache.append(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), R, on, entered)
        torch.cuda.synchronize()
        c, n = O.append(c, k, v, R, rows)
        assert entered.tolist() == n
        same(t, c)
    return c


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("length", [0, 1, 62, 63, 64, 127, 130])
@pytest.mark.parametrize("n", [1, 2, 65])
def test_rows_of_a_step(gpu, D, length, n):
    check_append(gpu, make(1, 2, 2, 3, D, 17, 5, [length, 33]), n, None)


@pytest.mark.parametrize("n", [63, 64, 128, 200, 1001])
def test_prompts(gpu, n):
    check_append(gpu, make(2, 1, 3, 2, 64, 60, 18, [0, 5, 64]), n, None)


def test_the_longest_prompt(gpu):
    check_append(gpu, make(3, 1, 1, 1, 128, 66, 65, [63]), 4096, None)


def test_lists(gpu):
    """Entries count up to the first that names no row; the same row may enter twice."""
    rows = [[3, 1, 1], [-1, 2, 2], [0, 4, 1], [2, 3, 9]]
    check_append(gpu, make(4, 3, 4, 2, 64, 20, 4, [61, 63, 62, 200]), 4, rows, calls=3)


def test_one_row_after_the_other(gpu):
    check_append(gpu, make(5, 1, 2, 1, 64, 9, 3, [0, 40]), 1, None, calls=150)


def test_no_room(gpu):
    """Whole streams or nothing: columns that are used up, a pool that is."""
    c = check_append(gpu, make(6, 1, 5, 2, 64, 4, 2, [191, 10, 60, 63, 0]), 8, [[0] * 8, [1] * 8, [2] * 8, [3] * 8, [4] * 8], calls=1)
    assert c["len"].tolist() == [191, 18, 68, 71, 8]
    c = check_append(gpu, make(7, 1, 5, 2, 64, 4, 4, [128, 10, 60, 63, 0]), 8, [[0] * 8, [1] * 8, [2] * 8, [3] * 8, [4] * 8], calls=1)
    assert c["len"].tolist() == [136, 18, 68, 71, 8]
    c = check_append(gpu, make(8, 1, 5, 2, 64, 4, 4, [60, 10, 130, 63, 0], used=[1]), 70, None)
    assert c["len"].tolist() == [60, 10, 130, 63, 0]      # (two pages are held, one is not free: the first finds one page of two)


def test_many_streams(gpu):
    rng = np.random.default_rng(9)
    lengths = [int(x) for x in rng.integers(0, 200, 1024)]
    check_append(gpu, make(9, 1, 1024, 1, 64, 5000, 4, lengths), 1, None, calls=2)
    check_append(gpu, make(10, 1, 1000, 1, 64, 9000, 5, [0] * 1000), 4, None, calls=1)


@pytest.mark.parametrize("S", [64, 65, 255, 256, 257])
@pytest.mark.parametrize("n", [1, 63, 64, 65])
def test_calls_of_one_launch_and_of_two(gpu, S, n):
    """Streams and rows at the borders, streams that fill a page beside others that do not, and a pool that ends among them."""
    if S * n > 4096:
        n = 4096 // S
    rng = np.random.default_rng(S + n)
    lengths = [int(x) for x in rng.integers(0, 130, S)]
    check_append(gpu, make(S, 1, S, 2, 64, 3 * S // 2 + 40, 4, lengths), n, None, calls=3)
    check_reorder(gpu, make(S, 1, S, 2, 64, 2 * S, 3, lengths), rng.integers(-1, S, S).tolist(), 20, 3, calls=3)


def test_pages_are_taken_from_the_lowest_on(gpu):
    """A pool of several looks, with holes; and one that has none."""
    used = [p for p in range(9001) if p % 4099 != 7 and p != 9000]
    c = check_append(gpu, make(11, 1, 2, 1, 64, 9001, 4, [63, 63], used=used), 65, None)
    assert sorted(c["table"][c["table"] >= 0].tolist()) == [7, 4106, 8205, 9000]
    c = check_append(gpu, make(12, 1, 2, 1, 64, 9001, 4, [63, 62], used=range(9001)), 1, None)
    assert c["len"].tolist() == [63, 63]


@pytest.mark.parametrize("S", [3, 60])
@pytest.mark.parametrize("free", [[], [0, 39999], [39998, 39999], [1023, 1024, 20000], [5, 8192 + 1024, 8192 + 1025], [33791, 33792, 33793], list(range(30000, 40000, 17))])
def test_few_free_pages_in_a_large_pool(gpu, S, free):
    c = make(62, 1, S, 1, 64, 40000, 5, [63, 3, 127] + [10] * (S - 3))
    c["refs"] += 1
    c["refs"][free] -= 1
    check_append(gpu, c, 1, None, calls=2)
    check_append(gpu, c, 64, None)
    check_append(gpu, c, 65, None)


@pytest.mark.parametrize("S", [3, 300])
@pytest.mark.parametrize("pages", [200, 8193, 8200])
def test_a_full_pool_is_searched_once(gpu, pages, S):
    """Three streams fill a page each, and two pages are free.  A search that came to the pool's end is not made again, until pages are given up: then
    those are found."""
    lib, _, torch = gpu
    most = (pages - 9) // 2
    c = make(63, 1, S, 1, 64, pages, most + 3, [64 * (pages - 9 - most) + 63, 64 * 7 + 63, 64 * most + 63] + [5] * (S - 3))
    given_up = sorted(c["table"][c["slot"][1], :7].tolist())
    assert np.count_nonzero(c["refs"] == 0) == 2
    t, cache = upload(gpu, c)
    k, v = (bits(np.random.default_rng(63), 1, S, 1, 64) for _ in range(2))
    on = [torch.from_numpy(x).cuda() for x in (k, v)]
    entered = torch.zeros(S, dtype=torch.int32).cuda()

    def check(c, n, ahead):
        torch.cuda.synchronize()
        assert entered.tolist() == n and cache.own[0].item() == ahead
        same(t, c)
        return c
    for _ in range(3):                                   # (the first two streams go on behind the pages that they got)
        cache.append(*on, 1, None, entered)
        c, n = O.append(c, k, v, 1)
        assert n == [1, 1, 0] + [1] * (S - 3)
        c = check(c, n, pages)
    given_up = sorted(given_up + [int(c["table"][c["slot"][1], 7])])
    source = [0, -1] + list(range(2, S))
    cache.reorder(torch.tensor(source, dtype=torch.int32).cuda())
    c = check(O.reorder(c, source), n, given_up[0])
    cache.append(*on, 1, None, entered)
    c, n = O.append(c, k, v, 1)
    assert n == [1] * S and c["table"][c["slot"][2], most] == given_up[0]
    check(c, n, given_up[0] + 1)                         # (behind the page taken)


def test_odd_numbers(gpu):
    """Zeros, subnormals, the largest, infinities, NaN; ties (127 x / m in halves)."""
    some = {0: 0x0000, 1: 0x8000, 2: 0x0001, 3: 0x807F, 4: 0x7F7F, 5: 0x7F80, 6: 0xFF80, 7: 0x7FC0, 8: 0x3F80, 9: 0xBF00, 10: 0x0080}
    for seed, pick in enumerate([[0, 1], [0, 2, 3], [2, 3, 10], [4, 8, 9], [8, 9], [5, 8], [6, 8], [7, 8], [4, 0, 2]]):
        def values(rng, shape):
            out = np.array([some[i] for i in pick], np.uint16)[rng.integers(0, len(pick), shape)]
            return np.ascontiguousarray(out).view(np.int16)
        check_append(gpu, make(20 + seed, 1, 1, 3, 64, 4, 3, [0]), 70, None, seed=seed, values=values)
    halves = lambda rng, shape: f32_to_bf16_bits((rng.integers(-254, 255, shape) / 2 * 2.0 ** -3).astype(np.float32)).view(np.int16)   # noqa: E731
    check_append(gpu, make(30, 1, 1, 3, 128, 4, 3, [0]), 128, None, values=halves)


def check_reorder(gpu, c, source, window=0, sink=0, calls=1):
    lib, _, torch = gpu
    t, cache = upload(gpu, c)
    on = None if source is None else torch.tensor(source, dtype=torch.int32).cuda()
    for _ in range(calls):
        cache.reorder(on, window, sink)
        torch.cuda.synchronize()
        c = O.reorder(c, source, window, sink)
        same(t, c)
    return c


@pytest.mark.parametrize("source", [[0, 1, 2, 3], [3, 2, 1, 0], [1, 1, 1, 1], [-1, -1, -1, -1], [2, -1, 2, 9], [1, 0, 0, 1], None])
@pytest.mark.parametrize("window,sink", [(0, 0), (1, 0), (70, 0), (100, 65), (5000, 1)])
def test_streams_become_others(gpu, source, window, sink):
    check_reorder(gpu, make(40, 2, 4, 2, 64, 40, 9, [300, 64, 63, 512]), source, window, sink, calls=3)


def test_empty_streams_and_long_tables(gpu):
    check_reorder(gpu, make(41, 1, 3, 1, 128, 700, 700, [0, 64 * 600 + 5, 64 * 20]), [1, 0, 1], 64 * 300, 130, calls=2)


def test_a_thousand_streams(gpu):
    rng = np.random.default_rng(42)
    check_reorder(gpu, make(42, 1, 1024, 1, 64, 2500, 4, [int(x) for x in rng.integers(0, 150, 1024)]), rng.integers(-3, 1030, 1024).tolist(), calls=2)


def check_copy(gpu, c, to, source):
    lib, _, torch = gpu
    t, cache = upload(gpu, c)
    o, other = upload(gpu, to)
    used = torch.full((1,), -5, dtype=torch.int32).cuda()
    for _ in range(2):
        other.copy_from(cache, torch.tensor(source, dtype=torch.int32).cuda(), used)
        torch.cuda.synchronize()
        to, n = O.copy(c, to, source)
        assert used.item() == n
        same(o, to)
        same(t, c)
    return to


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("source", [[0], [3, 1, 0], [2, 2, 2, 2, 2], [-1, 1, 77], [4]])
def test_copies(gpu, D, source):
    c = O.reorder(make(50, 2, 5, 3, D, 40, 9, [300, 64, 63, 512, 0]), [0, 0, 2, 3, 0])
    check_copy(gpu, c, make(51, 2, len(source), 3, D, 30, 11, [70] * len(source)), source)


@pytest.mark.parametrize("pages,table", [(41, 9), (60, 9), (500, 40)])
def test_copies_into_larger_pools(gpu, pages, table):
    c = O.reorder(make(56, 2, 5, 3, 64, 40, 9, [300, 64, 63, 512, 0]), [0, 0, 2, 3, 0])
    for source in ([0, 1, 2, 3, 4], [3, 3], [-1, 2]):
        to = check_copy(gpu, c, make(57, 2, len(source), 3, 64, pages, table, [70] * len(source)), source)
        assert to["len"].tolist() == [max(0, c["len"][i]) if i >= 0 else 0 for i in source]


@pytest.mark.parametrize("most", [1024, 4096, 4097, 9000])
def test_copies_out_of_large_pools(gpu, most):
    """Pages anywhere in the pool, the last one among them; more than one thread's share of entries."""
    c = make(58, 1, 3, 1, 64, 9000, 900, [64 * 700 + 3, 64 * 800, 64 * 5])
    rng = np.random.default_rng(most)
    to_page = rng.permutation(most)[:1505]
    to_page[0] = most - 1 if most - 1 not in to_page else to_page[0]
    if most < 1505:
        to_page = np.arange(1505) % most                                                 # (many held more than once)
    at = 0
    c["refs"][:], c["table"][:] = 0, -1
    for s, n in enumerate((700, 800, 5)):
        c["table"][c["slot"][s], :n] = to_page[at:at + n]
        at += n
    np.add.at(c["refs"], to_page, 1)
    check_copy(gpu, c, make(59, 1, 3, 1, 64, 1600, 900, [70, 3, 0]), [2, 0, 1])
    check_copy(gpu, c, make(59, 1, 2, 1, 64, 9000, 900, [70, 3]), [2, -1])


def test_copies_of_more_pages_than_blocks(gpu):
    c = make(60, 16, 2, 1, 64, 700, 400, [64 * 390 + 1, 64 * 210])
    check_copy(gpu, c, make(61, 16, 2, 1, 64, 650, 400, [70, 3]), [1, 0])


def test_copies_that_find_no_room(gpu):
    c = make(52, 1, 2, 2, 64, 40, 9, [300, 512])
    to = check_copy(gpu, c, make(53, 1, 2, 2, 64, 11, 9, [70, 3]), [0, 1])
    assert to["len"].tolist() == [0, 0] and to["refs"].max() == 0
    to = check_copy(gpu, c, make(54, 1, 2, 2, 64, 12, 7, [70, 3]), [0, 1])
    assert to["len"].tolist() == [0, 0]
    to = check_copy(gpu, c, make(55, 1, 2, 2, 64, 12, 8, [70, 3]), [0, 1])
    assert to["len"].tolist() == [300, 512]


def test_pages_that_no_table_should_name(gpu):
    """Entries outside the pool hold nothing: they are neither counted nor read."""
    c = make(56, 1, 3, 1, 64, 20, 6, [300, 200, 64])
    c["table"][c["slot"][0], 1], c["table"][c["slot"][1], 0] = 20, -9
    c["refs"][:] = np.bincount(c["table"][(c["table"] >= 0) & (c["table"] < 20)], minlength=20)
    check_reorder(gpu, c, [0, 0, 1], 0, 0)
    check_copy(gpu, c, O.empty_cache(1, 2, 1, 64, 20, 6), [1, 0])


@pytest.mark.parametrize("seed", range(4))
def test_a_life(gpu, seed):
    """Rows, reorderings and windows in any order, eager, and the whole of it again from a graph."""
    lib, _, torch = gpu
    rng = np.random.default_rng(60 + seed)
    L, S, H, D, R = 2, 6, 2, 64 * (1 + seed % 2), 40
    start = make(60 + seed, L, S, H, D, 30, 8, [int(x) for x in rng.integers(0, 130, S)])
    t, cache = upload(gpu, start)
    calls, c = [], start
    for _ in range(14):
        if rng.random() < 0.5:
            new = [bits(rng, L, S * R, H, D) for _ in range(2)]
            rows = rng.integers(0, R, (S, 37))
            rows[np.arange(37) >= rng.integers(0, 38, S)[:, None]] = -1
            on = [torch.from_numpy(x).cuda() for x in new] + [torch.from_numpy(rows.astype(np.int32)).cuda()]
            calls.append(lambda on=on: cache.append(on[0], on[1], R, on[2]))
            c = O.append(c, *new, R, rows.tolist())[0]
        else:
            source = rng.integers(-1, S, S)
            window, sink = int(rng.choice([0, 60, 150])), int(rng.choice([0, 3, 64]))
            on = torch.from_numpy(source.astype(np.int32)).cuda()
            calls.append(lambda on=on, window=window, sink=sink: cache.reorder(on, window, sink))
            c = O.reorder(c, source, window, sink)
        calls[-1]()
        torch.cuda.synchronize()
        same(t, c)
    again = torch.cuda.Stream()
    first = {n: torch.from_numpy(a.copy()).cuda() for n, a in start.items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=again):
        for n in O.FIELDS:
            t[n].copy_(first[n])
        cache.own[:1].zero_()                            # (refs was written: the search for free pages starts over)
        for call in calls:
            call()
    for _ in range(3):
        for n in O.FIELDS:
            t[n].fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        same(t, c)


def test_going_back_to_a_state_that_was_kept(gpu):
    """All tensors of the cache are written from outside: the pages below where the search for free ones had come to are found again, in a pool that
    has no others; eager and in a graph."""
    lib, _, torch = gpu
    start = make(72, 1, 3, 2, 64, 7, 5, [63, 64, 5])
    t, cache = upload(gpu, start)
    first = {n: x.clone() for n, x in t.items()}
    rng = np.random.default_rng(72)
    k, v = (bits(rng, 1, 3 * 63, 2, 64) for _ in range(2))
    on = [torch.from_numpy(x).cuda() for x in (k, v)]
    want, full = start, []
    for _ in range(3):
        want, n = O.append(want, k, v, 63)
        full.append(n)
    assert full == [[63, 63, 63], [63, 63, 63], [63, 0, 0]] and want["refs"].min() == 1

    def again():
        for n in O.FIELDS:
            t[n].copy_(first[n])
        cache.refs_written()
        for _ in range(3):
            cache.append(*on, 63)
    again()
    for _ in range(2):
        again()
        torch.cuda.synchronize()
        same(t, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        again()
    for _ in range(3):
        for n in O.FIELDS:
            t[n].fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        same(t, want)


def test_offsets_past_32_bits(gpu):
    """A pool of 2.3 GB of keys, all but its last pages taken."""
    lib, _, torch = gpu
    pages, H, D = 36000, 16, 64
    cache = lib.PageCache.empty(1, 2, H, D, pages, 3)
    cache.refs[:-3] = 1
    rng = np.random.default_rng(70)
    k, v = (bits(rng, 1, 2 * 70, H, D) for _ in range(2))
    cache.append(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), 70)
    other = lib.PageCache.empty(1, 1, H, D, 2, 3)
    other.copy_from(cache, torch.tensor([1], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    want, _ = O.append(O.empty_cache(1, 2, H, D, 3, 3), k, v, 70)
    for n in ("k", "v", "k_scale", "v_scale"):
        got = getattr(cache, n)[:, -3:].cpu().numpy()
        assert np.array_equal(got[:, :2], want[n][:, :2]), n
        assert np.array_equal(getattr(other, n)[:, 0].cpu().numpy(), want[n][:, 1]), n
    assert cache.table.tolist() == [[pages - 3, -1, -1], [pages - 2, -1, -1]] and other.table.tolist() == [[0, -1, -1]]
