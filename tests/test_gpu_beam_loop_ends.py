"""Beam search whose beams come to an end: finished beams and places without a candidate take no rows, and no page that another beam needs."""
import numpy as np
import pytest

from oracle import beams as O
from oracle import decoding_loop as D
from test_gpu_beam_loop import G, HEADS, KV, L, S, W, host, make_loop, of_cache, same, wide
from test_gpu_page_attention import bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sink", [(0, 0), (50, 3)])
def test_every_stage_while_beams_finish(gpu, window, sink):
    """Every stage against its definition, fed with what it read on the device; some beams finish on the way."""
    lib, device, torch = gpu
    loop, _ = make_loop(gpu, window=window, sink=sink)
    attn = {}
    for l, layer in enumerate(loop.layers):
        run = layer.attention.run

        def keep(q, out, dtype, ws, stream=None, l=l, run=run):
            run(q, out, dtype, ws, stream)
            attn[l] = (q.clone(), out.clone())
        layer.attention.run = keep
    said, ended, tokens_of = [[] for _ in range(S)], 0, np.zeros(S, np.int64)
    for step in range(140):
        before, score, length, done = of_cache(loop.cache), host(loop.score), host(loop.length), host(loop.finished)
        loop.step()
        torch.cuda.synchronize()
        angles = D.rope_angles(before["len"].astype(np.int64), 64, "plain", 10000.0)
        assert np.abs(host(loop.cos) - np.cos(angles)).max() <= 4 * 2.0 ** -24 and np.abs(host(loop.sin) - np.sin(angles)).max() <= 4 * 2.0 ** -24
        k_new, v_new = (host(t).reshape(L, S, KV, 64) for t in (loop.k_new, loop.v_new))
        if step % 13 == 0 or step in (63, 64, 65, 127, 128, 129):
            for l in range(L):
                q = host(attn[l][0]).reshape(S, HEADS, 64)
                want, size = O.attention(before, l, q, k_new[l], v_new[l], [-1] * S, 1, 0.125, window, sink)
                got = wide(attn[l][1]).reshape(S, HEADS, 64)
                assert np.all(np.abs(got - want) <= bound(size, O.bf16(q), 0.125, 64, 9, want, True) + np.abs(want) * 2.0 ** -8)
        want, ranks = O.beam_select(wide(loop.logits), score, length, done, W, 3, 3, float(np.float32(0.7)))
        for n in ("source", "token", "length", "finished"):
            assert np.array_equal(host({"token": loop.tokens}.get(n, getattr(loop, n, None))), want[n]), (step, n, ranks)
        rows = [[0] if np.isfinite(score[s]) and not done[s] else [-1] for s in range(S)]
        cache, entered = O.append(before, k_new, v_new, 1, rows)
        assert entered == [r[0] + 1 for r in rows] and host(loop.appended).tolist() == [1] * S
        same(of_cache(loop.cache), O.reorder(cache, want["source"], window, sink))
        tokens_of = (tokens_of + entered)[want["source"]]
        said = [said[int(want["source"][s])] + [int(want["token"][s])] for s in range(S)]
        assert np.array_equal(host(loop.cache.len), tokens_of) and np.array_equal(tokens_of, want["length"])
        ended = max(ended, int(done.sum()))
    assert ended == 2                                    # (of 6: what the test is about)
    found = loop.sequences()
    for s in range(S):
        tokens, total = found[s // W][s % W]
        assert tokens == said[s][:len(tokens)] and len(tokens) == host(loop.length)[s] and total == host(loop.score)[s]


def finish(torch, loop, which):
    """The named beams are finished, with scores that keep them where they are."""
    for s in which:
        loop.finished[s], loop.score[s] = 1, -1e-3 * (s % W)


def test_finished_beams_leave_the_pool_to_the_others(gpu):
    """Two of six are finished, and the pool has pages for the other four: the same sequences as with a large pool, and twice over in a graph."""
    lib, device, torch = gpu
    results = []
    for pages in (40, 4):
        loop, _ = make_loop(gpu, 5, pages=pages)
        for _ in range(6):
            loop.step()
        finish(torch, loop, (0, 1))
        held = [loop.cache.len[s].item() for s in (0, 1)]
        for _ in range(20):
            loop.step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            loop.step()
        for i in range(64):
            graph.replay() if i % 7 else loop.step()
        assert loop.finished.tolist()[:2] == [1, 1] and [loop.cache.len[s].item() for s in (0, 1)] == held
        results.append(loop.sequences())
        assert torch.count_nonzero(loop.cache.refs).item() <= 4
    assert results[0] == results[1]


def test_steps_behind_the_end_of_all_beams(gpu):
    """All beams are finished, and further steps go on past what their tables hold: nothing changes any more."""
    lib, device, torch = gpu
    loop, _ = make_loop(gpu, 6, pages=6, columns=1)
    for _ in range(5):
        loop.step()
    finish(torch, loop, range(S))
    loop.step()
    before, found = of_cache(loop.cache), loop.sequences()
    for _ in range(150):
        loop.step()
    same(of_cache(loop.cache), before)
    assert loop.sequences() == found and all(len(tokens) == 5 for group in found for tokens, _ in group)


def test_the_first_step_takes_a_page_for_a_group(gpu):
    """Behind a prompt of 63 tokens one row of each group fills a page; the other beams have no candidates yet, and need none."""
    lib, device, torch = gpu
    loop, bits = make_loop(gpu, 7, pages=G)
    loop.prompt(bits(L, G, 63, KV, 64), bits(L, G, 63, KV, 64))
    loop.start(torch.tensor([1, 2], dtype=torch.int32).cuda())
    loop.step()
    assert len(loop.sequences()) == G and loop.cache.len.tolist() == [64] * S and loop.cache.refs.tolist() == [W] * G


def test_live_beams_without_room_are_still_told(gpu):
    lib, device, torch = gpu
    loop, _ = make_loop(gpu, 5, pages=3)
    for _ in range(6):
        loop.step()
    finish(torch, loop, (0, 1))
    for _ in range(64):
        loop.step()
    with pytest.raises(lib.MloraError):
        loop.sequences()


def test_a_search_behind_a_finished_beam(gpu):
    """What a finished beam holds are its own tokens: a search that goes on from it gives the logits of the sequence without the steps that it sat out."""
    lib, device, torch = gpu
    out = []
    for sat in (0, 70):
        loop, _ = make_loop(gpu, 8)
        for _ in range(9):
            loop.step()
        finish(torch, loop, (0, W))
        for _ in range(sat):
            loop.step()
        loop.start(torch.tensor([7, 8], dtype=torch.int32).cuda())
        loop.step()
        out.append([loop.logits[s].clone() for s in (0, W)] + [loop.cache.len[s].item() for s in (0, W)])
    assert out[0][2:] == out[1][2:] and all(torch.equal(x, y) for x, y in zip(out[0][:2], out[1][:2]))


@pytest.mark.parametrize("pages,columns,most", [(40, 2, 191), (5, 6, 191), (4, 6, 191), (3, 6, 127), (1, 6, 63)])
def test_prompts_that_find_no_room(gpu, pages, columns, most):
    """The longest prompt that a table and the pool (one stream of each of two groups) hold, and one more: refused before anything changes."""
    lib, device, torch = gpu
    loop, bits = make_loop(gpu, 9, pages=pages, columns=columns)
    for _ in range(3):
        loop.step()
    before = of_cache(loop.cache)
    with pytest.raises(lib.MloraError):
        loop.prompt(bits(L, G, most + 1, KV, 64), bits(L, G, most + 1, KV, 64))
    same(of_cache(loop.cache), before)
    loop.step()
    assert len(loop.sequences()) == G
    loop.prompt(bits(L, G, most, KV, 64), bits(L, G, most, KV, 64))
    assert loop.least.tolist() == [1] * S and loop.cache.len.tolist() == [most] * S
