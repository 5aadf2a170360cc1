"""Beam search on a paged cache as a whole: every new stage of several steps against its definition, fed with what the stage read on the device;
the same steps replayed from a graph and run on another stream; prompts, windows, and pools that are too small."""
import numpy as np
import pytest

import workloads as wl
from oracle import beams as O
from oracle import decoding_loop as D
from test_gpu_page_attention import bound
from workloads.generate import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu

G, W, L, HEADS, KV, F, V = 2, 3, 2, 4, 2, 256, 517
S = G * W


def make_loop(gpu, seed=0, pages=40, columns=6, max_steps=200, **kw):
    lib, device, torch = gpu
    from paper_2604_18655_amd.beams import BeamLoop
    rng = np.random.default_rng(seed)
    H, KVN = 64 * HEADS, 64 * KV
    mk = lambda name, K, N, l, i: wl.make_problem(wl.ProjShape(name, K, N, 32, 8, 2, 2.0), 7000 + seed, l, i)   # noqa: E731
    up = device.upload_problem
    layers = [[up(mk("q", H, H, l, 0)), up(mk("k", H, KVN, l, 1)), up(mk("v", H, KVN, l, 2)), up(mk("o", H, H, l, 3)),
               up(wl.fuse_gate_up(mk("gate", H, F, l, 4), mk("up", H, F, l, 5))), up(mk("down", F, H, l, 6))] for l in range(L)]
    head = up(mk("head", H, V, 0, 7))
    bits = lambda *shape: torch.from_numpy(f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32)).view(np.int16)).cuda()   # noqa: E731
    adapters = torch.from_numpy(rng.integers(-1, 2, S).astype(np.int32)).cuda()
    loop = BeamLoop(layers, head, bits(V, H), G, W, pages, columns, max_steps, eos=3, length_power=0.7, row_adapter=adapters, **kw)
    loop.start(torch.tensor([5, 100], dtype=torch.int32).cuda())
    return loop, bits


host = lambda t: t.cpu().numpy()   # noqa: E731
wide = lambda t: bf16_bits_to_f32(host(t).view(np.uint16)).astype(np.float64)   # noqa: E731


def of_cache(c):
    import torch
    of = lambda t: t.view(torch.int16) if t.dtype == torch.bfloat16 else t   # noqa: E731
    return {n: host(of(getattr(c, n))).copy() for n in O.FIELDS}


def same(got, want):
    for n in O.FIELDS:
        assert np.array_equal(got[n], want[n]), n


@pytest.mark.parametrize("window,sink", [(0, 0), (50, 3)])
def test_every_stage_of_many_steps(gpu, window, sink):
    lib, device, torch = gpu
    loop, _ = make_loop(gpu, window=window, sink=sink)
    attn = {}
    for l, layer in enumerate(loop.layers):
        run = layer.attention.run

        def keep(q, out, dtype, ws, stream=None, l=l, run=run):
            run(q, out, dtype, ws, stream)
            attn[l] = (q.clone(), out.clone())
        layer.attention.run = keep
    said = [[] for _ in range(S)]
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
                assert np.all(np.abs(got - want) <= bound(size, O.bf16(q), 0.125, 64, 9, want, False))
        z = wide(loop.logits)
        want, ranks = O.beam_select(z, score, length, done, W, 3, 3, float(np.float32(0.7)))
        for n in ("source", "token", "length", "finished"):
            assert np.array_equal(host({"token": loop.tokens}.get(n, getattr(loop, n, None))), want[n]), (step, n, ranks)
        cache, entered = O.append(before, k_new, v_new, 1)
        assert host(loop.appended).tolist() == entered == [1] * S
        same(of_cache(loop.cache), O.reorder(cache, want["source"], window, sink))
        said = [said[int(want["source"][s])] + [int(want["token"][s])] for s in range(S)]
    found = loop.sequences()
    for s in range(S):
        tokens, total = found[s // W][s % W]
        assert tokens == said[s][:len(tokens)] and len(tokens) == host(loop.length)[s] and total == host(loop.score)[s]
    if window:
        held = of_cache(loop.cache)
        assert np.count_nonzero(held["refs"]) <= S * 2 + 1 and np.all(held["len"] == 140)


STATE = ("tokens", "score", "length", "finished", "source", "trace", "steps", "least")


def snapshot(loop):
    out = {n: getattr(loop, n).clone() for n in STATE}
    out.update({"cache." + n: getattr(loop.cache, n).clone() for n in O.FIELDS + ("own",)})
    return out


def restore(loop, state):
    for n, t in state.items():
        (getattr(loop.cache, n[6:]) if n.startswith("cache.") else getattr(loop, n)).copy_(t)


def test_replays_with_eager_work_between(gpu):
    lib, device, torch = gpu
    loop, _ = make_loop(gpu, 1)
    for _ in range(60):
        loop.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    start = snapshot(loop)
    for _ in range(12):
        loop.step()
    eager = snapshot(loop)
    restore(loop, start)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        loop.step()
    for _ in range(2):
        restore(loop, start)
        for i in range(12):
            if i % 5 == 4:
                loop.step()
            else:
                graph.replay()
            torch.cuda.synchronize()
            torch.zeros(1 << 16).cuda().sum().item()
        for n, t in snapshot(loop).items():
            if n != "cache.own":
                assert torch.equal(t, eager[n]), n


def test_steps_on_another_stream(gpu):
    lib, device, torch = gpu
    loop, _ = make_loop(gpu, 2)
    for _ in range(55):
        loop.step()
    start = snapshot(loop)
    for _ in range(15):
        loop.step()
    eager = snapshot(loop)
    restore(loop, start)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        for _ in range(15):
            loop.step()
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    for n, t in snapshot(loop).items():
        assert torch.equal(t, eager[n]), n


def test_prompts(gpu):
    """Prompts of 150 tokens: turned keys and values in the pages, once for all beams of a group; then steps behind them; then another prompt in their
    place."""
    lib, device, torch = gpu
    loop, bits = make_loop(gpu, 3)
    for N in (150, 64, 1):
        k, v = bits(L, G, N, KV, 64), bits(L, G, N, KV, 64)
        loop.prompt(k, v)
        torch.cuda.synchronize()
        c = of_cache(loop.cache)
        assert np.all(c["len"] == N) and np.count_nonzero(c["refs"]) == G * (N // 64) and (N < 64 or c["refs"].max() == W)
        angles = D.rope_angles(np.arange(N), 64, "plain", 10000.0)
        for l in range(L):
            for s in range(S):
                turned = D.rope(wide(k[l, s // W]), angles, 64, False)
                for h in range(KV):
                    where, keys, values = O.tokens_of(c, l, s, h)
                    assert np.array_equal(where, np.arange(N))
                    exact = wide(v[l, s // W])[:, h]
                    for i in range(0, N, 64):
                        full = i + 64 <= N
                        for got, want, off in ((keys, turned[:, h], 1), (values, exact, 0)):
                            x, y = got[i:i + 64], want[i:i + 64]
                            top = np.abs(y).max() * (1 + off * 2.0 ** -8)
                            # half a scale on full pages; the turned keys are rounded to bf16 before
                            assert np.all(np.abs(x - y) <= (0.5 * top / 127 * (1 + 255 * 2.0 ** -24) if full else 0) + off * (np.abs(y) * 2.0 ** -8 + 2.0 ** -20))
        loop.start(torch.tensor([1, 2], dtype=torch.int32).cuda())
        for _ in range(4):
            loop.step()
        torch.cuda.synchronize()
        assert torch.all(loop.cache.len == N + 4)
        assert all(len(tokens) <= 4 and np.isfinite(score) for group in loop.sequences() for tokens, score in group)
    for bad in ((bits(L, G, 0, KV, 64),) * 2, (bits(L, G, 5, KV, 64), bits(L, G, 4, KV, 64)), (bits(L, G + 1, 5, KV, 64),) * 2):
        with pytest.raises(lib.MloraError):
            loop.prompt(*bad)


def test_a_pool_that_is_too_small_is_told(gpu):
    lib, device, torch = gpu
    loop, _ = make_loop(gpu, 4, pages=2)
    for _ in range(70):
        loop.step()
    with pytest.raises(lib.MloraError):
        loop.sequences()
    loop.reset()
    loop.start(torch.tensor([1, 2], dtype=torch.int32).cuda())
    loop.step()
    assert len(loop.sequences()) == G
    loop, _ = make_loop(gpu, 4, max_steps=3)
    for _ in range(4):
        loop.step()
    with pytest.raises(lib.MloraError):
        loop.sequences()
