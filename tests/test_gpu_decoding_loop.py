"""The decoding loop on a bounded cache: every new stage of several steps against its definition, fed with what the stage read
on the device; the same steps replayed from a graph and run on another stream."""
import numpy as np
import pytest

import workloads as wl
from oracle import decoding_loop as D
from oracle import ds2d as oracle_ds2d
from workloads.generate import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu

S, L, HEADS, KV, F, V, M_FORECAST, BRANCH, BUDGET, P = 3, 2, 4, 2, 256, 517, 2, (3, 2), 24, 40


def make_loop(gpu, seed=0):
    lib, device, torch = gpu
    from paper_2604_18655_amd.decoding import DecodingLoop
    rng = np.random.default_rng(seed)
    H, KVN = 64 * HEADS, 64 * KV
    mk = lambda name, K, N, l, i: wl.make_problem(wl.ProjShape(name, K, N, 32, 8, 2, 2.0), 5000 + seed, l, i)   # noqa: E731
    up = device.upload_problem
    layers = [[up(mk("q", H, H, l, 0)), up(mk("k", H, KVN, l, 1)), up(mk("v", H, KVN, l, 2)), up(mk("o", H, H, l, 3)),
               up(wl.fuse_gate_up(mk("gate", H, F, l, 4), mk("up", H, F, l, 5))), up(mk("down", F, H, l, 6))] for l in range(L)]
    head = up(mk("head", H, V, 0, 7))
    bits = lambda *shape: torch.from_numpy(f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32)).view(np.int16)).cuda()   # noqa: E731
    adapters = torch.from_numpy(rng.integers(-1, 2, S * 30).astype(np.int32)).cuda()
    masks = rng.integers(0, 1 << 32, (1, (V + 31) // 32), dtype=np.uint32)
    rules = dict(repetition=torch.tensor([1.1, 1.3, 1.0]).cuda(), frequency=torch.tensor([0.1, 0.0, 0.2]).cuda(), presence=torch.tensor([0.0, 0.3, 0.1]).cuda(),
                 bias=torch.from_numpy(rng.standard_normal((1, V)).astype(np.float32)).cuda(), bias_row=torch.tensor([0, -1, 0], dtype=torch.int32).cuda(),
                 masks=torch.from_numpy(masks.view(np.int32)).cuda(),
                 mask_row=torch.tensor(([0] * 30) + ([-1] * 60), dtype=torch.int32).cuda())
    loop = DecodingLoop(layers, head, bits(V, H), bits(M_FORECAST, H), S, BRANCH, BUDGET, sink=2, recent=5, decay=0.97,
                        rope=lib.Rope(64, 64, lib.ROPE_HALF, lib.ROPE_TURNS, 500000.0, factor=8.0), k_prefill=bits(L, KV, P, 64), v_prefill=bits(L, KV, P, 64),
                        row_adapter=adapters, rules=rules)
    loop.start(torch.tensor([3, 100, 7], dtype=torch.int32).cuda())
    return loop, rules, bits


STATE = ("tokens", "emitted", "counts", "n_accepted", "accepted_rows")


def snapshot(loop):
    c = loop.cache
    out = {n: getattr(loop, n).clone() for n in STATE}
    out.update({n: getattr(c, n).clone() for n in ("k", "v", "mass", "slot_pos", "len", "next_pos")})
    out["mass_prefill"] = loop.mass_prefill.clone()
    return out


def restore(loop, state):
    for n in STATE:
        getattr(loop, n).copy_(state[n])
    for n in ("k", "v", "mass", "slot_pos", "len", "next_pos"):
        getattr(loop.cache, n).copy_(state[n])
    loop.mass_prefill.copy_(state["mass_prefill"])


def test_every_stage_of_several_steps(gpu):
    lib, device, torch = gpu
    loop, rules, _ = make_loop(gpu)
    host = lambda t: t.cpu().numpy()   # noqa: E731
    wide = lambda t: bf16_bits_to_f32(host(t).view(np.uint16)).astype(np.float64)   # noqa: E731
    logits = {}
    run_rules = loop.rules.run

    def keep_logits(z, tokens, out, new_tokens=None):
        logits["in"] = wide(z)
        run_rules(z, tokens, out, new_tokens=new_tokens)

    loop.rules.run = keep_logits
    emitted_all = []
    for step in range(30):                                               # (every step gives a row at least: from the 24th on the caches are full)
        before = {k: host(v) for k, v in snapshot(loop).items()}
        loop.step()
        torch.cuda.synchronize()
        # tables: the root stands at next_pos
        pos = (before["next_pos"].astype(np.int64)[:, None] + host(loop.offset)[None, :]).reshape(-1)
        angles = D.rope_angles(pos, 64, "turns", 500000.0, factor=8.0, low=1.0, high=4.0, context=8192.0)
        assert np.abs(host(loop.cos) - np.cos(angles)).max() <= 4 * 2.0 ** -24 and np.abs(host(loop.sin) - np.sin(angles)).max() <= 4 * 2.0 ** -24
        # rules: the tokens given out before are counted first
        kw = {n: host(t) for n, t in rules.items()}
        kw["masks"] = kw["masks"].view(np.uint32)
        want, counts = D.logit_rules(logits["in"], S, 30, 10, host(loop.parent), before["tokens"].tolist(), before["emitted"].tolist(), before["counts"], **kw)
        got = wide(loop.logits)
        assert np.array_equal(host(loop.counts), counts)
        with np.errstate(invalid="ignore"):
            size = np.abs(logits["in"]) * 1.3 + 0.2 * 30 + 0.3 + 4.0
            assert np.all((got == want) | (np.abs(got - want) <= size * 4 * 2.0 ** -24 + np.abs(want) * 2.0 ** -8))
        # the walk on these logits
        for s in range(S):
            ref = oracle_ds2d.step(BRANCH, BRANCH, M_FORECAST, got[s * 30:(s + 1) * 30], before["tokens"][s])
            n = len(ref["emitted"])
            assert host(loop.emitted)[s, :n].tolist() == ref["emitted"] and np.all(host(loop.emitted)[s, n:] == -1)
            assert host(loop.tokens)[s].tolist() == ref["next_tokens"]
            emitted_all.append(n)
        # the accepted rows in the caches (masses aside, which the weights change at once)
        rows = host(loop.accepted_rows).tolist()
        k_new, v_new = (host(t).reshape(L, S * 30, KV, 64) for t in (loop.k_new, loop.v_new))
        cache = {n: before[n] for n in ("k", "v", "mass", "slot_pos", "len", "next_pos")}
        ref = D.append(cache, k_new, v_new, 30, rows, BUDGET, 2, 5)
        for n in ("k", "v", "slot_pos", "len", "next_pos"):
            assert np.array_equal(host(getattr(loop.cache, n)), ref[n]), n
        # their weights
        as_wide = lambda a: bf16_bits_to_f32(np.ascontiguousarray(a).view(np.uint16)).astype(np.float64)   # noqa: E731
        k, q, kp = as_wide(ref["k"]), wide(loop.q).reshape(L, S * 30, HEADS, 64), wide(loop.keep[0])
        want, shared = D.attention_mass(k, ref["mass"], ref["slot_pos"], ref["len"], ref["next_pos"], q, 30, rows, loop.scale, float(np.float32(0.97)), kp,
                                        before["mass_prefill"])
        norm = lambda a: np.sqrt((a ** 2).sum(-1)).max()   # noqa: E731
        rel = 2 * 66 * 2.0 ** -23 * loop.scale * norm(q) * max(norm(k), norm(kp)) + (8 + 16) * 2.0 ** -23
        for g, w in ((host(loop.cache.mass), want), (host(loop.mass_prefill), shared)):
            assert np.all(np.abs(g - w) <= np.abs(w) * (rel + 2.0 ** -22) + 1e-37)
    assert int(loop.cache.len.min()) == BUDGET and int(loop.cache.next_pos.min()) >= 30


def run_steps(loop, n):
    given = []
    for _ in range(n):
        loop.step()
        given.append(loop.emitted.clone())
    return given


def test_steps_replayed_from_a_graph(gpu):
    """A captured step replayed, with eager steps and synchronisations in between, gives the eager run's bits."""
    lib, device, torch = gpu
    loop, _, _ = make_loop(gpu, 1)
    run_steps(loop, 20)                                                  # (caches nearly full)
    start = snapshot(loop)
    eager = run_steps(loop, 12)
    torch.cuda.synchronize()
    end = snapshot(loop)
    restore(loop, start)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.step()
    restore(loop, start)
    given = []
    for i in range(12):
        if i % 3 == 2:
            loop.step()
        else:
            graph.replay()
        given.append(loop.emitted.clone())
        if i % 4 == 1:
            torch.cuda.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(eager, given):
        assert torch.equal(a, b)
    for n, t in snapshot(loop).items():
        assert torch.equal(t, end[n]), n


def test_steps_on_another_stream(gpu):
    lib, device, torch = gpu
    loop, _, _ = make_loop(gpu, 2)
    run_steps(loop, 22)
    start = snapshot(loop)
    eager = run_steps(loop, 6)
    end = snapshot(loop)
    restore(loop, start)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        given = run_steps(loop, 6)
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, given))
    for n, t in snapshot(loop).items():
        assert torch.equal(t, end[n]), n


def test_a_prompt_enters_compressed(gpu):
    """Prompts of 70 tokens into caches of 24 slots: the turned keys of the heaviest, in order; then steps go on behind them."""
    lib, device, torch = gpu
    loop, _, bits = make_loop(gpu, 3)
    N, window = 70, 16
    q, k, v = bits(L, S, N, HEADS, 64), bits(L, S, N, KV, 64), bits(L, S, N, KV, 64)
    kept = loop.prompt(q, k, v, window).cpu().numpy()
    torch.cuda.synchronize()
    wide = lambda t: bf16_bits_to_f32(t.cpu().numpy().view(np.uint16)).astype(np.float64)   # noqa: E731
    angles = D.rope_angles(np.arange(N), 64, "turns", 500000.0, factor=8.0, low=1.0, high=4.0, context=8192.0)
    assert np.all(kept[..., 1:] > kept[..., :-1]) and np.all(kept[..., -5:] == np.arange(N - 5, N)) and np.all(kept[..., :2] == [0, 1])
    assert torch.all(loop.cache.len == BUDGET) and torch.all(loop.cache.next_pos == N)
    assert np.array_equal(loop.cache.slot_pos.cpu().numpy(), kept)
    cache_k, cache_v, mass = wide(loop.cache.k), wide(loop.cache.v), loop.cache.mass.cpu().numpy()
    for l in range(L):
        for s in range(S):
            turned = D.rope(wide(k[l, s]), angles, 64, False)
            tq = D.rope(wide(q[l, s]), angles, 64, False)
            for h in range(KV):
                at = kept[l, s, h]
                assert np.array_equal(cache_v[l, s, h], wide(v[l, s])[at, h])
                assert np.all(np.abs(cache_k[l, s, h] - turned[at, h]) <= np.abs(turned[at, h]) * 2.0 ** -8 + 2.0 ** -20)
                # the weights of the last rows, on keys and queries that were rounded to bf16: half a step each, 64 products
                got = np.zeros(N)
                for r in range(N - window, N):
                    for g in range(HEADS // KV):
                        x = turned[:r + 1, h] @ tq[r, h * (HEADS // KV) + g] * loop.scale
                        e = np.exp(x - x.max())
                        got[:r + 1] += e / e.sum()
                far = 2 * (2 * 2.0 ** -8) * loop.scale * 64 ** 0.5 * np.sqrt((turned ** 2).sum(-1)).max() * np.sqrt((tq ** 2).sum(-1)).max() / 8
                assert np.all(np.abs(mass[l, s, h] - got[at]) <= got[at] * (np.exp(far) - 1) + 1e-6)
                light = np.setdiff1d(np.arange(N), at)
                assert got[light].max() <= got[at[2:-5]].min() * np.exp(2 * far)
    loop.start(torch.tensor([1, 2, 3], dtype=torch.int32).cuda())
    run_steps(loop, 4)
    torch.cuda.synchronize()
    assert torch.all(loop.cache.next_pos >= N + 4) and torch.all(loop.cache.len == BUDGET)
