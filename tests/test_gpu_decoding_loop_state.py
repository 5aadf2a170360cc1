"""What a decoding loop keeps from call to call: where its rows stand beside a shared prefix, the weights that a prompt's slots enter with,
the normalised rows that the head takes, and a second generation on the same loop."""
import numpy as np
import pytest

import test_gpu_decoding_loop as T
import workloads as wl
from oracle import decoding_loop as D
from workloads.generate import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu

S, L, HEADS, KV, BUDGET = T.S, T.L, T.HEADS, T.KV, T.BUDGET
SCALING = dict(factor=8.0, low=1.0, high=4.0, context=8192.0)


def make_loop(gpu, monkeypatch, seed, P):
    monkeypatch.setattr(T, "P", P)
    return T.make_loop(gpu, seed)


def wide(t):
    return bf16_bits_to_f32(t.cpu().numpy().view(np.uint16)).astype(np.float64)


def angles(positions):
    return D.rope_angles(positions, 64, "turns", 500000.0, **SCALING)


@pytest.mark.parametrize("P", [40, 0])
def test_rows_stand_behind_the_prefix(gpu, monkeypatch, P):
    """The first token of a stream stands at position P: the prefix holds 0 .. P - 1."""
    lib, device, torch = gpu
    loop, _, _ = make_loop(gpu, monkeypatch, 4, P)
    depth = []
    for up in loop.parent.tolist()[:30]:
        depth.append(0 if up < 0 else depth[up] + 1)
    given = np.zeros(S, np.int64)
    for _ in range(4):
        loop.step()
        torch.cuda.synchronize()
        want = angles((P + given[:, None] + np.asarray(depth)[None, :]).reshape(-1))
        assert np.abs(loop.cos.cpu().numpy() - np.cos(want)).max() <= 4 * 2.0 ** -24
        assert np.abs(loop.sin.cpu().numpy() - np.sin(want)).max() <= 4 * 2.0 ** -24
        given += (loop.emitted >= 0).sum(1).cpu().numpy()


@pytest.mark.parametrize("P", [40, 0])
def test_a_prompts_keys_stand_behind_the_prefix(gpu, monkeypatch, P):
    """Turned by their places in one sequence of prefix and prompt; bf16's half step.  Steps go on behind them."""
    lib, device, torch = gpu
    loop, _, bits = make_loop(gpu, monkeypatch, 5, P)
    N = 70
    k = bits(L, S, N, KV, 64)
    kept = loop.prompt(bits(L, S, N, HEADS, 64), k, bits(L, S, N, KV, 64), 16).cpu().numpy()
    torch.cuda.synchronize()
    place, cache_k = angles(P + np.arange(N)), wide(loop.cache.k)
    for l in range(L):
        for s in range(S):
            turned = D.rope(wide(k[l, s]), place, 64, False)
            for h in range(KV):
                want = turned[kept[l, s, h], h]
                assert np.all(np.abs(cache_k[l, s, h] - want) <= np.abs(want) * 2.0 ** -8 + 2.0 ** -20)
    # the first two of the stream's own slots and its newest five are protected
    assert np.all(kept[..., -5:] == np.arange(N - 5, N)) and np.all(kept[..., :2] == [0, 1])
    loop.start(torch.tensor([1, 2, 3], dtype=torch.int32).cuda())
    loop.step()
    torch.cuda.synchronize()
    assert np.abs(loop.cos.cpu().numpy().reshape(S, 30, 32)[:, 0] - np.cos(angles(np.full(S, P + N)))).max() <= 4 * 2.0 ** -24


@pytest.mark.parametrize("P", [40, 0])
def test_a_prompt_beside_the_prefix_is_one_sequence(gpu, monkeypatch, P):
    """A row's weights run over the prefix and the prompt, taken as one sequence of P + N tokens.  Bounds: keys and queries are rounded
    to bf16 (half a step each), a weight is off by twice a score's error."""
    lib, device, torch = gpu
    loop, _, bits = make_loop(gpu, monkeypatch, 5, P)
    N, window = 70, 16
    q, k, v = bits(L, S, N, HEADS, 64), bits(L, S, N, KV, 64), bits(L, S, N, KV, 64)
    kept = loop.prompt(q, k, v, window).cpu().numpy()
    torch.cuda.synchronize()
    place, mass = angles(P + np.arange(N)), loop.cache.mass.cpu().numpy()
    prefix = wide(loop.keep[0]) if P else np.zeros((L, KV, 0, 64))
    shared = np.zeros((L, KV, P))
    norm = lambda a: np.sqrt((a ** 2).sum(-1)).max() if a.size else 0.0   # noqa: E731
    most = 0.0
    for l in range(L):
        for s in range(S):
            turned, tq = D.rope(wide(k[l, s]), place, 64, False), D.rope(wide(q[l, s]), place, 64, False)
            far = 2 * (2 * 2.0 ** -8) * loop.scale * max(norm(turned), norm(prefix)) * norm(tq)
            most = max(most, far)
            for h in range(KV):
                whole, got = np.concatenate([prefix[l, h], turned[:, h]]), np.zeros(P + N)
                for r in range(N - window, N):
                    for g in range(HEADS // KV):
                        x = whole[:P + r + 1] @ tq[r, h * (HEADS // KV) + g] * loop.scale
                        e = np.exp(x - x.max())
                        got[:P + r + 1] += e / e.sum()
                shared[l, h] += got[:P]
                at = P + kept[l, s, h]
                assert np.all(np.abs(mass[l, s, h] - got[at]) <= got[at] * (np.exp(far) - 1) + 1e-6)
    if P:
        assert np.all(np.abs(loop.mass_prefill.cpu().numpy() - shared) <= shared * (np.exp(most) - 1) + 1e-6)


def test_a_prompt_in_bfloat16(gpu, monkeypatch):
    lib, device, torch = gpu
    results = []
    for dtype in (torch.int16, torch.bfloat16):
        loop, _, bits = make_loop(gpu, monkeypatch, 6, 40)
        q, k, v = (t.view(dtype) for t in (bits(L, S, 50, HEADS, 64), bits(L, S, 50, KV, 64), bits(L, S, 50, KV, 64)))
        kept = loop.prompt(q, k, v, 9)
        torch.cuda.synchronize()
        results.append([kept] + [getattr(loop.cache, n) for n in ("k", "v", "mass", "slot_pos", "len", "next_pos")])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_prompts_that_do_not_fit_are_refused(gpu, monkeypatch):
    lib, device, torch = gpu
    loop, _, bits = make_loop(gpu, monkeypatch, 6, 40)
    q, k, v = bits(L, S, 20, HEADS, 64), bits(L, S, 20, KV, 64), bits(L, S, 20, KV, 64)
    before = T.snapshot(loop)
    for args, status in [((q, k, v, 0), -2), ((q, k, v, 21), -2), ((q[:, :2], k, v, 4), -2), ((q, k[:1], v, 4), -2), ((q, k, v[:, :, :19], 4), -2),
                         ((q[..., :1, :], k, v, 4), -2), ((q, k, v[0], 4), -2), ((q, k.float(), v, 4), -1), ((q.half(), k, v, 4), -1)]:
        with pytest.raises(lib.MloraError) as e:
            loop.prompt(*args)
        assert e.value.status == status
    for n, t in T.snapshot(loop).items():
        assert torch.equal(t, before[n]), n


def test_the_head_takes_normalised_rows(gpu, monkeypatch):
    """Logits before the rules: the head's product on the last layer's rows times 1 / rms.  Bound: bf16's half step, and both
    products' sums in fp32 (2^-12 of the row's largest covers 128 products and their roundings)."""
    lib, device, torch = gpu
    loop, _, _ = make_loop(gpu, monkeypatch, 7, 40)
    seen, run_rules = {}, loop.rules.run

    def keep_logits(z, tokens, out, new_tokens=None):
        seen["logits"] = wide(z)
        run_rules(z, tokens, out, new_tokens=new_tokens)

    loop.rules.run = keep_logits
    for _ in range(3):
        loop.step()
        torch.cuda.synchronize()
        plain = torch.empty((loop.M, T.V), device="cuda")
        lib.linear(loop.head, loop.final, loop.row_adapter, loop.M, plain, lib.Y_FP32, loop.head_ws)
        rows = wide(loop.final)
        want = plain.cpu().numpy().astype(np.float64) / np.sqrt((rows ** 2).mean(1) + 1e-5)[:, None]
        assert np.all(np.abs(seen["logits"] - want) <= np.abs(want) * 2.0 ** -8 + np.abs(want).max(1, keepdims=True) * 2.0 ** -12)


@pytest.mark.parametrize("prompt", [False, True])
def test_a_second_generation_is_as_the_first(gpu, monkeypatch, prompt):
    """Two generations in a row on one loop, and each of them on a loop of its own: the same tokens, positions and live slots."""
    lib, device, torch = gpu

    def generation(loop, i, bits):
        if prompt:
            g = torch.Generator().manual_seed(i)
            some = lambda *shape: torch.randn(shape, generator=g).to(torch.bfloat16).view(torch.int16).cuda()   # noqa: E731
            loop.prompt(some(L, S, 31 + i, HEADS, 64), some(L, S, 31 + i, KV, 64), some(L, S, 31 + i, KV, 64), 8)
        loop.start(torch.tensor([5 + i, 60, 7 * i], dtype=torch.int32).cuda())
        given = T.run_steps(loop, 9)
        torch.cuda.synchronize()
        live = torch.arange(BUDGET, device="cuda") < loop.cache.len[:, None, None]
        out = {n: getattr(loop.cache, n).clone() for n in ("len", "next_pos")}
        out.update({n: torch.where(live, getattr(loop.cache, n), 0) for n in ("mass", "slot_pos")})
        out.update({n: torch.where(live[..., None], getattr(loop.cache, n), 0) for n in ("k", "v")})
        out.update(emitted=torch.stack(given), counts=loop.counts.clone(), mass_prefill=loop.mass_prefill.clone(), tokens=loop.tokens.clone())
        return out

    one, _, bits = make_loop(gpu, monkeypatch, 8, 40)
    for i in range(2):
        alone, _, _ = make_loop(gpu, monkeypatch, 8, 40)
        got, want = generation(one, i, bits), generation(alone, i, bits)
        for n in want:
            assert torch.equal(got[n], want[n]), (i, n)


def test_tables_and_prefix_in_bfloat16(gpu, monkeypatch):
    """The same numbers handed in as bfloat16 and as their patterns."""
    lib, device, torch = gpu
    from paper_2604_18655_amd import decoding
    made, results = decoding.DecodingLoop, []
    for dtype in (torch.int16, torch.bfloat16):
        def loop_in(layers, head, embedding, forecast, *args, **kw):
            kw.update({n: kw[n].view(dtype) for n in ("k_prefill", "v_prefill")})
            return made(layers, head, embedding.view(dtype), forecast.view(dtype), *args, **kw)
        monkeypatch.setattr(decoding, "DecodingLoop", loop_in)
        loop, _, _ = make_loop(gpu, monkeypatch, 9, 40)
        results.append(T.run_steps(loop, 5) + [loop.h.clone(), loop.q.clone(), loop.logits.clone()])
    torch.cuda.synchronize()
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_tokens_outside_the_vocabulary(gpu, monkeypatch):
    """They are embedded as the nearest token; a place without a draft (-1) as the first."""
    lib, device, torch = gpu
    loop, _, _ = make_loop(gpu, monkeypatch, 10, 40)
    loop.start(torch.tensor([T.V, 1 << 30, -5], dtype=torch.int32).cuda())
    rows = loop.embedding[[T.V - 1, T.V - 1, 0]].clone()
    loop.step()
    torch.cuda.synchronize()
    assert torch.equal(loop.h.view(S, 30, -1)[:, 0], rows.view(torch.int16))
