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
