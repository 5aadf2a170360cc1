"""Host side of beam search on a paged cache (no GPU): every declared function is exported, what a host check can see is refused before
anything is launched (all pointers here are made up), and so is what the binding can see."""
import ctypes as C
import math
import os
import re

import pytest
import torch

import paper_2604_18655_amd as lib
from paper_2604_18655_amd import binding as B
from test_decoding_loop_binding import dev, recorder, refused

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, ESHAPE, EALIGN, EWORKSPACE = 0, -1, -2, -3, -4


def test_library_exports_the_headers():
    names = set()
    for header in ("mlora_page_cache.h", "mlora_page_attention.h", "mlora_beam.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names |= set(re.findall(r"\b(mlora_[a-z0-9_]+)\s*\(", text))
    assert names == set(lib.beam_symbols)
    for name in names:
        assert getattr(lib.load_library(), name) is not None


def cache(**kw):
    f = dict(n_layers=2, n_streams=4, n_kv_heads=2, head_dim=64, n_pages=10, max_pages=5)
    f.update({n: 0x10000 * (i + 1) for i, n in enumerate(("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "slot", "len", "table", "refs", "own"))})
    f.update(kw)
    return B._PageCacheStruct(**f)


BAD_CACHES = [(dict(head_dim=96), ESHAPE), (dict(n_layers=0), ESHAPE), (dict(n_streams=0), ESHAPE), (dict(n_streams=1025), ESHAPE), (dict(n_kv_heads=0), ESHAPE),
              (dict(n_pages=0), ESHAPE), (dict(n_pages=(1 << 20) + 1), ESHAPE), (dict(max_pages=0), ESHAPE), (dict(max_pages=(1 << 18) + 1), ESHAPE),
              (dict(n_layers=65536, n_streams=1, n_kv_heads=1), ESHAPE), (dict(n_layers=1 << 15, n_kv_heads=1 << 15), ESHAPE)]
BAD_CACHES += [({n: None}, EINVAL) for n in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "slot", "len", "table", "refs", "own")]
BAD_CACHES += [({n: 0x10008}, EALIGN) for n in ("k", "v", "k_tail", "v_tail")]
BAD_CACHES += [({n: 0x10002}, EALIGN) for n in ("k_scale", "v_scale", "slot", "len", "table", "refs", "own")]


@pytest.mark.parametrize("bad,want", BAD_CACHES)
def test_bad_caches(bad, want):
    cdll, c, good = lib.load_library(), C.byref(cache(**bad)), C.byref(cache(**{n: 0x1000000 for n in ("k",)}))
    assert cdll.mlora_page_cache_append(c, 0x1000, 0x2000, 4, None, 0, None, None) == want
    assert cdll.mlora_page_cache_reorder(c, 0x1000, 0, 0, None) == want
    assert cdll.mlora_page_cache_copy(c, good, 0x1000, None, None) == want
    assert cdll.mlora_page_cache_copy(good, c, 0x1000, None, None) == want
    t = attention(cache=cache(**bad))
    assert cdll.mlora_page_attention(C.byref(t), 0x1000, 0x2000, 0, 0x100000, 1 << 30, None) == want
    assert cdll.mlora_page_attention_workspace_bytes(C.byref(t)) == 0


def test_no_descriptors():
    cdll = lib.load_library()
    assert cdll.mlora_page_cache_append(None, 0x1000, 0x2000, 4, None, 0, None, None) == EINVAL
    assert cdll.mlora_page_cache_reorder(None, 0x1000, 0, 0, None) == EINVAL
    assert cdll.mlora_page_cache_copy(None, None, 0x1000, None, None) == EINVAL
    assert cdll.mlora_page_attention(None, 0x1000, 0x2000, 0, 0x100000, 1 << 30, None) == EINVAL
    assert cdll.mlora_page_attention_workspace_bytes(None) == 0 and cdll.mlora_page_attention_plan(None, (C.c_int32 * 3)()) == EINVAL
    assert cdll.mlora_beam_workspace_bytes(None) == 0
    assert cdll.mlora_beam_select(None, *[0x1000] * 10, 1 << 30, None) == EINVAL


def test_own_words():
    cdll = lib.load_library()
    assert cdll.mlora_page_cache_own_words(4, 10) >= 10
    for bad in ((0, 1), (1025, 1), (1, 0), (1, (1 << 20) + 1)):
        assert cdll.mlora_page_cache_own_words(*bad) == 0


def test_append_refusals():
    cdll, c = lib.load_library(), C.byref(cache())
    call = lambda k=0x1000, v=0x2000, R=4, rows=None, n=0, out=None: cdll.mlora_page_cache_append(c, k, v, R, rows, n, out, None)   # noqa: E731
    assert call(k=None) == EINVAL and call(v=None) == EINVAL
    assert call(k=0x1008) == EALIGN and call(v=0x2004) == EALIGN and call(rows=0x3001, n=1) == EALIGN and call(out=0x3002) == EALIGN
    assert call(R=0) == ESHAPE and call(R=1025) == ESHAPE and call(rows=0x3000, n=0) == ESHAPE and call(rows=0x3000, n=5) == ESHAPE


def test_reorder_and_copy_refusals():
    cdll, c = lib.load_library(), C.byref(cache())
    assert cdll.mlora_page_cache_reorder(c, 0x1002, 0, 0, None) == EALIGN
    assert cdll.mlora_page_cache_reorder(c, 0x1000, -1, 0, None) == ESHAPE and cdll.mlora_page_cache_reorder(c, None, 1, -1, None) == ESHAPE
    names = ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "slot", "len", "table", "refs", "own")
    other = {n: 0x1000000 + 0x10000 * i for i, n in enumerate(names)}
    copy = lambda to, source=0x1000, out=None: cdll.mlora_page_cache_copy(c, C.byref(to), source, out, None)   # noqa: E731
    assert copy(cache(**other), None) == EINVAL and copy(cache(**other), 0x1001) == EALIGN and copy(cache(**other), out=0x1001) == EALIGN
    for bad in (dict(n_layers=3), dict(n_kv_heads=3), dict(head_dim=128)):
        assert copy(cache(**dict(other, **bad))) == ESHAPE
    for n in names:
        assert copy(cache(**dict(other, **{n: getattr(cache(), n)}))) == EINVAL


def attention(**kw):
    f = dict(cache=cache(), layer=1, n_q_heads=8, rows_per_stream=3, scale=0.125, window=0, sink=0, k_new=0x100000, v_new=0x200000, parent=0x300000)
    f.update(kw)
    return B._PageAttnStruct(**f)


@pytest.mark.parametrize("bad,want", [(dict(layer=-1), ESHAPE), (dict(layer=2), ESHAPE), (dict(n_q_heads=0), ESHAPE), (dict(n_q_heads=7), ESHAPE),
                                      (dict(n_q_heads=18), ESHAPE), (dict(rows_per_stream=0), ESHAPE), (dict(rows_per_stream=65), ESHAPE),
                                      (dict(window=-1), ESHAPE), (dict(sink=-1), ESHAPE), (dict(k_new=None), EINVAL), (dict(v_new=None), EINVAL),
                                      (dict(parent=None), EINVAL), (dict(k_new=0x100008), EALIGN), (dict(v_new=0x100008), EALIGN), (dict(parent=0x100002), EALIGN),
                                      (dict(cache=cache(n_streams=1000), rows_per_stream=5), ESHAPE)])
def test_bad_attention(bad, want):
    cdll, t = lib.load_library(), attention(**bad)
    assert cdll.mlora_page_attention(C.byref(t), 0x1000, 0x2000, 0, 0x100000, 1 << 30, None) == want
    assert cdll.mlora_page_attention_workspace_bytes(C.byref(t)) == 0 and cdll.mlora_page_attention_plan(C.byref(t), (C.c_int32 * 3)()) == want


def test_attention_refusals():
    cdll, t = lib.load_library(), C.byref(attention())
    need = cdll.mlora_page_attention_workspace_bytes(t)
    call = lambda q=0x1000, out=0x2000, dtype=0, ws=0x100000, n=need: cdll.mlora_page_attention(t, q, out, dtype, ws, n, None)   # noqa: E731
    assert need > 0 and cdll.mlora_page_attention_plan(t, None) == EINVAL
    assert call(q=None) == EINVAL and call(out=None) == EINVAL and call(dtype=2) == EINVAL
    assert call(q=0x1008) == EALIGN and call(out=0x1008) == EALIGN and call(ws=0x100010) == EALIGN
    assert call(ws=None) == EWORKSPACE and call(n=need - 1) == EWORKSPACE


def beam(**kw):
    f = dict(n_groups=2, n_beams=4, vocab=1003, logits_dtype=0, eos=2, pad=0, length_power=0.5)
    f.update(kw)
    return B._BeamStruct(**f)


@pytest.mark.parametrize("bad,want", [(dict(n_groups=0), ESHAPE), (dict(n_beams=0), ESHAPE), (dict(n_beams=33), ESHAPE), (dict(n_groups=1025), ESHAPE),
                                      (dict(vocab=0), ESHAPE), (dict(vocab=(1 << 24) + 1), ESHAPE), (dict(logits_dtype=2), EINVAL),
                                      (dict(length_power=-0.1), EINVAL), (dict(length_power=math.nan), EINVAL), (dict(length_power=math.inf), EINVAL)])
def test_bad_beams(bad, want):
    cdll, d = lib.load_library(), beam(**bad)
    assert cdll.mlora_beam_select(C.byref(d), *[0x1000 * (i + 1) for i in range(9)], 0x100000, 1 << 30, None) == want
    assert cdll.mlora_beam_workspace_bytes(C.byref(d)) == 0


def test_beam_refusals():
    cdll, d = lib.load_library(), beam(logits_dtype=1)
    need = cdll.mlora_beam_workspace_bytes(C.byref(d))
    good = [0x1000 * (i + 1) for i in range(9)]
    call = lambda args, ws=0x100000, n=need: cdll.mlora_beam_select(C.byref(d), *args, ws, n, None)   # noqa: E731
    for i in range(9):
        assert call(good[:i] + [None] + good[i + 1:]) == EINVAL
        assert call(good[:i] + [good[i] + 2] + good[i + 1:]) == EALIGN
    assert call(good, None) == EWORKSPACE and call(good, n=need - 1) == EWORKSPACE and call(good, 0x100010) == EALIGN


# ------------------------------------------------------------------------------------------ the binding

bf16, f16, f32, i8, i32 = torch.bfloat16, torch.float16, torch.float32, torch.int8, torch.int32
SHAPES = dict(k=((2, 10, 3, 64, 64), i8), v=((2, 10, 3, 64, 64), i8), k_scale=((2, 10, 3), f32), v_scale=((2, 10, 3), f32), k_tail=((2, 4, 3, 64, 64), bf16),
              v_tail=((2, 4, 3, 64, 64), bf16), slot=((4,), i32), len=((4,), i32), table=((4, 5), i32), refs=((10,), i32))


def a_cache(**kw):
    t = {n: kw[n] if n in kw else dev(*shape, dtype=dtype) for n, (shape, dtype) in SHAPES.items()}
    calls = []
    c = lib.PageCache(*(t[n] for n in SHAPES))
    c.append_fn = c.reorder_fn = c.copy_fn = recorder(calls)
    return c, calls


def test_what_a_cache_is_made_of():
    a_cache()
    for n, (shape, dtype) in SHAPES.items():
        refused(lambda: a_cache(**{n: torch.zeros(shape, dtype=dtype)}))                                       # host memory
        refused(lambda: a_cache(**{n: dev(*shape, dtype=f16 if dtype != f16 else f32)}))                       # another type
        if n not in ("k", "k_tail", "table"):                                                                  # (these say how large the others are)
            refused(lambda: a_cache(**{n: dev(*shape[:-1], shape[-1] + 1, dtype=dtype)}), ESHAPE)
    refused(lambda: a_cache(k=dev(2, 10, 3, 32, 64, dtype=i8)), ESHAPE)
    refused(lambda: a_cache(k=dev(10, 3, 64, 64, dtype=i8)), ESHAPE)


def test_what_a_cache_is_called_with():
    c, calls = a_cache()
    new, rows, out = dev(2, 8, 3, 64, dtype=bf16), dev(4, 2), dev(4)
    refused(lambda: c.append(new, dev(2, 7, 3, 64, dtype=bf16), 2, stream=0), ESHAPE)
    refused(lambda: c.append(dev(2, 8, 3, 64, dtype=f16), new, 2, stream=0))
    refused(lambda: c.append(new, torch.zeros((2, 8, 3, 64), dtype=bf16), 2, stream=0))
    refused(lambda: c.append(new, new, 2, dev(7), stream=0), ESHAPE)
    refused(lambda: c.append(new, new, 2, dev(4, 0), stream=0), ESHAPE)
    refused(lambda: c.append(new, new, 2, dev(4, 2, dtype=f32), stream=0))
    refused(lambda: c.append(new, new, 2, rows, dev(3), stream=0), ESHAPE)
    refused(lambda: c.reorder(dev(3), stream=0), ESHAPE)
    refused(lambda: c.reorder(dev(4, dtype=torch.int64), stream=0))
    refused(lambda: c.reorder(torch.zeros(4, dtype=i32), stream=0))
    other, _ = a_cache()
    refused(lambda: c.copy_from(other, dev(5), stream=0), ESHAPE)
    refused(lambda: c.copy_from(other, dev(4, dtype=f32), stream=0))
    refused(lambda: c.copy_from(other, dev(4), dev(2), stream=0), ESHAPE)
    assert not calls
    c.append(new, new, 2, rows, out, stream=0)
    c.append(new, new, 2, stream=0)
    c.reorder(out, stream=0)
    c.reorder(stream=0)
    c.copy_from(other, out, dev(1), stream=0)
    assert [len(x) for x in calls] == [8, 8, 5, 5, 5] and calls[0][5] == 2 and calls[1][4] is None


def test_what_the_attention_takes():
    c, _ = a_cache()
    new, parent = dev(8, 3, 64, dtype=bf16), dev(8)
    refused(lambda: lib.PageAttention(c, 0, 6, 2, 0.125, dev(7, 3, 64, dtype=bf16), new, parent), ESHAPE)
    refused(lambda: lib.PageAttention(c, 0, 6, 2, 0.125, new, dev(8, 3, 64, dtype=f16), parent))
    refused(lambda: lib.PageAttention(c, 0, 6, 2, 0.125, new, new, dev(4)), ESHAPE)
    refused(lambda: lib.PageAttention(c, 0, 6, 2, 0.125, new, new, torch.zeros(8, dtype=i32)))
    op, calls = lib.PageAttention(c, 0, 6, 2, 0.125, new, new, parent, window=7, sink=1), []
    op.fn = recorder(calls)
    q, ws = dev(8, 6, 64, dtype=bf16), dev(1 << 16, dtype=torch.uint8)
    refused(lambda: op.run(dev(8, 5, 64, dtype=bf16), q, lib.Y_BF16, ws, stream=0), ESHAPE)
    refused(lambda: op.run(q, q, lib.Y_FP32, ws, stream=0))
    refused(lambda: op.run(q, dev(8, 6, 64, dtype=f32), lib.Y_BF16, ws, stream=0))
    refused(lambda: op.run(q, q, lib.Y_BF16, torch.zeros(1 << 16, dtype=torch.uint8), stream=0))
    assert not calls and op.struct.window == 7 and op.struct.sink == 1
    op.run(q, q, lib.Y_BF16, ws, stream=0)
    op.run(q, dev(8, 6, 64, dtype=f32), lib.Y_FP32, ws, stream=0)
    assert len(calls) == 2


def test_what_the_selection_takes():
    op, calls = lib.BeamSelect(2, 3, 11, lib.Y_BF16), []
    op.fn = recorder(calls)
    names = ("logits", "score", "length", "finished", "source", "token", "score_out", "length_out", "finished_out")
    good = dict(logits=dev(6, 11, dtype=bf16), **{n: dev(6, dtype=f32 if "score" in n else i32) for n in names[1:]})
    ws = dev(1 << 14, dtype=torch.uint8)
    run = lambda **kw: op.run(*(dict(good, **kw)[n] for n in names), ws, stream=0)   # noqa: E731
    refused(lambda: run(logits=dev(6, 10, dtype=bf16)), ESHAPE)
    refused(lambda: run(logits=dev(6, 11, dtype=f16)))
    for n in names[1:]:
        refused(lambda: run(**{n: dev(5, dtype=f32 if "score" in n else i32)}), ESHAPE)
        refused(lambda: run(**{n: dev(6, dtype=i32 if "score" in n else f32)}))
        refused(lambda: run(**{n: torch.zeros(6, dtype=f32 if "score" in n else i32)}))
    refused(lambda: op.run(*(good[n] for n in names), torch.zeros(1 << 14, dtype=torch.uint8), stream=0))
    assert not calls
    run()
    assert len(calls) == 1


def test_what_a_beam_loop_is_made_of():
    from paper_2604_18655_amd.beams import BeamLoop
    proj = lambda K, N: lib.Proj(K, N, 32, torch.zeros(16, dtype=torch.uint8))   # noqa: E731
    layer = [proj(128, 128), proj(128, 64), proj(128, 64), proj(128, 128), proj(128, 512), proj(256, 128)]
    embedding = torch.zeros((300, 128), dtype=torch.int16)
    make = lambda layers=(layer,), head=proj(128, 300), emb=embedding, W=2, **kw: BeamLoop(   # noqa: E731
        layers, head, emb, 2, W, 8, 4, kw.pop("max_steps", 5), device="cpu", **kw)
    refused(lambda: make(layers=()), ESHAPE)
    refused(lambda: make(head=proj(128, 301)), ESHAPE)
    refused(lambda: make(emb=torch.zeros((300, 64), dtype=torch.int16)), ESHAPE)
    refused(lambda: make(emb=torch.zeros((300, 128), dtype=torch.float32)))
    refused(lambda: make(W=33), ESHAPE)
    refused(lambda: make(max_steps=0), ESHAPE)
    refused(lambda: make(window=-1), ESHAPE)
    refused(lambda: make(sink=-1), ESHAPE)
    refused(lambda: make(row_adapter=dev(3)), ESHAPE)
    refused(lambda: make(row_adapter=torch.zeros(4, dtype=i32)))
    refused(lambda: make(rope=lib.Rope(64, 32, device="cpu")), ESHAPE)
