"""Host side of the decoding loop's calls (no GPU): every declared function is exported, and what a host check can see is
refused before anything is launched (all pointers here are made up)."""
import ctypes as C
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2604_18655_amd as lib
from oracle import decoding_loop as D
from paper_2604_18655_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, ESHAPE, EALIGN, EWORKSPACE = 0, -1, -2, -3, -4


def test_library_exports_the_loop_headers():
    names = set()
    for header in ("mlora_rope.h", "mlora_stream_cache.h", "mlora_logit_rules.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names |= set(re.findall(r"\b(mlora_[a-z0-9_]+)\s*\(", text))
    assert names == set(lib.loop_symbols)
    for name in names:
        assert getattr(lib.load_library(), name) is not None


def rope(**kw):
    f = dict(head_dim=64, rot=64, layout=0, scaling=0, theta=10000.0, factor=1.0, low=1.0, high=4.0, context=8192.0)
    f.update(kw)
    return B._RopeStruct(**f)


@pytest.mark.parametrize("scaling,name", [(0, "plain"), (1, "linear"), (2, "base"), (3, "turns")])
@pytest.mark.parametrize("rot", [4, 10, 64, 128])
def test_frequencies_match_the_definition(scaling, name, rot):
    out = (C.c_double * (rot // 2))()
    assert lib.load_library().mlora_rope_frequencies(C.byref(rope(head_dim=128, rot=rot, scaling=scaling, theta=500000.0, factor=8.0)), out) == OK
    want = [D.rope_frequency(i, rot, name, 500000.0, factor=8.0) * 2 / math.pi for i in range(rot // 2)]
    assert np.allclose(list(out), want, rtol=1e-14, atol=0)


def test_rope_refusals():
    cdll = lib.load_library()
    out = (C.c_double * 512)()
    for bad, want in [(dict(rot=63), ESHAPE), (dict(rot=66), ESHAPE), (dict(rot=0), ESHAPE), (dict(head_dim=514, rot=8), ESHAPE), (dict(layout=2), EINVAL),
                      (dict(scaling=4), EINVAL), (dict(theta=0.0), EINVAL), (dict(theta=math.nan), EINVAL), (dict(scaling=1, factor=0.0), EINVAL),
                      (dict(scaling=2, rot=2, factor=2.0), ESHAPE), (dict(scaling=3, low=4.0), EINVAL), (dict(scaling=3, context=math.inf), EINVAL)]:
        assert cdll.mlora_rope_frequencies(C.byref(rope(**bad)), out) == want, bad
    assert cdll.mlora_rope_frequencies(None, out) == EINVAL
    assert cdll.mlora_rope_frequencies(C.byref(rope()), None) == EINVAL

    def rows(**kw):
        f = dict(M=8, rows_per_stream=4, base=0x1000, offset=0x2000, quarter_turns=0x3000)
        f.update(kw)
        return B._RopeRowsStruct(**f)

    def tensor(**kw):
        f = dict(x=0x10000, y=0x20000, x_row=512, x_head=64, y_row=512, y_head=64, heads=8, rotate=1)
        f.update(kw)
        return B._RopeTensorStruct(**f)

    def apply(r=rope(), w=rows(), t=(tensor(),), n=None, dtype=0, inverse=0):
        arr = (B._RopeTensorStruct * max(1, len(t)))(*t)
        return cdll.mlora_rope_apply(C.byref(r), C.byref(w), arr, len(t) if n is None else n, dtype, inverse, None)

    assert apply(w=rows(M=0)) == OK                                     # an empty call: nothing is launched
    for bad, want in [(dict(M=7), ESHAPE), (dict(M=-4), ESHAPE), (dict(M=1 << 25), ESHAPE), (dict(rows_per_stream=0), ESHAPE), (dict(base=0x1002), EALIGN),
                      (dict(quarter_turns=0x3004), EALIGN), (dict(quarter_turns=None), EINVAL)]:
        assert apply(w=rows(**bad)) == want, bad
        assert cdll.mlora_rope_tables(C.byref(rope()), C.byref(rows(**bad)), 0x4000, 0x5000, None) == want
    assert cdll.mlora_rope_tables(C.byref(rope()), C.byref(rows()), None, 0x5000, None) == EINVAL
    assert cdll.mlora_rope_tables(C.byref(rope()), C.byref(rows()), 0x4002, 0x5000, None) == EALIGN
    assert cdll.mlora_rope_tables(C.byref(rope()), C.byref(rows(M=0)), 0x4000, 0x5000, None) == OK
    for bad, want in [(dict(x=None), EINVAL), (dict(y=0x20001), EALIGN), (dict(heads=0), ESHAPE), (dict(heads=4097), ESHAPE), (dict(x_row=-1), ESHAPE),
                      (dict(y=0x10000, y_row=1024), EINVAL)]:
        assert apply(t=(tensor(**bad),)) == want, bad
    assert apply(t=(tensor(x=0x10002),), dtype=1) == EALIGN             # aligned for bf16, not for fp32
    assert apply(t=(tensor(),) * 5) == EINVAL and apply(n=0) == EINVAL and apply(dtype=2) == EINVAL and apply(inverse=2) == EINVAL


def cache(**kw):
    f = dict(n_layers=2, n_streams=3, n_kv_heads=4, head_dim=64, cap=100, k=0x10000, v=0x20000, mass=0x30000, slot_pos=0x40000, len=0x50000,
             next_pos=0x60000, tickets=0x70000)
    f.update(kw)
    return B._StreamCacheStruct(**f)


BAD_CACHES = [(dict(head_dim=96), ESHAPE), (dict(cap=0), ESHAPE), (dict(cap=(1 << 24) + 1), ESHAPE), (dict(n_layers=0), ESHAPE),
              (dict(n_layers=1 << 11, n_streams=1 << 10), ESHAPE), (dict(k=None), EINVAL), (dict(k=0x10008), EALIGN), (dict(mass=0x30002), EALIGN),
              (dict(slot_pos=None), EINVAL), (dict(len=None), EINVAL)]


def test_stream_cache_refusals():
    cdll = lib.load_library()

    def append(c=cache(), k=0x100000, v=0x200000, R=8, rows=0x300000, n=3, budget=50, sink=4, recent=8):
        return cdll.mlora_stream_cache_append(C.byref(c), k, v, R, rows, n, budget, sink, recent, None)

    def compress(a=cache(), b=cache(k=0x11000, v=0x21000, mass=0x31000, slot_pos=0x41000, len=0x51000, next_pos=0x61000, tickets=0x71000), kept=0x400000,
                 budget=20, sink=4, recent=8):
        return cdll.mlora_stream_cache_compress(C.byref(a), C.byref(b), kept, budget, sink, recent, None)

    for bad, want in BAD_CACHES + [(dict(tickets=None), EINVAL), (dict(v=None), EINVAL)]:
        assert append(c=cache(**bad)) == want, bad
        assert compress(a=cache(**bad)) == want, bad
    for kw, want in [(dict(k=None), EINVAL), (dict(v=0x200004), EALIGN), (dict(rows=0x300001), EALIGN), (dict(R=0), ESHAPE), (dict(R=2000), ESHAPE),
                     (dict(n=0), ESHAPE), (dict(n=9), ESHAPE), (dict(budget=2), ESHAPE), (dict(budget=101), ESHAPE), (dict(sink=-1), ESHAPE),
                     (dict(recent=-1), ESHAPE), (dict(rows=None, budget=7), ESHAPE)]:
        assert append(**kw) == want, kw
    for kw, want in [(dict(kept=None), EINVAL), (dict(kept=0x400002), EALIGN), (dict(budget=0), ESHAPE), (dict(budget=101), ESHAPE), (dict(sink=-1), ESHAPE),
                     (dict(b=cache()), EINVAL), (dict(b=cache(k=0x11000, head_dim=128)), ESHAPE), (dict(b=cache(n_streams=2)), ESHAPE)]:
        assert compress(**kw) == want, kw
    assert cdll.mlora_stream_cache_append(None, 16, 16, 1, None, 0, 1, 0, 0, None) == EINVAL


def test_attention_mass_refusals():
    cdll = lib.load_library()

    def mass(c=None, **kw):
        f = dict(cache=c or cache(), n_q_heads=8, rows_per_stream=8, scale=0.125, k_prefill=0x80000, mass_prefill=0x90000, len_prefill=64, decay=1.0)
        f.update(kw)
        return B._AttentionMassStruct(**f)

    def call(d, q=0x100000, rows=0x300000, n=3, ws=0x400000, nbytes=1 << 30):
        return cdll.mlora_attention_mass_add(C.byref(d), q, rows, n, ws, nbytes, None)

    for bad, want in BAD_CACHES:
        assert call(mass(c=cache(**bad))) == want, bad
        assert cdll.mlora_attention_mass_workspace_bytes(C.byref(mass(c=cache(**bad))), 3) == 0
    for bad, want in [(dict(n_q_heads=6), ESHAPE), (dict(n_q_heads=36), ESHAPE), (dict(rows_per_stream=0), ESHAPE), (dict(rows_per_stream=2000), ESHAPE),
                      (dict(len_prefill=-1), ESHAPE), (dict(k_prefill=None), EINVAL), (dict(mass_prefill=None), EINVAL), (dict(k_prefill=0x80008), EALIGN)]:
        assert call(mass(**bad)) == want, bad
    d = mass()
    need = cdll.mlora_attention_mass_workspace_bytes(C.byref(d), 3)
    assert need > 0 and cdll.mlora_attention_mass_workspace_bytes(C.byref(d), 0) == cdll.mlora_attention_mass_workspace_bytes(C.byref(d), 8)
    assert cdll.mlora_attention_mass_workspace_bytes(C.byref(d), 9) == 0 and cdll.mlora_attention_mass_workspace_bytes(C.byref(d), -1) == 0
    for kw, want in [(dict(q=None), EINVAL), (dict(q=0x100008), EALIGN), (dict(rows=0x300002), EALIGN), (dict(n=0), ESHAPE), (dict(n=9), ESHAPE),
                     (dict(ws=None), EWORKSPACE), (dict(nbytes=need - 1), EWORKSPACE), (dict(ws=0x400010), EALIGN)]:
        assert call(d, **kw) == want, kw
    assert cdll.mlora_attention_mass_add(None, 16, None, 0, 256, 1, None) == EINVAL
    assert call(mass(k_prefill=None, mass_prefill=None, len_prefill=0), nbytes=1) == EWORKSPACE     # an empty segment needs no pointer


def test_logit_rules_refusals():
    cdll = lib.load_library()

    def rules(**kw):
        f = dict(n_streams=2, rows_per_stream=5, tokens_per_stream=3, vocab=100, logits_dtype=0, parent=0x1000, counts=0x2000, repetition=0x3000,
                 frequency=0x4000, presence=0x5000, bias=0x6000, bias_row=0x7000, n_bias=1, masks=0x8000, mask_row=0x9000, n_masks=2)
        f.update(kw)
        return B._LogitRulesStruct(**f)

    def call(d=rules(), logits=0x10000, tokens=0x20000, new=0x30000, n=2, out=0x40000):
        return cdll.mlora_logit_rules_apply(C.byref(d), logits, tokens, new, n, out, None)

    for bad, want in [(dict(n_streams=0), ESHAPE), (dict(rows_per_stream=65), ESHAPE), (dict(n_streams=1000), ESHAPE), (dict(tokens_per_stream=6), ESHAPE),
                      (dict(tokens_per_stream=0), ESHAPE), (dict(vocab=0), ESHAPE), (dict(vocab=(1 << 30) + 1), ESHAPE), (dict(logits_dtype=2), EINVAL),
                      (dict(parent=None), EINVAL), (dict(bias=None), EINVAL), (dict(mask_row=None), EINVAL), (dict(n_masks=-1), ESHAPE),
                      (dict(counts=0x2002), EALIGN), (dict(masks=0x8001), EALIGN)]:
        assert call(rules(**bad)) == want, bad
    for kw, want in [(dict(logits=None), EINVAL), (dict(tokens=None), EINVAL), (dict(out=None), EINVAL), (dict(new=None), EINVAL), (dict(n=-1), ESHAPE),
                     (dict(n=4097), ESHAPE), (dict(logits=0x10001), EALIGN), (dict(tokens=0x20002), EALIGN), (dict(d=rules(counts=None)), EINVAL),
                     (dict(d=rules(logits_dtype=1), out=0x40002), EALIGN)]:
        assert call(**kw) == want, kw
    assert cdll.mlora_logit_rules_apply(None, 16, 16, None, 0, 16, None) == EINVAL


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    """A pointer to host memory, or to fewer elements than the kernels read, never reaches the library."""
    def refused(make, status=EINVAL):
        with pytest.raises(lib.MloraError) as e:
            make()
        assert e.value.status == status

    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)   # noqa: E731
    f = lambda *shape: torch.zeros(shape)   # noqa: E731
    k = torch.zeros((1, 2, 3, 8, 64), dtype=torch.bfloat16)
    r = lib.Rope(64, 64, device="cpu")
    refused(lambda: lib.RopeTables(r, f(4, 32), f(4, 32), 4))
    refused(lambda: lib.RopeTensor(torch.zeros((4, 2, 64)), torch.zeros((4, 2, 64))))
    refused(lambda: lib.StreamCache(k, k, f(1, 2, 3, 8), i(1, 2, 3, 8), i(2), i(2)))
    refused(lambda: lib.StreamCache(k[0], k[0], f(2, 3, 8), i(2, 3, 8), i(2), i(2)), ESHAPE)
    refused(lambda: lib.LogitRules(2, 3, 3, 10, lib.Y_FP32, i(6)))
    with pytest.raises(lib.MloraError):
        lib.Rope(64, 63, device="cpu")
    meta = lambda t: t.to("meta")   # noqa: E731  (a device tensor's shape checks cannot run without a device)
    refused(lambda: lib.StreamCache(*(meta(t) for t in (k, k, f(1, 2, 3, 8), i(1, 2, 3, 8), i(2), i(2)))))


def test_rotated_rows_or_heads_that_overlap_are_refused():
    """y with a stride of less than a head is written by several blocks at once."""
    cdll = lib.load_library()

    def apply(M=8, heads=8, **kw):
        f = dict(x=0x10000, y=0x20000, x_row=0, x_head=0, y_row=512, y_head=64, heads=heads, rotate=1)
        f.update(kw)
        rows = B._RopeRowsStruct(M, max(1, M), None, None, 0x3000)
        return cdll.mlora_rope_apply(C.byref(rope()), C.byref(rows), (B._RopeTensorStruct * 1)(B._RopeTensorStruct(**f)), 1, 0, 0, None)

    for bad in (dict(y_row=0), dict(y_row=63), dict(y_head=0), dict(y_head=63), dict(y_row=0, M=2, heads=1), dict(x=0x20000, y_row=0, x_head=64)):
        assert apply(**bad) == EINVAL, bad
    assert apply(M=0, y_row=0) == OK
