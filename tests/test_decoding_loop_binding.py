"""What the Python side of the decoding loop's calls refuses before the library sees a pointer (no GPU: tensors that say they
are on the device, and a library that records its calls)."""
import pytest
import torch

import paper_2604_18655_amd as lib
from paper_2604_18655_amd import binding as B

EINVAL, ESHAPE = -1, -2


class OnDevice:
    """A tensor that says it is device memory."""

    def __init__(self, t):
        self.t = t

    is_cuda = True

    def __getattr__(self, name):
        return getattr(self.t, name)


def dev(*shape, dtype=torch.int32):
    return OnDevice(torch.zeros(shape, dtype=dtype))


def refused(make, status=EINVAL):
    with pytest.raises(lib.MloraError) as e:
        make()
    assert e.value.status == status


def a_cache(**kw):
    L, S, H, cap, D = 1, 2, 3, 8, 64
    t = dict(k=dev(L, S, H, cap, D, dtype=torch.bfloat16), v=dev(L, S, H, cap, D, dtype=torch.bfloat16), mass=dev(L, S, H, cap, dtype=torch.float32),
             slot_pos=dev(L, S, H, cap), len=dev(S), next_pos=dev(S))
    t.update(kw)
    return lib.StreamCache(*(t[n] for n in ("k", "v", "mass", "slot_pos", "len", "next_pos")))


def recorder(calls):
    def call(*args):
        calls.append(args)
        return 0
    return call


def a_mass(cache=None, **kw):
    op = lib.AttentionMass(cache or a_cache(), 6, 4, 0.125, **kw)
    calls = []
    op.fn = recorder(calls)
    return op, calls


def test_frequencies_on_the_host_are_refused():
    r = lib.Rope(64, 64, device="cpu")
    refused(lambda: r.rows(4, None, None, None))
    refused(lambda: lib.RopeTables(r, dev(4, 32, dtype=torch.float32), dev(4, 32, dtype=torch.float32), 4))
    refused(lambda: lib.RopePlan(r, [], 4, lib.Y_FP32))


def test_workspaces_on_the_host_or_with_gaps_are_refused():
    op, calls = a_mass()
    q = dev(1, 8, 6, 64, dtype=torch.bfloat16)
    for ws in (torch.zeros(1 << 16, dtype=torch.uint8), OnDevice(torch.zeros(1, dtype=torch.uint8).expand(1 << 16)),
               OnDevice(torch.zeros(1 << 17, dtype=torch.uint8)[::2])):
        refused(lambda: op.run(q, None, ws, stream=0))
    assert not calls
    op.run(q, None, dev(1 << 16, dtype=torch.uint8), stream=0)
    assert len(calls) == 1


def test_a_place_for_the_queries_of_another_size_is_refused():
    from paper_2604_18655_amd.decoder import DecoderLayerStep
    M, hidden = 6, 128
    proj = lambda K, N: lib.Proj(K, N, 32, torch.zeros(16, dtype=torch.uint8))   # noqa: E731
    projs = [proj(hidden, 128), proj(hidden, 64), proj(hidden, 64), proj(128, hidden), proj(hidden, 256), proj(128, hidden)]
    i32, i16 = (lambda *s: torch.zeros(s, dtype=torch.int32)), (lambda *s: torch.zeros(s, dtype=torch.int16))   # noqa: E731
    attention = lib.TreeAttention(2, 1, 64, 1, M, 0.125, None, None, None, None, None, None, None, i16(M, 64), i16(M, 64), i32(M),
                                  torch.zeros(M, dtype=torch.uint8), 0, 0, 0)
    table = torch.zeros(M, 32)
    step = lambda q: DecoderLayerStep(*projs, attention, i16(M, hidden), table, table, None, M, q=q)   # noqa: E731
    for q, status in ((i16(M - 1, 128), ESHAPE), (i16(M, 64), ESHAPE), (i16(128, M).t(), EINVAL), (torch.zeros((M, 128)), EINVAL), (i16(M, 128).to("meta"), EINVAL)):
        refused(lambda: step(q), status)
    mine = i16(M, 128)
    assert step(mine).q is mine and step(None).q.shape == (M, 128)


def test_lists_without_entries_are_refused():
    """Their pointer is null, which would mean all rows."""
    c, calls = a_cache(), []
    c.append_fn = recorder(calls)
    new = [dev(1, 8, 3, 64, dtype=torch.bfloat16) for _ in range(2)]
    refused(lambda: c.append(*new, 4, dev(2, 0), 8, stream=0), ESHAPE)
    op, mass_calls = a_mass(c)
    refused(lambda: op.run(dev(1, 8, 6, 64, dtype=torch.bfloat16), dev(2, 0), dev(1 << 16, dtype=torch.uint8), stream=0), ESHAPE)
    assert not calls and not mass_calls
    c.append(*new, 4, None, 8, stream=0)
    c.append(*new, 4, dev(2, 3), 8, stream=0)
    assert [x[4] is None for x in calls] == [True, False] and calls[1][5] == 3


def test_a_rotation_of_no_rows():
    """Tensors without elements have null pointers; nothing is launched, as the header says of M = 0."""
    r = lib.Rope(64, 32, device="cpu")
    r.quarter_turns = OnDevice(r.quarter_turns)
    none = lambda *shape: dev(0, *shape, dtype=torch.float32)   # noqa: E731
    lib.RopeTables(r, none(16), none(16), 0).run(stream=0)
    lib.RopePlan(r, [lib.RopeTensor(none(2, 64), none(2, 64))], 0, lib.Y_FP32).run(stream=0)
    lib.RopePlan(r, [lib.RopeTensor(none(2, 64), none(2, 64))], 0, lib.Y_FP32, rows_per_stream=4, base=dev(0), offset=dev(4)).run(stream=0)
    rows = B._RopeRowsStruct(4, 4, None, None, 0x3000)
    assert lib.load_library().mlora_rope_tables(r.struct, rows, None, None, None) == EINVAL


def test_a_prefix_of_no_tokens():
    """It needs no masses, as the header says of len 0."""
    none = dev(1, 3, 0, 64, dtype=torch.bfloat16)
    for kw in (dict(k_prefill=none), dict(k_prefill=none, mass_prefill=dev(1, 3, 0, dtype=torch.float32)), dict()):
        op, calls = a_mass(**kw)
        op.run(dev(1, 8, 6, 64, dtype=torch.bfloat16), None, dev(1 << 16, dtype=torch.uint8), stream=0)
        assert len(calls) == 1 and op.struct.len_prefill == 0
    refused(lambda: a_mass(k_prefill=dev(1, 3, 2, 64, dtype=torch.bfloat16)))
    refused(lambda: a_mass(k_prefill=none, mass_prefill=dev(1, 3, 1, dtype=torch.float32)), ESHAPE)


def test_elements_of_another_type_of_the_same_size_are_refused():
    bf16, f32, i32, f16, i16 = torch.bfloat16, torch.float32, torch.int32, torch.float16, torch.int16
    on = lambda shape, dtype: dev(*shape, dtype=dtype)   # noqa: E731
    for kw in (dict(k=f16), dict(v=f16), dict(mass=i32), dict(slot_pos=f32), dict(len=f32), dict(next_pos=f32)):
        (name, dtype), shapes = next(iter(kw.items())), dict(k=(1, 2, 3, 8, 64), v=(1, 2, 3, 8, 64), mass=(1, 2, 3, 8), slot_pos=(1, 2, 3, 8), len=(2,), next_pos=(2,))
        refused(lambda: a_cache(**{name: on(shapes[name], dtype)}))
    a_cache(k=on((1, 2, 3, 8, 64), i16))
    c, calls = a_cache(), []
    c.append_fn = c.compress_fn = recorder(calls)
    new = on((1, 8, 3, 64), bf16)
    refused(lambda: c.append(new, on((1, 8, 3, 64), f16), 4, None, 8, stream=0))
    refused(lambda: c.append(on((1, 8, 3, 64), f16), new, 4, None, 8, stream=0))
    refused(lambda: c.append(new, new, 4, on((2, 3), f32), 8, stream=0))
    refused(lambda: c.append(new, new, 4, on((2, 3), torch.int64), 8, stream=0))
    refused(lambda: c.append(new, new, 4, on((7,), i32), 8, stream=0), ESHAPE)
    refused(lambda: c.compress(a_cache(), on((1, 2, 3, 5), f32), 5, stream=0))
    ws = on((1 << 16,), torch.uint8)
    op, mass_calls = a_mass(c)
    refused(lambda: op.run(on((1, 8, 6, 64), f16), None, ws, stream=0))
    refused(lambda: op.run(on((1, 8, 6, 64), bf16), on((2, 3), f32), ws, stream=0))
    refused(lambda: a_mass(c, k_prefill=on((1, 3, 9, 64), f16), mass_prefill=on((1, 3, 9), f32)))
    refused(lambda: a_mass(c, k_prefill=on((1, 3, 9, 64), bf16), mass_prefill=on((1, 3, 9), i32)))
    assert not calls and not mass_calls
    c.append(on((1, 8, 3, 64), i16), new, 4, on((2, 3), i32), 8, stream=0)
    op.run(on((1, 8, 6, 64), i16), None, ws, stream=0)
    assert len(calls) == 1 and calls[0][5] == 3 and len(mass_calls) == 1

    r = lib.Rope(64, 64, device="cpu")
    r.quarter_turns = OnDevice(r.quarter_turns)
    table, x = on((4, 32), f32), on((4, 2, 64), f16)
    refused(lambda: lib.RopeTables(r, table, on((4, 32), i32), 4))
    refused(lambda: lib.RopeTables(r, table, table, 4, base=on((1,), f32)))
    refused(lambda: lib.RopeTables(r, table, table, 4, offset=on((4,), f32)))
    refused(lambda: lib.RopePlan(r, [lib.RopeTensor(x, x)], 4, lib.Y_BF16))
    refused(lambda: lib.RopePlan(r, [lib.RopeTensor(on((4, 2, 64), i32), on((4, 2, 64), i32))], 4, lib.Y_FP32))
    lib.RopePlan(r, [lib.RopeTensor(on((4, 2, 64), bf16), on((4, 2, 64), bf16))], 4, lib.Y_BF16)

    given = dict(counts=on((2, 40), i32), repetition=on((2,), f32), bias=on((1, 40), f32), bias_row=on((2,), i32), masks=on((1, 2), i32), mask_row=on((6,), i32))
    other = dict(counts=f32, repetition=i32, bias=i32, bias_row=f32, masks=f32, mask_row=f32)
    rules = lambda y=lib.Y_BF16, **kw: lib.LogitRules(2, 3, 2, 40, y, on((6,), i32), **dict(given, **kw))   # noqa: E731
    for name, dtype in other.items():
        refused(lambda: rules(**{name: on(tuple(given[name].shape), dtype)}))
    op, calls = rules(), []
    op.fn = recorder(calls)
    z, tokens = on((6, 40), bf16), on((2, 2), i32)
    for args in ((on((6, 40), f16), tokens, z), (z, tokens, on((6, 40), f16)), (z, on((2, 2), f32), z), (z, on((2, 1), torch.int64), z),
                 (z, tokens, z, on((2, 3), f32))):
        refused(lambda: op.run(*args, stream=0))
    assert not calls
    op.run(z, tokens, z, on((2, 3), i32), stream=0)
    op.run(z, tokens, z, on((2, 0), i32), stream=0)
    assert [x[4] for x in calls] == [3, 0]
    op = rules(lib.Y_FP32)
    refused(lambda: op.run(on((6, 40), i32), tokens, on((6, 40), i32), stream=0))


def loop_of(**kw):
    """Arguments that fit each other, but for what the caller changes.  Nothing here is on a device."""
    from paper_2604_18655_amd.decoding import DecodingLoop
    bits = lambda *shape: torch.zeros(shape, dtype=torch.int16)   # noqa: E731
    sizes = dict(q=(128, 256), k=(128, 64), v=(128, 64), o=(256, 128), gate_up=(128, 512), down=(256, 128), head=(128, 300))
    second = {n[1:]: kw.pop(n) for n in list(kw) if n.startswith("_")}
    proj = lambda n, over=(): lib.Proj(*dict(sizes, **dict(over))[n], 32, None)   # noqa: E731
    layers = [[proj(n) for n in list(sizes)[:6]], [proj(n, second) for n in list(sizes)[:6]]]
    args = dict(layers=layers, head=proj("head", {k: kw.pop(k) for k in ("head",) if k in kw}), embedding=bits(300, 128), forecast=bits(2, 128), n_streams=3,
                branch=(3, 2), budget=24)
    args.update(kw)
    return DecodingLoop(**args)


@pytest.mark.parametrize("bad", [dict(budget=2), dict(sink=-1), dict(recent=-1)])
def test_a_budget_below_a_step_is_refused(bad):
    refused(lambda: loop_of(**bad), ESHAPE)


@pytest.mark.parametrize("bad", [
    dict(layers=[]),
    dict(_q=(128, 320)), dict(_k=(128, 128)), dict(_v=(128, 128)), dict(_o=(256, 256)), dict(_o=(128, 128)), dict(_gate_up=(128, 1024)), dict(_down=(256, 256)),
    dict(_q=(256, 256)), dict(head=(256, 300)), dict(head=(128, 301)),
    dict(embedding=torch.zeros((300, 64), dtype=torch.int16)), dict(forecast=torch.zeros((2, 64), dtype=torch.int16)),
    dict(k_prefill=dev(2, 1, 9, 64, dtype=torch.int16)), dict(v_prefill=dev(2, 1, 9, 64, dtype=torch.int16)),
    dict(k_prefill=dev(2, 1, 9, 64, dtype=torch.int16), v_prefill=dev(2, 1, 8, 64, dtype=torch.int16)),
    dict(k_prefill=dev(1, 1, 9, 64, dtype=torch.int16), v_prefill=dev(1, 1, 9, 64, dtype=torch.int16)),
    dict(row_adapter=dev(3)),
    dict(row_adapter=dev(89)),
    dict(rope=lib.Rope(64, 64, lib.ROPE_INTERLEAVED, device="cpu")), dict(rope=lib.Rope(64, 32, device="cpu")), dict(rope=lib.Rope(128, 64, device="cpu")),
])
def test_parts_of_a_loop_that_do_not_fit_are_refused(bad):
    refused(lambda: loop_of(**bad), ESHAPE)


@pytest.mark.parametrize("bad", [
    dict(embedding=torch.zeros((300, 128), dtype=torch.float16)), dict(forecast=torch.zeros((2, 128))), dict(row_adapter=torch.zeros(90, dtype=torch.int32)), dict(row_adapter=dev(90, dtype=torch.float32)),
    dict(k_prefill=dev(2, 1, 9, 64, dtype=torch.int16), v_prefill=torch.zeros((2, 1, 9, 64), dtype=torch.int16)),
    dict(k_prefill=dev(2, 1, 9, 64, dtype=torch.int16), v_prefill=dev(2, 1, 9, 64, dtype=torch.float16)),
])
def test_parts_of_a_loop_in_other_memory_or_of_other_types_are_refused(bad):
    refused(lambda: loop_of(**bad))
