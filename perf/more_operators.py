"""Operators of beam search on a paged cache of 8 bits, as timed cases: selection over beams and vocabulary, rows that enter the
pages, streams that fork, move and give up what a window no longer sees, copies into another pool, attention over the pages.

A case is a dict of plain values.  Its "kind" names the public call it stands for:

    beam      binding.BeamSelect: the best continuations of every group of beams
    append    binding.PageCache.append behind a reorder: streams fork from one (or are emptied), then new rows enter their caches
    reorder   binding.PageCache.reorder: streams become others, pages are shared, counted and freed
    copy      binding.PageCache.copy_from: streams into another cache, their pages packed
    attention binding.PageAttention: rows of a step against pages, tail and each other, with and without a window

A page holds 64 tokens: int8 codes and a scale per layer and head, keys [64][dim], values [dim][64].  Where codes are outputs they are
returned as code * scale.  `own` chooses between the plain form of each operator (elementary torch operations) and the library's
call.  exact() computes the same outputs in float64, written separately.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
P = 64                                                    # tokens of a page


# ----------------------------------------------------------------------------------------------- cases

def _beam(name, groups, beams, vocab, dtype, power, done):
    return {"name": name, "kind": "beam", "groups": groups, "beams": beams, "vocab": vocab, "dtype": dtype, "power": power, "done": done}


def _append(name, layers, streams, kv_heads, dim, length, rows, accepted):
    return {"name": name, "kind": "append", "layers": layers, "streams": streams, "kv_heads": kv_heads, "dim": dim, "length": length,
            "rows": rows, "accepted": accepted}


def _reorder(name, layers, groups, beams, kv_heads, dim, shared, length, window, sink):
    return {"name": name, "kind": "reorder", "layers": layers, "groups": groups, "beams": beams, "kv_heads": kv_heads, "dim": dim, "shared": shared,
            "length": length, "window": window, "sink": sink}


def _copy(name, layers, groups, beams, kv_heads, dim, shared, length, taken):
    return {"name": name, "kind": "copy", "layers": layers, "groups": groups, "beams": beams, "kv_heads": kv_heads, "dim": dim, "shared": shared,
            "length": length, "taken": taken}


def _attention(name, groups, beams, rows, kv_heads, group, dim, shared, length, window, sink, dtype):
    return {"name": name, "kind": "attention", "groups": groups, "beams": beams, "rows": rows, "kv_heads": kv_heads, "group": group, "dim": dim,
            "shared": shared, "length": length, "window": window, "sink": sink, "dtype": dtype}


def listed():
    return [
        # one request with 4 beams, fp32 logits of an odd vocabulary: latency
        _beam("beam_token", 1, 4, 32003, "fp32", 0.0, 0.0),
        # 8 requests with 16 beams each over a large vocabulary, finished ones compete by a normalised score
        _beam("beam_groups", 8, 16, 128256, "bf16", 0.8, 0.1),
        # one layer: 3 samples fork from a prompt and each takes its first token
        _append("append_token", 1, 4, 8, 64, 333, 1, 1),
        # a prompt of 4096 tokens enters the caches of a layer, in place of an older sequence
        _append("append_prompt", 1, 1, 8, 128, 0, 4096, 0),
        # a beam step's reordering, 16 layers, 8 beams behind a shared prompt
        _reorder("reorder_beams", 16, 1, 8, 8, 64, 2048, 2500, 0, 0),
        # 16 requests with 4 beams each on long histories that a window with sinks leaves behind
        _reorder("reorder_window", 2, 16, 4, 8, 64, 1000, 16400, 4096, 4),
        # one of 4 beams is taken on, odd lengths, one layer
        _copy("copy_beam", 1, 1, 4, 5, 64, 700, 1003, 1),
        # half of 16 streams into another pool, packed, 2 layers
        _copy("copy_pool", 2, 4, 4, 8, 64, 2048, 4096, 8),
        # one token of one stream against an ordinary history: latency
        _attention("attention_token", 1, 1, 1, 8, 4, 64, 0, 333, 0, 0, "bf16"),
        # a beam step: 4 requests with 8 beams each on a shared prompt
        _attention("attention_beams", 4, 8, 1, 8, 4, 64, 4096, 4500, 0, 0, "bf16"),
        # draft trees of 30 rows in 8 streams that see a window and the first tokens, fp32 out
        _attention("attention_window", 8, 1, 30, 8, 4, 64, 0, 20000, 2048, 4, "fp32"),
        # one token against 200000: bytes
        _attention("attention_long", 1, 1, 1, 8, 4, 128, 0, 200000, 0, 0, "bf16"),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(["beam", "beam", "append", "append", "reorder", "copy", "attention", "attention", "attention"])
    kv_heads, group, dim = rng.choice([1, 2, 3, 4, 5, 8, 8]), rng.randint(1, 8), rng.choice([64, 64, 128])
    if kind == "beam":
        groups, beams = _spread(rng, 1, 16), _spread(rng, 1, 32)
        while groups * beams > 128:
            groups -= 1
        vocab = rng.choice([32000, 128256, _spread(rng, 1000, 128256)])
        dtype = rng.choice(["bf16", "bf16", "fp32"]) if groups * beams <= 64 else "bf16"
        c = _beam("", groups, beams, vocab, dtype, rng.choice([0.0, 0.6, 1.0]), rng.choice([0.0, 0.1, 0.4]))
    elif kind == "append":
        if rng.random() < 0.4:
            streams = rng.randint(1, 6)
            c = _append("", 1, streams, kv_heads, dim, 0, _spread(rng, 60, 4096 // streams), 0)
        else:
            accepted = rng.randint(1, 9)
            c = _append("", _spread(rng, 1, 8), rng.randint(2, 9), kv_heads, dim, _spread(rng, 1, 3000), rng.randint(accepted, 30), accepted)
            while c["layers"] > 1 and c["layers"] * kv_heads * dim * (c["length"] + c["streams"] * P) > 8 * 128 * 4096:
                c["layers"] //= 2
    elif kind == "attention":
        groups, beams, rows = _spread(rng, 1, 8), rng.choice([1, 1, 2, 4, 7]), rng.choice([1, 1, rng.randint(2, 30)])
        length = _spread(rng, 1, 60000)
        while groups * beams * length > 200000:
            groups, length = max(1, groups // 2), max(1, length * 2 // 3)
        while groups * beams * rows * group * length * kv_heads * dim > 8 * 120 * 2048 * 8 * 64:
            rows, length = max(1, rows // 2), max(1, length * 3 // 4)
        window = rng.choice([0, 0, _spread(rng, 1, 4096)])
        c = _attention("", groups, beams, rows, kv_heads, group, dim, rng.randint(0, length) if beams > 1 else 0, length, window,
                       rng.choice([0, rng.randint(1, 100)]) if window else 0, rng.choice(["bf16", "bf16", "fp32"]))
    else:
        groups, beams, layers, length = _spread(rng, 1, 16), rng.randint(2, 8), _spread(rng, 1, 8), _spread(rng, 1, 8000)
        shared = rng.randint(0, length)
        while layers * kv_heads * dim * groups * beams * (length - shared + shared / beams + P) > 16 * 8 * 64 * 8 * 800:
            groups, layers, length = max(1, groups // 2), max(1, layers // 2), max(1, length * 2 // 3)
            shared = min(shared, length)
        if kind == "reorder":
            window = rng.choice([0, 0, _spread(rng, 1, 4096)])
            c = _reorder("", layers, groups, beams, kv_heads, dim, shared, length, window, rng.choice([0, rng.randint(1, 100)]) if window else 0)
        else:
            c = _copy("", layers, groups, beams, kv_heads, dim, shared, length, rng.randint(1, groups * beams))
    del c["name"]
    return c


# ----------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32) * std).to(dtype)


def _codes(g, shape):
    """Codes of normal values: a page's largest of several thousand is about four deviations."""
    out = torch.empty(shape, dtype=torch.int8, device=DEVICE)
    for page in out.flatten(0, 1).split(1024):
        page.copy_((torch.randn(page.shape, generator=g, device=DEVICE) * 32.0).round_().clamp_(-127.0, 127.0))
    return out


def _upload(values):
    return torch.tensor(np.asarray(values, np.int32)).to(DEVICE)


def _cache(g, rng, layers, lengths, group_of, shared, kv_heads, dim, spare):
    """A cache in use: streams of one group share the pages of their first tokens; pages lie anywhere in the pool, a stream's data in any slot."""
    S, full = len(lengths), [n // P for n in lengths]
    both, want = {}, 0
    for s in range(S):
        both.setdefault(group_of[s], min(shared // P, full[s]))
        both[group_of[s]] = min(both[group_of[s]], full[s])
        want += full[s]
    pages = list(range(want + spare))
    rng.shuffle(pages)
    columns = max(full) + 2 + spare // S
    slot, table, refs, first = list(range(S)), np.full((S, columns), -1, np.int32), np.zeros(len(pages), np.int32), {}
    rng.shuffle(slot)
    for s in range(S):
        n = both[group_of[s]]
        head = first.setdefault(group_of[s], [pages.pop() for _ in range(n)])
        table[slot[s], :full[s]] = head + [pages.pop() for _ in range(full[s] - n)]
        np.add.at(refs, table[slot[s], :full[s]], 1)
    n = len(refs)
    scale = lambda: 0.02 + 0.02 * torch.rand((layers, n, kv_heads), generator=g, device=DEVICE)   # noqa: E731
    return {"k": _codes(g, (layers, n, kv_heads, P, dim)), "v": _codes(g, (layers, n, kv_heads, dim, P)), "k_scale": scale(), "v_scale": scale(),
            "k_tail": _normal(g, (layers, S, kv_heads, P, dim)), "v_tail": _normal(g, (layers, S, kv_heads, P, dim)),
            "slot": _upload(slot), "len": _upload(lengths), "table": _upload(table), "refs": _upload(refs)}


def _accepted(g, S, R, N):
    """Rows of the accepted path of every stream: the root, then rows further down, -1 beyond."""
    path = torch.rand((S, R), generator=g, device=DEVICE)
    path[:, 0] = -1.0
    rows = torch.sort(path.argsort(-1)[:, :N], -1)[0].to(torch.int32)
    n = torch.randint(1, N + 1, (S,), generator=g, device=DEVICE)
    return torch.where(torch.arange(N, device=DEVICE) < n[:, None], rows, -1).to(torch.int32).contiguous()


def _tree(g, S, R):
    """Parents of a random draft tree: row 0 is the root, every other row continues an earlier one."""
    p = (torch.rand((S, R), generator=g, device=DEVICE) * torch.arange(R, device=DEVICE)).floor()
    p[:, 0] = -1
    return p.to(torch.int32).contiguous()


def prepare(case, seed):
    c, g, rng = case, _generator(seed), random.Random(int(seed))
    st = {"case": c}
    if c["kind"] == "beam":
        G, W, V = c["groups"], c["beams"], c["vocab"]
        st["logits"] = _normal(g, (G * W, V), TYPES[c["dtype"]], 3.0)
        st["score"] = -5.0 * torch.rand((G * W,), generator=g, device=DEVICE) - 20.0
        st["finished"] = (torch.rand((G * W,), generator=g, device=DEVICE) < c["done"]).to(torch.int32)
        st["length"] = torch.where(st["finished"] > 0, torch.randint(3, 20, (G * W,), generator=g, device=DEVICE), 20).to(torch.int32)
        st["eos"] = 2
    else:
        L, H, D = c.get("layers", 1), c["kv_heads"], c["dim"]
        if c["kind"] == "append":
            S, R, N = c["streams"], c["rows"], c["accepted"]
            lengths, group_of, shared = [c["length"]] + [0] * (S - 1), [0] * S, 0
            spare = S * ((P - 1 + (N or R)) // P + 1) + 3
            if not N:                                     # an older, shorter sequence is in the way of each prompt
                lengths, group_of = [R * (s + 1) // (S + 1) for s in range(S)], list(range(S))
            st.update(_cache(g, rng, L, lengths, group_of, shared, H, D, spare))
            st["k_new"], st["v_new"] = (_normal(g, (L, S * R, H, D)) for _ in range(2))
            st["rows"], st["source"] = None, _upload([-1] * S)
            if N:
                st["rows"], st["source"] = _accepted(g, S, R, N), _upload([0] * S)
                st["rows"][0] = -1
        else:
            G, W = c["groups"], c["beams"]
            S, group_of = G * W, [s // W for s in range(G * W)]
            if c["kind"] == "attention" and W == 1:       # streams of their own lengths, one of them as long as said
                lengths = [c["length"]] + [rng.randint((c["length"] + 1) // 2, c["length"]) for _ in range(S - 1)]
            else:
                lengths = [c["length"] - g_ % 3 if c["length"] > 3 else c["length"] for g_ in group_of]
            st.update(_cache(g, rng, L, lengths, group_of, c["shared"], H, D, 5))
            if c["kind"] == "reorder":                    # beams of a group go on from each other; here and there the last has come to its end
                source = [s // W * W + rng.randrange(W - 1) for s in range(S)]
                st["source"] = _upload([-1 if s % W == W - 1 and rng.random() < 0.3 else source[s] for s in range(S)])
            elif c["kind"] == "copy":
                T = c["taken"]
                st["source"] = _upload(sorted(rng.sample(range(S), T)))
                n, columns = max(1, T * (c["length"] // P)), st["table"].shape[1]
                z = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device=DEVICE)   # noqa: E731
                st["to"] = {"k": z((L, n, H, P, D), torch.int8), "v": z((L, n, H, D, P), torch.int8), "k_scale": z((L, n, H), torch.float32),
                            "v_scale": z((L, n, H), torch.float32), "k_tail": z((L, T, H, P, D), torch.bfloat16), "v_tail": z((L, T, H, P, D), torch.bfloat16),
                            "slot": _upload(range(T)), "len": z((T,), torch.int32), "table": _upload(np.full((T, columns), -1)), "refs": z((n,), torch.int32)}
            else:
                st["q"] = _normal(g, (S * c["rows"], H * c["group"], D), std=1.5)
                st["k_new"], st["v_new"] = (_normal(g, (S * c["rows"], H, D)) for _ in range(2))
                st["parent"] = _tree(g, S, c["rows"])
    if own:
        _handles(st)
    return st


# ----------------------------------------------------------------------------------------------- the library's calls

FIELDS = ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "slot", "len", "table", "refs")


def _handles(st):
    """The descriptors, outputs and workspaces that a program keeps from step to step."""
    import paper_2604_18655_amd as lib
    c = st["case"]
    i32 = lambda n: torch.empty((n,), dtype=torch.int32, device=DEVICE)   # noqa: E731
    if c["kind"] == "beam":
        n = c["groups"] * c["beams"]
        st["op"] = lib.BeamSelect(c["groups"], c["beams"], c["vocab"], lib.Y_BF16 if c["dtype"] == "bf16" else lib.Y_FP32, eos=st["eos"],
                                  length_power=c["power"])
        st["out"] = {"source": i32(n), "token": i32(n), "score": torch.empty((n,), device=DEVICE), "length": i32(n), "finished": i32(n)}
        st["workspace"] = torch.empty(st["op"].workspace_bytes(), dtype=torch.uint8, device=DEVICE)
        return
    st["cache"] = lib.PageCache(*(st[n] for n in FIELDS))
    if c["kind"] == "append":
        st["appended"] = i32(c["streams"])
    elif c["kind"] == "copy":
        st["other"], st["used"] = lib.PageCache(*(st["to"][n] for n in FIELDS)), i32(1)
    elif c["kind"] == "attention":
        st["op"] = lib.PageAttention(st["cache"], 0, c["kv_heads"] * c["group"], c["rows"], c["dim"] ** -0.5, st["k_new"], st["v_new"], st["parent"],
                                     window=c["window"], sink=c["sink"])
        st["out"] = torch.empty(st["q"].shape, dtype=TYPES[c["dtype"]], device=DEVICE)
        st["workspace"] = torch.empty(st["op"].workspace_bytes(), dtype=torch.uint8, device=DEVICE)


def _own_run(st):
    import paper_2604_18655_amd as lib
    c = st["case"]
    if c["kind"] == "beam":
        o = st["out"]
        st["op"].run(st["logits"], st["score"], st["length"], st["finished"], o["source"], o["token"], o["score"], o["length"], o["finished"],
                     st["workspace"])
        return o
    if c["kind"] == "append":
        st["cache"].reorder(st["source"])
        st["cache"].append(st["k_new"], st["v_new"], c["rows"], st["rows"], st["appended"])
        return dict(_values(st), appended=st["appended"])
    if c["kind"] == "reorder":
        st["cache"].reorder(st["source"], c["window"], c["sink"])
        return {n: st[n] for n in FIELDS[4:]}
    if c["kind"] == "copy":
        st["other"].copy_from(st["cache"], st["source"], st["used"])
        return dict(_values(st["to"]), used=st["used"])
    st["op"].run(st["q"], st["out"], lib.Y_BF16 if c["dtype"] == "bf16" else lib.Y_FP32, st["workspace"])
    return st["out"]


# ----------------------------------------------------------------------------------------------- the plain forms

def _values(st):
    """A cache's contents, its codes as the values they stand for."""
    out = {n: st[n] for n in FIELDS[4:]}
    out["k"], out["v"] = st["k"] * st["k_scale"][..., None, None], st["v"] * st["v_scale"][..., None, None]
    return out


def _plain_beam(st):
    c = st["case"]
    G, W, V = c["groups"], c["beams"], c["vocab"]
    z = st["logits"].float()
    score, length = st["score"].double(), st["length"].double()
    top = z.amax(-1, keepdim=True)
    lse = (top.double() + torch.exp((z - top).double()).sum(-1, keepdim=True).log())
    order = torch.sort(z, dim=-1, descending=True, stable=True)[1][:, :W]                     # no more than W of a beam are taken
    total = score[:, None] + (z.gather(1, order).double() - lse)
    done = st["finished"][:, None] > 0
    first = torch.arange(W, device=DEVICE) == 0
    total = torch.where(done, torch.where(first, score[:, None], -math.inf), total)
    token = torch.where(done, 0, order)
    grown = torch.where(done, length[:, None], length[:, None] + 1)
    rank = total / torch.clamp(grown, min=1.0) ** c["power"]
    best = torch.sort(rank.view(G, W * W), dim=-1, descending=True, stable=True)[1][:, :W]
    beam = (best // W + W * torch.arange(G, device=DEVICE)[:, None]).view(-1)
    at = (beam, (best % W).view(-1))
    token = token[at].int()
    return {"source": beam.int(), "token": token, "score": total[at].float(), "length": grown.expand(-1, W)[at].int(),
            "finished": (st["finished"][beam] > 0).int() | (token == st["eos"]).int()}


def _held(st, stream_slot):
    """Table rows of the streams whose slots are given, -1 behind their pages; lengths go with them."""
    return st["table"][stream_slot.long()]


def _plain_reorder(st, window, sink):
    S, columns = st["table"].shape
    source, slot, length = st["source"].long(), st["slot"].long(), st["len"].long()
    stream = torch.arange(S, device=DEVICE)
    valid = (source >= 0) & (source < S)
    of = torch.where(valid, source, 0)
    same = (source[:, None] == source[None, :]) & (stream[None, :] < stream[:, None])
    keeps = valid & ~same.any(1)                                                              # the first that goes on from a stream keeps its slot
    kept_slot = torch.where(keeps, slot[of], S)
    taken = (kept_slot[None, :] == stream[:, None]).any(1)
    free_slots = torch.sort(taken.int(), stable=True)[1]                                      # the others take the free ones in order
    number = torch.cumsum((~keeps).int(), 0) - 1
    new_slot = torch.where(keeps, slot[of], free_slots[number.clamp(min=0)])
    new_len = torch.where(valid, length[of], 0)
    column = torch.arange(columns, device=DEVICE)
    rows = torch.where(column < (new_len // P)[:, None], _held(st, slot[of]), -1)
    if window:
        first = new_len[:, None] - window + 1                                                 # what the next row sees begins here
        rows = torch.where((P * (column + 1) <= first) & (P * column >= sink), -1, rows)
    tail = torch.arange(P, device=DEVICE)
    fresh = ((tail < (new_len % P)[:, None]) & ~keeps[:, None])[None, :, None, :, None]
    for n in ("k_tail", "v_tail"):
        st[n].index_copy_(1, new_slot, torch.where(fresh, st[n][:, slot[of]], st[n][:, new_slot]))
    st["table"].index_copy_(0, new_slot, rows.int())
    st["refs"].zero_()
    st["refs"].scatter_add_(0, rows.clamp(min=0).view(-1).long(), (rows >= 0).int().view(-1))
    st["slot"].copy_(new_slot)
    st["len"].copy_(new_len)


def _plain_append(st):
    c = st["case"]
    L, _, H, _, D = st["k"].shape
    S, R = c["streams"], c["rows"]
    _plain_reorder(st, 0, 0)
    N = c["accepted"] or R
    row = st["rows"] if c["accepted"] else torch.arange(R, dtype=torch.int32, device=DEVICE).expand(S, R)
    n = torch.cumprod(((row >= 0) & (row < R)).int(), -1).sum(-1)
    length, slot = st["len"].long(), st["slot"].long()
    full, t = length // P, length % P
    F = (P - 1 + N) // P
    wish = (t + n) // P
    wish = torch.where(full + wish <= st["table"].shape[1], wish, 0)
    offset = torch.cumsum(wish, 0) - wish
    enters = (full + (t + n) // P <= st["table"].shape[1]) & ((wish == 0) | (offset + wish <= (st["refs"] <= 0).sum()))
    n = torch.where(enters, n, 0)
    # the stream's unfinished page and its new rows, one after the other
    i = torch.arange((F + 1) * P, device=DEVICE)
    pick = (torch.arange(S, device=DEVICE)[:, None] * R + row.long().clamp(0, R - 1)).view(-1)
    at = torch.where(i < t[:, None], i, (P + i - t[:, None]).clamp(max=P + N - 1))
    tokens = {}
    for name in ("k", "v"):
        new = st[name + "_new"].index_select(1, pick).view(L, S, N, H, D).transpose(2, 3)
        both = torch.cat([st[name + "_tail"][:, slot], new], 3)
        tokens[name] = both.gather(3, at[None, :, None, :, None].expand(L, S, H, (F + 1) * P, D))
    # pages that fill: the lowest free ones, streams in order (other pairs rewrite what free pages hold)
    j = torch.arange(F, device=DEVICE)
    fills = (j < ((t + n) // P)[:, None])
    order = torch.sort((~fills).view(-1).int(), stable=True)[1]
    number = torch.empty_like(order).scatter_(0, order, torch.arange(S * F, device=DEVICE))
    free_pages = torch.sort((st["refs"] > 0).int(), stable=True)[1]
    page = free_pages[number.clamp(max=free_pages.numel() - 1)]
    write = fills.view(-1)
    for name in ("k", "v"):
        x = tokens[name][:, :, :, :F * P].reshape(L, S, H, F, P, D).permute(0, 1, 3, 2, 4, 5).reshape(L, S * F, H, P, D).float()
        top = x.abs().amax((-1, -2))
        code = torch.where(top[..., None, None] > 0, torch.round(127.0 * x / top[..., None, None]), 0.0).to(torch.int8)
        code = code if name == "k" else code.transpose(-1, -2)
        st[name].index_copy_(1, page, torch.where(write[:, None, None, None], code, st[name][:, page]))
        st[name + "_scale"].index_copy_(1, page, torch.where(write[:, None], top / 127.0, st[name + "_scale"][:, page]))
    st["refs"].scatter_add_(0, page, write.int())
    column = torch.where(fills, full[:, None] + j, st["table"].shape[1])
    wide = torch.cat([_held(st, slot), torch.zeros((S, 1), dtype=torch.int32, device=DEVICE)], 1)
    wide.scatter_(1, column.clamp(max=st["table"].shape[1]), page.view(S, F).int())
    st["table"].index_copy_(0, slot, wide[:, :-1].contiguous())
    # what is left is the new tail
    tail = torch.arange(P, device=DEVICE)
    rest = (P * ((t + n) // P)[:, None] + tail)[None, :, None, :, None].expand(L, S, H, P, D)
    live = (tail < ((t + n) % P)[:, None])[None, :, None, :, None]
    for name in ("k", "v"):
        st[name + "_tail"].index_copy_(1, slot, torch.where(live, tokens[name].gather(3, rest), st[name + "_tail"][:, slot]))
    st["len"].copy_(length + n)
    return dict(_values(st), appended=n.int())


def _plain_copy(st):
    to, source = st["to"], st["source"].long()
    T, columns = to["table"].shape
    slot, length = st["slot"].long()[source], st["len"][source]
    rows = _held(st, slot).long()
    n = st["refs"].numel()
    count = torch.zeros(n, dtype=torch.int32, device=DEVICE).scatter_add_(0, rows.clamp(min=0).view(-1), (rows >= 0).int().view(-1))
    used = count > 0
    number = torch.cumsum(used.int(), 0) - 1
    room = to["refs"].numel()
    order = torch.sort((~used).int(), stable=True)[1][:room]
    some = torch.arange(room, device=DEVICE) < used.sum()
    for name in FIELDS[:4]:
        shape = [1, room] + [1] * (st[name].dim() - 2)
        to[name].copy_(torch.where(some.view(shape), st[name].index_select(1, order), to[name]))
    to["refs"].copy_(torch.where(some, count[order], 0))
    to["table"].copy_(torch.where(rows >= 0, number[rows.clamp(min=0)], -1))
    live = (torch.arange(P, device=DEVICE) < (length % P)[:, None])[None, :, None, :, None]
    for name in ("k_tail", "v_tail"):
        to[name].copy_(torch.where(live, st[name][:, slot], to[name]))
    to["slot"].copy_(torch.arange(T, device=DEVICE))
    to["len"].copy_(length)
    return dict(_values(to), used=used.sum().int().view(1))


def _plain_attention(st):
    c = st["case"]
    S, R, H, G, D = st["len"].numel(), c["rows"], c["kv_heads"], c["group"], c["dim"]
    slot, length = st["slot"].long(), st["len"].long()
    full = length // P
    rows = _held(st, slot)[:, :-1]
    columns = rows.shape[1]
    page = rows.clamp(min=0).long()
    keys = (st["k"][0][page].float() * st["k_scale"][0][page][..., None, None]).permute(0, 2, 1, 3, 4).reshape(S, H, columns * P, D)
    values = (st["v"][0][page].float() * st["v_scale"][0][page][..., None, None]).permute(0, 2, 1, 4, 3).reshape(S, H, columns * P, D)
    keys = torch.cat([keys, st["k_tail"][0, slot].float(), st["k_new"].view(S, R, H, D).transpose(1, 2).float()], 2)
    values = torch.cat([values, st["v_tail"][0, slot].float(), st["v_new"].view(S, R, H, D).transpose(1, 2).float()], 2)
    # positions of the rows: one behind what they continue; of the keys: pages, tail, rows
    parent = st["parent"].long().view(S, R)
    row = torch.arange(R, device=DEVICE)
    up = torch.eye(R, device=DEVICE) + (parent[:, :, None] == row).float()
    continues = torch.linalg.matrix_power(up, 64) > 0 if R > 1 else torch.ones((S, 1, 1), dtype=torch.bool, device=DEVICE)
    at = length[:, None] + continues.sum(-1) - 1
    column, i = torch.arange(columns, device=DEVICE).repeat_interleave(P), torch.arange(P, device=DEVICE)
    where = torch.cat([(P * column + i.repeat(columns)).expand(S, -1), P * full[:, None] + i, at], 1)
    there = torch.cat([(column < full[:, None]) & (rows >= 0).repeat_interleave(P, 1), i < (length % P)[:, None]], 1)
    sees = torch.cat([there[:, None, :].expand(S, R, -1), continues], 2)
    if c["window"]:
        sees = sees & ((where[:, None, :] > at[:, :, None] - c["window"]) | (where[:, None, :] < c["sink"]))
    q = st["q"].float().view(S, R, H, G, D).permute(0, 2, 1, 3, 4).reshape(S, H, R * G, D)
    x = torch.matmul(q, keys.transpose(-1, -2).contiguous()) * D ** -0.5
    x = torch.where(sees[:, None, :, None, :].expand(S, H, R, G, -1).reshape(S, H, R * G, -1), x, -math.inf)
    w = torch.exp(x - x.amax(-1, keepdim=True))
    out = torch.matmul(w, values) / w.sum(-1, keepdim=True)
    return out.view(S, H, R, G, D).permute(0, 2, 1, 3, 4).reshape(S * R, H * G, D).to(TYPES[c["dtype"]])


def run(state):
    if own:
        return _own_run(state)
    c = state["case"]
    if c["kind"] == "reorder":
        _plain_reorder(state, c["window"], c["sink"])
        return {n: state[n] for n in FIELDS[4:]}
    return {"beam": _plain_beam, "append": _plain_append, "copy": _plain_copy, "attention": _plain_attention}[c["kind"]](state)


# ----------------------------------------------------------------------------------------------- floors

def work(case):
    c = case
    if c["kind"] == "beam":
        n = c["groups"] * c["beams"]
        alive = n * (1.0 - c["done"])
        return {"bytes": alive * c["vocab"] * (2 if c["dtype"] == "bf16" else 4) + 32 * n, "flops": 3 * alive * c["vocab"]}
    H, D = c["kv_heads"], c["dim"]
    if c["kind"] == "attention":
        S, R, G = c["groups"] * c["beams"], c["rows"], c["group"]
        length = c["length"] if c["beams"] > 1 else 0.75 * c["length"] + 0.25 * c["length"] / c["groups"]
        alone = length - (c["shared"] if c["beams"] > 1 else 0)
        seen = min(length, c["window"] + c["sink"]) if c["window"] else length
        read = min(alone, seen) * S + max(0, seen - alone) * c["groups"]          # tokens of pages that someone sees, shared ones once
        return {"bytes": H * (read * 2 * D + S * R * (4 * D + G * D * (4 if c["dtype"] == "bf16" else 6))), "flops": 4 * D * S * R * G * H * (seen + 1)}
    L, row = c["layers"], 2 * D
    if c["kind"] == "append":
        n = (c["accepted"] + 1) / 2 * (c["streams"] - 1) if c["accepted"] else c["streams"] * c["rows"]
        forked = (c["streams"] - 1) * (c["length"] % P) if c["accepted"] else 0
        pool = (c["length"] // P if c["accepted"] else c["streams"] * c["rows"] / 2 / P) + c["streams"] * (c["rows"] // P + 1)
        return {"bytes": L * H * (n * 2 * row + (n * 2 * row if c["accepted"] else n * row) + forked * 4 * row + pool * P * (row + 8 * D)),
                "flops": 3 * L * H * n * row}
    S = c["groups"] * c["beams"]
    if c["kind"] == "reorder":
        forks = 0.5 * S
        return {"bytes": L * H * forks * (c["length"] % P) * 4 * row + 8 * S * (c["length"] // P + 4), "flops": 0.0}
    share = min(1.0, c["taken"] / c["groups"])
    pages = (c["shared"] // P) * c["groups"] * share + ((c["length"] - c["shared"]) / P) * c["taken"]
    pool = (c["length"] // P) * c["taken"]
    return {"bytes": L * H * (pages * 2 * P * row + c["taken"] * (c["length"] % P) * 4 * row + pool * P * (row + 8 * D)), "flops": 0.0}


# ----------------------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"beam": _exact_beam, "append": _exact_append, "reorder": _exact_reorder, "copy": _exact_copy, "attention": _exact_attention}[case["kind"]](st)


def _exact_beam(st):
    """Every candidate of a group in one list."""
    c = st["case"]
    W, V = c["beams"], c["vocab"]
    got = []
    for group in range(c["groups"]):
        mine = slice(group * W, (group + 1) * W)
        logp = torch.log_softmax(st["logits"][mine].double(), -1) + st["score"][mine].double()[:, None]
        grown = (st["length"][mine].double() + 1).clamp(min=1) ** c["power"]
        done = st["finished"][mine] > 0
        rank = logp / grown[:, None]
        rank[done] = -math.inf
        rank[done, 0] = (st["score"][mine].double() / st["length"][mine].double().clamp(min=1) ** c["power"])[done]
        logp[done, 0] = st["score"][mine].double()[done]
        best = torch.topk(rank.view(-1), W)[1]
        got.append(logp.view(-1)[best])
    return {"source": None, "token": None, "score": torch.cat(got), "length": None, "finished": None}


def _sequences(st):
    """Every stream's tail in 64 bits, and its pages."""
    slot, length, table = (st[n].tolist() for n in ("slot", "len", "table"))
    tails = [[st[n][:, slot[s], :, :length[s] % P].double() for n in ("k_tail", "v_tail")] for s in range(len(slot))]
    return slot, length, [table[slot[s]][:length[s] // P] for s in range(len(slot))], tails


def _moved(st, source):
    """Streams that become others: the new slots, and tails where the first that goes on from a stream keeps its place."""
    slot, length, pages, tails = _sequences(st)
    S, new, left = len(slot), {}, set(range(len(slot)))
    for s in range(S):
        if 0 <= source[s] < S and source[s] not in source[:s]:
            new[s] = slot[source[s]]
            left.discard(new[s])
    for s in range(S):
        if s not in new:
            new[s] = min(left)
            left.discard(new[s])
    k, v = st["k_tail"].double(), st["v_tail"].double()
    for s in range(S):
        if 0 <= source[s] < S:
            n = length[source[s]] % P
            k[:, new[s], :, :n], v[:, new[s], :, :n] = tails[source[s]]
    old = [length[x] if 0 <= x < S else 0 for x in source]
    held = [pages[x] if 0 <= x < S else [] for x in source]
    return new, old, held, k, v


def _exact_reorder(st):
    _, _, _, k, v = _moved(st, st["source"].tolist())
    return {"k_tail": k, "v_tail": v, "slot": None, "len": None, "table": None, "refs": None}


def _exact_append(st):
    c = st["case"]
    source = st["source"].tolist()
    new, length, held, k_tail, v_tail = _moved(st, source)
    S, R = c["streams"], c["rows"]
    k, v = (st[n].double() * st[n + "_scale"].double()[..., None, None] for n in ("k", "v"))
    lists = [list(range(R))] * S if st["rows"] is None else [[r for r in x if r >= 0] for x in st["rows"].tolist()]
    used = {p for row in held for p in row}
    free_pages = [p for p in range(st["refs"].numel()) if p not in used]
    for s in range(S):
        t = length[s] % P
        mine = [s * R + r for r in lists[s]]
        for name, pool, tail in (("k", k, k_tail), ("v", v, v_tail)):
            rows = torch.cat([tail[:, new[s], :, :t], st[name + "_new"][:, mine].double().transpose(1, 2)], 2)
            n = rows.shape[2] // P
            for j in range(n):
                x = rows[:, :, j * P:(j + 1) * P]
                top = x.abs().amax((2, 3), keepdim=True)
                x = torch.round(127.0 * x / top) * (top / 127.0)
                pool[:, free_pages[j]] = x if name == "k" else x.transpose(2, 3)
            rest = rows[:, :, n * P:]
            tail[:, new[s], :, :rest.shape[2]] = rest
        free_pages = free_pages[(t + len(mine)) // P:]
    return {"k_tail": k_tail, "v_tail": v_tail, "slot": None, "len": None, "table": None, "refs": None, "k": k, "v": v, "appended": None}


def _exact_copy(st):
    _, length, pages, tails = _sequences(st)
    source, to = st["source"].tolist(), st["to"]
    used = sorted({p for s in source for p in pages[s]})
    out = {"k_tail": to["k_tail"].double(), "v_tail": to["v_tail"].double(), "slot": None, "len": None, "table": None, "refs": None}
    for i, s in enumerate(source):
        for name, tail in zip(("k_tail", "v_tail"), tails[s]):
            out[name][:, i, :, :tail.shape[2]] = tail
    for name in ("k", "v"):
        x = torch.zeros(to[name].shape, dtype=torch.float64, device=DEVICE)
        x[:, :len(used)] = st[name][:, used].double() * st[name + "_scale"][:, used].double()[..., None, None]
        out[name] = x
    return dict(out, used=None)


def _exact_attention(st):
    c = st["case"]
    R, H, G, D = c["rows"], c["kv_heads"], c["group"], c["dim"]
    _, length, pages, tails = _sequences(st)
    parent = st["parent"].view(-1, R).tolist()
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEVICE)
    for s in range(len(length)):
        T, held = length[s], torch.tensor(pages[s], dtype=torch.long, device=DEVICE)
        mine = slice(s * R, (s + 1) * R)
        paths = []
        for r in range(R):
            paths.append([r] + (paths[parent[s][r]] if 0 <= parent[s][r] < r else []))
        depth = torch.tensor([len(x) - 1 for x in paths], device=DEVICE)
        hidden = torch.ones((R, T + R), dtype=torch.bool, device=DEVICE)
        hidden[:, :T] = False
        for r in range(R):
            hidden[r, [T + x for x in paths[r]]] = False
        where = torch.cat([torch.arange(T, device=DEVICE), T + depth])
        if c["window"]:
            hidden |= (where[None, :] <= (T + depth)[:, None] - c["window"]) & (where >= c["sink"])
        for h in range(H):
            k = (st["k"][0, held, h].double() * st["k_scale"][0, held, h].double()[:, None, None]).reshape(-1, D)
            v = (st["v"][0, held, h].double() * st["v_scale"][0, held, h].double()[:, None, None]).transpose(1, 2).reshape(-1, D)
            k = torch.cat([k, tails[s][0][0, h], st["k_new"][mine, h].double()])
            v = torch.cat([v, tails[s][1][0, h], st["v_new"][mine, h].double()])
            x = torch.matmul(st["q"][mine, h * G:(h + 1) * G].double().reshape(R * G, D), k.t().contiguous()) / math.sqrt(D)
            x = x.view(R, G, T + R).masked_fill_(hidden[:, None, :], -math.inf)
            out[mine, h * G:(h + 1) * G] = torch.matmul(torch.softmax(x, -1).view(R * G, T + R), v).view(R, G, D)
    return out
