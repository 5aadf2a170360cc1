"""Operators of a decoding loop on a bounded cache, as timed cases: rotary positions, rows appended to the streams'
caches, accumulated attention weights, compression of a long segment to its heaviest slots, rules on logits.

A case is a dict of plain values.  Its "kind" names the public call it stands for:

    rope_tables   binding.RopeTables: cosines and sines of the rows' positions, as the fused projections read them
    rope          binding.RopePlan: rotation of query and key heads by the rows' positions
    append        binding.StreamCache.append: the accepted rows of a step, all layers in one call, evicting where the cache is full
    weights       binding.AttentionMass: attention weights of the newest rows added to what every slot has received so far
    compress      binding.StreamCache.compress: the heaviest slots of a segment, in order, into a smaller one
    rules         binding.LogitRules: penalties, biases and grammar masks on the rows of a draft tree

`own` chooses between the plain form of each operator (elementary torch operations) and the library's call.
exact() computes the same outputs in float64, written separately.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ----------------------------------------------------------------------------------------------- cases

def _rope(name, streams, rows, kv_heads, group, dim, rot, layout, scaling, dtype, inverse=False, into_cache=False, far=131072):
    return {"name": name, "kind": "rope", "streams": streams, "rows": rows, "kv_heads": kv_heads, "group": group, "dim": dim, "rot": rot,
            "layout": layout, "scaling": scaling, "dtype": dtype, "inverse": inverse, "into_cache": into_cache, "far": far}


def _tables(name, streams, rows, rot, scaling, far=131072):
    return {"name": name, "kind": "rope_tables", "streams": streams, "rows": rows, "rot": rot, "scaling": scaling, "far": far}


def _append(name, layers, streams, kv_heads, dim, cap, budget, rows, accepted, sink, recent, full):
    return {"name": name, "kind": "append", "layers": layers, "streams": streams, "kv_heads": kv_heads, "dim": dim, "cap": cap, "budget": budget,
            "rows": rows, "accepted": accepted, "sink": sink, "recent": recent, "full": full}


def _weights(name, layers, streams, kv_heads, group, dim, prefill, cap, rows, accepted, decay):
    return {"name": name, "kind": "weights", "layers": layers, "streams": streams, "kv_heads": kv_heads, "group": group, "dim": dim,
            "prefill": prefill, "cap": cap, "rows": rows, "accepted": accepted, "decay": decay}


def _compress(name, layers, streams, kv_heads, dim, cap, budget, sink, recent):
    return {"name": name, "kind": "compress", "layers": layers, "streams": streams, "kv_heads": kv_heads, "dim": dim, "cap": cap, "budget": budget,
            "sink": sink, "recent": recent}


def _rules(name, streams, rows, tokens, vocab, dtype, history, new):
    return {"name": name, "kind": "rules", "streams": streams, "rows": rows, "tokens": tokens, "vocab": vocab, "dtype": dtype,
            "history": history, "new": new}


def listed():
    return [
        # one token in each of 8 streams, the heads of a 1B-like layer, far positions with blended frequencies: latency
        _rope("rope_token", 8, 1, 8, 4, 64, 64, "half", "turns", "bf16"),
        # draft trees of 30 rows in fp32, a quarter of the head rotated back (the gradient's direction), neighbours paired
        _rope("rope_back", 8, 30, 8, 4, 128, 32, "interleaved", "linear", "fp32", inverse=True),
        # a long prompt: queries rotated, keys rotated into the cache segment, values moved there
        _rope("rope_prompt", 1, 4096, 8, 4, 128, 128, "half", "plain", "bf16", into_cache=True, far=1),
        # one layer, one stream, one token into a short cache with room and without
        _append("append_token", 1, 1, 8, 64, 200, 128, 1, 1, 4, 32, True),
        # a decoding step of a 16-layer stack: 8 streams, up to 3 accepted rows of a tree of 30, caches full
        _append("append_stack", 16, 8, 8, 64, 1088, 1024, 30, 3, 4, 64, True),
        # one token of one stream against its prompt and what it has produced
        _weights("weights_token", 1, 1, 8, 4, 64, 2048, 128, 1, 1, 1.0),
        # the step of the stack: a shared prompt, 8 streams, the accepted rows' weights
        _weights("weights_stack", 16, 8, 8, 4, 64, 2048, 1088, 30, 3, 0.98),
        # a chunk of a long prompt scoring everything before it
        _weights("weights_prompt", 1, 1, 8, 4, 128, 0, 16384, 512, 0, 1.0),
        # an odd segment of one layer
        _compress("compress_short", 1, 3, 5, 64, 1003, 257, 4, 64),
        # a prompt of a 16-layer stack to an eighth
        _compress("compress_prompt", 16, 1, 8, 128, 16384, 2048, 4, 64),
        # one token in each of 8 streams, fp32 logits of an odd vocabulary
        _rules("rules_token", 8, 1, 1, 32003, "fp32", 300, 1),
        # 8 streams x 30 rows of a draft tree over a large vocabulary
        _rules("rules_tree", 8, 30, 10, 128256, "bf16", 2048, 3),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "rope_tables", "append", "append", "weights", "weights", "compress", "compress", "rules", "rules"])
    scaling = rng.choice(["plain", "linear", "base", "turns"])
    kv_heads, group, dim = rng.choice([1, 2, 3, 4, 5, 8, 8]), rng.randint(1, 8), rng.choice([64, 64, 128])
    if kind == "rope_tables":
        c = _tables("", rng.randint(1, 8), _spread(rng, 1, 512), 2 * rng.randint(2, 64), scaling, _spread(rng, 16, 1 << 20))
    elif kind == "rope":
        prompt = rng.random() < 0.4
        dim = rng.choice([32, 64, 80, 96, 128, 128])
        rot = dim if rng.random() < 0.5 else 2 * rng.randint(2, dim // 2)
        streams = 1 if prompt else rng.randint(1, 16)
        rows = _spread(rng, 65, 3000) if prompt else _spread(rng, 1, 64)
        c = _rope("", streams, rows, kv_heads, min(group, 4), dim, rot, rng.choice(["half", "interleaved"]), scaling,
                  "bf16" if prompt else rng.choice(["bf16", "fp32"]), inverse=rng.random() < 0.3, into_cache=prompt and rng.random() < 0.7,
                  far=_spread(rng, 16, 1 << 20))
    elif kind == "append":
        accepted = rng.randint(1, 9)
        sink, recent = rng.randint(0, 8), rng.randint(0, 64)
        budget = accepted + sink + recent + _spread(rng, 8, 3000)
        layers, streams = _spread(rng, 1, 16), _spread(rng, 1, 8)
        while layers * streams * kv_heads * budget * dim > 16 * 8 * 8 * 1024 * 64:
            layers, streams = max(1, layers // 2), max(1, streams * 2 // 3)
        c = _append("", layers, streams, kv_heads, dim, budget + rng.randint(0, 70), budget, rng.randint(accepted, 30), accepted, sink, recent,
                    rng.random() < 0.7)
    elif kind == "weights":
        if rng.random() < 0.35:
            c = _weights("", 1, 1, kv_heads, min(group, 4), dim, 0, _spread(rng, 300, 12000), _spread(rng, 17, 300), 0, rng.choice([1.0, 0.95]))
        else:
            accepted = rng.randint(1, 9)
            c = _weights("", _spread(rng, 1, 8), _spread(rng, 1, 8), kv_heads, group, dim, rng.choice([0, _spread(rng, 1, 4000)]), _spread(rng, 16, 2000),
                         rng.randint(accepted, 30), accepted, rng.choice([1.0, 0.95]))
    elif kind == "compress":
        cap = _spread(rng, 40, 16000)
        sink, recent = rng.randint(0, 4), rng.randint(0, 16)
        budget = max(sink + recent + 1, int(cap * rng.uniform(0.05, 0.6)))
        layers, streams = _spread(rng, 1, 16), _spread(rng, 1, 4)
        while layers * streams * kv_heads * cap * dim > 16 * 8 * 16384 * 64:
            layers, streams = max(1, layers // 2), max(1, streams // 2)
        c = _compress("", layers, streams, kv_heads, dim, cap, budget, sink, recent)
    else:
        rows = _spread(rng, 1, 30)
        vocab = rng.choice([32000, 128256, _spread(rng, 1000, 128256)])
        c = _rules("", rng.randint(1, 8), rows, rng.randint(1, rows), vocab, rng.choice(["bf16", "bf16", "fp32"]) if rows <= 14 else "bf16",
                   _spread(rng, 1, 8000), rng.randint(0, 9))
    del c["name"]
    return c


# ----------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32) * std).to(dtype)


def _ints(g, low, high, shape):
    return torch.randint(low, high, shape, generator=g, device=DEVICE, dtype=torch.int32)


SCALES = {"plain": {}, "linear": {"factor": 4.0}, "base": {"factor": 8.0}, "turns": {"factor": 8.0, "low": 1.0, "high": 4.0, "context": 8192}}
THETA = 500000.0


def _frequencies(rot, scaling):
    """Radians per position of every pair, float64."""
    i, p = np.arange(rot // 2, dtype=np.float64), SCALES[scaling]
    if scaling == "base":
        return (THETA * p["factor"] ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
    f = THETA ** (-2.0 * i / rot)
    if scaling == "linear":
        return f / p["factor"]
    if scaling == "turns":
        share = np.clip((p["context"] * f / (2 * np.pi) - p["low"]) / (p["high"] - p["low"]), 0.0, 1.0)
        return (1.0 - share) * f / p["factor"] + share * f
    return f


def _positions(g, c):
    base = _ints(g, 0, c["far"], (c["streams"],))
    offset = torch.arange(c["rows"], dtype=torch.int32, device=DEVICE)
    if c["kind"] == "rope" and not c["into_cache"]:
        offset = torch.sort(_ints(g, 0, 9, (c["rows"],)))[0].to(torch.int32)   # levels of a draft tree
    return base, offset


def _cache(g, c, full=True, window=0):
    """K, V, accumulated weights, positions and lengths of the streams' slots.  The live slots hold the newest positions in
    any order (a slot that was evicted takes a newer row)."""
    L, S, H, cap, D = c["layers"], c["streams"], c["kv_heads"], c["cap"], c["dim"]
    top = c.get("budget", cap) if c["kind"] == "append" else cap
    length = torch.full((S,), top, dtype=torch.int32, device=DEVICE)
    if not full:
        length = _ints(g, max(1, window, top // 2), top + 1, (S,))
    older = _ints(g, 0, 5000, (S,)) if c["kind"] != "compress" else torch.zeros(S, dtype=torch.int32, device=DEVICE)
    slot = torch.arange(cap, device=DEVICE)
    if c["kind"] == "append" or c.get("accepted"):
        r = torch.rand((L, S, H, cap), generator=g, device=DEVICE)
        r = torch.where(slot < length[:, None, None], r, 2.0)
        order = r.argsort(-1).argsort(-1).to(torch.int32)
    else:
        order = slot.to(torch.int32).expand(L, S, H, cap).contiguous()      # a prompt: slots in order of position
    mass = torch.exp(1.5 * torch.randn((L, S, H, cap), generator=g, device=DEVICE)) * 0.1
    mass = mass * (torch.rand((L, S, H, cap), generator=g, device=DEVICE) > 0.05)          # some never attended to: ties
    return {"k": _normal(g, (L, S, H, cap, D)), "v": _normal(g, (L, S, H, cap, D)), "mass": mass,
            "slot_pos": (order + older[:, None, None]).to(torch.int32).contiguous(), "len": length, "next_pos": (older + length).to(torch.int32)}


def _accepted(g, c):
    """Rows of the accepted path of every stream: the root, then rows further down, -1 beyond."""
    S, R, N = c["streams"], c["rows"], c["accepted"]
    path = torch.rand((S, R), generator=g, device=DEVICE)
    path[:, 0] = -1.0
    rows = torch.sort(path.argsort(-1)[:, :N], -1)[0].to(torch.int32)
    n = _ints(g, 1, N + 1, (S,))
    return torch.where(torch.arange(N, device=DEVICE) < n[:, None], rows, -1).to(torch.int32).contiguous()


def _tree(g, c):
    """Parents of a random draft tree: row 0 is the root, every other row continues an earlier one (token rows stand first)."""
    S, R = c["streams"], c["rows"]
    row = torch.arange(R, device=DEVICE)
    p = (torch.rand((S, R), generator=g, device=DEVICE) * row).floor()
    p[:, 0] = -1
    return p.to(torch.int32).contiguous()


def prepare(case, seed):
    c, g = case, _generator(seed)
    st = {"case": c}
    if c["kind"] in ("rope", "rope_tables"):
        st["base"], st["offset"] = _positions(g, c)
        st["freq"] = torch.from_numpy(_frequencies(c["rot"], c["scaling"])).to(DEVICE)
        if c["kind"] == "rope":
            M, H, G, D = c["streams"] * c["rows"], c["kv_heads"], c["group"], c["dim"]
            st["q"], st["k"] = _normal(g, (M, H * G, D), TYPES[c["dtype"]]), _normal(g, (M, H, D), TYPES[c["dtype"]])
            if c["into_cache"]:
                st["v"] = _normal(g, (M, H, D), TYPES[c["dtype"]])
    elif c["kind"] == "append":
        st.update(_cache(g, c, c["full"]))
        M = c["streams"] * c["rows"]
        st["k_new"], st["v_new"] = (_normal(g, (c["layers"], M, c["kv_heads"], c["dim"])) for _ in range(2))
        st["rows"] = _accepted(g, c)
    elif c["kind"] == "weights":
        st.update(_cache(g, c, c["accepted"] == 0, c["accepted"]))
        L, H, P = c["layers"], c["kv_heads"], c["prefill"]
        st["q"] = _normal(g, (L, c["streams"] * c["rows"], H * c["group"], c["dim"]), std=1.5)
        st["rows"] = _accepted(g, c) if c["accepted"] else None
        st["k_prefill"] = _normal(g, (L, H, P, c["dim"])) if P else None
        st["mass_prefill"] = torch.rand((L, H, P), generator=g, device=DEVICE) if P else None
    elif c["kind"] == "compress":
        st.update(_cache(g, c))
    else:
        S, R, T, V = c["streams"], c["rows"], c["tokens"], c["vocab"]
        st["logits"] = _normal(g, (S * R, V), TYPES[c["dtype"]], 3.0)
        st["parent"] = _tree(g, c)
        zipf = lambda shape: (V * torch.rand(shape, generator=g, device=DEVICE) ** 4).to(torch.int32).clamp(max=V - 1)   # noqa: E731
        st["tokens"] = zipf((S, T))
        st["counts"] = torch.zeros((S, V), dtype=torch.int32, device=DEVICE)
        seen = zipf((S, c["history"])).long()
        st["counts"].scatter_add_(1, seen, torch.ones_like(seen, dtype=torch.int32))
        st["new"] = zipf((S, c["new"]))
        if c["new"]:
            st["new"][:, -1] = torch.where(_ints(g, 0, 2, (S,)) > 0, st["new"][:, -1], -1)
        st["repetition"] = 1.0 + torch.rand(S, generator=g, device=DEVICE)
        st["frequency"] = torch.rand(S, generator=g, device=DEVICE)
        st["presence"] = torch.rand(S, generator=g, device=DEVICE)
        some = torch.rand((2, V), generator=g, device=DEVICE) < 0.003
        st["bias"] = torch.where(some, torch.randn((2, V), generator=g, device=DEVICE) * 5.0, 0.0)
        st["bias_row"] = _ints(g, -1, 2, (S,))
        words = (V + 31) // 32
        full = torch.full((3, words), -1, dtype=torch.int32, device=DEVICE)
        hits = _ints(g, -2 ** 31, 2 ** 31 - 1, (3, words))
        keep = torch.rand((3, words), generator=g, device=DEVICE)
        few = torch.where(keep < 0.02, hits, 0)                        # a grammar that allows little, one that forbids little, half of all
        most = torch.where(keep < 0.02, hits, full)
        st["masks"] = torch.stack([few[0], most[1], hits[2]]).contiguous()
        st["mask_row"] = _ints(g, -1, 3, (S * R,))
    if own:
        _handles(st)
    return st


# ----------------------------------------------------------------------------------------------- the library's calls

def _handles(st):
    """The descriptors, plans, outputs and workspaces that a program keeps from step to step."""
    import paper_2604_18655_amd as lib
    c = st["case"]
    kind = c["kind"]
    if kind in ("rope", "rope_tables"):
        M = c["streams"] * c["rows"]
        names = {"plain": lib.ROPE_PLAIN, "linear": lib.ROPE_LINEAR, "base": lib.ROPE_BASE, "turns": lib.ROPE_TURNS}
        rope = lib.Rope(c.get("dim", c["rot"]), c["rot"], lib.ROPE_INTERLEAVED if c.get("layout") == "interleaved" else lib.ROPE_HALF,
                        names[c["scaling"]], THETA, device=DEVICE, **SCALES[c["scaling"]])
        at = dict(rows_per_stream=c["rows"], base=st["base"], offset=st["offset"])
        if kind == "rope_tables":
            out = [torch.empty((M, c["rot"] // 2), device=DEVICE) for _ in range(2)]
            st["plan"] = lib.RopeTables(rope, out[0], out[1], M, **at)
        else:
            out = [torch.empty_like(st["q"])]
            moves = [lib.RopeTensor(st["q"], out[0])]
            if c["into_cache"]:
                out += [torch.empty((c["kv_heads"], M, c["dim"]), dtype=st["k"].dtype, device=DEVICE) for _ in range(2)]
                moves += [lib.RopeTensor(st["k"], out[1].permute(1, 0, 2)), lib.RopeTensor(st["v"], out[2].permute(1, 0, 2), rotate=False)]
            else:
                out += [torch.empty_like(st["k"])]
                moves += [lib.RopeTensor(st["k"], out[1])]
            st["plan"] = lib.RopePlan(rope, moves, M, lib.Y_BF16 if c["dtype"] == "bf16" else lib.Y_FP32, inverse=c["inverse"], **at)
        st["out"] = out
    elif kind in ("append", "weights", "compress"):
        cache = lib.StreamCache(st["k"], st["v"], st["mass"], st["slot_pos"], st["len"], st["next_pos"])
        st["cache"] = cache
        if kind == "weights":
            st["mass_op"] = lib.AttentionMass(cache, c["kv_heads"] * c["group"], c["rows"], c["dim"] ** -0.5, k_prefill=st["k_prefill"],
                                              mass_prefill=st["mass_prefill"], decay=c["decay"])
            st["workspace"] = torch.empty(max(256, st["mass_op"].workspace_bytes(c["accepted"])), dtype=torch.uint8, device=DEVICE)
        elif kind == "compress":
            L, S, H, B, D = c["layers"], c["streams"], c["kv_heads"], c["budget"], c["dim"]
            to = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=DEVICE)   # noqa: E731
            st["to"] = {"k": to((L, S, H, B, D), st["k"].dtype), "v": to((L, S, H, B, D), st["v"].dtype), "mass": to((L, S, H, B), torch.float32),
                        "slot_pos": to((L, S, H, B), torch.int32), "len": to((S,), torch.int32), "next_pos": to((S,), torch.int32)}
            st["smaller"] = lib.StreamCache(*(st["to"][n] for n in ("k", "v", "mass", "slot_pos", "len", "next_pos")))
            st["kept"] = to((L, S, H, B), torch.int32)
    else:
        st["rules"] = lib.LogitRules(c["streams"], c["rows"], c["tokens"], c["vocab"], lib.Y_BF16 if c["dtype"] == "bf16" else lib.Y_FP32, st["parent"],
                                     counts=st["counts"], repetition=st["repetition"], frequency=st["frequency"], presence=st["presence"],
                                     bias=st["bias"], bias_row=st["bias_row"], masks=st["masks"], mask_row=st["mask_row"])
        st["out"] = torch.empty_like(st["logits"])


def _own_run(st):
    c = st["case"]
    kind = c["kind"]
    if kind in ("rope", "rope_tables"):
        st["plan"].run()
        return st["out"]
    if kind == "append":
        st["cache"].append(st["k_new"], st["v_new"], c["rows"], st["rows"], c["budget"], c["sink"], c["recent"])
        return {n: st[n] for n in ("k", "v", "mass", "slot_pos", "len", "next_pos")}
    if kind == "weights":
        st["mass_op"].run(st["q"], st["rows"], st["workspace"])
        return [st["mass"]] + ([st["mass_prefill"]] if c["prefill"] else [])
    if kind == "compress":
        st["cache"].compress(st["smaller"], st["kept"], c["budget"], c["sink"], c["recent"])
        return dict(st["to"], kept=st["kept"])
    st["rules"].run(st["logits"], st["tokens"], st["out"], new_tokens=st["new"])
    return {"logits": st["out"], "counts": st["counts"]}


# ----------------------------------------------------------------------------------------------- the plain forms

def _rows_positions(st):
    return (st["base"].long()[:, None] + st["offset"].long()[None, :]).reshape(-1)


def _rotate(x, cos, sin, rot, interleaved):
    y = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, w = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, w
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = u, w
    return y


def _plain_rope(st):
    c = st["case"]
    angle = _rows_positions(st).double()[:, None] * st["freq"][None, :]
    cos, sin = torch.cos(angle), torch.sin(angle)
    if c["kind"] == "rope_tables":
        return [cos.float(), sin.float()]
    cos, sin = cos.float()[:, None, :], (-sin if c["inverse"] else sin).float()[:, None, :]
    out = [_rotate(st[n].float(), cos, sin, c["rot"], c["layout"] == "interleaved").to(st[n].dtype) for n in ("q", "k")]
    if c["into_cache"]:
        out = [out[0], out[1].permute(1, 0, 2).contiguous(), st["v"].permute(1, 0, 2).contiguous()]
    return out


def _order(st, sink, recent):
    """Rank of every live slot: protected ones first, then the heavier, then the lower slot; NaN behind every number."""
    L, S, H, cap = st["mass"].shape
    slot = torch.arange(cap, device=DEVICE)
    live = (slot < st["len"][:, None, None]).expand(L, S, H, cap)
    kept = (st["slot_pos"] >= (st["next_pos"] - recent)[:, None, None]) | (st["slot_pos"] < sink)
    nan = torch.isnan(st["mass"])
    group = torch.where(~live, -1, torch.where(kept, 2, torch.where(nan, 0, 1)))
    weight = torch.where(nan | kept, 0.0, st["mass"])
    by_weight = torch.sort(weight, dim=-1, descending=True, stable=True)[1]
    by_group = torch.sort(group.gather(-1, by_weight), dim=-1, descending=True, stable=True)[1]
    order = by_weight.gather(-1, by_group)
    rank = torch.empty_like(order)
    rank.scatter_(-1, order, slot.expand(L, S, H, cap))
    return rank, live


def _listed_rows(rows, R, S):
    """(row of each entry, whether it counts): the entries before the first that names no row."""
    if rows is None:
        return torch.arange(R, device=DEVICE).expand(S, R), torch.ones((S, R), dtype=torch.bool, device=DEVICE)
    ok = torch.cumprod(((rows >= 0) & (rows < R)).int(), -1).bool()
    return torch.where(ok, rows, 0).long(), ok


def _plain_append(st):
    c = st["case"]
    L, S, H, cap, D = st["k"].shape
    R = c["rows"]
    rows, ok = _listed_rows(st["rows"], R, S)
    N, n = rows.shape[1], ok.sum(-1)
    T = st["len"].long()
    top = torch.clamp(T, min=c["budget"])
    evict = torch.clamp(T + n - top, min=0)
    room = n - evict
    rank, live = _order(st, c["sink"], c["recent"])
    gone = live & (rank >= (T - evict)[:, None, None])
    number = torch.cumsum(gone.long(), -1) - 1
    j = torch.arange(N, device=DEVICE)
    target = (T[:, None] + j)[None, :, None, :].expand(L, S, H, N)
    target = torch.cat([target, target[..., :1]], -1)                                     # the last column takes what is not evicted
    at = torch.where(gone, number + room[:, None, None], N)
    target = target.scatter(-1, at, torch.arange(cap, device=DEVICE).expand(L, S, H, cap))[..., :N]
    use = torch.where(ok, j, 0)                                                           # entries that do not count repeat the first
    target = target.gather(-1, use[None, :, None, :].expand(L, S, H, N)).contiguous()
    pick = (torch.arange(S, device=DEVICE)[:, None] * R + rows.gather(1, use)).reshape(-1)
    for name in ("k", "v"):
        new = st[name + "_new"].index_select(1, pick).view(L, S, N, H, D).transpose(2, 3)
        st[name].scatter_(3, target[..., None].expand(L, S, H, N, D), new)
    st["mass"].scatter_(-1, target, 0.0)
    st["slot_pos"].scatter_(-1, target, (st["next_pos"][:, None] + use.int())[None, :, None, :].expand(L, S, H, N).contiguous())
    st["len"].copy_(T + room)
    st["next_pos"].add_(n.int())
    return {n: st[n] for n in ("k", "v", "mass", "slot_pos", "len", "next_pos")}


def _plain_weights(st):
    c = st["case"]
    L, S, H, cap, D = st["k"].shape
    R, G, P = c["rows"], c["group"], c["prefill"]
    rows, ok = _listed_rows(st["rows"], R, S)
    N = rows.shape[1]
    pick = (torch.arange(S, device=DEVICE)[:, None] * R + rows).reshape(-1)
    q = st["q"].index_select(1, pick).view(L, S, N, H, G, D).permute(0, 1, 3, 2, 4, 5).reshape(L, S, H, N * G, D).float()
    pos = st["next_pos"].long()[:, None] - ok.sum(-1)[:, None] + torch.arange(N, device=DEVICE)
    live = torch.arange(cap, device=DEVICE) < st["len"][:, None, None]                    # [S][1][cap]
    visible = live[None, :, :, None, :] & (st["slot_pos"][:, :, :, None, :] <= pos[None, :, None, :, None]) & ok[None, :, None, :, None]
    s = torch.matmul(q, st["k"].float().transpose(-1, -2)) * D ** -0.5
    s = torch.where(visible[:, :, :, :, None, :].expand(L, S, H, N, G, cap).reshape(L, S, H, N * G, cap), s, -math.inf)
    top = s.amax(-1, keepdim=True)
    if P:
        t = torch.matmul(q.transpose(1, 2).reshape(L, H, S * N * G, D), st["k_prefill"].float().transpose(-1, -2)) * D ** -0.5
        t = t.view(L, H, S, N * G, P).transpose(1, 2)
        t = torch.where(ok[None, :, None, :, None, None].expand(L, S, H, N, G, P).reshape(L, S, H, N * G, P), t, -math.inf)
        top = torch.maximum(top, t.amax(-1, keepdim=True))
    top = torch.where(torch.isinf(top), 0.0, top)
    s = torch.exp(s - top)
    total = s.sum(-1, keepdim=True)
    if P:
        t = torch.exp(t - top)
        total = total + t.sum(-1, keepdim=True)
    inv = torch.where(total > 0, 1.0 / total, 0.0)
    st["mass"].copy_(torch.where(live, c["decay"] * st["mass"] + (s * inv).sum(-2), st["mass"]))
    if P:
        st["mass_prefill"].mul_(c["decay"]).add_((t * inv).sum((1, 3)))
    return [st["mass"]] + ([st["mass_prefill"]] if P else [])


def _plain_compress(st):
    c = st["case"]
    L, S, H, cap, D = st["k"].shape
    B = c["budget"]
    rank, live = _order(st, c["sink"], c["recent"])
    slot = torch.arange(cap, device=DEVICE)
    kept = torch.sort(torch.where(live & (rank < B), slot, cap), -1)[0][..., :B]
    rows = kept[..., None].expand(L, S, H, B, D)
    return {"k": st["k"].gather(3, rows), "v": st["v"].gather(3, rows), "mass": st["mass"].gather(3, kept), "slot_pos": st["slot_pos"].gather(3, kept),
            "len": torch.clamp(st["len"], max=B), "next_pos": st["next_pos"].clone(), "kept": kept.int()}


def _plain_rules(st):
    c = st["case"]
    S, R, T, V = c["streams"], c["rows"], c["tokens"], c["vocab"]
    new = st["new"].long()
    st["counts"].scatter_add_(1, new.clamp(0, V - 1), ((new >= 0) & (new < V)).int())
    parent = st["parent"].long()
    up = torch.eye(R, device=DEVICE) + (parent[:, :, None] == torch.arange(R, device=DEVICE)).float()
    above = torch.linalg.matrix_power(up, 64) > 0                                        # row r continues row t, or is it
    on_path = above[:, :, :T] & (torch.arange(T, device=DEVICE) > 0)
    count = st["counts"].float()[:, None, :].repeat(1, R, 1)
    count.scatter_add_(2, st["tokens"].long()[:, None, :].expand(S, R, T), on_path.float())
    z = st["logits"].float().view(S, R, V)
    rep = st["repetition"][:, None, None]
    z = torch.where(count > 0, torch.where(z > 0, z / rep, z * rep), z)
    z = z - (st["frequency"][:, None, None] * count + st["presence"][:, None, None] * (count > 0))
    row = st["bias_row"].long()
    z = z + torch.where(row[:, None] >= 0, st["bias"][row.clamp(min=0)], 0.0)[:, None, :]
    bits = ((st["masks"][:, :, None] >> torch.arange(32, device=DEVICE)) & 1).reshape(st["masks"].shape[0], -1)[:, :V].bool()
    row = st["mask_row"].long().view(S, R)
    z = torch.where(bits[row.clamp(min=0)] | (row[..., None] < 0), z, -math.inf)
    return {"logits": z.view(S * R, V).to(st["logits"].dtype), "counts": st["counts"]}


def run(state):
    if own:
        return _own_run(state)
    kind = state["case"]["kind"]
    if kind in ("rope", "rope_tables"):
        return _plain_rope(state)
    return {"append": _plain_append, "weights": _plain_weights, "compress": _plain_compress, "rules": _plain_rules}[kind](state)


# ----------------------------------------------------------------------------------------------- floors

def work(case):
    c = case
    kind = c["kind"]
    if kind == "rope_tables":
        M = c["streams"] * c["rows"]
        return {"bytes": 4 * M * c["rot"] + 4 * (c["streams"] + c["rows"]), "flops": 4 * M * c["rot"]}
    if kind == "rope":
        M = c["streams"] * c["rows"]
        n = M * c["kv_heads"] * (c["group"] + (2 if c["into_cache"] else 1)) * c["dim"]
        return {"bytes": n * 2 * (2 if c["dtype"] == "bf16" else 4) + 4 * (c["streams"] + c["rows"]), "flops": 3 * n}
    if kind == "rules":
        S, R, V = c["streams"], c["rows"], c["vocab"]
        return {"bytes": S * R * V * 2 * (2 if c["dtype"] == "bf16" else 4) + S * V * 4 + 2 * V * 4 + 3 * V // 8, "flops": 4 * S * R * V}
    heads = c["layers"] * c["streams"] * c["kv_heads"]
    row = 2 * c["dim"]
    if kind == "append":
        n = (c["accepted"] + 1) / 2
        live = c["budget"] if c["full"] else 0.75 * c["budget"]
        return {"bytes": heads * (live * 8 + n * (4 * row + 8)), "flops": heads * live}
    if kind == "compress":
        return {"bytes": heads * (c["cap"] * 8 + c["budget"] * (4 * row + 12)), "flops": heads * c["cap"]}
    n = (c["accepted"] + 1) / 2 if c["accepted"] else c["rows"]
    live = 0.75 * c["cap"] if c["accepted"] else c["cap"]
    shared = c["layers"] * c["kv_heads"] * c["prefill"]
    seen = live - (n / 2 if not c["accepted"] else 0)
    return {"bytes": (heads * live + shared) * row + heads * live * 12 + shared * 8 + heads * n * c["group"] * row,
            "flops": 2 * n * c["group"] * c["dim"] * heads * (seen + c["prefill"])}


# ----------------------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rope", "rope_tables"):
        return _exact_rope(st)
    return {"append": _exact_append, "weights": _exact_weights, "compress": _exact_compress, "rules": _exact_rules}[kind](st)


def _exact_rope(st):
    """Complex numbers: a pair times e^(i angle)."""
    c = st["case"]
    pos = (st["base"].cpu().numpy().astype(np.float64)[:, None] + st["offset"].cpu().numpy()[None, :]).reshape(-1)
    angle = np.outer(pos, _frequencies(c["rot"], c["scaling"]))
    turn = torch.from_numpy(np.exp((-1j if c.get("inverse") else 1j) * angle)).to(DEVICE)
    if c["kind"] == "rope_tables":
        return [turn.real.contiguous(), turn.imag.contiguous()]
    half, out = c["rot"] // 2, []
    for name in ("q", "k"):
        x = st[name].double()
        pairs = x[..., :c["rot"]]
        z = torch.complex(pairs[..., ::2].contiguous(), pairs[..., 1::2].contiguous()) if c["layout"] == "interleaved" else torch.complex(
            pairs[..., :half].contiguous(), pairs[..., half:].contiguous())
        z = z * turn[:, None, :]
        y = torch.stack([z.real, z.imag], -1).flatten(-2) if c["layout"] == "interleaved" else torch.cat([z.real, z.imag], -1)
        out.append(torch.cat([y, x[..., c["rot"]:]], -1))
    if c["into_cache"]:
        out = [out[0], out[1].transpose(0, 1).contiguous(), st["v"].double().transpose(0, 1).contiguous()]
    return out


def _ranked(mass, pos, sink, newest):
    """Slots of one head in the order in which they are kept."""
    slots = range(len(mass))
    protected = (pos >= newest) | (pos < sink)
    return sorted(slots, key=lambda t: (not protected[t], 0.0 if protected[t] else -mass[t], t))


def _exact_append(st):
    c = st["case"]
    if st["mass"].numel() > 3_000_000:
        return None
    k, v, mass = (st[n].double() for n in ("k", "v", "mass"))
    where, weights = st["slot_pos"].cpu().numpy(), st["mass"].cpu().numpy()
    length, nxt, rows = (st[n].cpu().numpy() for n in ("len", "next_pos", "rows"))
    L, S, H = mass.shape[:3]
    index, source = [], []
    for s in range(S):
        mine = []
        for r in rows[s]:
            if not 0 <= r < c["rows"]:
                break
            mine.append(int(r))
        free = list(range(int(length[s]), max(c["budget"], int(length[s]))))[:len(mine)]
        out = len(mine) - len(free)
        for l in range(L):
            for h in range(H):
                w, p = weights[l, s, h, :length[s]], where[l, s, h, :length[s]]
                slots = free + (sorted(_ranked(w, p, c["sink"], nxt[s] - c["recent"])[int(length[s]) - out:]) if out else [])
                index += [(l, s, h, t) for t in slots]
                source += [(l, s * c["rows"] + r, h) for r in mine]
    to, of = (tuple(torch.tensor(x, device=DEVICE).t()) for x in (index, source))
    k[to], v[to], mass[to] = st["k_new"].double()[of], st["v_new"].double()[of], 0.0
    return {"k": k, "v": v, "mass": mass, "slot_pos": None, "len": None, "next_pos": None}


def _exact_compress(st):
    c = st["case"]
    if st["mass"].numel() > 3_000_000:
        return None
    where, weights = st["slot_pos"].cpu().numpy(), st["mass"].cpu().numpy()
    nxt = st["next_pos"].cpu().numpy()
    L, S, H = weights.shape[:3]
    kept = np.array([[[sorted(_ranked(weights[l, s, h], where[l, s, h], c["sink"], nxt[s] - c["recent"])[:c["budget"]]) for h in range(H)]
                      for s in range(S)] for l in range(L)])
    l, s, h = (torch.from_numpy(x).to(DEVICE) for x in np.ogrid[:L, :S, :H])
    kept = torch.from_numpy(kept).to(DEVICE)
    at = (l[..., None], s[..., None], h[..., None], kept)
    return {"k": st["k"][at].double(), "v": st["v"][at].double(), "mass": st["mass"][at].double(), "slot_pos": None, "len": None, "next_pos": None,
            "kept": None}


def _exact_weights(st):
    c = st["case"]
    L, S, H, cap, D = st["k"].shape
    P, G, R = c["prefill"], c["group"], c["rows"]
    mass = st["mass"].double()
    shared = st["mass_prefill"].double() * c["decay"] if P else None
    length, nxt = st["len"].tolist(), st["next_pos"].tolist()
    lists = [list(range(R))] * S if st["rows"] is None else [[r for r in x if r >= 0] for x in st["rows"].tolist()]
    for s in range(S):
        T, n = length[s], len(lists[s])
        at = torch.tensor(lists[s], device=DEVICE) + s * R
        pos = torch.arange(nxt[s] - n, nxt[s], device=DEVICE)
        for h in range(H):
            q = st["q"][:, at, h * G:(h + 1) * G].double()                                # [L][n][G][D]
            keys = st["k"][:, s, h, :T].double()
            if P:
                keys = torch.cat([st["k_prefill"][:, h].double(), keys], 1)
            x = torch.matmul(q.reshape(L, n * G, D), keys.transpose(1, 2)).view(L, n, G, P + T) / math.sqrt(D)
            hidden = torch.zeros((L, n, P + T), dtype=torch.bool, device=DEVICE)
            hidden[:, :, P:] = st["slot_pos"][:, s, h, None, :T] > pos[None, :, None]
            got = torch.softmax(x.masked_fill_(hidden[:, :, None], -math.inf), -1).nan_to_num_(0.0).sum((1, 2))
            mass[:, s, h, :T] = c["decay"] * mass[:, s, h, :T] + got[:, P:]
            if P:
                shared[:, h] += got[:, :P]
    return [mass] + ([shared] if P else [])


def _exact_rules(st):
    c = st["case"]
    S, R, T, V = c["streams"], c["rows"], c["tokens"], c["vocab"]
    parent, tokens, new = (st[n].tolist() for n in ("parent", "tokens", "new"))
    out = torch.empty((S * R, V), dtype=torch.float64, device=DEVICE)
    masks = np.unpackbits(st["masks"].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :V]
    allowed = torch.from_numpy(masks).to(DEVICE) > 0
    rows, tables = st["mask_row"].tolist(), st["bias_row"].tolist()
    for s in range(S):
        seen = st["counts"][s].double()
        for t in new[s]:
            if 0 <= t < V:
                seen[t] += 1
        rep, freq, pres = (float(st[n][s]) for n in ("repetition", "frequency", "presence"))
        for r in range(R):
            count, at = seen.clone(), r
            while at > 0:
                if at < T:
                    count[tokens[s][at]] += 1
                at = parent[s][at]
            z = st["logits"][s * R + r].double()
            hit = count > 0
            z = torch.where(hit & (z > 0), z / rep, torch.where(hit, z * rep, z)) - freq * count - pres * hit
            if tables[s] >= 0:
                z = z + st["bias"][tables[s]]
            if rows[s * R + r] >= 0:
                z[~allowed[rows[s * R + r]]] = -math.inf
            out[s * R + r] = z
    return {"logits": out, "counts": None}
