"""Plain float64 / plain Python definitions of beam search on a paged cache of 8 bits: rows entering the pages, streams that become
others, copies into another cache, attention over pages, tail and rows of the step, selection over beams and vocabulary.  Written from
the definitions in include/mlora_page_cache.h, mlora_page_attention.h and mlora_beam.h; used by the tests only.

A cache is a dict of numpy arrays with the header's names; bf16 numbers are int16 patterns."""
from __future__ import annotations

import math

import numpy as np

P = 64
FIELDS = ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "slot", "len", "table", "refs")


def bf16(patterns):
    """int16 / uint16 patterns -> float64."""
    return (np.ascontiguousarray(patterns).view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def empty_cache(L, S, H, D, pages, columns):
    return {"k": np.zeros((L, pages, H, P, D), np.int8), "v": np.zeros((L, pages, H, D, P), np.int8),
            "k_scale": np.zeros((L, pages, H), np.float32), "v_scale": np.zeros((L, pages, H), np.float32),
            "k_tail": np.zeros((L, S, H, P, D), np.int16), "v_tail": np.zeros((L, S, H, P, D), np.int16),
            "slot": np.arange(S, dtype=np.int32), "len": np.zeros(S, np.int32), "table": np.full((S, columns), -1, np.int32),
            "refs": np.zeros(pages, np.int32)}


def copy_of(c):
    return {n: a.copy() for n, a in c.items()}


def quantise(x):
    """float64 numbers -> (codes, scale)."""
    if not np.all(np.isfinite(x)):
        return np.zeros(x.shape, np.int8), np.float32(math.nan)
    m = np.max(np.abs(x))
    if m == 0:
        return np.zeros(x.shape, np.int8), np.float32(0)
    return np.rint(127.0 * x / m).astype(np.int8), np.float32(np.float32(m) / np.float32(127))


def count_of(row, R):
    """Rows of a list before the first entry that names none."""
    n = 0
    while n < len(row) and 0 <= row[n] < R:
        n += 1
    return n


def append(c, k_new, v_new, R, rows=None):
    """k_new, v_new int16 [L][S * R][H][D]; rows: lists per stream.  Returns (cache, rows that entered per stream)."""
    c = copy_of(c)
    L, pages, H, _, D = c["k"].shape
    S, columns = c["table"].shape
    rows = [list(range(R))] * S if rows is None else rows
    entered, out_of_pages = [], False
    for s in range(S):
        n, slot, length = count_of(rows[s], R), int(c["slot"][s]), int(c["len"][s])
        t, full = length % P, length // P
        want = (t + n) // P
        if full + want > columns:
            n = want = 0
        if want:
            free = [p for p in range(pages) if c["refs"][p] <= 0][:want]
            out_of_pages = out_of_pages or len(free) < want
            if out_of_pages:
                n = want = 0
        entered.append(n)
        if n == 0:
            continue
        mine = [s * R + r for r in rows[s][:n]]
        for name in ("k", "v"):
            new = {"k": k_new, "v": v_new}[name][:, mine].transpose(0, 2, 1, 3)                 # [L][H][n][D]
            both = np.concatenate([c[name + "_tail"][:, slot, :, :t], new], 2)
            for j in range(want):
                for l in range(L):
                    for h in range(H):
                        code, scale = quantise(bf16(both[l, h, j * P:(j + 1) * P]))
                        c[name][l, free[j], h] = code if name == "k" else code.T
                        c[name + "_scale"][l, free[j], h] = scale
            left = t + n - want * P
            at = 0 if want else t
            c[name + "_tail"][:, slot, :, at:left] = both[:, :, want * P + at:]
        for j in range(want):
            c["table"][slot, full + j] = free[j]
            c["refs"][free[j]] = 1
        c["len"][s] = length + n
    return c, entered


def reorder(c, source=None, window=0, sink=0):
    old, c = c, copy_of(c)
    S, columns = c["table"].shape
    source = list(range(S)) if source is None else [int(x) for x in source]
    valid = [0 <= x < S for x in source]
    keeps = [valid[s] and source[s] not in source[:s] for s in range(S)]
    taken = {int(old["slot"][source[s]]) for s in range(S) if keeps[s]}
    left = [x for x in range(S) if x not in taken]
    owner = {int(old["slot"][s]): s for s in range(S)}
    for s in range(S):
        src = int(old["slot"][source[s]]) if valid[s] else None
        to = src if keeps[s] else left.pop(0)
        length = int(old["len"][source[s]]) if valid[s] else 0
        had = int(old["len"][owner[to]]) // P
        row = [int(old["table"][src][i]) if valid[s] and i < length // P else -1 for i in range(columns)]
        for i in range(columns):
            if i < length // P and window > 0 and (i + 1) * P <= length - window + 1 and i * P >= sink:
                row[i] = -1
            if i < max(had, length // P):
                c["table"][to][i] = row[i]
        if valid[s] and not keeps[s]:
            for name in ("k_tail", "v_tail"):
                c[name][:, to, :, :length % P] = old[name][:, src, :, :length % P]
        c["slot"][s], c["len"][s] = to, length
    held = c["table"][(c["table"] >= 0) & (c["table"] < len(c["refs"]))]
    c["refs"][:] = np.bincount(held, minlength=len(c["refs"]))
    return c


def copy(c, to, source):
    """Returns (what `to` becomes, pages that the streams hold)."""
    to = copy_of(to)
    S, T = len(c["len"]), len(to["len"])
    valid = [0 <= int(x) < S for x in source]
    rows = [[int(p) for p in c["table"][c["slot"][x]][:int(c["len"][x]) // P]] if ok else [] for x, ok in zip(source, valid)]
    used = sorted({p for row in rows for p in row if 0 <= p < len(c["refs"])})
    place = {p: i for i, p in enumerate(used)}
    to["slot"][:], to["len"][:], to["table"][:], to["refs"][:] = np.arange(T), 0, -1, 0
    if len(used) > len(to["refs"]) or any(len(r) > to["table"].shape[1] for r in rows):
        return to, len(used)
    for name in ("k", "v", "k_scale", "v_scale"):
        to[name][:, :len(used)] = c[name][:, used]
    for i in range(T):
        if not valid[i]:
            continue
        n = int(c["len"][source[i]])
        to["len"][i] = n
        for j, p in enumerate(rows[i]):
            to["table"][i, j] = place.get(p, -1)
            if p in place:
                to["refs"][place[p]] += 1
        for name in ("k_tail", "v_tail"):
            to[name][:, i, :, :n % P] = c[name][:, c["slot"][source[i]], :, :n % P]
    return to, len(used)


def paths_of(parent):
    """Rows of every row's path, itself first."""
    paths = []
    for r, up in enumerate(parent):
        paths.append([r] + (paths[up] if 0 <= up < r else []))
    return paths


def tokens_of(c, layer, s, h):
    """Positions, keys and values (float64) of the tokens that stream s has in a head."""
    slot, length = int(c["slot"][s]), int(c["len"][s])
    D = c["k"].shape[-1]
    where, keys, values = [], [], []
    for i in range(length // P):
        p = int(c["table"][slot, i])
        if not 0 <= p < len(c["refs"]):
            continue
        where += range(i * P, (i + 1) * P)
        keys.append(c["k"][layer, p, h].astype(np.float64) * np.float64(c["k_scale"][layer, p, h]))
        values.append(c["v"][layer, p, h].T.astype(np.float64) * np.float64(c["v_scale"][layer, p, h]))
    n = length % P
    where += range(length - n, length)
    keys.append(bf16(c["k_tail"][layer, slot, h, :n]).reshape(n, D))
    values.append(bf16(c["v_tail"][layer, slot, h, :n]).reshape(n, D))
    return np.array(where, np.int64), np.concatenate(keys), np.concatenate(values)


def softmax_sum(x, v):
    """Weights of the scores x [n] (all of them count) applied to v [n][D]; NaN as IEEE arithmetic has it."""
    with np.errstate(all="ignore"):
        w = np.exp(x - np.max(x))
        return (w[:, None] * v).sum(0) / w.sum()


def attention(c, layer, q, k_new, v_new, parent, R, scale, window=0, sink=0):
    """q int16 [S * R][Hq][D], k_new and v_new int16 [S * R][H][D] -> float64 [S * R][Hq][D], and a bound of every output's size of
    error (see the caller): the largest |value|, sum |q k| scale and |key| of what each row sees."""
    S, H = len(c["len"]), c["k"].shape[2]
    Hq, D = q.shape[1:]
    G = Hq // H
    out = np.empty(q.shape)
    size = np.zeros((q.shape[0], Hq, 3))
    for s in range(S):
        paths = paths_of([int(x) for x in parent[s * R:(s + 1) * R]])
        length = int(c["len"][s])
        for h in range(H):
            where, keys, values = tokens_of(c, layer, s, h)
            kn, vn = bf16(k_new[s * R:(s + 1) * R, h]), bf16(v_new[s * R:(s + 1) * R, h])
            for r in range(R):
                at = length + len(paths[r]) - 1
                pos = np.array([length + len(paths[x]) - 1 for x in paths[r]])
                see = lambda t: (t > at - window) | (t < sink) if window else np.ones(len(t), bool)   # noqa: E731
                k = np.concatenate([keys[see(where)], kn[paths[r]][see(pos)]])
                v = np.concatenate([values[see(where)], vn[paths[r]][see(pos)]])
                for g in range(G):
                    x = bf16(q[s * R + r, h * G + g])
                    with np.errstate(all="ignore"):
                        out[s * R + r, h * G + g] = softmax_sum(scale * (k @ x), v) if np.all(np.isfinite(x)) else math.nan
                        size[s * R + r, h * G + g] = np.max(np.abs(v)), abs(scale) * np.max(np.abs(k) @ np.abs(x)), np.max(np.abs(k).sum(1))
    return out, size


def beam_select(logits, score, length, finished, W, eos=-1, pad=0, power=0.0):
    """logits float64 [rows][V].  Returns dict(source, token, score, length, finished) and the ranked scores of all candidates of
    each group, best first (what the choice turned on)."""
    rows, V = logits.shape
    out = {"source": np.arange(rows, dtype=np.int32), "token": np.full(rows, pad, np.int32), "score": np.full(rows, -math.inf),
           "length": np.zeros(rows, np.int32), "finished": np.zeros(rows, np.int32)}
    ranks = []
    for g in range(rows // W):
        found = []
        for b in range(g * W, (g + 1) * W):
            base = float(score[b])
            if not math.isfinite(base):
                continue
            if finished[b]:
                found.append((base / max(1, int(length[b])) ** power, b, 0.0, pad, base, int(length[b]), 1))
                continue
            z = logits[b]
            if np.any(np.isnan(z)) or np.max(z) == math.inf or np.max(z) == -math.inf:
                continue
            top = np.max(z)
            lse = top + math.log(math.fsum(np.exp(z - top)))
            n = int(length[b]) + 1
            order = np.lexsort((np.arange(V), -z))[:W]
            for v in order:
                if z[v] > -math.inf:
                    total = base + (z[v] - lse)
                    found.append((total / max(1, n) ** power, b, z[v], int(v), total, n, int(v == eos)))
        found.sort(key=lambda x: (-x[0], x[1], -x[2], x[3]))
        ranks.append([(x[0], x[1]) for x in found])
        for i, x in enumerate(found[:W]):
            at = g * W + i
            out["source"][at], out["token"][at], out["score"][at], out["length"][at], out["finished"][at] = x[1], x[3], x[4], x[5], x[6]
    return out, ranks
