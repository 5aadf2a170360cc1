"""Plain float64 / plain Python definitions of what a decoding loop does around the projections and the attention: rotary
positions, rows entering a bounded cache, accumulated attention weights, the heaviest slots of a segment, rules on logits.
Written from the definitions in include/mlora_rope.h, mlora_stream_cache.h and mlora_logit_rules.h, one element after the
other; used by the tests only."""
from __future__ import annotations

import math

import numpy as np


# ------------------------------------------------------------------------------------------ rotary positions

def rope_frequency(i, rot, scaling, theta, factor=1.0, low=1.0, high=4.0, context=8192.0):
    """Radians per position of pair i."""
    t = theta ** (-2.0 * i / rot)
    if scaling == "plain":
        return t
    if scaling == "linear":
        return t / factor
    if scaling == "base":
        return (theta * factor ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
    turns = context * t / (2 * math.pi)                   # full turns within the context
    if turns <= low:
        return t / factor
    if turns >= high:
        return t
    u = (turns - low) / (high - low)
    return (1 - u) * t / factor + u * t


def rope_angles(positions, rot, scaling, theta, **kw):
    """float64 [rows][rot / 2], the product in extended precision, reduced to one turn."""
    f = np.array([rope_frequency(i, rot, scaling, theta, **kw) for i in range(rot // 2)], np.longdouble)
    turn = 2 * np.longdouble("3.14159265358979323846264338327950288")
    return np.asarray(np.remainder(np.asarray(positions, np.longdouble)[:, None] * f[None, :], turn), np.float64)


def rope(x, angles, rot, interleaved, inverse=False):
    """x float64 [rows][heads][dim]."""
    y = np.array(x, np.float64)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = np.cos(angles[:, i])[:, None], np.sin(angles[:, i])[:, None] * (-1 if inverse else 1)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


# ------------------------------------------------------------------------------------------ the bounded cache

def listed(row, R):
    out = []
    for r in row:
        if not 0 <= int(r) < R:
            break
        out.append(int(r))
    return out


def ranked(mass, pos, live, next_pos, sink, recent):
    """The live slots, the one to keep first in front."""
    def key(t):
        if pos[t] >= next_pos - recent or pos[t] < sink:
            return (0, 0.0, t)
        return (2, 0.0, t) if math.isnan(mass[t]) else (1, -float(mass[t]), t)
    return sorted(range(live), key=key)


def append(cache, k_new, v_new, R, rows, budget, sink, recent):
    """cache: dict of arrays k, v [L][S][H][cap][D], mass, slot_pos [L][S][H][cap], len, next_pos [S]; returns a new one.
    rows: a list per stream."""
    c = {n: np.array(a) for n, a in cache.items()}
    L, S, H, cap, _ = c["k"].shape
    for s in range(S):
        mine, live, nxt = listed(rows[s], R), min(max(int(c["len"][s]), 0), cap), int(c["next_pos"][s])
        free = list(range(live, max(live, budget)))[:len(mine)]
        out = len(mine) - len(free)
        for l in range(L):
            for h in range(H):
                order = ranked(c["mass"][l, s, h], c["slot_pos"][l, s, h], live, nxt, sink, recent)
                for j, (slot, r) in enumerate(zip(free + sorted(order[live - out:]), mine)):
                    c["k"][l, s, h, slot], c["v"][l, s, h, slot] = k_new[l, s * R + r, h], v_new[l, s * R + r, h]
                    c["mass"][l, s, h, slot], c["slot_pos"][l, s, h, slot] = 0.0, nxt + j
        c["len"][s], c["next_pos"][s] = live + len(free), nxt + len(mine)
    return c


def compress(cache, to, budget, sink, recent):
    """(a new version of `to`, kept [L][S][H][budget])."""
    t = {n: np.array(a) for n, a in to.items()}
    L, S, H, cap, _ = cache["k"].shape
    kept = np.full((L, S, H, budget), -1, np.int32)
    for s in range(S):
        live, nxt = min(max(int(cache["len"][s]), 0), cap), int(cache["next_pos"][s])
        for l in range(L):
            for h in range(H):
                slots = sorted(ranked(cache["mass"][l, s, h], cache["slot_pos"][l, s, h], live, nxt, sink, recent)[:budget])
                kept[l, s, h, :len(slots)] = slots
                for n in ("k", "v", "mass", "slot_pos"):
                    t[n][l, s, h, :len(slots)] = cache[n][l, s, h][slots]
        t["len"][s], t["next_pos"][s] = min(live, budget), nxt
    return t, kept


def attention_mass(k, mass, slot_pos, length, next_pos, q, R, rows, scale, decay, k_prefill=None, mass_prefill=None):
    """(mass, mass_prefill) in float64.  k [L][S][H][cap][D], q [L][S * R][Hq][D] float64; rows: a list per stream."""
    L, S, H, cap, D = k.shape
    G = q.shape[2] // H
    P = 0 if k_prefill is None else k_prefill.shape[2]
    out = np.array(mass, np.float64)
    shared = None if P == 0 else decay * np.array(mass_prefill, np.float64)
    for l in range(L):
        for s in range(S):
            live = min(max(int(length[s]), 0), cap)
            mine = listed(rows[s], R)
            for h in range(H):
                got = np.zeros(P + live)
                for j, r in enumerate(mine):
                    at = int(next_pos[s]) - len(mine) + j
                    see = [("p", t) for t in range(P)] + [("s", t) for t in range(live) if slot_pos[l, s, h, t] <= at]
                    if not see:
                        continue
                    keys = np.array([k_prefill[l, h, t] if kind == "p" else k[l, s, h, t] for kind, t in see])
                    where = [t if kind == "p" else P + t for kind, t in see]
                    for g in range(G):
                        x = scale * (keys @ q[l, s * R + r, h * G + g])
                        if x.max() == -np.inf:                   # (NaN is not)
                            continue
                        e = np.exp(x - x.max())
                        got[where] += e / e.sum()
                out[l, s, h, :live] = decay * out[l, s, h, :live] + got[P:]
                if P:
                    shared[l, h] += got[:P]
    return out, shared


# ------------------------------------------------------------------------------------------ rules on logits

def logit_rules(z, S, R, T, parent, tokens, new=None, counts=None, repetition=None, frequency=None, presence=None, bias=None,
                bias_row=None, masks=None, mask_row=None):
    """(out float64 [S * R][V], counts).  z float64; masks uint32 [n][(V + 31) / 32]."""
    V = z.shape[1]
    counts = None if counts is None else np.array(counts)
    out = np.empty((S * R, V))
    for s in range(S):
        for t in ([] if new is None else new[s]):
            if 0 <= t < V:
                counts[s, t] += 1
        for r in range(R):
            c, at = np.zeros(V) if counts is None else counts[s].astype(np.float64), r
            while at > 0:
                if at < T and 0 <= tokens[s][at] < V:
                    c[tokens[s][at]] += 1
                up = int(parent[s * R + at])
                at = up if up < at else 0
            y = np.array(z[s * R + r], np.float64)
            for v in np.nonzero(c)[0]:
                if c[v] > 0 and repetition is not None:
                    y[v] = y[v] / repetition[s] if y[v] > 0 else y[v] * repetition[s]
                if frequency is not None:
                    y[v] -= frequency[s] * c[v]
                if presence is not None and c[v] > 0:
                    y[v] -= presence[s]
            if bias is not None and 0 <= bias_row[s] < len(bias):
                y += bias[bias_row[s]]
            if masks is not None and 0 <= mask_row[s * R + r] < len(masks):
                words = masks[mask_row[s * R + r]]
                for v in range(V):
                    if not int(words[v // 32]) >> (v % 32) & 1:
                        y[v] = -math.inf
            out[s * R + r] = y
    return out, counts
