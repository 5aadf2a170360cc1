"""A decoding loop on a bounded cache as a sequence of library calls: several output streams, a draft tree with forecast
embeddings per stream (Sections 3.4 and 3.5 of the paper), and stream caches that keep to a budget.

    prompt   rope (queries and keys turned, keys and values into a long segment), attention weights of its last rows on the
             shared prefix and on the segment, compression of the segment to its heaviest slots
    step     rope tables for the rows' positions behind the prefix, the decoder layers (decoder.py), the head's logits from
             rows normalised by the sums of squares that the last layer leaves, rules on them
             (penalties, biases, grammar masks), verification and next drafts (DS2D), the accepted rows into the caches of all
             layers, their attention weights added to the slots they saw

Argument marshalling only, apart from torch's look-up of embeddings.  A step reads nothing back: positions, lengths, accepted
rows and tokens stay on the device, so steps can follow each other without a synchronisation, or be captured into a graph.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as B
from .decoder import DecoderLayerStep

HEAD_DIM = 64                                            # the fused projections turn heads of 64 features


def _fitting(layers, head, embedding, forecast, k_prefill, v_prefill) -> None:
    """Refuses parts of a loop that do not fit each other: what a call writes or reads has the size of another part's."""
    hidden, wide, narrow = head.K, 0, 0
    ok = len(layers) > 0 and embedding.dim() == 2 and forecast.dim() == 2
    ok = ok and embedding.shape[0] >= head.N and embedding.shape[1] == forecast.shape[1] == hidden
    for q, k, v, o, gate_up, down in layers:
        wide, narrow = wide or q.N, narrow or k.N
        ok = ok and q.K == k.K == v.K == gate_up.K == o.N == down.N == hidden and q.N == o.K == wide and k.N == v.N == narrow
        ok = ok and wide % HEAD_DIM == narrow % HEAD_DIM == 0 and gate_up.N == 2 * down.K
    ok = ok and (k_prefill is None) == (v_prefill is None)
    if not ok:
        raise B.MloraError(B._ESHAPE, "decoding loop")
    for t in () if k_prefill is None else (k_prefill, v_prefill):
        B._buffer(t, "decoding loop", B._AS_BF16, (len(layers), narrow // HEAD_DIM, k_prefill.shape[2] if k_prefill.dim() == 4 else -1, HEAD_DIM))


def _patterns(t):
    """A bf16 tensor as the int16 patterns of its numbers (which it may be already)."""
    if not B._AS_BF16.takes(t.dtype):
        raise B.MloraError(B._EINVAL, "decoding loop")
    return t.view(torch.int16)


class DecodingLoop:
    def __init__(self, layers: Sequence[Sequence[B.Proj]], head: B.Proj, embedding, forecast, n_streams: int, branch: Sequence[int],
                 budget: int, sink: int = 4, recent: int = 32, decay: float = 1.0, rope: Optional[B.Rope] = None, k_prefill=None,
                 v_prefill=None, row_adapter=None, rules: Optional[dict] = None, device="cuda:0"):
        """layers: (q, k, v, o, gate_up, down) of each layer; head: hidden -> vocabulary, the last normalisation's weight folded in;
        embedding bf16 [V][hidden] and forecast bf16 [m][hidden] (or their int16 patterns, like all bf16 here); k_prefill, v_prefill
        bf16 [L][H][P][64], shared by the streams, keys turned by their positions 0 .. P - 1.  A stream's own positions (next_pos
        and slot_pos of its cache, sink) count from its first token, which is turned as the one at position P.  rules: keyword
        arguments of binding.LogitRules (counts and parent are made here).  Stream caches have room for `budget` slots."""
        L, S, m = len(layers), int(n_streams), int(forecast.shape[0])
        self.T, self.R = B.ds2d_rows(branch, m)
        embedding, forecast = _patterns(embedding), _patterns(forecast)
        _fitting(layers, head, embedding, forecast, k_prefill, v_prefill)
        if rope is not None and (rope.struct.head_dim, rope.struct.rot, rope.struct.layout) != (HEAD_DIM, HEAD_DIM, B.ROPE_HALF):
            raise B.MloraError(B._ESHAPE, "decoding loop")          # (what the fused projections turn)
        if row_adapter is not None:
            B._buffer(row_adapter, "decoding loop", B._AS_INT32)
        short = row_adapter is not None and row_adapter.numel() < S * self.R
        if short or budget < m + 1 or sink < 0 or recent < 0:        # (a step appends up to m + 1 rows)
            raise B.MloraError(B._ESHAPE, "decoding loop")
        parent, is_forecast, _ = B.ds2d_layout(branch, m)
        M, V, hidden = S * self.R, head.N, head.K
        kv, heads = layers[0][1].N // HEAD_DIM, layers[0][0].N // HEAD_DIM
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)   # noqa: E731
        i16 = lambda *shape: torch.zeros(shape, dtype=torch.int16, device=device)   # noqa: E731
        self.S, self.L, self.M, self.heads, self.kv = S, L, M, heads, kv
        self.budget, self.sink, self.recent, self.decay = int(budget), int(sink), int(recent), float(decay)
        self.scale = HEAD_DIM ** -0.5
        self.rope = rope or B.Rope(HEAD_DIM, HEAD_DIM, device=device)
        self.cache = self._cache(self.budget, device)
        P = 0 if k_prefill is None else int(k_prefill.shape[2])
        self.mass_prefill = torch.zeros((L, kv, P), device=device) if P else None

        # rows: the tree's tokens, then their forecast embeddings; a row stands one position behind the one it continues, and a
        # stream's first token behind the P of the prefix
        depth = []
        for up in parent:
            depth.append(0 if up < 0 else depth[up] + 1)
        self.prefix = P
        self.offset = torch.tensor([P + d for d in depth], dtype=torch.int32).to(device)
        self.parent = torch.tensor(parent * S, dtype=torch.int32).to(device)
        self.is_forecast = torch.tensor(is_forecast * S, dtype=torch.uint8).to(device)
        self.cos, self.sin = (torch.empty((M, HEAD_DIM // 2), device=device) for _ in range(2))
        self.tables = B.RopeTables(self.rope, self.cos, self.sin, M, rows_per_stream=self.R, base=self.cache.next_pos, offset=self.offset)
        self.embedding = embedding
        self.h = i16(M, hidden)
        self.h.view(S, self.R, hidden)[:, self.T:] = forecast.repeat(self.T, 1)     # (the same in every step)

        self.q, self.k_new, self.v_new = i16(L, M, heads * HEAD_DIM), i16(L, M, kv * HEAD_DIM), i16(L, M, kv * HEAD_DIM)
        self.layers, h, sq = [], self.h, None
        for l, proj in enumerate(layers):
            attention = B.TreeAttention(heads, kv, HEAD_DIM, S, self.R, self.scale, None if P == 0 else k_prefill[l],
                                        None if P == 0 else v_prefill[l], None, None, self.cache.k[l], self.cache.v[l], self.cache.len,
                                        self.k_new[l], self.v_new[l], self.parent, self.is_forecast, P, 0, self.budget)
            step = DecoderLayerStep(*proj, attention, h, self.cos, self.sin, row_adapter, M, h_sq=sq, q=self.q[l])
            self.layers.append(step)
            h, sq = step.out, step.out_sq
        self.head, self.final, self.row_adapter = head, h, row_adapter
        self.head_ws = torch.zeros(max(256, B.workspace_bytes([head], M)), dtype=torch.uint8, device=device)
        self.logits = i16(M, V)
        # (the last normalisation: 1 / rms from the sums of squares that the last layer leaves, as between the layers)
        self.to_logits = B.LayerPlanFused([head], [B.Epilogue(sq_in=sq, sq_parts=(hidden + 63) // 64, sq_eps=self.layers[-1].eps)], [h], [self.logits],
                                          row_adapter, M, B.Y_BF16, self.head_ws)

        self.counts = i32(S, V)
        self.rules = B.LogitRules(S, self.R, self.T, V, B.Y_BF16, self.parent, counts=self.counts, **(rules or {}))
        self.ds2d = B.Ds2dStep(S, m, branch, branch, V, B.Y_BF16)
        self.ds2d_ws = torch.empty(max(16, self.ds2d.workspace_bytes()), dtype=torch.uint8, device=device)
        self.tokens, self.next_tokens = i32(S, self.T), i32(S, self.T)
        self.n_accepted, self.accepted_rows, self.emitted = i32(S), i32(S, m + 1), i32(S, m + 1)
        self.mass = B.AttentionMass(self.cache, heads, self.R, self.scale, k_prefill=k_prefill, mass_prefill=self.mass_prefill, decay=decay)
        self.mass_ws = torch.empty(max(256, self.mass.workspace_bytes(m + 1)), dtype=torch.uint8, device=device)
        self.keep = (k_prefill, v_prefill)
        self.prompted = False                            # the caches hold a prompt that no generation has started on

    def _cache(self, cap: int, device) -> B.StreamCache:
        shape = (self.L, self.S, self.kv, cap)
        i32 = lambda s: torch.zeros(s, dtype=torch.int32, device=device)   # noqa: E731
        return B.StreamCache(*(torch.zeros(shape + (HEAD_DIM,), dtype=torch.int16, device=device) for _ in range(2)),
                             torch.zeros(shape, device=device), i32(shape), i32((self.S,)), i32((self.S,)))

    def reset(self) -> None:
        """Empties the caches and forgets the prefix's masses: the next token is a stream's first."""
        self.cache.len.zero_()
        self.cache.next_pos.zero_()
        if self.mass_prefill is not None:
            self.mass_prefill.zero_()
        self.prompted = False

    def start(self, tokens, counts=None) -> None:
        """A new generation, behind the prompt if there has been one since the last start and otherwise on empty caches.
        tokens int32 [S]: every stream's newest token, the root of its first tree (which has no drafts yet); one outside the
        vocabulary is embedded as the nearest."""
        if not self.prompted:
            self.reset()
        self.prompted = False
        self.tokens.fill_(-1)
        self.tokens[:, 0] = tokens
        self.emitted.fill_(-1)
        self.emitted[:, 0] = tokens
        if counts is None:
            self.counts.zero_()
        else:
            self.counts.copy_(counts)

    def prompt(self, q, k, v, window: int) -> torch.Tensor:
        """Every stream's own prompt of N tokens, not yet turned: q bf16 [L][S][N][heads][64], k and v [L][S][N][kv][64].  Its last
        `window` rows weigh what they see, the prefix and the slots, the heaviest of which stay.  Returns the slots that were
        kept, [L][S][kv][budget]."""
        q, k, v = _patterns(q), _patterns(k), _patterns(v)
        N, device = int(k.shape[2]) if k.dim() == 5 else 0, k.device
        for t, heads in ((q, self.heads), (k, self.kv), (v, self.kv)):
            if tuple(t.shape) != (self.L, self.S, N, heads, HEAD_DIM) or not 1 <= window <= N:
                raise B.MloraError(B._ESHAPE, "decoding loop's prompt")
        long = self._cache(N, device)
        weigh = B.AttentionMass(long, self.heads, window, self.scale, k_prefill=self.keep[0], mass_prefill=self.mass_prefill, decay=self.decay)
        ws = torch.empty(weigh.workspace_bytes(), dtype=torch.uint8, device=device)
        if ws.numel() == 0:                              # (more rows than a call takes)
            raise B.MloraError(B._ESHAPE, "decoding loop's prompt")
        self.reset()
        turned = torch.empty((self.L, self.S, window) + tuple(q.shape[3:]), dtype=q.dtype, device=device)
        first, at = (torch.tensor([self.prefix + n], dtype=torch.int32).to(device) for n in (0, N - window))
        for l in range(self.L):
            for s in range(self.S):
                B.RopePlan(self.rope, [B.RopeTensor(k[l, s], long.k[l, s].transpose(0, 1)),
                                       B.RopeTensor(v[l, s], long.v[l, s].transpose(0, 1), rotate=False)], N, B.Y_BF16, base=first).run()
                B.RopePlan(self.rope, [B.RopeTensor(q[l, s, N - window:], turned[l, s])], window, B.Y_BF16, base=at).run()
        long.slot_pos.copy_(torch.arange(N, dtype=torch.int32, device=device).expand(long.slot_pos.shape))
        long.len.fill_(N)
        long.next_pos.fill_(N)
        weigh.run(turned.view(self.L, self.S * window, self.heads, HEAD_DIM), None, ws)
        kept = torch.empty((self.L, self.S, self.kv, self.budget), dtype=torch.int32, device=device)
        long.compress(self.cache, kept, self.budget, self.sink, self.recent)
        self.prompted = True
        return kept

    def step(self) -> None:
        """One step of all streams: emitted (int32 [S][m + 1], -1 beyond) holds the tokens given out, tokens the next tree."""
        S, T, hidden = self.S, self.T, self.h.shape[1]
        rows = torch.index_select(self.embedding, 0, self.tokens.view(-1).clamp(0, self.embedding.shape[0] - 1))
        self.h.view(S, self.R, hidden)[:, :T].copy_(rows.view(S, T, hidden))
        self.tables.run()
        for layer in self.layers:
            layer.run()
        self.to_logits.run()
        self.rules.run(self.logits, self.tokens, self.logits, new_tokens=self.emitted)
        self.ds2d.run(self.logits, self.tokens, self.n_accepted, self.accepted_rows, self.emitted, self.next_tokens, self.ds2d_ws)
        self.cache.append(self.k_new, self.v_new, self.R, self.accepted_rows, self.budget, self.sink, self.recent)
        self.mass.run(self.q, self.accepted_rows, self.mass_ws)
        self.tokens.copy_(self.next_tokens)
