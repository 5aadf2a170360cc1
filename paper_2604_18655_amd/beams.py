"""Beam search as a sequence of library calls: groups (requests) of beams, each a stream of a paged cache of 8 bits that shares the pages
of what it has in common with others.

    prompt   keys turned and, with the values, into the pages of a group's first beam; the others of the group continue it
    step     rope tables, the decoder layers (decoder.py) with attention over the pages, the head's logits, selection over beams
             and vocabulary, the rows into the caches, and every beam becomes the continuation of the one it was chosen from

Finished beams, and places without a candidate, take no further rows: a finished beam's cache holds its tokens but the last, and neither takes
a page that another beam needs.

Argument marshalling only, apart from torch's look-up of embeddings and small copies.  A step reads nothing back, so steps can follow each other
without a synchronisation, or be captured into a graph.  What each step chose is kept on the device (trace); sequences() reads it back.
"""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import torch

from . import binding as B
from .decoder import DecoderLayerStep
from .decoding import HEAD_DIM, _fitting, _patterns


class BeamLoop:
    def __init__(self, layers: Sequence[Sequence[B.Proj]], head: B.Proj, embedding, n_groups: int, n_beams: int, n_pages: int, max_pages: int,
                 max_steps: int, eos: int = -1, length_power: float = 0.0, window: int = 0, sink: int = 0, rope: Optional[B.Rope] = None,
                 row_adapter=None, device="cuda:0"):
        """layers, head and embedding as of decoding.DecodingLoop; n_pages of the pool, max_pages of a beam; window and sink as of
        PageAttention (pages that the window leaves behind go back to the pool); row_adapter int32 [n_groups * n_beams]: the adapter of each
        place, which a beam changes when it is chosen into another place.  A request that is to be answered by one adapter has it in all places
        of its group; with several, a beam goes on with its new place's on the keys and values that the old one's made."""
        L, G, W = len(layers), int(n_groups), int(n_beams)
        S = G * W
        embedding = _patterns(embedding)
        _fitting(layers, head, embedding, embedding, None, None)
        if rope is not None and (rope.struct.head_dim, rope.struct.rot, rope.struct.layout) != (HEAD_DIM, HEAD_DIM, B.ROPE_HALF):
            raise B.MloraError(B._ESHAPE, "beam loop")              # (what the fused projections turn)
        if row_adapter is not None:
            B._buffer(row_adapter, "beam loop", B._AS_INT32)
        if max_steps < 1 or window < 0 or sink < 0 or (row_adapter is not None and row_adapter.numel() < S):
            raise B.MloraError(B._ESHAPE, "beam loop")
        V, hidden = head.N, head.K
        kv, heads = layers[0][1].N // HEAD_DIM, layers[0][0].N // HEAD_DIM
        self.select = B.BeamSelect(G, W, V, B.Y_BF16, eos=eos, pad=max(0, eos) if eos < V else 0, length_power=length_power)
        select_bytes = self.select.workspace_bytes()
        if select_bytes == 0:
            raise B.MloraError(B._ESHAPE, "beam loop")
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)   # noqa: E731
        i16 = lambda *shape: torch.zeros(shape, dtype=torch.int16, device=device)   # noqa: E731
        self.G, self.W, self.S, self.L, self.kv, self.window, self.sink = G, W, S, L, kv, int(window), int(sink)
        self.rope = rope or B.Rope(HEAD_DIM, HEAD_DIM, device=device)
        self.cache = B.PageCache.empty(L, S, kv, HEAD_DIM, n_pages, max_pages, device)
        self.embedding, self.row_adapter = embedding, row_adapter
        self.h, self.logits = i16(S, hidden), i16(S, V)
        self.cos, self.sin = (torch.empty((S, HEAD_DIM // 2), device=device) for _ in range(2))
        self.tables = B.RopeTables(self.rope, self.cos, self.sin, S, rows_per_stream=1, base=self.cache.len)
        self.k_new, self.v_new, self.alone = i16(L, S, kv * HEAD_DIM), i16(L, S, kv * HEAD_DIM), i32(S) - 1
        self.layers, h, sq = [], self.h, None
        for l, proj in enumerate(layers):
            attention = B.PageAttention(self.cache, l, heads, 1, HEAD_DIM ** -0.5, self.k_new[l], self.v_new[l], self.alone, self.window, self.sink)
            step = DecoderLayerStep(*proj, attention, h, self.cos, self.sin, row_adapter, S, h_sq=sq)
            self.layers.append(step)
            h, sq = step.out, step.out_sq
        self.head_ws = torch.zeros(max(256, B.workspace_bytes([head], S)), dtype=torch.uint8, device=device)
        # (the last normalisation: 1 / rms from the sums of squares that the last layer leaves, as between the layers)
        self.to_logits = B.LayerPlanFused([head], [B.Epilogue(sq_in=sq, sq_parts=(hidden + 63) // 64, sq_eps=self.layers[-1].eps)], [h], [self.logits],
                                          row_adapter, S, B.Y_BF16, self.head_ws)
        self.select_ws = torch.empty(select_bytes, dtype=torch.uint8, device=device)
        self.tokens, self.source, self.length, self.finished = i32(S), i32(S), i32(S), i32(S)
        # of a step: what enters (0: the beam's row, 1: nothing, as there is no row 1), and whether that found its place
        self.rows, self.appended = i32(S, 1), i32(S)
        self.score = torch.zeros((S,), device=device)
        # what the steps chose, [0] sources and [1] tokens, how many steps there were, and whether all rows that enter found their places
        self.trace = i32(max_steps, 2, S)
        self.steps = torch.zeros((1,), dtype=torch.int64, device=device)
        self.least = torch.ones((S,), dtype=torch.int32, device=device)
        first = [-1] + [g * W for g in range(G)]
        self.first = torch.tensor(first[1:], dtype=torch.int64).to(device)
        self.fork = torch.tensor([s // W * W for s in range(S)], dtype=torch.int32).to(device)
        self.nobody = torch.full((S,), -1, dtype=torch.int32).to(device)

    def reset(self) -> None:
        """Empties all beams: their pages go back to the pool."""
        self.cache.reorder(self.nobody)
        self.least.fill_(1)

    def prompt(self, k, v) -> None:
        """Prompts of N tokens for all groups, in place of what the beams held: k and v bf16 [L][G][N][kv][64], keys not yet
        turned.  All beams of a group continue its prompt.  Refused, with nothing changed, if a table or the pool has no room for them."""
        k, v = _patterns(k), _patterns(v)
        N = int(k.shape[2]) if k.dim() == 5 else 0
        for t in (k, v):
            if tuple(t.shape) != (self.L, self.G, N, self.kv, HEAD_DIM) or N < 1:
                raise B.MloraError(B._ESHAPE, "beam loop's prompt")
        tokens = B.PAGE_TOKENS
        if N >= tokens * (self.cache.struct.max_pages + 1) or self.G * (N // tokens) > self.cache.struct.n_pages:
            raise B.MloraError(B._ESHAPE, "beam loop's prompt")
        self.reset()
        at_once = min(N, 4096 // self.S)                            # (rows that a call takes)
        for n0 in range(0, N, at_once):
            n = min(at_once, N - n0)
            rows = [torch.zeros((self.L, self.S, n, self.kv, HEAD_DIM), dtype=torch.int16, device=k.device) for _ in range(2)]
            at = torch.tensor([n0], dtype=torch.int32).to(k.device)
            for l in range(self.L):
                for g in range(self.G):
                    pairs = [B.RopeTensor(x[l, g, n0:n0 + n], to[l, g * self.W], rotate=i == 0) for i, (x, to) in enumerate(zip((k, v), rows))]
                    B.RopePlan(self.rope, pairs, n, B.Y_BF16, base=at).run()
            lists = torch.full((self.S, n), -1, dtype=torch.int32)
            lists[::self.W] = torch.arange(n, dtype=torch.int32)
            self.cache.append(rows[0].view(self.L, self.S * n, self.kv, HEAD_DIM), rows[1].view(self.L, self.S * n, self.kv, HEAD_DIM), n,
                              lists.to(k.device), self.appended)
            self.least[self.first] = torch.minimum(self.least[self.first], self.appended[self.first])
        self.cache.reorder(self.fork, self.window, self.sink)

    def start(self, tokens) -> None:
        """A new search from one beam of every group, behind what the beams hold (a prompt's, or nothing after reset()).  tokens int32 [G]: every
        group's newest token."""
        self.tokens.view(self.G, self.W).copy_(tokens.view(self.G, 1).expand(self.G, self.W))
        self.score.fill_(-float("inf"))
        self.score[self.first] = 0.0
        self.length.zero_()
        self.finished.zero_()
        self.steps.zero_()

    def step(self) -> None:
        """One token of every beam: tokens int32 [G * W], score, length and finished hold the new beams, best first in each group."""
        torch.index_select(self.embedding, 0, self.tokens.clamp(0, self.embedding.shape[0] - 1), out=self.h)
        self.tables.run()
        for layer in self.layers:
            layer.run()
        self.to_logits.run()
        torch.logical_or(self.finished, self.score - self.score, out=self.rows.view(self.S))     # (no number: the score of a place without a candidate)
        self.select.run(self.logits, self.score, self.length, self.finished, self.source, self.tokens, self.score, self.length, self.finished,
                        self.select_ws)
        self.cache.append(self.k_new, self.v_new, 1, self.rows, self.appended)
        self.appended.add_(self.rows.view(self.S))
        torch.minimum(self.least, self.appended, out=self.least)
        self.cache.reorder(self.source, self.window, self.sink)
        last = self.trace.shape[0] - 1
        self.trace.index_copy_(0, self.steps.clamp(max=last), torch.stack([self.source, self.tokens]).unsqueeze(0))
        self.steps.add_(1)

    def sequences(self) -> List[List[Tuple[List[int], float]]]:
        """The tokens and score of every beam of every group, best first (waits for the device).  Steps beyond max_steps are not traced, and rows that
        found no place in a cache would make what followed wrong: both are refused here."""
        steps = int(self.steps.item())
        if steps > self.trace.shape[0] or int(self.least.min().item()) < 1:
            raise B.MloraError(B._EWORKSPACE, "beam loop")
        trace, length, score = self.trace[:steps].tolist(), self.length.tolist(), self.score.tolist()
        out = []
        for s in range(self.S):
            tokens, at = [], s
            for source, token in reversed(trace):
                tokens.append(token[at])
                at = source[at]
            out.append((tokens[::-1][:length[s]], score[s]))
        return [out[g * self.W:(g + 1) * self.W] for g in range(self.G)]
