"""The cache-managed inference cycle around the refresh pass (Sec. 3.2, algorithm summary).

A sequence's cache holds up to J + h entries: the J kept by the last refresh followed by
the entries appended since.  `append` adds new entries (their keys and values for every
cache layer, token ids, original positions, and the per-entry rows the scoring mode
needs: queries for the given-query fast variant, the activations entering the last
layer for the exact fast variant).  `refresh` runs one memory-refresh cycle: the
counter-causal score of every cached entry, selection of the J highest (kept in their
original order), and compaction of keys, values, ids, positions and rows.  `run_stream`
drives a prompt and a decode phase, refreshing every h tokens (chunked mode) or once at
the end of the prompt (prefill-end mode).

Everything here is orchestration on the caller's stream; every step of the pass runs in
libcc.  Entries keep the absolute positions they were appended with.

The cache holds bf16, or 8 bits (cache="e4m3": E4M3 codes with a power-of-two scale for each
block of entries and head, half the bytes): the same cycle on cc_append_kv8, cc_attention_kv8
and cc_compact_kv8.  An 8-bit cache scores the given-query fast variants, and `attend` runs
the inference cycle's own attention over it.
"""
from __future__ import annotations

import dataclasses
from typing import Callable, Optional

import torch

from . import cc


@dataclasses.dataclass
class Model:
    """Shapes and weights the scoring pass needs (device tensors in bf16)."""
    mode: str                         # "last_layer" (queries given), "last_layer_fused" (queries
                                      # given, w_lm = W_lm W_o) or "last_layer_h"
    n_layers: int                     # cache layers
    n_heads_q: int
    n_heads_kv: int
    head_dim: int
    hidden: int
    vocab: int
    w_lm: torch.Tensor
    w_o: Optional[torch.Tensor] = None          # last_layer
    layer: Optional[dict] = None                # last_layer_h: the last layer's weights
    final_norm: Optional[torch.Tensor] = None   # last_layer_h
    ffn: int = 0
    rope_theta: float = 5e5
    rms_eps: float = 1e-5
    w_lm_packed: Optional[torch.Tensor] = None  # cc_pack_lmhead(w_lm): the packed LM head

    @property
    def row_width(self) -> int:
        """Elements of the per-entry row the mode scores from (Q or H)."""
        return self.hidden if self.mode == "last_layer_h" else self.n_heads_q * self.head_dim


class RefreshLoop:
    """One sequence's cache under counter-causal memory management."""

    def __init__(self, model: Model, J: int, h: int, device="cuda",
                 capacity: Optional[int] = None, cache: str = "bf16", scale_block: int = 16):
        """cache: "bf16" or "e4m3" (scale_block entries a scale: a power of two from 16 to 128)."""
        if model.mode not in ("last_layer", "last_layer_fused", "last_layer_h"):
            raise ValueError("mode must be last_layer, last_layer_fused or last_layer_h")
        if J < 1 or h < 1:
            raise ValueError("J and h must be positive")
        if cache not in ("bf16", "e4m3"):
            raise ValueError("cache must be bf16 or e4m3")
        if cache == "e4m3" and model.mode == "last_layer_h":
            raise ValueError("an 8-bit cache scores given queries (last_layer or last_layer_fused)")
        if cache == "e4m3" and scale_block not in (16, 32, 64, 128):
            raise ValueError("scale_block must be 16, 32, 64 or 128")
        self.m, self.J, self.h = model, J, h
        self.cache = cache
        self.device = torch.device(device)
        cap = capacity if capacity is not None else J + h   # chunked mode needs J + h
        self.cap = cap
        L, hkv, d = model.n_layers, model.n_heads_kv, model.head_dim
        bf = torch.bfloat16
        self.k = torch.zeros((L, hkv, cap, d), dtype=torch.uint8 if cache == "e4m3" else bf, device=self.device)
        self.v = torch.zeros_like(self.k)
        self.ids = torch.zeros(cap, dtype=torch.int32, device=self.device)
        self.pos = torch.zeros(cap, dtype=torch.int32, device=self.device)
        self.rows = torch.zeros((cap, model.row_width), dtype=bf, device=self.device)
        self.n = 0
        if cache == "e4m3":
            blocks = -(-cap // scale_block)
            self.k_scale = torch.zeros((L, hkv, blocks), dtype=torch.uint8, device=self.device)
            self.v_scale = torch.zeros_like(self.k_scale)
            self.cached = torch.zeros(1, dtype=torch.int32, device=self.device)   # n, for appending
            self.kv = cc.kv8_contiguous(self.k, self.v, self.k_scale, self.v_scale, n_layers=L,
                                        layer_stride=hkv * cap * d, head_stride=cap * d, tok_stride=d,
                                        scale_block=scale_block, scale_layer_stride=hkv * blocks,
                                        scale_head_stride=blocks)
        else:
            self.kv = cc.kv_contiguous(self.k, self.v, n_layers=L, layer_stride=hkv * cap * d,
                                       head_stride=cap * d, tok_stride=d)
        self.refreshes = 0

    # ---------------------------------------------------------------- inference side
    def append(self, k: torch.Tensor, v: torch.Tensor, ids: torch.Tensor, pos: torch.Tensor,
               rows: torch.Tensor) -> None:
        """Append m entries: k, v [L][Hkv][m][d]; ids, pos [m]; rows [m][row_width]."""
        m = int(ids.shape[0])
        if self.n + m > self.cap:
            raise ValueError(f"cache holds {self.n} of {self.cap}; refresh before appending {m}")
        sl = slice(self.n, self.n + m)
        if self.cache == "e4m3":
            if m == 0:
                return
            # (lengths written by the stream, as in _queued_problem)
            self.cached.fill_(self.n)
            cc.cc_append_kv8(self._queued_problem(m), self.kv, k.transpose(1, 2), v.transpose(1, 2), self.cached,
                             capacity=self.cap, n_layers=self.m.n_layers, rotate=False)
        else:
            self.k[:, :, sl].copy_(k)
            self.v[:, :, sl].copy_(v)
        self.ids[sl].copy_(ids)
        self.pos[sl].copy_(pos)
        self.rows[sl].copy_(rows)
        self.n += m

    # ---------------------------------------------------------------- refresh cycle
    def problem(self, cu_device: Optional[torch.Tensor] = None, n: Optional[int] = None) -> cc.Problem:
        m = self.m
        return cc.problem(dtype="bf16", cu_seqlens=[0, self.n if n is None else n], n_heads_q=m.n_heads_q,
                          n_heads_kv=m.n_heads_kv, head_dim=m.head_dim, hidden=m.hidden,
                          vocab=m.vocab, device=self.device, mode=m.mode, ffn=m.ffn,
                          rope_theta=m.rope_theta, rms_eps=m.rms_eps,
                          lmhead_packed=m.w_lm_packed is not None, cu_device=cu_device)

    def _queued_problem(self, n: Optional[int] = None) -> cc.Problem:
        """problem(), its device lengths written by the current stream: no wait for a copy
        (2% of a pass of 768 entries when passes follow each other)."""
        cu = torch.zeros(2, dtype=torch.int32, device=self.device)
        cu[1:].fill_(self.n if n is None else n)
        return self.problem(cu, n)

    def attend(self, layer: int, q: torch.Tensor) -> torch.Tensor:
        """Causal attention of the last m entries' queries q [m][Hq][head_dim] (rotated) over cache
        layer `layer` (8-bit caches): the inference cycle's attention after its append."""
        if self.cache != "e4m3":
            raise ValueError("attend runs on 8-bit caches")
        m = int(q.shape[0])
        if m > self.n:
            raise ValueError(f"{m} queries for {self.n} entries")
        lens = torch.full((1,), self.n, dtype=torch.int32, device=self.device)
        return cc.cc_attention_kv8(self._queued_problem(m), q, self.kv, layer, lens, self.n)

    def _scores8(self) -> torch.Tensor:
        """scores() on an 8-bit cache, step by step: attention, W_o, LM head."""
        m, n = self.m, self.n
        p = self._queued_problem()
        q = self.rows[:n].view(n, m.n_heads_q, m.head_dim)
        u = cc.cc_attention_kv8(p, q, self.kv, m.n_layers - 1, p.cu_d[1:], n, mask="counter").view(n, m.row_width)
        if m.mode == "last_layer":
            u = cc.cc_linear("bf16", u, m.w_o, torch.empty((n, m.hidden), dtype=u.dtype, device=u.device))
        else:   # the LM head's input is as wide as the queries
            p.struct.hidden = m.row_width
        s = torch.empty(n, dtype=torch.float32, device=self.device)
        if m.w_lm_packed is not None:
            return cc.cc_lmhead_score_packed(p, u, m.w_lm_packed, self.ids, s)
        return cc.cc_lmhead_score(p, u, m.w_lm, self.ids, s)

    def inputs(self) -> cc.Inputs:
        m, n = self.m, self.n
        if m.mode in ("last_layer", "last_layer_fused"):
            return cc.inputs(kv=self.kv, token_ids=self.ids, w_lm=m.w_lm, w_o=m.w_o,
                             q=self.rows[:n], w_lm_packed=m.w_lm_packed)
        return cc.inputs(kv=self.kv, token_ids=self.ids, w_lm=m.w_lm, layers=[m.layer],
                         final_norm=m.final_norm, h_last=self.rows[:n], pos_ids=self.pos,
                         w_lm_packed=m.w_lm_packed)

    def scores(self) -> torch.Tensor:
        """Counter-causal surprise of every cached entry (the last one is +inf)."""
        if self.cache == "e4m3":
            return self._scores8()
        s = torch.empty(self.n, dtype=torch.float32, device=self.device)
        cc.cc_score(self._queued_problem(), self.inputs(), s)
        return s

    def refresh(self, hook: Optional[Callable] = None) -> torch.Tensor:
        """One memory-refresh cycle; returns the keep list (indices into the entries as
        they were).  `hook(scores, keep)` sees both before the cache is rewritten."""
        if self.n <= self.J:
            return torch.arange(self.n, dtype=torch.int32, device=self.device)
        p = self._queued_problem()
        s = self.scores()
        keep = torch.empty(self.J, dtype=torch.int32, device=self.device)
        cc.cc_select_keep(s, [0], [self.n], [self.J], keep)
        if hook is not None:
            hook(s, keep)
        compact = cc.cc_compact_kv8 if self.cache == "e4m3" else cc.cc_compact_kv
        compact(p, self.kv, keep, [self.J], 0, token_ids=self.ids, pos_ids=self.pos)
        cc.cc_compact_rows(p, self.rows, keep, [self.J], 0)
        self.n = self.J
        self.refreshes += 1
        return keep


def run_stream(loop: RefreshLoop, entry: Callable, T_prompt: int, T_total: int,
               chunked: bool = True, hook: Optional[Callable] = None) -> None:
    """Drive a stream of T_total tokens through the cache.  `entry(t0, t1)` returns the
    (k, v, ids, pos, rows) of tokens t0..t1-1 (the inference cycle's new keys, values,
    token ids, positions and rows).  Chunked mode refreshes whenever the token count
    reaches a multiple of h: the prompt is appended in batches up to each refresh point,
    the decode phase one token at a time.  Prefill-end mode appends the whole prompt,
    refreshes once, then decodes without refreshing (the cache must hold the prompt and
    the decoded tokens)."""
    h = loop.h
    t = 0
    while t < T_prompt:
        t1 = min(T_prompt, (t // h + 1) * h) if chunked else T_prompt
        loop.append(*entry(t, t1))
        t = t1
        if chunked and t % h == 0:
            loop.refresh(hook)
    if not chunked:
        loop.refresh(hook)
    while t < T_total:
        loop.append(*entry(t, t + 1))
        t += 1
        if chunked and t % h == 0:
            loop.refresh(hook)
