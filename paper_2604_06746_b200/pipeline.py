"""Sequencing of the C-ABI calls over one prompt (the control flow of Algorithm 1
replayed over per-layer tensors): score every layer, detect the pivot, rebuild
the centrality at the pivot, select both budgets, compact K/V, hidden states
and position ids; and over the tokens that follow it (Decode).  All arithmetic happens
inside the library's kernels; this file only owns buffers and call order.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import torch

from . import binding

PAPER_LAMBDA = 0.9
PAPER_WEIGHTS = (0.2, 0.3, 0.5)


class Prefill:
    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, window: int,
                 seq: int, kv_budget: int, struct_budget: int, dtype: torch.dtype,
                 hidden_dim: int = 0, device: str = "cuda:0", lam: float = PAPER_LAMBDA,
                 weights: Sequence[float] = PAPER_WEIGHTS, l_limit: int = -1, flags: int = 0,
                 keep_kv: bool = True, defer_head_stats: bool = True):
        self.L, self.H, self.Hkv, self.d, self.w, self.N = n_layers, n_q_heads, n_kv_heads, head_dim, window, seq
        self.kv_budget, self.struct_budget = kv_budget, struct_budget
        self.lam, self.weights, self.l_limit, self.flags = lam, tuple(weights), l_limit, flags
        self.dtype, self.device = dtype, torch.device(device)
        self.ctx = binding.Context(n_q_heads, n_kv_heads, head_dim, window, seq, dtype, device)
        dev = self.device
        f32, i32 = torch.float32, torch.int32
        self.s_hist = torch.zeros((n_layers, seq), dtype=f32, device=dev)
        self.metrics = torch.zeros((n_layers, 3), dtype=f32, device=dev)
        self.c_running = torch.zeros((seq,), dtype=f32, device=dev)
        self.c_star = torch.zeros((seq,), dtype=f32, device=dev)
        self.i_kv = torch.zeros((n_layers, kv_budget), dtype=i32, device=dev)
        self.i_struct = torch.zeros((struct_budget,), dtype=i32, device=dev)
        n_kv_out = n_layers if keep_kv else 1
        self.keep_kv = keep_kv
        # compacted K and V of a layer sit in one allocation [2, H_kv, B, d]: when the source K and V
        # are laid out the same way, one gather launch serves both
        self.kv_out = torch.empty((n_kv_out, 2, n_kv_heads, kv_budget, head_dim), dtype=dtype, device=dev)
        self.k_out = self.kv_out[:, 0]
        self.v_out = self.kv_out[:, 1]
        self.hidden_out = (torch.empty((struct_budget, hidden_dim), dtype=torch.bfloat16, device=dev)
                           if hidden_dim else None)
        self.pos_out = torch.empty((struct_budget,), dtype=i32, device=dev)
        self.pivot = -1
        self.transition: List[float] = []
        # Eq. 5-6 of all layers in one batched call before the pivot (instead of a chain of short
        # dependent launches after every layer): the pooled per-head attention of every layer is kept
        self.defer = bool(defer_head_stats) and not (flags & binding.FLAG_NO_HEAD_STATS) and n_layers <= 128
        self.head_cols = (torch.empty((n_layers, n_q_heads, seq), dtype=f32, device=dev) if self.defer else None)
        self._stats_done = 0
        self._layers_ws = None
        self._plan = None

    def rotate(self, q_win: torch.Tensor, k: torch.Tensor, rope: binding.Rope, positions: torch.Tensor) -> None:
        """Eq. 12's f_RoPE, in place: a layer's keys ``[H_kv, N, d]`` at ``positions [N]`` (int32) and its window queries ``[H, w, d]`` at the
        last of them, as the scorer takes them."""
        self.ctx.rotate(k.transpose(0, 1)[None], positions, rope)
        self.ctx.rotate(q_win.transpose(0, 1)[None], positions[-q_win.shape[1]:], rope)

    # -- Algorithm 1 lines 3-6 for one layer
    def score(self, layer: int, q_win: torch.Tensor, k: torch.Tensor, scale: float,
              head_cols_out: Optional[torch.Tensor] = None) -> None:
        if layer == 0:
            self.c_running.zero_()
            self._stats_done = 0
        if self.defer:
            self.ctx.score_layer(q_win, k, scale, self.s_hist[layer], self.metrics[layer],
                                 c_inout=self.c_running, lam=self.lam, head_cols_out=self.head_cols[layer],
                                 flags=self.flags | binding.FLAG_NO_HEAD_STATS)
            if head_cols_out is not None:
                head_cols_out.copy_(self.head_cols[layer])
            return
        self.ctx.score_layer(q_win, k, scale, self.s_hist[layer], self.metrics[layer],
                             c_inout=self.c_running, lam=self.lam, head_cols_out=head_cols_out,
                             flags=self.flags)

    def score_all(self, layers: Sequence[Dict[str, torch.Tensor]]) -> None:
        """Algorithm 1 lines 3-6 for resident layers.  Where the pooled per-head attention of every layer
        is kept anyway (head statistics in one batched call) and the layers' K tensors share one layout,
        all layers go through one structkv_score_layers call, which interleaves the scorer passes of
        neighbouring layers; otherwise layer after layer."""
        L = len(layers)
        k0 = layers[0]["k"]
        same = all(t["k"].shape == k0.shape and t["k"].stride() == k0.stride() for t in layers)
        if not (self.defer and same and L == self.L and self.flags in (0, binding.FLAG_INPUTS_READY)):
            for l, t in enumerate(layers):
                self.score(l, t["q_win"], t["k"], t["scale"])
            return
        if self._layers_ws is None:
            self._layers_ws = self.ctx.layers_workspace(self.L)
        self.c_running.zero_()
        self._stats_done = 0
        self.ctx.score_layers([t["q_win"] for t in layers], [t["k"] for t in layers],
                              [t["scale"] for t in layers], self.s_hist, self.metrics, self.head_cols,
                              self._layers_ws, c_inout=self.c_running, lam=self.lam)

    def finish_scores(self, n_scored: Optional[int] = None) -> None:
        """Sparsity and variance (Eq. 5-6) of the layers scored so far, in one batched call."""
        L = self.L if n_scored is None else n_scored
        if self.defer and self._stats_done < L:
            self.ctx.head_stats(self.head_cols[self._stats_done:L], self.metrics[self._stats_done:L])
            self._stats_done = L

    # -- Algorithm 1 lines 7-10 and 16: pivot, centrality at the pivot, both index sets
    def detect_and_select(self, n_scored: Optional[int] = None) -> int:
        L = self.L if n_scored is None else n_scored
        self.finish_scores(L)
        self.pivot, self.transition = self.ctx.pivot_select(
            self.s_hist[:L], self.metrics[:L], self.weights, self.l_limit, self.lam, self.w, self.kv_budget, self.i_kv[:L],
            self.struct_budget, self.c_star, self.i_struct)
        return self.pivot

    # -- Algorithm 1 line 17 for one layer
    def compact_kv(self, layer: int, k: torch.Tensor, v: torch.Tensor,
                   kv: Optional[torch.Tensor] = None) -> None:
        """``kv`` (optional) is the joint storage ``[2, H_kv, N, d]`` whose halves are ``k`` and ``v``."""
        slot = layer if self.keep_kv else 0
        if kv is not None:
            self.ctx.compact(kv.view(2 * self.Hkv, kv.shape[2], self.d), self.i_kv[layer],
                             self.kv_out[slot].view(2 * self.Hkv, self.kv_budget, self.d))
            return
        self.ctx.compact(k, self.i_kv[layer], self.k_out[slot])
        self.ctx.compact(v, self.i_kv[layer], self.v_out[slot])

    def compact_all_kv(self, layers: Sequence[Dict[str, torch.Tensor]]) -> None:
        """Algorithm 1 line 17 for resident layers: one launch for all of them when every layer keeps
        K and V in one joint allocation, else one gather per layer."""
        if self.keep_kv and len(layers) <= 128 and all("kv" in t for t in layers):
            self.ctx.compact_layers([t["kv"].view(2 * self.Hkv, t["kv"].shape[2], self.d) for t in layers],
                                    self.i_kv[:len(layers)],
                                    self.kv_out[:len(layers)].view(len(layers), 2 * self.Hkv, self.kv_budget, self.d))
            return
        for l, t in enumerate(layers):
            if "v" in t:
                self.compact_kv(l, t["k"], t["v"], t.get("kv"))

    # -- Algorithm 1 line 13
    def compact_hidden(self, hidden: torch.Tensor, positions: torch.Tensor) -> None:
        self.ctx.compact(hidden[None], self.i_struct, self.hidden_out[None])
        self.ctx.compact(positions[None, :, None], self.i_struct, self.pos_out[None, :, None])

    # -- Algorithm 1 past the pivot (Eq. 11-13 on the reduced sequence)
    def enable_reduced(self) -> None:
        """Buffers for layers scored after the truncation: K gathered at I_struct, the saliency of
        the reduced sequence, its selection, and that selection as original position ids."""
        dev, f32, i32 = self.device, torch.float32, torch.int32
        nr = self.struct_budget
        self.k_red = torch.empty((self.Hkv, nr, self.d), dtype=self.dtype, device=dev)
        self.s_red = torch.zeros((self.L, nr), dtype=f32, device=dev)
        self.metrics_red = torch.zeros((self.L, 3), dtype=f32, device=dev)
        self.i_red = torch.zeros((self.L, self.kv_budget), dtype=i32, device=dev)
        self.i_kv_pos = torch.zeros((self.L, self.kv_budget), dtype=i32, device=dev)
        self.recovery = torch.zeros((self.L,), dtype=f32, device=dev)

    def score_reduced(self, layer: int, q_win: torch.Tensor, k: torch.Tensor, scale: float) -> None:
        """Layer ``layer`` > L* on the keys that survived the truncation: gather K at I_struct
        (Eq. 11), score the reduced sequence (the window is its tail, so the queries are unchanged)."""
        self.ctx.compact(k, self.i_struct, self.k_red)
        self.ctx.score_layer(q_win, self.k_red, scale, self.s_red[layer], self.metrics_red[layer],
                             flags=self.flags)

    def select_reduced(self, first: int, last: int) -> None:
        """Eq. 13 on the reduced sequences of layers ``first .. last - 1`` (one batched launch), then
        each index list mapped back to original positions through the gathered position ids
        (Eq. 12; ``compact_hidden`` must have filled ``pos_out``)."""
        if last <= first:
            return
        self.ctx.select(self.s_red[first:last], self.kv_budget, self.w, self.i_red[first:last])
        # every layer gathers from the same position ids: one launch for (up to 128 of) them
        pos = self.pos_out[None, :, None]
        for lo in range(first, last, 128):
            hi = min(last, lo + 128)
            self.ctx.compact_layers([pos] * (hi - lo), self.i_red[lo:hi], self.i_kv_pos[lo:hi, None, :, None])

    def run(self, layers: Sequence[Dict[str, torch.Tensor]], hidden: Optional[torch.Tensor] = None,
            positions: Optional[torch.Tensor] = None) -> int:
        """Whole path over resident per-layer tensors (dicts with q_win, k, v, scale): one library call where every
        layer keeps K and V in one joint allocation and all share one layout, otherwise step by step."""
        args = self._prefill_args(layers, hidden, positions)
        if args is not None:
            self.pivot, self.transition = self.ctx.prefill(args)
            self._stats_done = self.L
            return self.pivot
        self.score_all(layers)
        self.detect_and_select(len(layers))
        self.compact_all_kv(layers)
        if hidden is not None:
            self.compact_hidden(hidden, positions)
        return self.pivot

    def _prefill_args(self, layers, hidden, positions) -> Optional[binding.PrefillArgs]:
        """The argument block of the one-call path (None: these tensors are not in that form).  Only the block's own
        memory is kept: every field is checked and written for every call, so that new tensors, other
        hyper-parameters and replaced output buffers are seen, and no tensor outlives its call here."""
        L, N, Hkv, d, dt = len(layers), self.N, self.Hkv, self.d, self.dtype
        if not (self.defer and self.keep_kv and L == self.L and L <= 128 and self.flags in (0, binding.FLAG_INPUTS_READY)):
            return None
        if self._plan is None or self._plan.n_layers != L:
            self._plan = binding.PrefillArgs.for_layers(L)
        a = self._plan
        sizes = (self.H, Hkv, N, d, self.w, self.kv_budget, self.struct_budget, self.l_limit)
        if not binding.fill_prefill(a, layers, hidden, positions, self.s_hist, self.head_cols, self.metrics, self.c_running,
                                    self.c_star, self.i_kv, self.i_struct, self.kv_out, self.hidden_out, self.pos_out,
                                    self._layers_ws, sizes, dt, self.lam, self.weights):
            return None
        if self._layers_ws is None:
            self._layers_ws = self.ctx.layers_workspace(L)
            a.layers_workspace, a.layers_workspace_bytes = self._layers_ws.data_ptr(), self._layers_ws.numel()
        return a


class Decode:
    """Decoding over what a Prefill kept (the paper stops at the compacted cache).  A token's step is ``step`` for every layer, then
    ``advance``; drafted tokens, a tree of them or a chain, are looked at by ``verify`` for every layer, then ``accept`` keeps
    some.  Cached tokens gather the attention weight that new ones give them, multiplied by ``decay`` once a ``step`` and once an
    ``accept``, however many tokens that keeps; with a ``budget`` every KV head keeps its ``recent`` newest tokens and the
    heaviest others.  All layers of all sequences are in one cache (sequence ``layer * batch +
    b``), so that commit and eviction are one launch each; every call can be captured into a graph.  Lengths live on the device:
    a KV head that has no room for new tokens is left as it is, and ``ctx.poll_device_status`` says so."""

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, capacity: int, dtype: torch.dtype,
                 batch: int = 1, budget: int = 0, recent: int = 0, max_new: int = 1, softcap: float = 0.0,
                 slopes: Optional[torch.Tensor] = None, decay: float = 1.0, device: str = "cuda:0"):
        if not 1 <= max_new <= binding.MAX_NEW:
            raise ValueError(f"max_new: 1 to {binding.MAX_NEW} new tokens")
        if budget < 0 or recent < 0 or (budget or 1) + max_new > capacity:
            raise ValueError("capacity: room for the budget and max_new tokens behind it")
        self.L, self.B, self.max_new = n_layers, batch, max_new
        self.budget, self.recent, self.softcap, self.slopes, self.decay = budget, recent, softcap, slopes, decay
        self.ctx = binding.Context(n_q_heads, n_kv_heads, head_dim, 8, 8, dtype, device)
        dev, f32, i32 = torch.device(device), torch.float32, torch.int32
        rows = (n_layers * batch, n_kv_heads, capacity)
        k, v = (torch.empty(rows + (head_dim,), dtype=dtype, device=dev) for _ in range(2))
        positions, weights = torch.zeros(rows, dtype=i32, device=dev), torch.zeros(rows, dtype=f32, device=dev)
        lengths = torch.zeros(rows[:2], dtype=i32, device=dev)
        self.cache = binding.Cache(k, v, positions, weights, lengths)
        self._weighed = torch.empty_like(lengths)              # lengths as accept() weighs by them
        self.layers, self._weighing = ([binding.Cache(*(t[l * batch:(l + 1) * batch] for t in (k, v, positions, weights, n)))
                                        for l in range(n_layers)] for n in (lengths, self._weighed))
        few = (batch, n_kv_heads, max_new)                     # (accept() asks whether its counts and paths are well-formed)
        self._asked = binding.Cache(*(torch.zeros(few + (head_dim,), dtype=dtype, device=dev) for _ in range(2)),
                                    torch.zeros(few, dtype=i32, device=dev), None, torch.zeros(few[:2], dtype=i32, device=dev))
        self._nth, self._one = torch.arange(max_new, dtype=i32, device=dev), torch.ones(1, dtype=torch.int64, device=dev)
        self._none = torch.full((1,), -1, dtype=i32, device=dev)
        self.lse = torch.empty((n_layers, batch, max_new, n_q_heads), dtype=f32, device=dev)
        self._ws = self.ctx.attend_workspace(self.layers[0], 1)
        for t in range(2, max_new + 1):                      # (not always more for more tokens)
            if self.ctx.attend_workspace_bytes(self.layers[0], t) > self._ws.numel():
                self._ws = self.ctx.attend_workspace(self.layers[0], t)
        self._seen: List[Optional[tuple]] = [None] * n_layers

    def take(self, prefill: Prefill, sequence: int = 0, positions: Optional[torch.Tensor] = None) -> None:
        """Sequence ``sequence`` begins with the prompt that ``prefill`` compacted: its K and V, its tokens' positions (``positions
        [L, kv_budget]`` int32; None: the prompt's indices) and, as the weight that they start with, the saliency that selected
        them."""
        n = prefill.kv_budget
        if not prefill.keep_kv or (prefill.L, prefill.Hkv, prefill.d, prefill.dtype) != (
                self.L, self.cache.n_kv_heads, self.cache.head_dim, self.cache.dtype):
            raise ValueError("take: a Prefill of these layers, heads and type that keeps K and V")
        if prefill.i_kv.device != self.cache.device:
            raise ValueError("take: a Prefill on the cache's device")
        if n > self.cache.capacity - self.max_new:
            raise ValueError("take: capacity for the prompt's tokens and max_new behind them")
        if not 0 <= sequence < self.B:
            raise ValueError("take: no such sequence")
        at = slice(sequence, None, self.B)
        c, start = self.cache, torch.empty((self.L, 1, n, 1), dtype=torch.float32, device=self.cache.device)
        for lo in range(0, self.L, 128):
            hi = min(self.L, lo + 128)
            prefill.ctx.compact_layers([s[None, :, None] for s in prefill.s_hist[lo:hi]], prefill.i_kv[lo:hi], start[lo:hi])
        c.k[at, :, :n], c.v[at, :, :n] = prefill.k_out, prefill.v_out
        c.positions[at, :, :n] = (prefill.i_kv if positions is None else positions)[:, None]
        c.weights[at, :, :n] = start[:, :, :, 0]
        c.lengths[at] = n

    def step(self, layer: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, positions: torch.Tensor,
             scale: float, out: torch.Tensor) -> None:
        """One token a sequence, ``q``, ``out [batch, 1, H, d]``, ``k_new``, ``v_new [batch, 1, H_kv, d]``: it is appended, attends,
        and its attention weight is added."""
        self.ctx.attend(self.layers[layer], q, scale, out, self._ws, k_new=k_new, v_new=v_new, positions=positions,
                        softcap=self.softcap, slopes=self.slopes, accumulate=True, decay=self.decay)

    def advance(self, n_new: int = 1) -> None:
        """After the last layer: the new tokens stay, and every KV head goes back to its budget."""
        self.ctx.commit(self.cache, n_new)
        self._evict()

    def verify(self, layer: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, positions: torch.Tensor,
               scale: float, out: torch.Tensor, tree: Optional[torch.Tensor] = None) -> None:
        """Drafted tokens, ``max_new`` of a sequence at most, see the cache and one another as ``tree`` says (None: those before
        them).  ``q`` and ``tree`` are looked at again by ``accept``."""
        n_new = q.shape[1]
        if n_new > self.max_new:
            raise ValueError("verify: more tokens than max_new")
        lse = self.lse[layer].view(-1)[:self.B * n_new * q.shape[2]].view(self.B, n_new, q.shape[2])
        self.ctx.attend(self.layers[layer], q, scale, out, self._ws, k_new=k_new, v_new=v_new, positions=positions, tree=tree,
                        softcap=self.softcap, slopes=self.slopes, lse=lse)
        self._seen[layer] = (q, scale, lse, tree)

    def accept(self, counts: torch.Tensor, path: torch.Tensor) -> None:
        """After ``verify`` of every layer: sequence b keeps the ``counts[b]`` drafted tokens that ``path[b]`` names, ascending
        (int32 ``[batch]`` and ``[batch, n_new]``); they give their attention weight, the others leave nothing.  A sequence whose
        count is not 0 .. n_new, or whose path does not ascend within them, is left as it is, and ``ctx.poll_device_status`` says so."""
        n_new, kind = path.shape[1] if path.dim() == 2 else 0, (torch.int32, self.cache.device)
        if counts.shape != (self.B,) or path.shape != (self.B, n_new) or (counts.dtype, counts.device) != kind or (path.dtype, path.device) != kind:
            raise ValueError("accept: counts [batch] and path [batch, n_new], int32 on the cache's device")
        if any(s is None or s[0].shape[1] != n_new for s in self._seen):
            raise ValueError("accept: verify of every layer comes first, of as many tokens")
        # What commit refuses must not weigh either: it is asked first, over caches without tokens, and what it leaves so has no lengths.
        self._asked.lengths.zero_()
        self.ctx.commit(self._asked, n_new, counts=counts.contiguous(), path=path.contiguous())
        torch.where(self._asked.lengths == counts[:, None], self.cache.lengths.view(self.L, self.B, -1), self._none,
                    out=self._weighed.view(self.L, self.B, -1))
        words = torch.where(self._nth[:n_new] < counts[:, None], self._one << path, 0).sum(1)
        for cache, (q, scale, lse, tree) in zip(self._weighing, self._seen):
            self.ctx.weigh(cache, q, scale, lse, words, tree=tree, softcap=self.softcap, slopes=self.slopes, decay=self.decay)
        self.ctx.commit(self.cache, n_new, counts=counts.repeat(self.L), path=path.repeat(self.L, 1))
        self._seen = [None] * self.L
        self._evict()

    def _evict(self) -> None:
        if self.budget:
            self.ctx.evict(self.cache, self.budget, self.recent)


class PagedDecode:
    """Decoding over a paged cache in 8 bits, for what a Prefill kept or for prompts whose keys come here.  Pages are shared out by
    ``reserve`` and given back by ``release``; page numbers, table and lengths are the same for all layers, of which each has storage of its
    own.  A step is ``step`` for every layer, with one new token a sequence or up to ``max_new``, then ``advance`` by as many as stay:
    tokens behind ``lengths`` do not count, and the next ones take their slots.  Only ``take``, ``advance`` and ``release`` move ``lengths``, ``advance`` within
    the pages that a sequence has.  With a ``rope`` new keys and queries come without positions
    and are rotated on the way.  Every call but ``reserve`` and ``release`` can be captured into a graph.  A sequence without room is left
    as it is, and ``ctx.poll_device_status`` says so.  Rows that are dropped leave something: where one raised the scale of the 16 slots that
    kept tokens share with it, those keep the raised scale and the codes that were rounded to it."""

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, pages: int, columns: int, dtype: torch.dtype,
                 batch: int = 1, page_size: int = 64, max_new: int = 1, rope: Optional[binding.Rope] = None, softcap: float = 0.0,
                 device: str = "cuda:0"):
        if not 1 <= max_new <= binding.MAX_NEW:
            raise ValueError(f"max_new: 1 to {binding.MAX_NEW} new tokens")
        if pages < 1 or columns < 1 or batch < 1 or n_layers < 1:
            raise ValueError("layers, pages, columns and sequences: one at least")
        self.L, self.B, self.max_new, self.rope, self.softcap, self.page_size = n_layers, batch, max_new, rope, softcap, page_size
        self.ctx = binding.Context(n_q_heads, n_kv_heads, head_dim, 8, 8, dtype, device)
        dev = torch.device(device)
        self.table = torch.full((batch, columns), -1, dtype=torch.int32, device=dev)
        self.lengths = torch.zeros((batch,), dtype=torch.int32, device=dev)
        self.layers = [binding.Pages.empty(pages, n_kv_heads, page_size, head_dim, self.table, self.lengths) for _ in range(n_layers)]
        self._of = [[self._part(p, b) for b in range(batch)] for p in self.layers]     # a sequence by itself
        self._q = torch.empty((batch * max_new * n_q_heads * head_dim,), dtype=dtype, device=dev) if rope is not None else None
        self._ws = self.ctx.attend_pages_workspace(self.layers[0], 1)
        for t in range(2, max_new + 1):                      # (not always more for more tokens)
            ws = self.ctx.attend_pages_workspace(self.layers[0], t)
            self._ws = ws if ws.numel() > self._ws.numel() else self._ws
        self._free, self._have = list(range(pages)), [[] for _ in range(batch)]
        self._room = torch.zeros((batch,), dtype=torch.int32, device=dev)             # slots of the pages that a sequence has
        self._nth = torch.arange(1, max_new + 1, dtype=torch.int32, device=dev)
        self._counts = torch.zeros((max_new, batch), dtype=torch.int32, device=dev)   # row n - 1: n where a sequence has pages, else 0
        one = (batch, n_kv_heads, 1)                            # (by which advance() tells the status word; never a token in it)
        self._asked = binding.Cache(*(torch.zeros(one + (head_dim,), dtype=dtype, device=dev) for _ in range(2)),
                                    torch.zeros(one, dtype=torch.int32, device=dev), None, torch.zeros(one[:2], dtype=torch.int32, device=dev))

    def _part(self, p: binding.Pages, b: int) -> binding.Pages:
        return binding.Pages(p.k, p.v, p.k_scales, p.v_scales, self.table[b:b + 1], self.lengths[b:b + 1])

    def reserve(self, sequence: int, tokens: int) -> None:
        """Pages for ``tokens`` tokens of a sequence in all, those that it has among them."""
        have, need = self._have[sequence], -(-tokens // self.page_size)
        if need > self.table.shape[1] or need - len(have) > len(self._free):
            raise ValueError("reserve: more pages than a sequence can have, or than are free")
        more = [self._free.pop() for _ in range(need - len(have))]
        if more:
            self.table[sequence, len(have):need] = torch.tensor(more, dtype=torch.int32, device=self.table.device)
            have += more
            self._room[sequence] = need * self.page_size
            self._counts[:, sequence] = self._nth

    def release(self, sequence: int) -> None:
        """The sequence ends: its pages are free again.  (Calls that read them were made before, on the same stream.)"""
        self._free += self._have[sequence]
        self._have[sequence] = []
        self.table[sequence] = -1
        self.lengths[sequence] = 0
        self._room[sequence] = 0
        self._counts[:, sequence] = 0

    def take(self, prefill: Prefill, sequence: int = 0) -> None:
        """The sequence begins with the prompt that ``prefill`` compacted: its K (rotated, as it was scored) and V.  ``reserve`` comes first."""
        c = self.ctx.cfg
        if not prefill.keep_kv or (prefill.L, prefill.Hkv, prefill.d, prefill.dtype) != (self.L, c.n_kv_heads, c.head_dim, self.ctx.dtype):
            raise ValueError("take: a Prefill of these layers, heads and type that keeps K and V")
        if prefill.kv_out.device != self.table.device:
            raise ValueError("take: a Prefill on the pages' device")
        if len(self._have[sequence]) * self.page_size < prefill.kv_budget:
            raise ValueError("take: pages for the prompt's tokens are reserved first")
        self.lengths[sequence] = 0
        for l in range(self.L):
            self.ctx.append_pages(self._of[l][sequence], prefill.k_out[l].transpose(0, 1)[None], prefill.v_out[l].transpose(0, 1)[None])
        self.lengths[sequence] = prefill.kv_budget

    def keep(self, layer: int, sequence: int, k: torch.Tensor, v: torch.Tensor, index: Optional[torch.Tensor] = None,
             positions: Optional[torch.Tensor] = None) -> None:
        """Rows of one layer's K and V ``[H_kv, N, d]`` go behind the sequence's tokens: those that ``index`` (int32, one list for all heads)
        names, or all; with ``positions [N]`` (and a rope) K is rotated on the way.  ``advance`` comes after the last layer."""
        if positions is not None and self.rope is None:
            raise ValueError("keep: positions come with a rope")
        rope = self.rope if positions is not None else None
        self.ctx.append_pages(self._of[layer][sequence], k.transpose(0, 1)[None], v.transpose(0, 1)[None], positions=positions, rope=rope, index=index)

    def step(self, layer: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, positions: Optional[torch.Tensor], scale: float,
             out: torch.Tensor, counts: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None) -> None:
        """New tokens, ``q``, ``out [batch, n_new, H, d]``, ``k_new``, ``v_new [batch, n_new, H_kv, d]``, ``counts [batch]`` of them for each
        sequence (None: all, of the sequences that have pages): they are rotated (with a rope), appended, and see the cache and those before
        them."""
        b, n, h, d = q.shape
        if n > self.max_new:
            raise ValueError("step: more tokens than max_new")
        if counts is None and n:
            counts = self._counts[n - 1]
        if self.rope is not None:
            if positions is None:
                raise ValueError("step: positions come with a rope")
            rotated = self._q[:b * n * h * d].view(b, n, h, d)
            self.ctx.append_pages(self.layers[layer], k_new, v_new, positions=positions, rope=self.rope, counts=counts, q=q, q_out=rotated)
            q = rotated
        else:
            self.ctx.append_pages(self.layers[layer], k_new, v_new, counts=counts)
        self.ctx.attend_pages(self.layers[layer], q, scale, out, self._ws, counts=counts, softcap=self.softcap, lse=lse)

    def advance(self, n_new) -> None:
        """After the last layer: the first ``n_new`` of the new tokens stay: a number, for every sequence that has pages, or int32 ``[batch]``
        on the device.  A sequence whose pages do not hold as many is left as it is, and ``ctx.poll_device_status`` says so."""
        # (int64 where a number is multiplied: what 32 bits do not hold is refused too)
        n = n_new if isinstance(n_new, torch.Tensor) and n_new.dim() else (self._room > 0) * n_new
        grown = self.lengths + n
        fits = (grown >= 0) & (grown <= self._room)
        self.lengths += fits * n
        self.ctx.commit(self._asked, 1, counts=fits.to(torch.int32) - 1)       # (commit refuses a count of -1, and does nothing for 0)
