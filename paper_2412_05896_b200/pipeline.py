"""The call a user makes: one object that owns the device buffers of a batch (torch tensors for
memory and streams only) and drives the four library entry points in order.

    sess = XkvSession(...); sess.prefill(q_win, k, v, total=...); sess.decode(q, k_new, v_new)

Every computation happens inside libxkv.so; this file allocates, copies and calls.
"""
from __future__ import annotations

import ctypes
import math
import time

import numpy as np
import torch

from . import xkv


class XkvSession:
    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, window: int,
                 pool_kernel: int, lengths: list[int], pool_mode: int = xkv.POOL_MAX, page_size: int = 16,
                 max_new_tokens: int = 0, max_budget: int | None = None, total_budget: int | None = None,
                 curve_len: int | None = None, device="cuda:0", scale: float = 0.0,
                 decode_chunk_rows: int = 0, n_lanes: int = 6, head_level: bool = False,
                 kv_format: int = xkv.KV_BF16, pages_on_demand: bool = False):
        """head_level: budgets, cache lengths and page lists per (layer, sequence, KV head) instead of per (layer,
        sequence); total_budget and the solver's total then count prefix tokens over all heads of all layers, and
        max_budget bounds one head.
        pages_on_demand: caches take pages from the pool as they grow (planned on the device, `append`); otherwise the
        pages of all max_new_tokens are set aside when the budgets are known."""
        self.L, self.Hq, self.Hkv, self.d, self.W = n_layers, n_q_heads, n_kv_heads, head_dim, window
        self.head_level = bool(head_level)
        # xkv.KV_INT8: the reduced caches hold 8-bit codes and row scales; xkv.KV_E4M3: 8-bit floats and block scales
        self.kv_format = kv_format
        self.pages_on_demand = bool(pages_on_demand)
        self.G = n_q_heads // n_kv_heads
        self.B = len(lengths)
        self.lengths = list(lengths)
        self.device = torch.device(device)
        self.page_size = page_size
        self.max_new = max_new_tokens
        cu = [0]
        for t in lengths:
            cu.append(cu[-1] + t)
        self.T = cu[-1]
        self.max_seqlen = max(lengths)
        self.prefix = [max(t - window, 0) for t in lengths]
        self.max_prefix = max(self.prefix)
        self.cu_host = np.asarray(cu, dtype=np.int32)
        self.cu = torch.tensor(cu, dtype=torch.int32, device=self.device)
        self.dims = xkv.Dims(self.B, n_q_heads, n_kv_heads, head_dim, window, pool_kernel, pool_mode, scale,
                             n_kv_heads * head_dim, head_dim)

        # per-layer scores, their sort and the curves (kept for all layers: the solver needs every curve
        # before the first layer can be compacted)
        # (a multiple of four ranks, so that every layer's slice of the stacked arrays starts on a 16-byte boundary;
        # ranks beyond the longest prefix read zero)
        self.curve_len = (max(1, min(curve_len or self.max_prefix, max(self.max_prefix, 1))) + 3) // 4 * 4
        f32 = dict(dtype=torch.float32, device=self.device)
        self._layer_stride = (n_kv_heads * self.T + 3) // 4 * 4           # floats between the layers' score arrays
        self.scores = torch.empty(n_layers, self._layer_stride, **f32)[:, : n_kv_heads * self.T].view(
            n_layers, n_kv_heads, self.T)
        self.sorted = torch.empty(n_layers, self._layer_stride, **f32)[:, : n_kv_heads * self.T].view(
            n_layers, n_kv_heads, self.T)
        self.gains = torch.empty(n_layers, self.B, self.curve_len, **f32)
        # what crosses to the host for the solver: one curve per layer (the batch mean, formed on the device);
        # the per-sequence curves cross only when every sequence gets its own list
        # units of the solver: layers, or (layer, KV head) pairs with head-level budgets
        self.n_solver_units = n_layers * (n_kv_heads if self.head_level else 1)
        self.head_gains = torch.empty(n_layers, n_kv_heads, self.B, self.curve_len, **f32) if self.head_level else None
        self.layer_gains = torch.empty(self.n_solver_units, self.curve_len, **f32)
        self.layer_gains_host = torch.empty(self.n_solver_units, self.curve_len, dtype=torch.float32, pin_memory=True)
        self.gains_host = None
        # Layers are independent in the scoring and in the eviction phase, so consecutive layers go to
        # n_lanes side streams, each with its own workspace: the short latency-bound kernels of one layer
        # (sort, curves, selection) then run under the HBM-bound ones of the next.
        self.n_lanes = max(1, n_lanes)
        self.lanes = [torch.cuda.Stream(device=self.device) for _ in range(self.n_lanes)] if self.n_lanes > 1 else []
        n_ws = max(1, self.n_lanes)
        self.ws_score = [self._ws(xkv.workspace_bytes(xkv.OP_SCORE, self.dims, self.max_seqlen, self.T))
                         for _ in range(n_ws)]
        self.ws_select = [self._ws(xkv.workspace_bytes(xkv.OP_SELECT_COMPACT, self.dims, self.max_seqlen, self.T))
                          for _ in range(n_ws)]
        self._lanes_busy = False
        self.ws_prefill = None

        # ragged paged cache: a pool large enough for any split of the global budget
        per_layer_cap = min(max_budget if max_budget else self.max_prefix, self.max_prefix)
        self.max_cache_len = per_layer_cap + window + max_new_tokens
        self.max_pages_per_seq = max(1, math.ceil(self.max_cache_len / page_size))
        n_units = self.n_solver_units
        if total_budget is None:
            total_budget = n_units * per_layer_cap
        total_budget = min(total_budget, n_units * per_layer_cap)
        # caches per layer and the KV heads one page holds: B caches of Hkv heads, or B*Hkv caches of one head
        self.n_caches = self.B * (n_kv_heads if self.head_level else 1)
        page_heads = 1 if self.head_level else n_kv_heads
        n_pages = 0
        for P, t in zip(self.prefix, lengths):
            rows = min(total_budget, n_units * P) + n_units * (min(window, t) + max_new_tokens + page_size)
            n_pages += math.ceil(rows / page_size)
        self.n_pages = max(n_pages, 1)
        bf16 = dict(dtype=torch.bfloat16, device=self.device)
        page_dtype = torch.bfloat16 if kv_format == xkv.KV_BF16 else torch.uint8
        self.k_pages = torch.zeros(self.n_pages, page_heads, page_size, head_dim, dtype=page_dtype, device=self.device)
        self.v_pages = torch.zeros(self.n_pages, page_heads, page_size, head_dim, dtype=page_dtype, device=self.device)
        self.k_scales = self.v_scales = None
        if kv_format != xkv.KV_BF16:
            n_scales = page_size if kv_format == xkv.KV_INT8 else page_size // xkv.SCALE_BLOCK
            self.k_scales = torch.zeros(self.n_pages, page_heads, n_scales, **f32)
            self.v_scales = torch.zeros(self.n_pages, page_heads, n_scales, **f32)
        self.block_table = torch.zeros(n_layers, self.n_caches, self.max_pages_per_seq, dtype=torch.int32,
                                       device=self.device)
        self.seq_lens = torch.zeros(n_layers, self.n_caches, dtype=torch.int32, device=self.device)
        self.cache = xkv.Cache(self.k_pages.data_ptr(), self.v_pages.data_ptr(), self.block_table.data_ptr(),
                               self.seq_lens.data_ptr(), n_layers, page_size, self.max_pages_per_seq,
                               self.n_pages, None if self.k_scales is None else self.k_scales.data_ptr(),
                               None if self.v_scales is None else self.v_scales.data_ptr(), kv_format, 0)
        # decode sees the head-level caches as B*Hkv sequences of one KV head with G query heads each
        self.dec_dims = self.dims if not self.head_level else xkv.Dims(
            self.n_caches, self.G, 1, head_dim, window, pool_kernel, pool_mode, scale, head_dim, head_dim)
        self.ws_plan = self.ws_store = None
        if self.pages_on_demand:
            self.pages_used = torch.zeros(1, dtype=torch.int32, device=self.device)
            self.one_each = torch.ones(self.n_caches, dtype=torch.int32, device=self.device)   # a step's new rows
            self.ws_plan = self._ws(xkv.workspace_bytes(xkv.OP_PLAN_APPEND, self.dec_dims, n_layers=n_layers))
            self.ws_store = self._ws(xkv.workspace_bytes(xkv.OP_STORE_ROWS, self.dec_dims))
        self.chunk_rows = decode_chunk_rows
        self.ws_decode = self._ws(xkv.workspace_bytes(xkv.OP_DECODE_ATTN, self.dec_dims, n_layers=n_layers,
                                                      max_cache_len=self.max_pages_per_seq * page_size,
                                                      chunk_rows=decode_chunk_rows))
        self.out = torch.empty(n_layers, self.B, n_q_heads, head_dim, **bf16)
        self.lse = torch.empty(n_layers, self.B, n_q_heads, **f32)
        self.budgets: np.ndarray | None = None
        self.last_solver_ms: float | None = None      # host time of the last xkv_alloc_budgets call
        self.r_avg: float | None = None

    def _ws(self, nbytes: int) -> torch.Tensor:
        return torch.zeros(nbytes, dtype=torch.uint8, device=self.device)   # status word reads OK before first use

    def _to_device(self, a: np.ndarray, dtype=np.int32) -> torch.Tensor:
        """Host integers on the device without waiting for it, by a staging buffer of their own, which no later call
        overwrites while the copy is still to come."""
        a = np.ascontiguousarray(a, dtype=dtype)
        return torch.from_numpy(a).pin_memory().to(self.device, non_blocking=True)

    # ------------------------------------------------------------------ prefill
    def _lane(self, layer: int, *tensors):
        """(stream, workspace index) of a layer; the side stream first waits for what the caller's stream holds,
        and the caller's tensors are marked as in use on it (they may be temporaries)."""
        if not self.lanes:
            return torch.cuda.current_stream(), 0
        i = layer % self.n_lanes
        self.lanes[i].wait_stream(torch.cuda.current_stream())
        for t in tensors:
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(self.lanes[i])
        self._lanes_busy = True
        return self.lanes[i], i

    def join(self) -> None:
        """The caller's stream waits for the layers queued on the side streams."""
        if self._lanes_busy:
            cur = torch.cuda.current_stream()
            for s in self.lanes:
                cur.wait_stream(s)
            self._lanes_busy = False

    def score_layer(self, layer: int, q_win: torch.Tensor, k: torch.Tensor, want_curves: bool = True,
                    mass: torch.Tensor | None = None, lse: torch.Tensor | None = None) -> None:
        """lse: fp32 [Hq, T] row normalisers of the layer's prefill attention (prefill_attention's second result);
        with them the scores take one pass over the keys instead of two."""
        stream, i = self._lane(layer, q_win, k, mass, lse)
        srt = self.sorted[layer] if want_curves else None
        gains = self.gains[layer] if want_curves else None
        if lse is None:
            xkv.score(self.dims, q_win, k, self.cu, self.T, self.max_seqlen, self.scores[layer], srt, gains, mass,
                      self.curve_len, self.ws_score[i], stream=stream)
        else:
            xkv.score_lse(self.dims, q_win, k, self.cu, self.T, self.max_seqlen, lse, self.scores[layer], srt, gains,
                          mass, self.curve_len, self.ws_score[i], stream=stream)
        if self.head_level and want_curves:
            xkv.head_curves(self.dims, self.scores[layer], self.sorted[layer], self.cu, self.T, self.max_seqlen,
                            self.head_gains[layer], self.curve_len, stream=stream)

    def score_layers(self, q_win: list[torch.Tensor], k: list[torch.Tensor],
                     lse: list[torch.Tensor] | None = None) -> None:
        """score_layer for every layer, with one fork and one join of the side streams for the whole phase (the
        inputs of all layers must be ready on the caller's stream at the call)."""
        cur = torch.cuda.current_stream()
        streams = self.lanes if self.lanes else [cur]
        for s in self.lanes:
            s.wait_stream(cur)
        lib, dims, cu = xkv.lib(), ctypes.byref(self.dims), self.cu.data_ptr()
        esz = self._layer_stride * 4
        gsz = self.gains[0].numel() * 4
        for l in range(self.L):
            i = l % len(streams)
            ws = self.ws_score[i]
            if lse is None:
                st = lib.xkv_score(dims, q_win[l].data_ptr(), k[l].data_ptr(), cu, self.T, self.max_seqlen,
                                   self.scores.data_ptr() + l * esz, self.sorted.data_ptr() + l * esz,
                                   self.gains.data_ptr() + l * gsz, None, self.curve_len, ws.data_ptr(), ws.numel(),
                                   streams[i].cuda_stream)
            else:
                st = lib.xkv_score_lse(dims, q_win[l].data_ptr(), k[l].data_ptr(), cu, self.T, self.max_seqlen,
                                       lse[l].data_ptr(), self.scores.data_ptr() + l * esz,
                                       self.sorted.data_ptr() + l * esz, self.gains.data_ptr() + l * gsz, None,
                                       self.curve_len, ws.data_ptr(), ws.numel(), streams[i].cuda_stream)
            if st < 0:
                raise xkv.XkvError(st, "xkv_score")
            if self.head_level:
                xkv.head_curves(self.dims, self.scores[l], self.sorted[l], self.cu, self.T, self.max_seqlen,
                                self.head_gains[l], self.curve_len, stream=streams[i])
        self._lanes_busy = bool(self.lanes)
        self.join()

    def prefill_attention(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor | None = None,
                          lse: torch.Tensor | None = None):
        """Causal attention of one layer's prompt: q [T, Hq, d], k/v [T, Hkv, d] -> (out [T, Hq, d] bf16,
        lse [Hq, T] fp32).  The lse goes to score_layer(..., lse=) of that layer."""
        if out is None:
            out = torch.empty_like(q)
        if lse is None:
            lse = torch.empty(self.Hq, self.T, dtype=torch.float32, device=self.device)
        if self.ws_prefill is None:
            self.ws_prefill = self._ws(xkv.workspace_bytes(xkv.OP_PREFILL_ATTN, self.dims))
        xkv.prefill_attn(self.dims, q, k, v, self.cu, self.T, self.max_seqlen, out, lse, self.ws_prefill)
        return out, lse

    def select_layers(self, budgets, k: list[torch.Tensor], v: list[torch.Tensor]) -> None:
        """select_layer for every layer under one budget per layer ([L]), or per (layer, KV head) ([L, Hkv]) with
        head-level budgets; forked and joined once like score_layers."""
        cur = torch.cuda.current_stream()
        streams = self.lanes if self.lanes else [cur]
        for s in self.lanes:
            s.wait_stream(cur)
        lib, dims, cu, cache = xkv.lib(), ctypes.byref(self.dims), self.cu.data_ptr(), ctypes.byref(self.cache)
        esz = self._layer_stride * 4
        if self.head_level:
            # the same count for every sequence: [L, Hkv] -> [L, B, Hkv]; kept alive until the streams are joined
            b32 = np.ascontiguousarray(np.broadcast_to(np.asarray(budgets, dtype=np.int32).reshape(self.L, 1, self.Hkv),
                                                       (self.L, self.B, self.Hkv)))
            mode, step = xkv.BUDGET_PER_HEAD, 4 * self.B * self.Hkv
        else:
            b32 = np.ascontiguousarray(budgets, dtype=np.int32)
            mode, step = xkv.BUDGET_PER_LAYER, 4
        self._budget_keepalive = b32
        for l in range(self.L):
            i = l % len(streams)
            ws = self.ws_select[i]
            st = lib.xkv_select_compact(dims, l, b32.ctypes.data + step * l, mode, self.scores.data_ptr() + l * esz,
                                        self.sorted.data_ptr() + l * esz, k[l].data_ptr(), v[l].data_ptr(), cu,
                                        self.T, self.max_seqlen, cache, None, 0, ws.data_ptr(), ws.numel(),
                                        streams[i].cuda_stream)
            if st < 0:
                raise xkv.XkvError(st, "xkv_select_compact")
        self._lanes_busy = bool(self.lanes)
        self.join()

    def solve_budgets(self, total: int | None = None, r_target: float = 0.0, n_min: int = 0, n_max: int = 0,
                      per_sequence: bool = False, head_shards: int = 1, exchange=None):
        """Curves device -> host (the one crossing of the prefill), then Algorithm 1 on the host.  For one list per
        batch the curves are averaged over the sequences on the device first, so L x curve_len numbers cross.

        head_shards > 1: this session holds one of that many equal shares of the model's KV heads (one rank of a
        KV-head-sharded run).  The layers' curves are then combined over the shards before the solver -- summed
        (every shard contributes its heads' share of the layer mean), or with head-level budgets gathered, since
        each (layer, KV head) unit lives on one shard -- and every shard solves the same problem; `total` counts
        the whole model.  exchange(tensor) -> tensor does the combining: by default the torch.distributed
        collectives of `replicas`; a test on one GPU passes a function that stands in for the other shards.
        Returns this shard's budgets ([L], or [L, Hkv_local] with head-level budgets)."""
        self.join()
        if per_sequence and (self.head_level or head_shards > 1):
            raise ValueError("per-sequence lists are not combined with head-level budgets or head shards here")
        if per_sequence:
            if self.gains_host is None:
                self.gains_host = torch.empty(self.L, self.B, self.curve_len, dtype=torch.float32, pin_memory=True)
            self.gains_host.copy_(self.gains, non_blocking=True)
            torch.cuda.current_stream().synchronize()
            gains, prefix = self.gains_host.numpy(), np.asarray(self.prefix, dtype=np.int32)
        else:
            from . import replicas
            src = self.head_gains if self.head_level else self.gains        # [units, B, curve_len] either way
            # layer curves: a shard's mean over its heads is 1/head_shards of the layer's mean over all heads
            divisor = self.B * (1 if self.head_level else head_shards)
            xkv.batch_curves(src, self.n_solver_units, self.B, self.curve_len, divisor, self.layer_gains)
            curves = self.layer_gains
            if head_shards > 1:
                if self.head_level:
                    local = curves.view(self.L, self.Hkv, self.curve_len)
                    curves = (exchange or replicas.gather_unit_curves)(local).reshape(-1, self.curve_len)
                else:
                    curves = (exchange or replicas.sum_curves_over_ranks)(curves)
            n_units = curves.shape[0]
            if n_units == self.n_solver_units:
                self.layer_gains_host.copy_(curves, non_blocking=True)
                host = self.layer_gains_host
            else:
                host = torch.empty(n_units, self.curve_len, dtype=torch.float32, pin_memory=True)
                host.copy_(curves, non_blocking=True)
            torch.cuda.current_stream().synchronize()
            gains = host.numpy().reshape(n_units, 1, self.curve_len)
            prefix = np.asarray([self.max_prefix], dtype=np.int32)
        t0 = time.perf_counter()
        budgets, r_avg = xkv.alloc_budgets(gains, prefix, per_sequence=per_sequence,
                                           total=-1 if total is None else total,
                                           r_target=r_target, n_min=n_min, n_max=n_max)
        self.last_solver_ms = 1e3 * (time.perf_counter() - t0)
        if self.head_level:
            budgets = budgets.reshape(self.L, -1)                # one count per (layer, KV head of the whole model)
            if head_shards > 1:
                from . import replicas
                rank = replicas.env_ranks()[0] if exchange is None else getattr(exchange, "rank", 0)
                budgets = np.ascontiguousarray(budgets[:, rank * self.Hkv: (rank + 1) * self.Hkv])
        self.budgets, self.r_avg = budgets, r_avg
        return budgets, r_avg

    def assign_pages(self, budgets) -> None:
        """Hand consecutive pool pages to every (layer, sequence) for its kept rows plus new tokens: the runs are
        computed here (2 x L x B integers), the page table is expanded from them on the device."""
        budgets = np.asarray(budgets)
        prefix = np.asarray(self.prefix)[None, :]
        window = np.minimum(self.W, np.asarray(self.lengths))[None, :]
        if self.head_level:                                  # budgets [L, Hkv] -> one cache per (layer, b, g)
            k_lb = np.broadcast_to(budgets.reshape(self.L, 1, self.Hkv), (self.L, self.B, self.Hkv))
            rows = (np.minimum(k_lb, prefix[:, :, None]) + window[:, :, None]).reshape(self.L, -1)
        else:
            k_lb = budgets.T if budgets.ndim == 2 else np.broadcast_to(budgets[:, None], (self.L, self.B))   # [L, B]
            rows = np.minimum(k_lb, prefix) + window
        if self.pages_on_demand:                             # the kept rows only: tables and lengths from nothing
            n = -(-rows // self.page_size)
            if int(n[n <= self.max_pages_per_seq].sum()) > self.n_pages:   # (longer caches get nothing: select_layer's status)
                raise RuntimeError("page pool too small for these budgets")
            xkv.plan_append(self.cache, self.n_caches, self._to_device(rows), self.n_caches, None, None, self.n_pages, None,
                            self.pages_used, None, 0, self.ws_plan)
            return
        rows = rows + self.max_new
        n = np.minimum(-(-rows // self.page_size), self.max_pages_per_seq).astype(np.int64)               # pages
        start = np.concatenate([[0], np.cumsum(n.ravel())[:-1]]).reshape(self.L, self.n_caches)
        if int(start.ravel()[-1] + n.ravel()[-1]) > self.n_pages:
            raise RuntimeError("page pool too small for these budgets")
        # every (layer, cache): its first page and its number of pages, each from a 16-byte boundary on; expanded on the device
        runs = np.zeros((2, -(-n.size // 4) * 4), dtype=np.int32)
        runs[0, :n.size], runs[1, :n.size] = start.ravel(), n.ravel()
        runs = self._to_device(runs)
        xkv.build_block_table(runs[0], runs[1], self.cache, self.n_caches)

    def select_layer(self, layer: int, budget, k: torch.Tensor, v: torch.Tensor, sel: torch.Tensor | None = None,
                     per_sequence: bool = False) -> None:
        """budget: one count, [B] with per_sequence, or [Hkv] / [B, Hkv] in a head-level session."""
        stream, i = self._lane(layer, k, v, sel)
        if self.head_level:
            budget = np.ascontiguousarray(np.broadcast_to(np.asarray(budget, dtype=np.int32), (self.B, self.Hkv)))
            per_sequence = xkv.BUDGET_PER_HEAD
        xkv.select_compact(self.dims, layer, budget, per_sequence, self.scores[layer], self.sorted[layer], k, v,
                           self.cu, self.T, self.max_seqlen, self.cache, sel,
                           0 if sel is None else sel.shape[-1], self.ws_select[i], stream=stream)

    def prefill(self, q_win: list[torch.Tensor], k: list[torch.Tensor], v: list[torch.Tensor],
                budgets=None, total: int | None = None, n_min: int = 0, n_max: int = 0):
        """Score every layer, split the budget (unless given), evict and compact every layer."""
        self.score_layers(q_win, k)
        if budgets is None:
            budgets, _ = self.solve_budgets(total=total, n_min=n_min, n_max=n_max)
        else:
            self.budgets = np.asarray(budgets, dtype=np.int32)
        self.assign_pages(budgets)
        self.select_layers(budgets, k, v)
        return budgets

    # ------------------------------------------------------------------ generation
    def append(self, k: torch.Tensor, v: torch.Tensor, n_new) -> torch.Tensor:
        """Stores n_new[b] more rows of every sequence in every layer (a further turn of a conversation, a generated
        token): k, v bf16 [L, T, Hkv, d], the sequences' tokens one after the other, T = sum(n_new) (host integers).
        Needs pages_on_demand.  Returns the slots, int64 [L, T] ([L, T*Hkv] in a head-level session); a cache that cannot
        grow keeps its length and its tokens get slot -1 (device_status("append"))."""
        if not self.pages_on_demand:
            raise ValueError("append needs a session with pages_on_demand=True")
        n_new = np.asarray(n_new, dtype=np.int32)
        if n_new.shape != (self.B,) or int(n_new.min()) < 0:
            raise ValueError("append: n_new is one count per sequence")
        T = int(n_new.sum())
        self._check_rows(k, v, T)
        counts = n_new
        if self.head_level:                                  # caches (b, g): a sequence's tokens head by head
            counts = np.repeat(n_new, self.Hkv)
            if T:
                first = np.concatenate([[0], np.cumsum(n_new)[:-1]])
                order = np.concatenate([((first[b] + np.arange(n_new[b]))[None, :] * self.Hkv +
                                         np.arange(self.Hkv)[:, None]).ravel() for b in range(self.B)])
                order = self._to_device(order, np.int64)
                k, v = (x.reshape(self.L, T * self.Hkv, self.d)[:, order] for x in (k, v))
        return self._store_new(k, v, self._to_device(counts), int(counts.sum()))

    def _check_rows(self, k, v, T: int) -> None:
        for x in (k, v):
            if not isinstance(x, torch.Tensor) or tuple(x.shape) != (self.L, T, self.Hkv, self.d) \
                    or x.dtype != torch.bfloat16 or x.device != self.k_pages.device:
                raise ValueError(f"new rows are bf16 [{self.L}, {T}, {self.Hkv}, {self.d}] tensors on {self.k_pages.device}")

    def _store_new(self, k: torch.Tensor, v: torch.Tensor, counts: torch.Tensor, n_tokens: int) -> torch.Tensor:
        """counts: dev int32, rows to come of each of a layer's caches; k, v: [L, n_tokens, ..] in that order."""
        self.join()
        slots = torch.empty(self.L, n_tokens, dtype=torch.int64, device=self.device)
        xkv.plan_append(self.cache, self.n_caches, counts, 0, self.seq_lens, None, self.n_pages, self.pages_used,
                        self.pages_used, slots if n_tokens else None, n_tokens, self.ws_plan)
        # the layers' tokens are one list: their rows lie one after the other and so do their slots
        if n_tokens:
            xkv.store_rows(self.dec_dims, self.cache, k.contiguous(), v.contiguous(), slots, self.L * n_tokens,
                           self.ws_store)
        return slots

    def decode(self, q: torch.Tensor, k_new: torch.Tensor | None, v_new: torch.Tensor | None,
               out: torch.Tensor | None = None, lse: torch.Tensor | None = None, layer_begin: int = 0,
               layer_end: int | None = None, chunk_rows: int | None = None) -> torch.Tensor:
        self.join()
        out = self.out if out is None else out
        layer_end = self.L if layer_end is None else layer_end
        if self.pages_on_demand and k_new is not None:
            if (layer_begin, layer_end) != (0, self.L):
                raise ValueError("with pages_on_demand a step plans all layers: append first, then decode layer by layer")
            # one row a cache, head by head in a head-level session: the order in which the rows lie
            self._check_rows(k_new, v_new, self.B)
            self._store_new(k_new, v_new, self.one_each, self.n_caches)
            k_new = v_new = None
        xkv.decode_attn(self.dec_dims, self.cache, layer_begin, layer_end, q, k_new, v_new, out,
                        self.lse if lse is None else lse,
                        self.chunk_rows if chunk_rows is None else chunk_rows, self.ws_decode)
        return out

    def device_status(self, which: str = "decode") -> int:
        """First error any call of that kind recorded since the last check (the status words are sticky and
        reading resets them), XKV_OK otherwise."""
        self.join()
        ws = {"decode": [self.ws_decode], "score": self.ws_score, "select": self.ws_select,
              "prefill": [] if self.ws_prefill is None else [self.ws_prefill],
              "append": [] if self.ws_plan is None else [self.ws_plan, self.ws_store]}[which]
        first = xkv.OK
        for w in ws:
            st = xkv.read_device_status(w)
            if st != xkv.OK and first == xkv.OK:
                first = st
        return first
