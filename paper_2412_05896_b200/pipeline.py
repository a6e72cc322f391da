"""The call a user makes: one object that owns the device buffers of a batch (torch tensors for
memory and streams only) and drives the four library entry points in order.

    sess = XkvSession(...); sess.prefill(q_win, k, v, total=...); sess.decode(q, k_new, v_new)

Every computation happens inside libxkv.so; this file allocates, copies and calls (and lays out a few counts).
"""
from __future__ import annotations

import ctypes
import math
import time

import numpy as np
import torch

from . import xkv


class XkvSession:
    free_pages = shares = None                               # with pages_on_demand: the list and the counters, in place from the start
    _steps: dict | None = None                               # steps of some sequences, see _step_of_some

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
        self.ws_plan = self.ws_store = self.ws_fork = self.ws_compact = self.ws_copy = None
        self.live = [True] * self.B                          # sequences that take part in a step with new rows
        if self.pages_on_demand:
            self.pages_used = torch.zeros(1, dtype=torch.int32, device=self.device)
            self.one_each = torch.ones(self.n_caches, dtype=torch.int32, device=self.device)   # a step's new rows
            self.ws_plan = self._ws(xkv.workspace_bytes(xkv.OP_PLAN_APPEND, self.dec_dims, n_layers=n_layers))
            self.ws_store = self._ws(xkv.workspace_bytes(xkv.OP_STORE_ROWS, self.dec_dims))
            # (a step that is captured before the first fork hands pages out by the list that the fork changes, and a fork can be
            # captured without one before it)
            self._reset_pages()
            self._page_workspaces()
        self.chunk_rows = decode_chunk_rows
        # one workspace for both kinds of heads, made here: one that is made while a step is captured is zero only once the step is
        # replayed, and a call before that would find whatever lies there
        self.ws_decode = self.ws_diff_decode = self._ws(max(
            xkv.workspace_bytes(op, self.dec_dims, n_layers=n_layers, max_cache_len=self.max_pages_per_seq * page_size,
                                chunk_rows=decode_chunk_rows) for op in (xkv.OP_DECODE_ATTN, xkv.OP_DIFF_DECODE_ATTN)))
        self.out = torch.empty(n_layers, self.B, n_q_heads, head_dim, **bf16)
        self.lse = torch.empty(n_layers, self.B, n_q_heads, **f32)
        self.ws_diff_prefill = self._ws(xkv.workspace_bytes(xkv.OP_DIFF_PREFILL_ATTN, self.dims))
        self.diff_lse = None
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

    def diff_prefill_attention(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lam: torch.Tensor,
                               gain: torch.Tensor | None = None, eps: float = 1e-5, out: torch.Tensor | None = None,
                               lse: torch.Tensor | None = None):
        """prefill_attention of heads that attend by the difference of two softmax maps: rows of q [q1 | q2], of k
        [k1 | k2]; lam fp32 [Hq], gain fp32 [d] (the heads' norm) or None -> (out [T, Hq, d] bf16, lse [Hq, 2, T] fp32).  The lse
        is not for score_layer: there are no scores of differential heads (see diff_decode)."""
        self._check_diff(lam, gain, (self.Hq,), (self.d,))
        if out is None:
            out = torch.empty_like(q)
        if lse is None:
            lse = torch.empty(self.Hq, 2, self.T, dtype=torch.float32, device=self.device)
        xkv.diff_prefill_attn(self.dims, q, k, v, lam, gain, eps, self.cu, self.T, self.max_seqlen, out, lse,
                              self.ws_diff_prefill)
        return out, lse

    def _check_diff(self, lam, gain, heads: tuple, norm: tuple) -> None:
        for x, shape, name in ((lam, heads, "lam"), (gain, norm, "gain")):
            if x is None and name == "gain":
                continue
            if not isinstance(x, torch.Tensor) or tuple(x.shape) != shape or x.dtype != torch.float32 \
                    or x.device != self.k_pages.device or not x.is_contiguous():
                raise ValueError(f"{name} is a contiguous fp32 {list(shape)} tensor on {self.k_pages.device}")

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
            self.live = [True] * self.B
            if self.free_pages is not None:                  # all pages are free again
                self._reset_pages()
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
        if not all(self.live):                               # (an append of 1024 sequences is 0.1 ms shorter on the host for it)
            self.live = [a or n > 0 for a, n in zip(self.live, n_new.tolist())]
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
        xkv.plan_append(self.cache, self.n_caches, counts, 0, self.seq_lens, self.free_pages, self.n_pages, self.pages_used,
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
        k_new, v_new = self._store_step(k_new, v_new, layer_begin, layer_end)
        xkv.decode_attn(self.dec_dims, self.cache, layer_begin, layer_end, q, k_new, v_new, out,
                        self.lse if lse is None else lse,
                        self.chunk_rows if chunk_rows is None else chunk_rows, self.ws_decode)
        return out

    def _store_step(self, k_new, v_new, layer_begin: int, layer_end: int):
        """A step's new rows: stored here with pages_on_demand (those of live sequences), else left to the attention."""
        if not self.pages_on_demand or k_new is None:
            return k_new, v_new
        if (layer_begin, layer_end) != (0, self.L):
            raise ValueError("with pages_on_demand a step plans all layers: append first, then decode layer by layer")
        self._check_rows(k_new, v_new, self.B)
        if all(self.live):
            # one row a cache, head by head in a head-level session: the order in which the rows lie
            self._store_new(k_new, v_new, self.one_each, self.n_caches)
        elif any(self.live):
            rows, counts, n = self._step_of_some()
            self._store_new(k_new[:, rows], v_new[:, rows], counts, n)
        return None, None

    KEPT_STEPS = 64

    def _step_of_some(self):
        """(live sequences, new rows of every cache, their sum) of a step, the first two on the device.  A captured step holds their
        addresses, so those of a set of sequences that was captured stay for good; of others the last KEPT_STEPS sets do."""
        key, captured = tuple(self.live), self._capturing()
        if self._steps is None:
            self._steps = {}
        step = self._steps.pop(key, None)
        if step is None:
            if captured:                                     # (its copy from the host would be part of the graph)
                raise RuntimeError("a step of some sequences can be captured after one of the same sequences has run")
            counts = np.repeat(np.asarray(self.live, dtype=np.int32), self.n_caches // self.B)
            step = [False, self._to_device(np.flatnonzero(self.live), np.int64), self._to_device(counts), int(counts.sum())]
            spare = [k for k, other in self._steps.items() if not other[0]]
            if len(spare) >= self.KEPT_STEPS:
                del self._steps[spare[0]]
        if captured:
            step[0] = True
        elif step[1].is_cuda:                                # (it may be dropped under a step on another stream)
            for t in step[1:3]:
                t.record_stream(torch.cuda.current_stream())
        self._steps[key] = step                              # the last one used at the end
        return step[1:]

    def _capturing(self) -> bool:
        return self.device.type == "cuda" and torch.cuda.is_current_stream_capturing()

    def diff_decode(self, q: torch.Tensor, k_new: torch.Tensor | None, v_new: torch.Tensor | None, lam: torch.Tensor,
                    gain: torch.Tensor | None = None, eps: float = 1e-5, out: torch.Tensor | None = None,
                    lse: torch.Tensor | None = None, layer_begin: int = 0, layer_end: int | None = None,
                    chunk_rows: int | None = None) -> torch.Tensor:
        """decode of heads that attend by the difference of two softmax maps: q rows [q1 | q2], cached K rows [k1 | k2];
        lam fp32 [layers, Hq], gain fp32 [layers, d] (the heads' norm) or None, lse fp32 [layers, B, Hq, 2].
        It reads the caches as they are.  The rows that prefill keeps are chosen by scores of ordinary maps of the whole row,
        softmax(scale * q . k), which a differential head does not have; a budget of a whole prompt keeps every row."""
        if self.head_level:
            raise ValueError("diff_decode: lam is given per head of a layer, head-level caches are read as sequences of their own")
        self.join()
        layer_end = self.L if layer_end is None else layer_end
        n = layer_end - layer_begin
        self._check_diff(lam, gain, (n, self.Hq), (n, self.d))
        out = self.out if out is None else out
        if lse is None and self.diff_lse is None:
            self.diff_lse = torch.empty(self.L, self.B, self.Hq, 2, dtype=torch.float32, device=self.device)
        k_new, v_new = self._store_step(k_new, v_new, layer_begin, layer_end)
        xkv.diff_decode_attn(self.dec_dims, self.cache, layer_begin, layer_end, q, k_new, v_new, lam, gain, eps, out,
                             self.diff_lse if lse is None else lse,
                             self.chunk_rows if chunk_rows is None else chunk_rows, self.ws_diff_decode)
        return out

    # ------------------------------------------------------------------ caches that share pages
    def _reset_pages(self) -> None:
        if self.free_pages is None:
            self.free_pages = torch.empty(self.n_pages, dtype=torch.int32, device=self.device)
            self.shares = torch.empty(self.n_pages, dtype=torch.int32, device=self.device)
        torch.arange(self.n_pages, out=self.free_pages)      # in place: captured steps hold their addresses
        self.shares.zero_()

    def _page_workspaces(self) -> None:
        sizes = dict(max_seqlen=self.max_pages_per_seq, total_tokens=self.n_pages, n_layers=self.L)
        self.ws_fork = self._ws(xkv.workspace_bytes(xkv.OP_FORK_CACHES, self.dec_dims, **sizes))
        self.ws_compact = self._ws(xkv.workspace_bytes(xkv.OP_COMPACT_PAGES, self.dec_dims, **sizes))

    def _per_cache(self, x, name: str, layers: bool) -> torch.Tensor:
        """Host integers or a dev int32 tensor, [B] (or [L, B]), as dev int32 of a layer's caches."""
        if isinstance(x, torch.Tensor):
            if x.dtype != torch.int32 or x.device != self.k_pages.device:
                raise ValueError(f"{name}: host integers or an int32 tensor on {self.k_pages.device}")
        else:
            x = np.asarray(x)
            if x.dtype.kind not in "iu":
                raise ValueError(f"{name}: integers")
        if tuple(x.shape) != (self.B,) and not (layers and tuple(x.shape) == (self.L, self.B)):
            raise ValueError(f"{name}: one count per sequence" + (" or per layer and sequence" if layers else ""))
        x = x if isinstance(x, torch.Tensor) else self._to_device(np.clip(x, -1, 2 ** 31 - 1))
        return x.repeat_interleave(self.Hkv, dim=-1) if self.head_level else x.contiguous()

    def fork(self, parent, keep=None) -> None:
        """Sequence b goes on as sequence parent[b] (samples of one prompt, beams, a request that starts from another's
        cache), sharing its pages; -1 frees it.  keep: rows of a cache that stay, [B] or [L, B], negative: all.  Host
        integers or dev int32 tensors.  A freed sequence takes no part in later steps until it goes on as another one or
        append gives it rows -- where parent is host integers: a tensor is not read here, and then every sequence takes part
        (a freed one begins again with the next step's row).  A captured step keeps the sequences that it was captured with.
        Needs pages_on_demand; device_status("pages")."""
        if not self.pages_on_demand:
            raise ValueError("fork needs a session with pages_on_demand=True")
        live = [True] * self.B
        if not isinstance(parent, torch.Tensor):
            parent = np.asarray(parent)
            if parent.shape == (self.B,) and (int(parent.min()) < -1 or int(parent.max()) >= self.B):
                raise ValueError("fork: a parent is a sequence of the batch, or -1")
            live = [int(a) >= 0 and self.live[int(a)] for a in parent.ravel()]
        par = self._per_cache(parent, "fork: parent", layers=False)
        if self.head_level:
            heads = torch.arange(self.Hkv, dtype=torch.int32, device=self.device).repeat(self.B)
            par = torch.where(par == -1, par, par * self.Hkv + heads)
        kept = None if keep is None else self._per_cache(keep, "fork: keep", layers=True)
        self._fork(par, kept)
        self.live = live

    def cut(self, n_rows) -> None:
        """The last n_rows[b] rows of every cache of sequence b are taken back (drafted tokens that were rejected): host
        integers or a dev int32 tensor [B].  Needs pages_on_demand; device_status("pages")."""
        if not self.pages_on_demand:
            raise ValueError("cut needs a session with pages_on_demand=True")
        if not isinstance(n_rows, torch.Tensor) and np.asarray(n_rows).size and int(np.asarray(n_rows).min()) < 0:
            raise ValueError("cut: counts are not negative")
        drop = self._per_cache(n_rows, "cut", layers=False)
        same = torch.arange(self.n_caches, dtype=torch.int32, device=self.device)
        self.join()
        self._fork(same, (self.seq_lens - drop.clamp(min=0)).clamp(min=0))

    def _fork(self, parent: torch.Tensor, keep: torch.Tensor | None) -> None:
        self.join()
        if self.free_pages is None:
            self._reset_pages()
        stride = 0 if keep is None or keep.dim() == 1 else self.n_caches
        xkv.fork_caches(self.dec_dims, self.cache, parent, keep, stride, self.shares, self.free_pages, self.n_pages,
                        self.pages_used, self.ws_fork)

    def compact(self) -> None:
        """Moves the pages in use to the front of the pool.  Needs pages_on_demand; device_status("pages")."""
        if not self.pages_on_demand:
            raise ValueError("compact needs a session with pages_on_demand=True")
        self.join()
        xkv.compact_pages(self.dec_dims, self.cache, self.block_table, self.shares, self.shares, self.free_pages,
                          self.pages_used, self.ws_compact)

    def resize_pool(self, n_pages: int) -> None:
        """The pages in use in a new pool of n_pages, the old one given up (waits for the device).  Steps captured before it may not
        be replayed any more: they read and write memory that is no longer the session's.  Needs pages_on_demand; ValueError,
        and the pool as it was, when the pages do not fit; an error that device_status("pages") has not reported yet is raised."""
        self.compact()
        used, st = int(self.pages_used.item()), self.device_status("pages")
        if st != xkv.OK:
            raise xkv.XkvError(st, "resize_pool")
        if not max(used, 1) <= n_pages < 2 ** 31:
            raise ValueError(f"resize_pool: {used} pages are in use")
        old, old_cache = (self.k_pages, self.v_pages, self.k_scales, self.v_scales), self.cache
        new = [None if x is None else torch.zeros(n_pages, *x.shape[1:], dtype=x.dtype, device=x.device) for x in old]
        ptrs = [None if x is None else x.data_ptr() for x in new]
        cache = xkv.Cache(ptrs[0], ptrs[1], self.block_table.data_ptr(), self.seq_lens.data_ptr(), self.L, self.page_size,
                          self.max_pages_per_seq, n_pages, ptrs[2], ptrs[3], self.kv_format, 0)
        ids = torch.arange(n_pages, dtype=torch.int32, device=self.device)
        if used:
            if self.ws_copy is None:
                self.ws_copy = self._ws(xkv.workspace_bytes(xkv.OP_COPY_PAGES, self.dec_dims))
            xkv.copy_pages(self.dec_dims, old_cache, ids, cache, ids, used, self.ws_copy)
        self.k_pages, self.v_pages, self.k_scales, self.v_scales = new
        shares = torch.zeros(n_pages, dtype=torch.int32, device=self.device)
        shares[:used] = self.shares[:used]
        for t in (*old, self.free_pages, self.shares, self.ws_fork, self.ws_compact):
            if t is not None:                                # given up while the copy is still to come, on whatever stream
                t.record_stream(torch.cuda.current_stream())
        self.cache, self.n_pages, self.free_pages, self.shares = cache, n_pages, ids, shares
        self._page_workspaces()                              # sized by the pool

    def device_status(self, which: str = "decode") -> int:
        """First error any call of that kind recorded since the last check (the status words are sticky and
        reading resets them), XKV_OK otherwise."""
        self.join()
        some = lambda *ws: [w for w in ws if w is not None]  # noqa: E731
        ws = {"decode": some(self.ws_decode, self.ws_diff_decode), "score": self.ws_score, "select": self.ws_select,
              "prefill": some(self.ws_prefill, self.ws_diff_prefill), "append": some(self.ws_plan, self.ws_store),
              "pages": some(self.ws_fork, self.ws_compact, self.ws_copy)}[which]
        first = xkv.OK
        for w in ws:
            st = xkv.read_device_status(w)
            if st != xkv.OK and first == xkv.OK:
                first = st
        return first
