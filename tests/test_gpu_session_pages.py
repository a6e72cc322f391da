"""A run of the operators together through the session: prefill, eviction, forks that share pages, generation with differential
heads, drafts taken back, sequences freed, the pool compacted and resized.  What every cache holds is followed row by row."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import xkv_oracle as O
from paper_2412_05896_b200 import workloads as WL
from paper_2412_05896_b200 import xkv
from paper_2412_05896_b200.pipeline import XkvSession

from diff_util import DEV, FORMATS, check_causal, check_head, small_weight, weights
from gpu_util import f64, require_lib

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Run:
    def __init__(self, fmt, head_level=False, d=64, **kw):
        require_lib()
        self.fmt, self.head_level = fmt, head_level
        w = replace(WL.CONFIGS["mistral_7b_gqa"], n_layers=3, n_q_heads=8, n_kv_heads=2, head_dim=d, batch=4, prompt=(40, 300),
                    window=16, avg_budget=60, n_min=8, n_max=256)
        self.w, self.lengths = w, WL.prompt_lengths(w)
        self.L, self.B, self.H, self.Hq, self.d = w.n_layers, w.batch, w.n_kv_heads, w.n_q_heads, d
        self.tens = [WL.layer_tensors(w, l, DEV, self.lengths, stress=True) for l in range(self.L)]
        self.s = XkvSession(self.L, self.Hq, self.H, d, w.window, w.pool_kernel, self.lengths, max_new_tokens=60,
                            max_budget=w.n_max, curve_len=w.n_max, device=DEV, head_level=head_level, kv_format=FORMATS[fmt],
                            pages_on_demand=True, **kw)
        self.gen = torch.Generator().manual_seed(3)
        self.lam, self.gain = (t.to(DEV) for t in weights(self.L, self.Hq, d, 5))
        self.budgets = np.array([60, 100, 81])
        if head_level:
            self.budgets = np.array([[60, 33], [100, 7], [81, 20]])
        self.s.prefill(*([t[i] for t in self.tens] for i in range(3)), budgets=self.budgets)
        self.rows = self.held()
        self.status()

    def status(self):
        for which in ("score", "select", "append", "decode", "pages"):
            assert self.s.device_status(which) == xkv.OK, which

    def held(self):
        """{(l, b, g, x)}: the rows of a cache as values in 64 bits."""
        s, res, self.scales = self.s, {}, {}
        lens, table = s.seq_lens.cpu().numpy(), s.block_table.cpu().numpy()
        pages = [x.float().cpu().numpy() if self.fmt == "bf16" else x.cpu().numpy() for x in (s.k_pages, s.v_pages)]
        scales = [None if x is None else x.cpu().numpy().astype(np.float64) for x in (s.k_scales, s.v_scales)]
        for l in range(self.L):
            for b in range(self.B):
                for g in range(self.H):
                    ci, hp = (b * self.H + g, 0) if self.head_level else (b, g)
                    at = np.arange(lens[l, ci])
                    pg, off = table[l, ci][at // s.page_size], at % s.page_size
                    for i, x in enumerate("kv"):
                        r = pages[i][pg, hp, off]
                        if self.fmt == "int8":
                            r = (r.astype(np.float64) - 128) * scales[i][pg, hp, off][:, None]
                        elif self.fmt == "e4m3":
                            self.scales[l, b, g, x] = scales[i][pg, hp, off // 16][:, None]
                            r = O.e4m3_values(r) * self.scales[l, b, g, x]
                        res[l, b, g, x] = r.astype(np.float64)
        return res

    def expect(self, rows, new=None):
        """The caches hold `rows`, new {(l, b, g, x): rows} behind them; the page lists agree with the tables."""
        now = self.held()
        for key, r in rows.items():
            got, n = now[key], len(r)
            more = None if new is None else new.get(key)
            assert len(got) == n + (0 if more is None else len(more)), key
            more = np.zeros((0, self.d)) if more is None else more
            # stored anew: bf16 exact; int8 half a step of the row's scale; e4m3 half a step, 2^-4 relative or 2^-10 of the
            # block's scale (its least step is 2^-9 of that) -- also for the open block's earlier rows, whose scale may grow
            whole = n // 16 * 16 if self.fmt == "e4m3" and len(more) else n
            assert np.array_equal(got[:whole], r[:whole]), key
            was = np.concatenate([r[whole:], more])
            if self.fmt == "bf16":
                bound = 0.0 * was
            elif self.fmt == "int8":
                bound = np.abs(was).max(1, keepdims=True) / 254 * (1 + 2.0 ** -10) if len(was) else 0.0 * was
            else:
                bound = 2.0 ** -4 * np.abs(was) + 2.0 ** -10 * self.scales[key][whole:]
            assert np.all(np.abs(got[whole:] - was) <= bound), key
        self.rows = now
        s = self.s
        if s.free_pages is None:
            return
        lens, table, shares, free = (x.cpu().numpy() for x in (s.seq_lens, s.block_table, s.shares, s.free_pages))
        held = np.concatenate([table[l, c, :-(-lens[l, c] // s.page_size)] for l in range(self.L) for c in range(s.n_caches)])
        count = np.bincount(held.astype(np.int64), minlength=s.n_pages)
        used = int(s.pages_used.item())
        assert np.array_equal(shares, np.maximum(count - 1, 0)) and used == int((count > 0).sum())
        assert sorted(free[used:].tolist()) == np.flatnonzero(count == 0).tolist()

    def forked(self, parent, keep=None):
        rows = {}
        for (l, b, g, x) in self.rows:
            r = self.rows[l, parent[b], g, x] if parent[b] >= 0 else np.zeros((0, self.d))
            k = -1 if keep is None else int(np.asarray(keep)[l, b] if np.ndim(keep) == 2 else keep[b])
            rows[l, b, g, x] = r if k < 0 else r[:k]
        return rows

    def new_rows(self, n_new):
        T = int(sum(n_new))
        k, v = (torch.randn(self.L, T, self.H, self.d, generator=self.gen).to(torch.bfloat16).to(DEV) for _ in "kv")
        at, new = 0, {}
        for b, n in enumerate(n_new):
            for l in range(self.L):
                for g in range(self.H):
                    new[l, b, g, "k"], new[l, b, g, "v"] = f64(k[l, at:at + n, g]), f64(v[l, at:at + n, g])
            at += n
        return k, v, new

    def step(self, live):
        """One step of generation; every head's output against the definition over what its cache holds."""
        k, v, new = self.new_rows([1] * self.B)
        q = torch.randn(self.L, self.B, self.Hq, self.d, generator=self.gen).to(torch.bfloat16).to(DEV)
        before = self.rows
        if self.head_level:
            out = self.s.decode(q, k, v)
        else:
            out = self.s.diff_decode(q, k, v, self.lam, self.gain, EPS)
        torch.cuda.synchronize()
        self.status()
        self.expect(before, {key: r for key, r in new.items() if live[key[1]]})
        q64, o64 = f64(q), f64(out)
        lse = None if self.head_level else self.s.diff_lse.double().cpu().numpy()
        for l in range(self.L):
            for b in range(self.B):
                for h in range(self.Hq):
                    K, V = (self.rows[l, b, h // (self.Hq // self.H), x] for x in "kv")
                    if not self.head_level:
                        check_head(o64[l, b, h], lse[l, b, h], q64[l, b, h], K, V, float(self.lam[l, h]),
                                   self.gain[l].double().cpu().numpy(), EPS, None, f"layer {l} sequence {b} head {h}",
                                   small_weight(self.fmt, len(K)))
                    elif len(K):
                        z, _ = O.decode_attention(q64[l, b, h], K, V)
                        assert np.all(np.abs(o64[l, b, h] - z) <= 2e-2 + 1e-2 * np.abs(z)), (l, b, h)
                    else:
                        assert not o64[l, b, h].any()


@pytest.mark.parametrize("fmt,head_level,d", [("bf16", False, 64), ("int8", False, 128), ("e4m3", False, 64), ("bf16", True, 64),
                                              ("e4m3", True, 128)])
def test_a_run_together(fmt, head_level, d):
    r = Run(fmt, head_level, d)
    s = r.s
    if not head_level:                                        # the prompt's attention
        q = torch.randn(s.T, r.Hq, d, generator=r.gen).to(torch.bfloat16).to(DEV)
        k, v = (t.contiguous() for t in r.tens[1][1:3])
        out, lse = s.diff_prefill_attention(q, k, v, r.lam[1], r.gain[1])
        torch.cuda.synchronize()
        assert s.device_status("prefill") == xkv.OK
        lo, hi = int(s.cu_host[1]), int(s.cu_host[2])
        check_causal(f64(out[lo:hi, 5]), lse[5, :, lo:hi].double().cpu().numpy(), f64(q[lo:hi, 5]), f64(k[lo:hi, 1]),
                     f64(v[lo:hi, 1]), float(r.lam[1, 5]), r.gain[1].double().cpu().numpy(), EPS)
    r.step([True] * 4)
    want = r.forked([0, 0, 2, -1])                            # a sample more of the first prompt, the last request is done
    s.fork([0, 0, 2, -1])
    r.expect(want)
    for _ in range(3):
        r.step([True, True, True, False])
    k, v, new = r.new_rows([4, 0, 7, 2])                      # drafts; another request in the free place
    before = r.rows
    s.append(k, v, [4, 0, 7, 2])
    r.expect(before, new)
    want = {(l, b, g, x): t[:len(t) - [2, 0, 7, 1][b]] for (l, b, g, x), t in r.rows.items()}
    s.cut([2, 0, 7, 1])
    r.expect(want)
    r.step([True] * 4)
    parent = [1, 1, 0, 2]                                     # beams, cut to a different length in every layer
    keep = np.array([[30, -1, 17, 3], [0, 48, 64, 1], [15, 16, -1, 33]])
    want = r.forked(parent, keep)
    s.fork(torch.tensor(parent, dtype=torch.int32, device=DEV), torch.tensor(keep, dtype=torch.int32, device=DEV))
    r.expect(want)
    r.step([True] * 4)
    want = r.forked([-1, 1, 2, 3])
    s.fork([-1, 1, 2, 3])
    r.expect(want)
    s.compact()
    r.expect(want)
    used = int(s.pages_used.item())
    assert int(s.block_table.cpu()[r.s.seq_lens.cpu() > 0][:, 0].max()) < used
    with pytest.raises(ValueError):
        s.resize_pool(used - 1)
    r.expect(want)
    s.resize_pool(used + 40)
    assert s.k_pages.shape[0] == used + 40 == s.n_pages
    r.expect(want)
    r.step([False, True, True, True])
    r.status()
    # a batch that begins anew finds the whole pool free again
    s.resize_pool(4000)
    s.prefill(*([t[i] for t in r.tens] for i in range(3)), budgets=r.budgets)
    torch.cuda.synchronize()
    r.rows = r.held()
    r.expect(r.rows)
    r.step([True] * 4)


def test_a_pool_that_ends_is_reported():
    r = Run("bf16")
    s = r.s
    s.compact()
    s.resize_pool(int(s.pages_used.item()) + 1)
    s.fork([0, 0, 0, 0])                                      # copies of open pages: every layer wants three
    lens = s.seq_lens.cpu().numpy()
    whole = lens[:, :1] // 16 * 16
    assert np.all((lens == lens[:, :1]) | (lens == whole))
    assert int((lens[:, 1:] == lens[:, :1]).sum()) == 1 and lens[0, 0] % 16      # the page that was left
    assert s.device_status("pages") == xkv.ERR_CAPACITY
    s.compact()
    assert s.device_status("pages") == xkv.OK


def test_a_captured_step_with_a_fork():
    """A beam's step, fork by a tensor and generation, captured once and replayed, against the same steps one by one."""
    one, two = Run("bf16"), Run("bf16")
    parent = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device=DEV)
    q, k, v = (torch.randn(3, 4, n, 64, generator=one.gen).to(torch.bfloat16).to(DEV) for n in (8, 2, 2))
    for r in (one, two):                                      # workspaces and lists are made by first calls
        r.s.fork(parent)
        r.s.diff_decode(q, k, v, r.lam, r.gain, EPS)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.s.fork(parent)
        out = one.s.diff_decode(q, k, v, one.lam, one.gain, EPS)
    for p in ([0, 0, 1, 3], [3, 2, 1, 0], [1, 1, 1, -1], [0, 2, 2, 2]) * 6:
        parent.copy_(torch.tensor(p, dtype=torch.int32))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=one.gen).to(torch.bfloat16))
        graph.replay()
        two.s.fork(parent)
        want = two.s.diff_decode(q, k, v, two.lam, two.gain, EPS)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(one.s.seq_lens, two.s.seq_lens)
        assert torch.equal(one.s.shares, two.s.shares) and torch.equal(one.s.pages_used, two.s.pages_used)
    parent.copy_(torch.tensor([1, 1, 3, 2], dtype=torch.int32))
    for r in (one, two):                                      # another batch in the same session: the captured step goes on with it
        r.s.prefill(*([t[i] for t in r.tens] for i in range(3)), budgets=r.budgets)
    for _ in range(3):
        graph.replay()
        two.s.fork(parent)
        want = two.s.diff_decode(q, k, v, two.lam, two.gain, EPS)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(one.s.block_table, two.s.block_table)
        assert torch.equal(one.s.shares, two.s.shares) and torch.equal(one.s.pages_used, two.s.pages_used)
    one.status()
    two.status()


def test_a_run_on_another_stream():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        test_a_run_together("int8", False, 64)


def test_two_sessions_at_once():
    """Two sessions on two streams, their steps issued in turn without waiting, against one that runs alone."""
    def play(r, i):
        s = r.s
        q, k, v = (torch.randn(3, 4, n, 64, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).to(DEV) for n in (8, 2, 2))
        if i % 5 == 2:
            s.fork([[0, 0, 2, 3], [3, 1, 1, 0], [2, 2, -1, 1]][i % 3])
        if i % 5 == 4:
            s.cut([i % 3, 1, 0, 2])
        if i % 7 == 6:
            s.compact()
        return s.diff_decode(q, k, v, r.lam, r.gain, EPS).clone()

    alone, *both = (Run("bf16") for _ in range(3))
    want = [play(alone, i) for i in range(40)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    outs = [[], []]
    for i in range(40):
        for r, st, o in zip(both, streams, outs):
            with torch.cuda.stream(st):
                o.append(play(r, i))
    torch.cuda.synchronize()
    for r, o in zip(both, outs):
        assert all(torch.equal(a, b) for a, b in zip(o, want))
        assert torch.equal(r.s.seq_lens, alone.s.seq_lens) and torch.equal(r.s.pages_used, alone.s.pages_used)
        r.status()


def test_a_captured_step_of_some_sequences():
    one, two = Run("int8"), Run("int8")
    q, k, v = (torch.randn(3, 4, n, 64, generator=one.gen).to(torch.bfloat16).to(DEV) for n in (8, 2, 2))
    for r in (one, two):
        r.s.fork([0, -1, 2, 2])
        r.s.diff_decode(q, k, v, r.lam, r.gain, EPS)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one.s.diff_decode(q, k, v, one.lam, one.gain, EPS)
    for _ in range(20):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=one.gen).to(torch.bfloat16))
        graph.replay()
        want = two.s.diff_decode(q, k, v, two.lam, two.gain, EPS)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(one.s.seq_lens, two.s.seq_lens) and not one.s.seq_lens[:, 1].any()
    one.status()
    two.status()
