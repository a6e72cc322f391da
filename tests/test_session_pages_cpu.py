"""What a session checks and lays out on the host before caches are forked, cut, compacted or read by differential heads."""
import numpy as np
import pytest
import torch

from paper_2412_05896_b200 import xkv
from paper_2412_05896_b200.pipeline import XkvSession


def session(monkeypatch, head_level=False, on_demand=True):
    """A session of 2 layers, 3 sequences, 2 KV heads without a device; calls collects what reaches the library."""
    s = XkvSession.__new__(XkvSession)
    s.L, s.B, s.Hkv, s.Hq, s.d, s.page_size, s.n_pages, s.max_pages_per_seq = 2, 3, 2, 4, 64, 16, 20, 5
    s.head_level, s.pages_on_demand, s.device, s.lanes, s._lanes_busy = head_level, on_demand, torch.device("cpu"), [], False
    s.n_caches, s.live, s.chunk_rows = s.B * (s.Hkv if head_level else 1), [True] * 3, 0
    s.k_pages = s.v_pages = torch.zeros(20, 2, 16, 64, dtype=torch.bfloat16)
    s.seq_lens = torch.arange(s.L * s.n_caches, dtype=torch.int32).view(s.L, s.n_caches) * 5
    s._to_device = lambda a, dtype=np.int32: torch.from_numpy(np.ascontiguousarray(a, dtype=dtype))
    s.dims = s.dec_dims = s.cache = s.block_table = s.ws_fork = s.ws_compact = s.ws_diff_decode = s.diff_lse = None
    s.pages_used = torch.zeros(1, dtype=torch.int32)
    s.out = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    s.calls = []
    monkeypatch.setattr(xkv, "workspace_bytes", lambda *a, **k: 256)
    for name in ("fork_caches", "compact_pages", "diff_decode_attn", "plan_append", "store_rows"):
        monkeypatch.setattr(xkv, name, lambda *a, _n=name, **k: s.calls.append((_n, a)))
    return s


def test_parents_and_counts(monkeypatch):
    s = session(monkeypatch)
    s.fork([2, 0, -1], keep=[[1, 2, 3], [-1, 10 ** 12, 0]])
    name, a = s.calls[-1]
    assert name == "fork_caches" and a[2].tolist() == [2, 0, -1] and a[3].tolist() == [[1, 2, 3], [-1, 2 ** 31 - 1, 0]] and a[4] == 3
    assert s.live == [True, True, False] and s.free_pages.tolist() == list(range(20)) and not s.shares.any()
    s.fork([2, 2, 1])                                         # from a freed one: freed as well
    assert s.live == [False, False, True] and s.calls[-1][1][3] is None and s.calls[-1][1][4] == 0
    s.fork(torch.tensor([0, 1, 2], dtype=torch.int32), keep=[4, 5, 6])
    assert s.live == [True] * 3 and s.calls[-1][1][3].tolist() == [4, 5, 6] and s.calls[-1][1][4] == 0
    s.cut([1, 0, 100])
    assert s.calls[-1][1][2].tolist() == [0, 1, 2] and s.calls[-1][1][3].tolist() == [[0, 5, 0], [14, 20, 0]]


def test_head_level_caches(monkeypatch):
    s = session(monkeypatch, head_level=True)
    s.fork([2, -1, 0], keep=[1, -1, 3])
    assert s.calls[-1][1][2].tolist() == [4, 5, -1, -1, 0, 1] and s.calls[-1][1][3].tolist() == [1, 1, -1, -1, 3, 3]
    s.fork([2, 1, 0], keep=[[1, 2, 3], [4, 5, 6]])
    assert s.calls[-1][1][3].tolist() == [[1, 1, 2, 2, 3, 3], [4, 4, 5, 5, 6, 6]] and s.calls[-1][1][4] == 6
    s.cut([0, 3, 0])
    assert s.calls[-1][1][3].tolist() == [[0, 5, 7, 12, 20, 25], [30, 35, 37, 42, 50, 55]]


def test_steps_of_some_sequences(monkeypatch):
    s = session(monkeypatch)
    s.ws_plan = s.ws_store = None
    s.one_each = torch.ones(3, dtype=torch.int32)
    k = torch.arange(2 * 3 * 2 * 64).view(2, 3, 2, 64).to(torch.bfloat16)
    lam = torch.zeros(2, 4)
    s.fork([0, -1, 2])
    s.diff_decode(s.out, k, k, lam)
    plan, store, attend = s.calls[-3:]
    assert [c[0] for c in (plan, store, attend)] == ["plan_append", "store_rows", "diff_decode_attn"]
    assert plan[1][2].tolist() == [1, 0, 1] and plan[1][5] is s.free_pages and torch.equal(store[1][2], k[:, [0, 2]])
    assert attend[1][5] is None                               # the rows are stored
    s.append(k[:, :1], k[:, :1], [0, 1, 0])                   # a request in the free place
    s.diff_decode(s.out, k, k, lam)
    assert s.live == [True] * 3 and s.calls[-3][1][2] is s.one_each


@pytest.mark.parametrize("call", [
    lambda s: s.fork([0, 1]), lambda s: s.fork([0, 1, 3]), lambda s: s.fork([0, 1, -2]), lambda s: s.fork([0.0, 1.0, 2.0]),
    lambda s: s.fork([[0, 1, 2]] * 2), lambda s: s.fork(torch.tensor([0, 1, 2])), lambda s: s.fork([0, 1, 2], keep=[1, 2]),
    lambda s: s.fork([0, 1, 2], keep=[[1, 2, 3]] * 3), lambda s: s.fork([0, 1, 2], keep=[0.5, 1, 2]),
    lambda s: s.cut([1, 2]), lambda s: s.cut([1, 2, -1]), lambda s: s.cut([[1, 2, 3]] * 2),
    lambda s: s.diff_decode(s.out, None, None, torch.zeros(2, 3)),
    lambda s: s.diff_decode(s.out, None, None, torch.zeros(2, 4, dtype=torch.float64)),
    lambda s: s.diff_decode(s.out, None, None, torch.zeros(4, 2).t()),
    lambda s: s.diff_decode(s.out, None, None, torch.zeros(2, 4), torch.ones(64)),
    lambda s: s.diff_decode(s.out, None, None, torch.zeros(2, 4), layer_end=1),
    lambda s: s.diff_decode(s.out, s.out[:, :, :2], s.out[:, :, :2], torch.zeros(1, 4), layer_end=1),
    lambda s: s.diff_prefill_attention(None, None, None, torch.zeros(1, 4)),
])
def test_refusals(monkeypatch, call):
    s = session(monkeypatch)
    with pytest.raises(ValueError):
        call(s)
    assert not s.calls and s.live == [True] * 3


def test_sessions_that_cannot(monkeypatch):
    s = session(monkeypatch, on_demand=False)
    for call in (lambda: s.fork([0, 1, 2]), lambda: s.cut([0, 0, 0]), s.compact, lambda: s.resize_pool(20)):
        with pytest.raises(ValueError, match="pages_on_demand"):
            call()
    s = session(monkeypatch, head_level=True)
    with pytest.raises(ValueError, match="head-level"):
        s.diff_decode(s.out, None, None, torch.zeros(2, 4))
    assert not s.calls
