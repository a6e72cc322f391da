"""Serving on a reduced cache, host side: limits that the entry points refuse and what a session decides on the host."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2412_05896_b200 import build, xkv


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def test_plan_append_refuses_slot_maps_of_2_31_tokens():
    """Token counts of a layer saturate at 2^31 - 1, so a map has to be shorter than that."""
    cache = xkv.Cache(256, 512, 768, 1024, 4, 16, 8, 100)

    def call(stride):
        return xkv.lib().xkv_plan_append(ctypes.byref(cache), 3, 16, 0, None, None, 10, None, None, 16, stride, 256, 0, None)

    assert call(2 ** 31 - 1) == xkv.ERR_INVALID_ARG
    assert call(2 ** 31 - 2) == xkv.ERR_WORKSPACE             # (the next check)


def test_decode_refuses_more_blocks_than_it_can_count():
    """The caches of a call, as long as their tables allow, in blocks of 16 rows: fewer than 2^31."""
    cache = xkv.Cache(256, 512, 768, 1024, 8, 256, 1 << 13, 100, 2048, 4096, xkv.KV_E4M3, 0)      # 2^21 rows a table

    dims = xkv.Dims(64, 32, 32, 128, 1, 1, 0, 0.0, 32 * 128, 128)
    assert xkv.lib().xkv_decode_attn(ctypes.byref(dims), ctypes.byref(cache), 0, 8, 16, None, None, 16, None, 0, 256, 1 << 40,
                                     None) == xkv.ERR_UNSUPPORTED                          # 2^14 caches of 2^17 blocks


def _session(head_level, on_demand, n_pages):
    """A session of 2 layers, 2 sequences, 2 KV heads as assign_pages sees it, without a device."""
    from paper_2412_05896_b200.pipeline import XkvSession
    s = XkvSession.__new__(XkvSession)
    s.L, s.B, s.Hkv, s.W, s.max_new, s.page_size = 2, 2, 2, 4, 8, 16
    s.lengths, s.prefix, s.head_level, s.pages_on_demand = [100, 50], [96, 46], head_level, on_demand
    s.n_caches, s.n_pages, s.max_pages_per_seq = s.B * (s.Hkv if head_level else 1), n_pages, 7
    s._to_device = lambda a, dtype=np.int32: torch.from_numpy(np.ascontiguousarray(a, dtype=dtype))
    s.cache = s.pages_used = s.ws_plan = None
    return s


@pytest.mark.parametrize("head_level", [False, True])
@pytest.mark.parametrize("on_demand", [False, True])
def test_assign_pages_refuses_budgets_beyond_the_pool(monkeypatch, head_level, on_demand):
    """Caches without pages would be compacted through stale table entries into other caches' pages."""
    planned = []
    monkeypatch.setattr(xkv, "plan_append", lambda *a, **k: planned.append(a))
    monkeypatch.setattr(xkv, "build_block_table", lambda *a, **k: planned.append(a))
    budgets = np.array([[60, 20], [9, 44]]) if head_level else np.array([60, 28])
    kept = (np.minimum(budgets[:, None, :], np.array([96, 46])[None, :, None]) + 4).reshape(2, -1) if head_level else (
        np.minimum(budgets[:, None], np.array([[96, 46]])) + 4)
    need = int((-(-(kept + (0 if on_demand else 8)) // 16)).sum())
    _session(head_level, on_demand, need).assign_pages(budgets)
    assert len(planned) == 1
    with pytest.raises(RuntimeError, match="page pool too small"):
        _session(head_level, on_demand, need - 1).assign_pages(budgets)
    assert len(planned) == 1                                  # nothing was planned


def test_assign_pages_on_demand_counts_no_pages_for_caches_beyond_their_table(monkeypatch):
    planned = []
    monkeypatch.setattr(xkv, "plan_append", lambda *a, **k: planned.append(a))
    s = _session(False, True, 4 + 1 + 1)
    s.max_pages_per_seq = 6                                   # 96 rows: the first cache keeps 100 and gets no page
    s.assign_pages(np.array([96, 6]))
    assert len(planned) == 1 and planned[0][2].tolist() == [[100, 50], [10, 10]]
