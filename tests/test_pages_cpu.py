"""Pages copied, shared, given back and moved, host side: the plain definitions pinned by small cases and by what must hold
over random histories, and what the entry points refuse before anything is launched."""
import ctypes

import numpy as np
import pytest

from oracle import xkv_oracle as O
from paper_2412_05896_b200 import build, xkv

from test_serve_cpu import _cache, _dims


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _holders(table, lens, page, n_pages):
    n = np.zeros(n_pages, dtype=int)
    for row, m in zip(np.asarray(table).reshape(-1, np.asarray(table).shape[-1]), np.asarray(lens).ravel()):
        np.add.at(n, row[: -(-int(m) // page)], 1)
    return n


def test_fork_definition_by_hand():
    table = np.array([[[4, 2, -1], [-1, -1, -1], [0, -1, -1]]])
    t, n, s, free, used, copies, ok = O.fork_caches([0, 0, -1], None, [[20, 0, 3]], table, 16, [0] * 6, [0, 2, 4, 5, 1, 3], 3)
    assert ok and n.tolist() == [[20, 20, 0]] and copies == [(2, 5, 4)]
    assert t.tolist() == [[[4, 2, -1], [4, 5, -1], [0, -1, -1]]]
    assert s.tolist() == [0, 0, 0, 0, 1, 0]                # page 4 twice; page 0 came back, page 5 went out
    assert used == 3 and free.tolist() == [0, 2, 4, 0, 1, 3]


def test_fork_definition_keeps_its_counts():
    rng = np.random.default_rng(3)
    L, B, cols, page, n_pages = 2, 5, 4, 16, 90
    table, lens = np.full((L, B, cols), -1), np.zeros((L, B), dtype=int)
    shares, free, used = np.zeros(n_pages, dtype=int), rng.permutation(n_pages), 0
    for _ in range(60):
        new = np.minimum(rng.integers(0, 30, (L, B)), cols * page - lens)
        table, lens, _, used, ok = O.plan_append(new, lens, table, page, free, used)
        assert ok
        parent = rng.integers(-1, B, B)
        keep = rng.integers(-1, cols * page + 1, (L, B)) if rng.random() < 0.7 else None
        was = lens.copy()
        table, lens, shares, free, used, copies, ok = O.fork_caches(parent, keep, lens, table, page, shares, free, used)
        assert ok
        for b in range(B):
            most = was[:, parent[b]] if parent[b] >= 0 else np.zeros(L, dtype=int)
            cut = most if keep is None else np.where(keep[:, b] >= 0, np.minimum(most, keep[:, b]), most)
            assert np.array_equal(lens[:, b], cut)
        held = _holders(table, lens, page, n_pages)
        assert np.array_equal(shares, np.maximum(held - 1, 0))
        assert sorted(free[used:].tolist()) == np.flatnonzero(held == 0).tolist()
        for l in range(L):                                  # nobody else holds a page that rows will be added to
            for b in range(B):
                if lens[l, b] % page:
                    assert held[table[l, b, lens[l, b] // page]] == 1


def test_compact_definition():
    table = np.array([[[7, 3, -1], [7, 0, 5]]])
    t, s, n_live, moves = O.compact_pages(table, [[20, 48]], 16, np.array([0, 0, 0, 0, 0, 0, 0, 1]), 8)
    assert n_live == 4 and moves == {5: 1, 7: 2}
    assert t.tolist() == [[[2, 3, -1], [2, 0, 1]]] and s.tolist() == [0, 0, 1, 0, 0, 0, 0, 0]


def test_fork_caches_refuses():
    lib = xkv.lib()

    def call(d=None, c=None, parent=16, keep=None, stride=0, shares=16, free=16, n_free=10, used=16, ws=256, nb=1 << 30):
        return lib.xkv_fork_caches(ctypes.byref(d or _dims()), ctypes.byref(c or _cache()), parent, keep, stride, shares, free,
                                   n_free, used, ws, nb, None)

    for bad in (dict(parent=None), dict(shares=None), dict(free=None), dict(used=None), dict(ws=None), dict(parent=4),
                dict(keep=8), dict(shares=8), dict(free=4), dict(used=4), dict(ws=64), dict(n_free=-1), dict(stride=-1),
                dict(stride=1), dict(d=_dims(batch=0)), dict(d=_dims(n_kv_heads=3)), dict(c=_cache(page_size=24)),
                dict(c=_cache(k_pages=None)), dict(c=_cache(block_table=None)), dict(c=_cache(seq_lens=4)),
                dict(c=_cache(k_scales=None)), dict(c=_cache(kv_format=7)), dict(c=_cache(n_pages=0)),
                dict(c=_cache(max_pages_per_seq=0))):
        assert call(**bad) == xkv.ERR_INVALID_ARG, bad
    assert call(d=_dims(head_dim=96)) == xkv.ERR_UNSUPPORTED
    assert call(d=_dims(batch=16385)) == xkv.ERR_UNSUPPORTED
    assert call(nb=256) == xkv.ERR_WORKSPACE
    size = lambda **kw: lib.xkv_workspace_bytes(xkv.OP_FORK_CACHES, ctypes.byref(_dims()), kw.get("cols", 8),   # noqa: E731
                                                kw.get("pages", 100), kw.get("layers", 4), 0, 0)
    assert size() >= 256 + 4 * 2 * 8 * 4
    assert size(cols=0) == size(pages=0) == size(layers=0) == size(pages=1 << 31) == 0


def test_compact_pages_refuses():
    lib = xkv.lib()

    def call(d=None, c=None, before=16, sb=16, s=16, free=16, used=16, ws=256, nb=1 << 30):
        return lib.xkv_compact_pages(ctypes.byref(d or _dims()), ctypes.byref(c or _cache()), before, sb, s, free, used, ws, nb,
                                     None)

    for bad in (dict(before=None), dict(used=None), dict(ws=None), dict(sb=None), dict(s=None), dict(before=4), dict(sb=4),
                dict(s=4), dict(free=4), dict(used=4), dict(ws=16), dict(c=_cache(v_pages=None)), dict(c=_cache(page_size=8)),
                dict(d=_dims(batch=-1))):
        assert call(**bad) == xkv.ERR_INVALID_ARG, bad
    assert call(nb=256) == xkv.ERR_WORKSPACE
    assert lib.xkv_workspace_bytes(xkv.OP_COMPACT_PAGES, ctypes.byref(_dims()), 0, 0, 0, 0, 0) == 0


def test_copy_pages_refuses():
    lib = xkv.lib()

    def call(d=None, a=None, b=None, src=16, dst=16, n=4, ws=256, nb=1 << 20):
        return lib.xkv_copy_pages(ctypes.byref(d or _dims()), ctypes.byref(a or _cache()), src, ctypes.byref(b or _cache()), dst,
                                  n, ws, nb, None)

    for bad in (dict(src=None), dict(dst=None), dict(ws=None), dict(src=4), dict(dst=8), dict(ws=16), dict(n=-1), dict(n=1 << 31),
                dict(a=_cache(k_pages=None)), dict(b=_cache(v_pages=4)), dict(b=_cache(page_size=32)), dict(a=_cache(n_pages=0)),
                dict(b=_cache(kv_format=xkv.KV_INT8)), dict(a=_cache(k_scales=None)), dict(d=_dims(n_kv_heads=3))):
        assert call(**bad) == xkv.ERR_INVALID_ARG, bad
    assert call(d=_dims(head_dim=32)) == xkv.ERR_UNSUPPORTED
    assert call(nb=8) == xkv.ERR_WORKSPACE
    assert call(n=0) == xkv.OK                              # nothing to copy, nothing launched


def test_diff_decode_attn_refuses():
    lib = xkv.lib()

    def call(d=None, c=None, l0=0, l1=2, q=16, kn=None, vn=None, lam=16, gain=16, eps=1e-5, out=16, lse=16, chunk=0, ws=256,
             nb=1 << 32):
        return lib.xkv_diff_decode_attn(ctypes.byref(d or _dims()), ctypes.byref(c or _cache()), l0, l1, q, kn, vn, lam, gain,
                                        eps, out, lse, chunk, ws, nb, None)

    for bad in (dict(q=None), dict(out=None), dict(lam=None), dict(ws=None), dict(q=8), dict(lam=2), dict(gain=8), dict(lse=4),
                dict(out=2), dict(ws=16), dict(kn=16), dict(vn=16), dict(kn=16, vn=8), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(l0=-1), dict(l1=0), dict(l1=5), dict(chunk=32), dict(chunk=-64),
                dict(c=_cache(k_scales=None)), dict(c=_cache(page_size=40)), dict(d=_dims(n_kv_heads=3)), dict(d=_dims(scale=-1.0))):
        assert call(**bad) == xkv.ERR_INVALID_ARG, bad
    assert call(d=_dims(head_dim=96)) == xkv.ERR_UNSUPPORTED
    assert call(d=_dims(n_q_heads=18)) == xkv.ERR_UNSUPPORTED          # nine heads a KV head
    assert call(nb=256) == xkv.ERR_WORKSPACE
    one = xkv.workspace_bytes(xkv.OP_DECODE_ATTN, _dims(), n_layers=2, max_cache_len=1024)
    two = xkv.workspace_bytes(xkv.OP_DIFF_DECODE_ATTN, _dims(), n_layers=2, max_cache_len=1024)
    assert two > one                                                   # partial results of both maps
