"""Serving on a reduced cache, host side: the plain definitions (block-scaled 8-bit floats, page bookkeeping of a step)
pinned by small cases, and what the entry points refuse before anything is launched."""
import ctypes
import itertools

import numpy as np
import pytest

from oracle import xkv_oracle as O
from paper_2412_05896_b200 import build, xkv


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def test_e4m3_grid_is_the_nearest_code():
    codes = np.arange(256)
    vals = O.e4m3_values(codes)
    fin = np.unique(vals[np.isfinite(vals)])
    assert fin.max() == 448.0 and fin[fin > 0].min() == 2.0 ** -9
    assert np.array_equal(O.e4m3_grid(fin), fin)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-460, 460, 2000), rng.normal(0, 1e-2, 2000)])
    got = O.e4m3_grid(x)
    assert np.array_equal(np.abs(got - np.clip(x, -448, 448)), np.abs(fin[:, None] - np.clip(x, -448, 448)).min(0))
    mids = (fin[1:] + fin[:-1]) / 2                       # ties go to the even code: its mantissa's last bit is 0
    back = {v: c for c, v in zip(codes.tolist(), vals.tolist()) if np.isfinite(v) and v != 0}
    back[0.0] = 0
    assert all(back[g] % 2 == 0 for g in O.e4m3_grid(mids).tolist())


@pytest.mark.parametrize("top,want", [(448.0, 1.0), (448.5, 2.0), (0.875, 2.0 ** -9), (0.0, 2.0 ** -100), (1.0, 2.0 ** -8),
                                      (1.7e-40, 2.0 ** -100), (3.3e38, 2.0 ** 120)])
def test_block_scale(top, want):
    assert O.e4m3_block_scale(np.array([[top, -top / 3, np.inf, np.nan]])) == want


def test_block_cache_keeps_codes_when_the_scale_grows():
    c = O.BlockCache(2)
    c.append(np.array([[1.0, 0.5]]))
    assert c.scales == [2.0 ** -8] and np.array_equal(c.values(), [[1.0, 0.5]])
    c.append(np.array([[300.0, 2.0]]))
    assert c.scales == [1.0] and np.array_equal(c.values(), [[1.0, 0.5], [288.0, 2.0]])   # 300 rounds to 288
    c.append(np.ones((14, 2)))
    c.append(np.full((1, 2), 1e-3))                       # a new block starts anew
    assert len(c.scales) == 2 and c.scales[1] == 2.0 ** -18


def test_plan_oracle_against_brute_force():
    for ps, used, new in itertools.product((16, 32), (0, 3), (0, 1, 17)):
        lens = np.array([[0, 15, 16], [31, 1, 40]])
        n_new = np.full((2, 3), new)
        free = list(range(100, 140))
        table = np.full((2, 3, 6), -5)
        t, l, s, u, ok = O.plan_append(n_new, lens, table, ps, free, used)
        assert ok and np.array_equal(l, lens + new)
        took = [int(p) for p in t.ravel() if p >= 100]
        assert took == free[used:u]                       # in order, each once
        for i, j in itertools.product(range(2), range(3)):
            have, need = -(-lens[i, j] // ps), -(-(lens[i, j] + new) // ps)
            assert np.all(t[i, j, :have] == -5) and np.all(t[i, j, need:] == -5)


def _dims(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, window=1, pool_kernel=1, pool_mode=0, scale=0.0,
                kv_stride_token=256, kv_stride_head=128)
    base.update(kw)
    return xkv.Dims(**base)


def _cache(**kw):
    base = dict(k_pages=256, v_pages=512, block_table=768, seq_lens=1024, n_layers=4, page_size=16, max_pages_per_seq=8,
                n_pages=100, k_scales=2048, v_scales=4096, kv_format=xkv.KV_E4M3, reserved=0)
    base.update(kw)
    return xkv.Cache(*base.values())


def test_store_rows_refuses():
    lib = xkv.lib()

    def call(d=None, c=None, k=16, v=16, slots=16, n=4, ws=256, nb=4096):
        return lib.xkv_store_rows(ctypes.byref(d or _dims()), ctypes.byref(c or _cache()), k, v, slots, n, ws, nb, None)

    for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(ws=None), dict(k=24), dict(slots=8), dict(ws=64),
                dict(n=-1), dict(n=1 << 31), dict(c=_cache(page_size=24)), dict(c=_cache(page_size=512)),
                dict(c=_cache(k_scales=None)), dict(c=_cache(v_scales=4)), dict(c=_cache(kv_format=3)),
                dict(c=_cache(k_pages=None)), dict(c=_cache(n_pages=0)), dict(d=_dims(kv_stride_head=124)),
                dict(d=_dims(kv_stride_token=128)), dict(d=_dims(kv_stride_token=260)), dict(d=_dims(n_kv_heads=3))):
        assert call(**bad) == xkv.ERR_INVALID_ARG, bad
    assert call(d=_dims(head_dim=96)) == xkv.ERR_UNSUPPORTED
    assert call(nb=64) == xkv.ERR_WORKSPACE
    assert call(n=0) == xkv.OK                            # nothing to store, nothing launched


def test_plan_append_refuses():
    lib = xkv.lib()

    def call(c=None, batch=3, n_new=16, stride=0, lens=None, free=None, n_free=10, ub=None, ua=None, slots=16, ss=8, ws=256,
             nb=1 << 20):
        return lib.xkv_plan_append(ctypes.byref(c or _cache()), batch, n_new, stride, lens, free, n_free, ub, ua, slots, ss,
                                   ws, nb, None)

    for bad in (dict(n_new=None), dict(n_new=4), dict(lens=4), dict(free=8), dict(ub=4), dict(ua=4), dict(slots=8),
                dict(ws=None), dict(ws=16), dict(batch=0), dict(stride=2), dict(stride=-1), dict(ss=0), dict(ss=1 << 31),
                dict(n_free=-1), dict(c=_cache(page_size=20)), dict(c=_cache(block_table=None)), dict(c=_cache(seq_lens=None)),
                dict(c=_cache(n_layers=0)), dict(c=_cache(max_pages_per_seq=0)), dict(c=_cache(n_pages=0)),
                dict(c=_cache(page_size=256, max_pages_per_seq=1 << 23))):
        assert call(**bad) == xkv.ERR_INVALID_ARG, bad
    assert call(batch=16385) == xkv.ERR_UNSUPPORTED
    assert call(c=_cache(n_layers=70000)) == xkv.ERR_UNSUPPORTED
    assert call(nb=256) == xkv.ERR_WORKSPACE
    assert xkv.workspace_bytes(xkv.OP_PLAN_APPEND, _dims(), n_layers=4) >= 256 + 4 * 2 * 4
    assert lib.xkv_workspace_bytes(xkv.OP_PLAN_APPEND, ctypes.byref(_dims()), 0, 0, 0, 0, 0) == 0
    assert xkv.workspace_bytes(xkv.OP_STORE_ROWS, _dims()) >= 4


def test_decode_refuses_block_scaled_caches_without_scales():
    lib = xkv.lib()
    d = _dims()
    for bad in (_cache(k_scales=None), _cache(v_scales=None), _cache(k_scales=8), _cache(kv_format=9)):
        assert lib.xkv_decode_attn(ctypes.byref(d), ctypes.byref(bad), 0, 1, 16, None, None, 16, None, 0, 256, 1 << 30,
                                   None) == xkv.ERR_INVALID_ARG
    # the allocation-free variant reads 16-bit caches only
    assert lib.xkv_decode_attn_static(ctypes.byref(d), ctypes.byref(_cache()), 0, 1, 16, None, None, 16, None, 64, None,
                                      None) == xkv.ERR_UNSUPPORTED
    # more than eight query heads a KV head
    assert lib.xkv_decode_attn(ctypes.byref(_dims(n_q_heads=18)), ctypes.byref(_cache()), 0, 1, 16, None, None, 16, None, 0,
                               256, 1 << 30, None) == xkv.ERR_UNSUPPORTED
