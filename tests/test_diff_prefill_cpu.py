"""What xkv_diff_prefill_attn refuses, without a device."""
import ctypes
import math

import pytest

from paper_2412_05896_b200 import build, xkv


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


GOOD = dict(q=16, k=32, v=48, lam=4, gain=64, eps=1e-5, cu=80, T=100, longest=60, out=96, lse=112, ws=256, nbytes=4096)


def call(dims=None, **kw):
    a = {**GOOD, **kw}
    d = dims or xkv.Dims(2, 8, 4, 64, 1, 1, 0, 0.0, 256, 64)
    return xkv.lib().xkv_diff_prefill_attn(ctypes.byref(d), a["q"], a["k"], a["v"], a["lam"], a["gain"], a["eps"], a["cu"], a["T"],
                                           a["longest"], a["out"], a["lse"], a["ws"], a["nbytes"], None)


@pytest.mark.parametrize("kw", [
    *({n: None} for n in ("q", "k", "v", "lam", "cu", "out", "ws")),
    *({n: GOOD[n] + 8} for n in ("q", "k", "v", "gain", "cu", "out", "lse", "ws")), {"lam": 6},
    {"eps": -1.0}, {"eps": math.inf}, {"eps": math.nan},
    {"T": 0}, {"T": -1}, {"T": 1 << 31}, {"longest": 0}, {"longest": 101},
])
def test_bad_arguments(kw):
    assert call(**kw) == xkv.ERR_INVALID_ARG


@pytest.mark.parametrize("dims,status", [
    ((0, 8, 4, 64, 1, 1, 0, 0.0, 256, 64), xkv.ERR_INVALID_ARG), ((2, 8, 3, 64, 1, 1, 0, 0.0, 256, 64), xkv.ERR_INVALID_ARG),
    ((2, 8, 4, 64, 1, 1, 0, 0.0, 248, 64), xkv.ERR_INVALID_ARG), ((2, 8, 4, 64, 1, 1, 0, 0.0, 260, 64), xkv.ERR_INVALID_ARG),
    ((2, 8, 4, 64, 1, 1, 0, 0.0, 256, 56), xkv.ERR_INVALID_ARG), ((2, 8, 4, 64, 1, 1, 0, 0.0, 288, 68), xkv.ERR_INVALID_ARG),
    ((2, 8, 4, 96, 1, 1, 0, 0.0, 384, 96), xkv.ERR_UNSUPPORTED),
])
def test_bad_dims(dims, status):
    assert call(xkv.Dims(*dims)) == status


def test_workspace():
    dims = xkv.Dims(2, 8, 4, 64, 1, 1, 0, 0.0, 256, 64)
    need = xkv.workspace_bytes(xkv.OP_DIFF_PREFILL_ATTN, dims)
    assert call(nbytes=need - 1) == xkv.ERR_WORKSPACE
    with pytest.raises(xkv.XkvError):
        xkv.workspace_bytes(xkv.OP_DIFF_PREFILL_ATTN, xkv.Dims(2, 8, 3, 64, 1, 1, 0, 0.0, 256, 64))
