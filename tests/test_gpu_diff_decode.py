"""Differential attention of single tokens over paged caches of every format, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2412_05896_b200 import xkv

from diff_util import DEV, RowCache, check_head, small_weight, weights
from gpu_util import f64, require_lib

pytestmark = pytest.mark.gpu
EPS = 1e-5


def attend(c, Hq, q, lam, gain, k_new=None, v_new=None, l0=0, l1=None, chunk=0, ws=None, scale=0.0, lse=True, eps=EPS):
    l1 = c.L if l1 is None else l1
    dims = xkv.Dims(c.B, Hq, c.H, c.d, 1, 1, 0, scale, c.H * c.d, c.d)
    if ws is None:
        ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DIFF_DECODE_ATTN, dims, n_layers=l1 - l0, max_cache_len=c.cols * c.page,
                                             chunk_rows=chunk), dtype=torch.uint8, device=DEV)
    out = torch.full((l1 - l0, c.B, Hq, c.d), float("nan"), dtype=torch.bfloat16, device=DEV)
    sums = torch.full((l1 - l0, c.B, Hq, 2), float("nan"), device=DEV) if lse else None
    xkv.diff_decode_attn(dims, c.handle(), l0, l1, q, k_new, v_new, lam, gain, eps, out, sums, chunk, ws)
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) == xkv.OK
    return out, sums


def check(c, Hq, q, lam, gain, out, sums, l0=0, every=1, eps=EPS, scale=None):
    G = Hq // c.H
    q64, o64, lam64 = f64(q), f64(out), lam.double().cpu().numpy()
    s64 = None if sums is None else sums.double().cpu().numpy()
    g64 = None if gain is None else gain.double().cpu().numpy()
    for i in range(q.shape[0]):
        for b in range(0, c.B, every):
            for h in range(Hq):
                K, V = c.rows(l0 + i, b, h // G)
                check_head(o64[i, b, h], None if s64 is None else s64[i, b, h], q64[i, b, h], K, V, lam64[i, h],
                           None if g64 is None else g64[i], eps, scale, f"layer {i} sequence {b} head {h}",
                           small_weight(c.fmt, len(K)))


def queries(L, B, Hq, d, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(L, B, Hq, 2, d // 2, generator=g) * torch.exp(torch.rand(L, B, Hq, 2, 1, generator=g) * 1.5 - 0.5)
    return x.reshape(L, B, Hq, d).to(torch.bfloat16).to(DEV)


CASES = [  # L, B, KV heads, group, d, page, lengths
    (1, 1, 1, 1, 64, 16, [1]),
    (2, 3, 2, 1, 128, 16, [[17, 0, 33], [64, 1, 16]]),
    (2, 2, 4, 2, 64, 32, [[300, 129], [15, 700]]),
    (1, 3, 2, 3, 128, 48, [[1000, 3, 127]]),
    (3, 2, 1, 4, 128, 16, [[257, 2], [0, 0], [511, 513]]),
    (1, 2, 2, 5, 64, 64, [[400, 31]]),
    (1, 2, 1, 6, 128, 16, [[40, 1030]]),
    (1, 2, 2, 7, 128, 256, [[90, 777]]),
    (2, 1, 1, 8, 64, 128, [[2100], [5]]),
]


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("L,B,H,G,d,page,lens", CASES)
@pytest.mark.parametrize("norm,chunk", [(True, 0), (True, 64), (False, 0)])
def test_against_definition(fmt, L, B, H, G, d, page, lens, norm, chunk):
    c = RowCache(fmt, L, B, H, d, lens, page, seed=L + G)
    lam, gain = weights(L, H * G, d, 7, norm)
    q = queries(L, B, H * G, d, 11)
    lam, gain = lam.to(DEV), None if gain is None else gain.to(DEV)
    out, sums = attend(c, H * G, q, lam, gain, chunk=chunk)
    check(c, H * G, q, lam, gain, out, sums)
    again, _ = attend(c, H * G, q, lam, gain, lse=False, chunk=chunk)
    assert torch.equal(out, again)


@pytest.mark.parametrize("fmt,chunk", [("bf16", 64), ("bf16", 128), ("int8", 64), ("e4m3", 64), ("e4m3", 0)])
@pytest.mark.parametrize("G", [1, 4, 6])
def test_cut_caches_are_joined(fmt, chunk, G):
    d = 128
    c = RowCache(fmt, 1, 2, 2, d, [[5000, 261]], 32, seed=3)
    lam, gain = (t.to(DEV) for t in weights(1, 2 * G, d, 5))
    q = queries(1, 2, 2 * G, d, 6)
    out, sums = attend(c, 2 * G, q, lam, gain, chunk=chunk)
    check(c, 2 * G, q, lam, gain, out, sums)


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("G,chunk", [(2, 0), (8, 0), (2, 256), (8, 64)])
def test_new_rows_are_appended_first(fmt, G, chunk):
    """As xkv_decode_attn appends: the same pages, scales and lengths behind it, and the new row takes part."""
    L, B, H, d, page = 2, 4, 2, 64, 16
    lens = [[0, 15, 16, 31], [100, 1, 47, 64]]
    c, twin = (RowCache(fmt, L, B, H, d, lens, page, extra=2, seed=9) for _ in range(2))
    g = torch.Generator().manual_seed(1)
    lam, gain = (t.to(DEV) for t in weights(L, H * G, d, 5))
    q, q1 = queries(L, B, H * G, d, 6), torch.zeros(L, B, H, d, dtype=torch.bfloat16, device=DEV)
    dims = xkv.Dims(B, H, H, d, 1, 1, 0, 0.0, H * d, d)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DECODE_ATTN, dims, n_layers=L, max_cache_len=c.cols * page), dtype=torch.uint8,
                     device=DEV)
    for _ in range(2):
        kn, vn = (torch.randn(L, B, H, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
        out, sums = attend(c, H * G, q, lam, gain, kn, vn, chunk=chunk)
        xkv.decode_attn(dims, twin.handle(), 0, L, q1, kn, vn, torch.empty_like(q1), None, 0, ws)
        torch.cuda.synchronize()
        assert torch.equal(c.d_lens, twin.d_lens)
        for a, b in zip(c.pages + c.scales, twin.pages + twin.scales):
            if a is not None:
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        after, _ = attend(c, H * G, q, lam, gain, chunk=chunk)           # the rows are in the pages now: the same values
        assert torch.equal(after, out)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_some_layers_scale_and_many_units(fmt):
    L, B, H, G, d, page = 5, 500, 1, 2, 64, 16              # more units than the attention plans by itself
    rng = np.random.default_rng(0)
    c = RowCache(fmt, L, B, H, d, rng.integers(0, 40, (L, B)), page, seed=2)
    lam, gain = (t.to(DEV) for t in weights(L, G, d, 5))
    q = queries(L, B, G, d, 6)
    out, sums = attend(c, G, q, lam, gain, scale=0.3)
    check(c, G, q, lam, gain, out, sums, every=17, scale=float(np.float32(0.3)))
    args = q[2:4].contiguous(), lam[2:4].contiguous(), gain[2:4].contiguous()
    part, ps = attend(c, G, *args, l0=2, l1=4, scale=0.3)              # (fewer caches: not the same kernel for every format)
    check(c, G, *args, part, ps, l0=2, every=17, scale=float(np.float32(0.3)))
    out, sums = attend(c, G, q, lam, gain, scale=0.3, chunk=64)        # with chunks given, one kernel serves both
    part, ps = attend(c, G, *args, l0=2, l1=4, scale=0.3, chunk=64)
    assert torch.equal(part, out[2:4]) and torch.equal(ps, sums[2:4])


def test_one_map_is_ordinary_attention():
    """lambda = 0 leaves the first map: ordinary attention of queries whose second half is zero."""
    c = RowCache("bf16", 2, 3, 2, 128, [[700, 5, 0], [64, 129, 300]], 16, seed=4)
    q = queries(2, 3, 8, 128, 3)
    lam = torch.zeros(2, 8, device=DEV)
    out, sums = attend(c, 8, q, lam, None)
    half = q.clone()
    half[..., 64:] = 0
    dims = xkv.Dims(3, 8, 2, 128, 1, 1, 0, 0.125, 256, 128)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DECODE_ATTN, dims, n_layers=2, max_cache_len=c.cols * 16), dtype=torch.uint8,
                     device=DEV)
    want, ws_lse = torch.empty_like(out), torch.empty(2, 3, 8, device=DEV)
    xkv.decode_attn(dims, c.handle(), 0, 2, half, None, None, want, ws_lse, 0, ws)
    torch.cuda.synchronize()
    # both round weights and output once: twice the bound of one
    assert float((out.float() - want.float()).abs().max()) <= 4 * 2.0 ** -8 * float(want.float().abs().max())
    fin = torch.isfinite(ws_lse)
    assert torch.equal(fin, torch.isfinite(sums[..., 0])) and torch.allclose(sums[..., 0][fin], ws_lse[fin], atol=2e-5)


def test_equal_maps_cancel_to_zero_and_stay_finite():
    """q1 = q2, k1 = k2 and lambda = 1: y is zero up to roundings and its norm must not blow up to NaN; a cache of one row is
    exactly zero."""
    require_lib()
    c = RowCache("bf16", 1, 2, 1, 64, [[1, 50]], 16, seed=4)
    c.pages[0][..., 32:] = c.pages[0][..., :32]
    q = queries(1, 2, 2, 64, 3)
    q[..., 32:] = q[..., :32]
    lam, gain = torch.ones(1, 2, device=DEV), torch.ones(1, 64, device=DEV)
    for eps in (0.0, EPS):
        out, sums = attend(c, 2, q, lam, gain, eps=eps)
        assert torch.isfinite(out.float()).all() and float(out[0, 0].abs().max()) == 0.0
        assert torch.equal(sums[..., 0], sums[..., 1])


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_captured_and_replayed(fmt):
    L, B, H, G, d, page = 2, 3, 2, 4, 128, 16
    c = RowCache(fmt, L, B, H, d, [[300, 1, 64], [47, 2000, 9]], page, seed=8)
    lam, gain = (t.to(DEV) for t in weights(L, H * G, d, 5))
    q = queries(L, B, H * G, d, 6)
    want, want_lse = attend(c, H * G, q, lam, gain)
    dims = xkv.Dims(B, H * G, H, d, 1, 1, 0, 0.0, H * d, d)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DIFF_DECODE_ATTN, dims, n_layers=L, max_cache_len=c.cols * page),
                     dtype=torch.uint8, device=DEV)
    out, sums = torch.zeros_like(want), torch.zeros_like(want_lse)
    handle = c.handle()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xkv.diff_decode_attn(dims, handle, 0, L, q, None, None, lam, gain, EPS, out, sums, 0, ws)
    for _ in range(30):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(sums, want_lse)
    assert xkv.read_device_status(ws) == xkv.OK


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_one_workspace_for_small_and_large_calls(fmt):
    """Calls that take the kernel for few rows and the streaming one in turn, layer by layer and all at once, share a workspace."""
    L, B, H, G, d, page = 3, 1, 2, 3, 64, 16
    small = RowCache(fmt, L, B, H, d, [[300], [1000], [129]], page, seed=1)
    large = RowCache(fmt, L, 40, H, d, np.random.default_rng(1).integers(1, 900, (L, 40)), page, seed=2)
    lam, gain = (t.to(DEV) for t in weights(L, H * G, d, 5))
    qs, ql = queries(L, B, H * G, d, 6), queries(L, 40, H * G, d, 7)
    dims = xkv.Dims(40, H * G, H, d, 1, 1, 0, 0.0, H * d, d)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DIFF_DECODE_ATTN, dims, n_layers=L, max_cache_len=1024), dtype=torch.uint8,
                     device=DEV)
    want_s, want_l = attend(small, H * G, qs, lam, gain), attend(large, H * G, ql, lam, gain)
    check(small, H * G, qs, lam, gain, *want_s)
    for _ in range(5):
        got = attend(small, H * G, qs, lam, gain, ws=ws)
        assert torch.equal(got[0], want_s[0]) and torch.equal(got[1], want_s[1])
        got = attend(large, H * G, ql, lam, gain, ws=ws)
        assert torch.equal(got[0], want_l[0]) and torch.equal(got[1], want_l[1])
        for l in range(L):
            got = attend(small, H * G, qs[l:l + 1].contiguous(), lam[l:l + 1].contiguous(), gain[l:l + 1].contiguous(), l0=l,
                         l1=l + 1, ws=ws)
            assert torch.equal(got[0][0], want_s[0][l])


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
@pytest.mark.parametrize("L,B,H,G,d,page,longest", [
    (1, 1, 1, 4, 128, 64, 20000),       # one long cache, cut up
    (1, 3, 8, 4, 64, 16, 900),          # few caches in chunks, tickets of the workspace's head
    (1, 8, 8, 2, 128, 32, 1000),        # 64 of them: cleared tickets
    (2, 60, 4, 8, 64, 32, 300),         # four warps a CTA, two streamings of a KV head
    (1, 160, 4, 3, 128, 64, 2200),      # bf16: eight warps and a cache a chunk; int8: cut for an even last wave
    (4, 80, 2, 1, 128, 16, 90),         # short ones
])
def test_ways_to_cut_a_call(fmt, L, B, H, G, d, page, longest):
    """One size of each way in which the rows are handed out; lengths from nothing to what the tables hold."""
    rng = np.random.default_rng(L + B)
    lens = rng.integers(0, longest + 1, (L, B))
    lens.flat[0], lens.flat[-1] = longest, lens.flat[-1] // 16 * 16
    c = RowCache(fmt, L, B, H, d, lens, page, seed=3)
    lam, gain = (t.to(DEV) for t in weights(L, H * G, d, 5))
    q = queries(L, B, H * G, d, 6)
    out, sums = attend(c, H * G, q, lam, gain)
    check(c, H * G, q, lam, gain, out, sums, every=max(1, B // 4))
    for _ in range(3):
        again, s = attend(c, H * G, q, lam, gain)
        assert torch.equal(out, again) and torch.equal(sums, s)


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_pages_that_start_on_16_bytes(fmt):
    c = RowCache(fmt, 2, 3, 2, 64, [[100, 0, 33], [257, 16, 90]], 16, seed=3)
    lam, gain = (t.to(DEV) for t in weights(2, 4, 64, 5))
    q = queries(2, 3, 4, 64, 6)
    for i in range(2):
        x = c.pages[i]
        room = torch.empty(x.numel() * x.element_size() + 32, dtype=torch.uint8, device=DEV)
        moved = room[16:-16].view(x.dtype).view(x.shape)
        moved.copy_(x)
        c.pages[i] = moved
        assert moved.data_ptr() % 32 == 16
    out, sums = attend(c, 4, q, lam, gain)
    check(c, 4, q, lam, gain, out, sums)


@pytest.mark.parametrize("power", [-24, -14, 12, 30])
def test_row_scales_of_any_size(power):
    """8-bit V rows whose scales are far from 1, and a block of rows whose scales are far from the others'."""
    c = RowCache("int8", 1, 3, 2, 128, [[400, 37, 1000]], 16, seed=3)
    c.scales[1] *= 2.0 ** power
    c.values[1] *= 2.0 ** power
    first = c.table[0, :, 0].long()
    c.scales[1][first] *= 2.0 ** -20
    c.values[1][first] *= 2.0 ** -20
    lam, gain = (t.to(DEV) for t in weights(1, 8, 128, 5))
    q = queries(1, 3, 8, 128, 6)
    for g in (gain, None):
        out, sums = attend(c, 8, q, lam, g, eps=0.0)
        check(c, 8, q, lam, g, out, sums, eps=0.0)


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_a_long_cache_among_short_ones(fmt):
    """Tables much longer than most caches: chunks that find nothing, one cache in many pieces."""
    lens = np.random.default_rng(1).integers(0, 200, (1, 24))
    lens[0, 5] = 17001
    c = RowCache(fmt, 1, 24, 2, 64, lens, 64, seed=3)
    lam, gain = (t.to(DEV) for t in weights(1, 8, 64, 5))
    q = queries(1, 24, 8, 64, 6)
    out, sums = attend(c, 8, q, lam, gain)
    check(c, 8, q, lam, gain, out, sums)
    again, _ = attend(c, 8, q, lam, gain)
    assert torch.equal(out, again)
