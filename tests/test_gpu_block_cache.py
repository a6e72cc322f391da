"""Caches of 8-bit floats with one scale per block of 16 slots and KV head: rows stored by slot, the page bookkeeping of a
step, decode attention, and the three together, against plain 64-bit definitions.  Codes, scales, tables and slots are
compared exactly; attention with bounds counted from its roundings (check_decode)."""
import math

import numpy as np
import pytest
import torch

from oracle import xkv_oracle as O
from paper_2412_05896_b200 import xkv

from gpu_util import f64, require_lib

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16_HALF = 2.0 ** -8           # half a step of bf16, relative


@pytest.fixture(scope="module", autouse=True)
def _lib():
    require_lib()


def values(codes, scales, page):
    """What pages [.., page, d] and scales [.., page / 16] stand for (float64)."""
    return O.e4m3_values(codes) * np.repeat(np.asarray(scales, dtype=np.float64), O.SCALE_BLOCK, axis=-1)[..., None]


class Pool:
    """A page pool of block-scaled 8-bit floats filled by numpy (not by the library): random codes and power-of-two
    scales, pages of every (layer, sequence) in shuffled order, NaN codes and NaN scales behind the last row."""

    def __init__(self, lens, H, d, page, seed=0, spare_rows=0, spread=3, big_k_row=None, any_code=False):
        self.lens = np.asarray(lens, dtype=np.int64)
        L, B = self.lens.shape
        rng = np.random.default_rng(seed)
        self.H, self.d, self.page, self.L, self.B = H, d, page, L, B
        self.cols = max(1, -(-(int(self.lens.max()) + spare_rows) // page))
        self.n_pages = L * B * self.cols + 3
        self.table = rng.permutation(self.n_pages)[: L * B * self.cols].reshape(L, B, self.cols)
        nb = page // O.SCALE_BLOCK
        self.codes, self.scales = {}, {}
        for x in "kv":
            if any_code:                                 # every finite code alike
                sign_mag = rng.integers(0, 0x7F, (self.n_pages, H, page, d), dtype=np.uint8)
                sign_mag |= rng.integers(0, 2, sign_mag.shape, dtype=np.uint8) << 7
            else:
                sign_mag = self._bytes(O.e4m3_grid(rng.normal(0, 60, (self.n_pages, H, page, d))))
            s = 2.0 ** rng.integers(-7 - spread, -6 + spread, (self.n_pages, H, nb))
            for l in range(L):
                for b in range(B):
                    n = int(self.lens[l, b])
                    for i in range(self.cols):
                        pg, live = self.table[l, b, i], min(max(n - i * page, 0), page)
                        sign_mag[pg, :, live:] = 0x7F
                        s[pg, :, -(-live // O.SCALE_BLOCK):] = np.nan
            self.codes[x], self.scales[x] = sign_mag, s.astype(np.float32)
        if big_k_row is not None:                        # one row of every cache draws most of the attention
            for l in range(L):
                for b in range(B):
                    r = big_k_row % max(1, int(self.lens[l, b]))
                    if self.lens[l, b]:
                        pg, sl = self.table[l, b, r // page], (r % page) // O.SCALE_BLOCK
                        self.scales["k"][pg, :, sl] *= 4.0
        self.dev = {x: torch.from_numpy(self.codes[x]).to(DEV) for x in "kv"}
        self.dev_s = {x: torch.from_numpy(self.scales[x]).to(DEV) for x in "kv"}
        self.bt = torch.from_numpy(self.table.astype(np.int32)).to(DEV)
        self.seq_lens = torch.from_numpy(self.lens.astype(np.int32)).to(DEV)

    @staticmethod
    def _bytes(vals):
        """Bytes of values that lie on the grid."""
        allv = O.e4m3_values(np.arange(127))
        idx = np.searchsorted(allv, np.abs(vals))
        return (idx + np.where(np.signbit(vals), 128, 0)).astype(np.uint8)

    def handle(self):
        return xkv.Cache(self.dev["k"].data_ptr(), self.dev["v"].data_ptr(), self.bt.data_ptr(), self.seq_lens.data_ptr(),
                         self.L, self.page, self.cols, self.n_pages, self.dev_s["k"].data_ptr(),
                         self.dev_s["v"].data_ptr(), xkv.KV_E4M3, 0)

    def rows(self, x, l, b, g, n):
        s = np.arange(n)
        pg, off = self.table[l, b, s // self.page], s % self.page
        codes, scales = self.dev[x].cpu().numpy(), self.dev_s[x].cpu().numpy()
        return O.e4m3_values(codes[pg, g, off]) * scales[pg, g, off // O.SCALE_BLOCK].astype(np.float64)[:, None]


def check_decode(q, K, V, scale, out, lse, what):
    """One head's output against softmax(scale q K^T) V in 64 bits.

    Bounds: a logit is a sum of d exact products accumulated in fp32 (at most d + 1 roundings or truncations of one
    ulp 2^-23 of the running sum, itself at most sum|q k|) and multiplied three times: dz <= (d + 8) 2^-23 scale max_c
    sum|q k|; the query's second code leaves 2^-21 of its largest element.  A weight moves by dz (relative), by 2^-8 as
    a sum of two codes, by 2^-21 in the exponential; tiny weights by 2^-22 of the largest, at most 128 per tile.  The
    output rounds to bf16."""
    z = scale * (K @ q)
    m = z.max()
    p = np.exp(z - m)
    ref = (p @ V) / p.sum()
    mag = (p @ np.abs(V)) / p.sum()
    absqk = scale * (np.abs(K) @ np.abs(q))
    dz = (len(q) + 8) * 2.0 ** -23 * absqk.max() + 2.0 ** -21 * scale * np.abs(q).max() * np.abs(K).sum(1).max()
    assert np.all(np.isfinite(out)), what
    vmax = np.abs(V).max()
    bound = (2 * dz + BF16_HALF + 2.0 ** -20) * mag + 2.0 ** -14 * vmax * p.max() / p.sum() + BF16_HALF * np.abs(ref) + 1e-30
    worst = (np.abs(out - ref) / bound).max()
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"
    want = m + math.log(p.sum())
    assert abs(lse - want) <= dz + 2.0 ** -21 * (1 + abs(want)), f"{what}: lse {lse} for {want}"


def run_decode(pool, Hq, q, chunk=0, layers=None, kn=None, vn=None, scale=0.0, stream=None, ws=None):
    l0, l1 = layers or (0, pool.L)
    dims = xkv.Dims(pool.B, Hq, pool.H, pool.d, 1, 1, 0, scale, pool.H * pool.d, pool.d)
    if ws is None:
        ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DECODE_ATTN, dims, n_layers=l1 - l0, max_cache_len=pool.cols * pool.page,
                                             chunk_rows=chunk), dtype=torch.uint8, device=DEV)
    out = torch.full((l1 - l0, pool.B, Hq, pool.d), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((l1 - l0, pool.B, Hq), float("nan"), device=DEV)
    torch.cuda.synchronize()
    xkv.decode_attn(dims, pool.handle(), l0, l1, q, kn, vn, out, lse, chunk, ws, stream=stream)
    torch.cuda.synchronize()
    status = xkv.read_device_status(ws)
    return out, lse, status


def check_all(pool, Hq, q, out, lse, lens, l0=0, scale=0.0, what=""):
    G, sc = Hq // pool.H, scale or 1.0 / math.sqrt(pool.d)
    qf, of, lf = f64(q), f64(out), f64(lse)
    for l in range(out.shape[0]):
        for b in range(pool.B):
            n = int(lens[l0 + l][b])
            for g in range(pool.H):
                if n == 0:
                    assert np.all(of[l, b, g * G:(g + 1) * G] == 0) and np.all(np.isneginf(lf[l, b, g * G:(g + 1) * G]))
                    continue
                K, V = pool.rows("k", l0 + l, b, g, n), pool.rows("v", l0 + l, b, g, n)
                for h in range(g * G, (g + 1) * G):
                    check_decode(qf[l, b, h], K, V, sc, of[l, b, h], lf[l, b, h], f"{what} l{l} b{b} h{h} n{n}")


def queries(L, B, Hq, d, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(L, B, Hq, d, generator=g) * torch.exp(torch.rand(L, B, Hq, 1, generator=g) * 2 - 1) * size
    return q.to(torch.bfloat16).to(DEV)


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8])
def test_decode_groups(d, G):
    H = 2
    pool = Pool([[1, 15, 16, 17], [127, 128, 129, 300]], H, d, 16, seed=G)
    q = queries(2, 4, H * G, d, G)
    out, lse, st = run_decode(pool, H * G, q)
    assert st == xkv.OK
    check_all(pool, H * G, q, out, lse, pool.lens, what=f"d{d} G{G}")


@pytest.mark.parametrize("page", [16, 32, 48, 64, 80, 112, 128, 144, 256])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_pages_and_lengths(page, d):
    lens = [[0, 1, 2, 31, 33], [63, 64, 65, page, page + 1], [2 * page - 1, 255, 256, 257, 1000]]
    pool = Pool(lens, 1, d, page, seed=page)
    q = queries(3, 5, 4, d, page)
    out, lse, st = run_decode(pool, 4, q)
    assert st == xkv.OK
    check_all(pool, 4, q, out, lse, pool.lens, what=f"page {page}")
    # a range of layers, another logit scale
    out, lse, st = run_decode(pool, 4, q[1:2].contiguous(), layers=(1, 2), scale=0.31)
    assert st == xkv.OK
    check_all(pool, 4, q[1:2], out, lse, pool.lens, l0=1, scale=0.31, what=f"page {page} layer 1")


@pytest.mark.parametrize("chunk", [0, 64, 128, 192, 1024])
@pytest.mark.parametrize("H,G,d", [(1, 8, 128), (3, 1, 64), (2, 4, 128)])
def test_decode_long_caches_are_split(chunk, H, G, d):
    pool = Pool([[5000, 0, 129], [1, 2049, 4096]], H, d, 32, seed=chunk, big_k_row=1234)
    q = queries(2, 3, H * G, d, chunk)
    out, lse, st = run_decode(pool, H * G, q, chunk=chunk)
    assert st == xkv.OK
    check_all(pool, H * G, q, out, lse, pool.lens, what=f"chunk {chunk}")
    again, lse2, st = run_decode(pool, H * G, q, chunk=chunk)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("G", [1, 2, 3, 5, 8])
def test_decode_tiles_of_narrow_heads(G):
    """Heads of 64 elements: caches that end before, at and behind the middle and the end of a tile of 256 rows."""
    pool = Pool([[383, 384, 385, 511, 512], [513, 640, 641, 769, 3969]], 2, 64, 48, seed=40 + G, big_k_row=600)
    q = queries(2, 5, 2 * G, 64, 40 + G)
    out, lse, st = run_decode(pool, 2 * G, q)
    assert st == xkv.OK
    check_all(pool, 2 * G, q, out, lse, pool.lens, what=f"G {G}")


@pytest.mark.parametrize("G", [1, 7])
def test_decode_many_caches_per_block(G):
    """More caches than thread blocks, of one and of two tiles, so that queues of them run through every block."""
    lens = [[84 + (37 * i + 11 * l) % 74 for i in range(12)] for l in range(3)]
    pool = Pool(lens, 32, 128, 48, seed=50 + G)
    q = queries(3, 12, 32 * G, 128, 50 + G)
    out, lse, st = run_decode(pool, 32 * G, q)
    assert st == xkv.OK
    check_all(pool, 32 * G, q, out, lse, pool.lens, what=f"G {G}")


def test_decode_small_weights_of_many_rows_count():
    """One row takes almost all of a tile's weight while thousands of rows far below it hold most of the mass."""
    n, d = 20000, 128
    pool = Pool([[n]], 1, d, 16, seed=3, spread=0)
    vals = np.zeros((pool.n_pages, 1, 16, d))
    vals[..., 0] = 1.0
    pg = pool.table[0, 0]
    vals[pg[0], 0, 0, 0] = 448.0
    kb = Pool._bytes(vals)
    pool.dev["k"].copy_(torch.from_numpy(kb))
    pool.dev_s["k"].fill_(2.0 ** -5)                        # keys 14 and 1/32 along one direction
    q = torch.zeros(1, 1, 2, d, dtype=torch.bfloat16, device=DEV)
    q[0, 0, 0, 0] = 7.75                                    # logits 108.5 scale .. -> about 9.6 and 0.02
    q[0, 0, 1, 0] = 10.0
    out, lse, st = run_decode(pool, 2, q)
    assert st == xkv.OK
    check_all(pool, 2, q, out, lse, pool.lens, what="sink")


def test_decode_nothing_cached():
    pool = Pool([[0, 0], [0, 0]], 2, 64, 16, seed=1)
    q = queries(2, 2, 6, 64, 1)
    out, lse, st = run_decode(pool, 6, q)
    assert st == xkv.OK
    check_all(pool, 6, q, out, lse, pool.lens, what="empty")


def test_decode_bad_pages():
    """Table entries outside the pool are read as its nearest page: no fault, and the other sequences are untouched."""
    pool = Pool([[40, 300, 77]], 2, 128, 16, seed=17)
    q = queries(1, 3, 8, 128, 17)
    want, _, _ = run_decode(pool, 8, q)
    pool.bt[0, 1, 3], pool.bt[0, 1, 5] = -7, 1 << 30
    got, _, st = run_decode(pool, 8, q)
    assert st == xkv.OK and torch.equal(got[0, 0], want[0, 0]) and torch.equal(got[0, 2], want[0, 2])


def test_decode_extreme_scales_and_queries():
    """Scales at both ends within one cache, queries that are zero, tiny and huge; a NaN query gives a NaN row alone."""
    pool = Pool([[300, 40]], 2, 128, 16, seed=9)
    for x in "kv":
        s = pool.dev_s[x].cpu().numpy()
        rng = np.random.default_rng(5)
        s = np.where(np.isnan(s), s, s * 2.0 ** rng.integers(-20, 1, s.shape)).astype(np.float32)
        pool.dev_s[x].copy_(torch.from_numpy(s))
    q = queries(1, 2, 8, 128, 4)
    q[0, 0, 0] = 0.0
    q[0, 0, 1] *= 2.0 ** -60
    q[0, 1, 2] *= 2.0 ** 6
    q[0, 1, 3, 5:] = 0.0
    out, lse, st = run_decode(pool, 8, q)
    assert st == xkv.OK
    check_all(pool, 8, q, out, lse, pool.lens, what="extreme")
    q2 = q.clone()
    q2[0, 0, 6, 17] = float("nan")
    q2[0, 1, 5, 1] = float("inf")
    out2, lse2, _ = run_decode(pool, 8, q2)
    bad = torch.zeros(1, 2, 8, dtype=torch.bool, device=DEV)
    bad[0, 0, 6] = bad[0, 1, 5] = True
    assert torch.isnan(out2[bad]).all() and torch.equal(out2[~bad], out[~bad]) and torch.equal(lse2[~bad], lse[~bad])


def test_decode_many_units():
    lens = np.random.default_rng(1).integers(0, 40, (24, 130))
    pool = Pool(lens, 1, 64, 16, seed=8)
    q = queries(24, 130, 1, 64, 8)
    out, lse, st = run_decode(pool, 1, q)
    assert st == xkv.OK
    check_all(pool, 1, q, out, lse, lens, what="many")


def test_decode_in_a_graph_and_on_another_stream():
    pool = Pool([[700, 33], [128, 2000]], 2, 128, 16, seed=2)
    q = queries(2, 2, 8, 128, 2)
    want, want_lse, _ = run_decode(pool, 8, q)
    side = torch.cuda.Stream(device=DEV)
    with torch.cuda.stream(side):
        got, got_lse, st = run_decode(pool, 8, q, stream=side)
    assert st == xkv.OK and torch.equal(got, want) and torch.equal(got_lse, want_lse)
    dims = xkv.Dims(2, 8, 2, 128, 1, 1, 0, 0.0, 256, 128)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DECODE_ATTN, dims, n_layers=2, max_cache_len=pool.cols * 16),
                     dtype=torch.uint8, device=DEV)
    out = torch.empty_like(want)
    handle = pool.handle()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xkv.decode_attn(dims, handle, 0, 2, q, None, None, out, None, 0, ws)
    for _ in range(3):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    pool.seq_lens.copy_(torch.tensor([[699, 1], [0, 1999]], dtype=torch.int32))      # lengths are read at replay
    graph.replay()
    torch.cuda.synchronize()
    again, _, _ = run_decode(pool, 8, q)
    assert torch.equal(out, again) and not torch.equal(out, want)


@pytest.mark.parametrize("d,page", [(128, 16), (64, 48)])
def test_decode_appends_first(d, page):
    H, G = 2, 3
    pool = Pool([[0, 15, 16], [page - 1, page, 77]], H, d, page, seed=6, spare_rows=20)
    ref = {}
    lens = pool.lens.copy()
    for l in range(2):
        for b in range(3):
            for g in range(H):
                for x in "kv":
                    c = O.BlockCache(d)
                    n = int(lens[l, b])
                    s = np.arange(n)
                    pg, off = pool.table[l, b, s // page], s % page
                    c.n, c.codes = n, O.e4m3_values(pool.codes[x][pg, g, off]).reshape(n, d)
                    blocks = np.arange(-(-n // 16)) * 16
                    c.scales = [float(v) for v in
                                pool.scales[x][pool.table[l, b, blocks // page], g, (blocks % page) // 16]]
                    ref[l, b, g, x] = c
    for step in range(18):
        gen = torch.Generator().manual_seed(100 + step)
        kn, vn = ((torch.randn(2, 3, H, d, generator=gen) * 2.0 ** (step % 5)).to(torch.bfloat16).to(DEV) for _ in "kv")
        q = queries(2, 3, H * G, d, step, size=0.1)
        out, lse, st = run_decode(pool, H * G, q, kn=kn, vn=vn)
        assert st == xkv.OK
        lens += 1
        assert np.array_equal(pool.seq_lens.cpu().numpy(), lens)
        for (l, b, g, x), c in ref.items():
            c.append(f64((kn if x == "k" else vn)[l, b, g])[None])
            assert np.array_equal(pool.rows(x, l, b, g, c.n), c.values()), (step, l, b, g, x)
        check_all(pool, H * G, q, out, lse, lens, what=f"step {step}")


def test_decode_append_beyond_the_page_table():
    pool = Pool([[31, 32, 5]], 1, 64, 16, seed=1)             # two pages a sequence: the second one is full
    before = {x: pool.dev[x].clone() for x in "kv"}
    kn = torch.ones(1, 3, 1, 64, dtype=torch.bfloat16, device=DEV)
    q = queries(1, 3, 1, 64, 1)
    out, lse, st = run_decode(pool, 1, q, kn=kn, vn=kn)
    assert st == xkv.ERR_CAPACITY
    assert pool.seq_lens.tolist() == [[32, 32, 6]]
    full = pool.table[0, 1]
    assert torch.equal(pool.dev["k"][full], before["k"][full])
    check_all(pool, 1, q, out, lse, [[32, 32, 6]], what="full")


def test_decode_two_calls_at_once():
    """Two streams, a workspace each."""
    pool = Pool(np.random.default_rng(3).integers(1, 2500, (2, 6)), 2, 128, 16, seed=21)
    qs = [queries(2, 6, 8, 128, 30 + i) for i in range(2)]
    want = [run_decode(pool, 8, q)[:2] for q in qs]
    dims = xkv.Dims(6, 8, 2, 128, 1, 1, 0, 0.0, 256, 128)
    nbytes = xkv.workspace_bytes(xkv.OP_DECODE_ATTN, dims, n_layers=2, max_cache_len=pool.cols * 16)
    ws = [torch.zeros(nbytes, dtype=torch.uint8, device=DEV) for _ in qs]
    outs = [torch.empty_like(want[0][0]) for _ in qs]
    streams = [torch.cuda.Stream(device=DEV) for _ in qs]
    handle = pool.handle()
    torch.cuda.synchronize()
    for _ in range(20):
        for q, w, o, s in zip(qs, ws, outs, streams):
            xkv.decode_attn(dims, handle, 0, 2, q, None, None, o, None, 0, w, stream=s)
    torch.cuda.synchronize()
    for o, w, (ref, _) in zip(outs, ws, want):
        assert xkv.read_device_status(w) == xkv.OK and torch.equal(o, ref)


def test_decode_waits_that_expire():
    """One CTA's copies are never issued: its waits run out after a millisecond, the launch returns and says so, and
    workspace and cache stay usable."""
    pool = Pool([[3000, 40], [17, 5000]], 2, 128, 16, seed=12)
    q = queries(2, 2, 8, 128, 12)
    want, want_lse, st = run_decode(pool, 8, q)
    assert st == xkv.OK
    dims = xkv.Dims(2, 8, 2, 128, 1, 1, 0, 0.0, 256, 128)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DECODE_ATTN, dims, n_layers=2, max_cache_len=pool.cols * 16),
                     dtype=torch.uint8, device=DEV)
    try:
        xkv.test_hooks(wait_limit_ns=1_000_000, withhold_decode_item=1)
        _, _, st = run_decode(pool, 8, q, ws=ws)
    finally:
        xkv.test_hooks()
    assert st == xkv.ERR_TIMEOUT
    got, got_lse, st = run_decode(pool, 8, q, ws=ws)
    assert st == xkv.OK and torch.equal(got, want) and torch.equal(got_lse, want_lse)


def test_decode_profile_events():
    pool = Pool([[500, 40]], 2, 64, 16, seed=13)
    q = queries(1, 2, 4, 64, 13)
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    stop.record()
    try:
        xkv.profile_events(start, stop)
        out, lse, st = run_decode(pool, 4, q)
    finally:
        xkv.profile_events(None, None)
    assert st == xkv.OK and 0.0 < start.elapsed_time(stop) < 100.0
    check_all(pool, 4, q, out, lse, pool.lens, what="timed")


def test_decode_repeats_bit_for_bit():
    lens = np.random.default_rng(2).integers(1, 3000, (3, 9))
    pool = Pool(lens, 2, 128, 32, seed=14)
    q = queries(3, 9, 10, 128, 14)
    want, want_lse, st = run_decode(pool, 10, q)
    assert st == xkv.OK
    for _ in range(30):
        got, got_lse, _ = run_decode(pool, 10, q)
        assert torch.equal(got, want) and torch.equal(got_lse, want_lse)


# ------------------------------------------------------------------ rows stored by slot
def store(pool, k, v, slots, dims=None):
    dims = dims or xkv.Dims(1, pool.H, pool.H, pool.d, 1, 1, 0, 0.0, pool.H * pool.d, pool.d)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_STORE_ROWS, dims), dtype=torch.uint8, device=DEV)
    xkv.store_rows(dims, pool.handle(), k, v, slots, slots.numel(), ws)
    torch.cuda.synchronize()
    return xkv.read_device_status(ws)


def expect_store(pool, x, rows, slots):
    """The pool's values of K or V after the rows (float64 [T, H, d]) are stored, token runs in order."""
    codes, scales = O.e4m3_values(pool.codes[x]), pool.scales[x].astype(np.float64)
    page = pool.page
    i = 0
    while i < len(slots):
        s = int(slots[i])
        if s < 0:
            i += 1
            continue
        n = 1
        while i + n < len(slots) and slots[i + n] == s + n and (s + n) % 16:
            n += 1
        pg, sub, first = s // page, (s % page) // 16, s % 16
        new, lo = rows[i:i + n].transpose(1, 0, 2), sub * 16                     # [H, n, d]
        top = np.where(np.isfinite(new), np.abs(new), 0).max((1, 2))
        m, e = np.frexp(top)                                                     # top = m 2^e, 448 = 0.875 2^9
        sc = np.where(top > 0, np.ldexp(1.0, np.clip(np.where(m <= 0.875, e - 9, e - 8), -100, 120)), 2.0 ** -100)
        if first:
            was = scales[pg, :, sub]
            sc = np.where(was >= sc, was, sc)
            codes[pg, :, lo:lo + first] = O.e4m3_grid(codes[pg, :, lo:lo + first] * (was / sc)[:, None, None])
        scales[pg, :, sub] = sc
        codes[pg, :, lo + first:lo + first + n] = O.e4m3_grid(new / sc[:, None, None])
        i += n
    return codes, scales


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


@pytest.mark.parametrize("d,H,page,lens,new", [
    (128, 2, 16, [0, 5, 16, 30], [1, 1, 1, 1]),
    (64, 3, 48, [0, 17, 95, 250], [48, 16, 1, 133]),
    (128, 8, 64, [0, 0, 0], [700, 1, 64]),
    (64, 1, 256, [3, 260, 15], [512, 0, 2]),
    (128, 1, 112, [111], [2000]),
    (128, 8, 16, [7, 0], [4300, 333]),                       # many tokens: a warp looks for runs among sixteen
    (64, 8, 32, [i % 37 for i in range(720)], [1] * 720),    # a step of many sequences: among four
    (64, 16, 16, [i % 29 for i in range(2400)], [1] * 2400),  # of more: among sixteen
])
@pytest.mark.parametrize("pad", [0, 37])
def test_store_rows(d, H, page, lens, new, pad):
    lens, new = np.asarray(lens), np.asarray(new)
    pool = Pool([lens], H, d, page, seed=len(lens) + pad, spare_rows=int(new.max()), any_code=True)
    slots = np.concatenate([pool.table[0, b, (n + np.arange(a)) // page] * page + (n + np.arange(a)) % page
                            for b, (n, a) in enumerate(zip(lens, new))] + [np.full(pad, -1)]).astype(np.int64)
    T = len(slots)
    gen = torch.Generator().manual_seed(T)
    # K and V are slices of one projection's rows: wider token strides, heads interleaved with other columns
    qkv = torch.randn(T, H, 3, d, generator=gen) * torch.exp2(torch.randint(-6, 7, (T, H, 3, 1), generator=gen).float())
    qkv = qkv.to(torch.bfloat16).to(DEV)
    k, v = qkv[:, :, 1], qkv[:, :, 2]
    dims = xkv.Dims(1, H, H, d, 1, 1, 0, 0.0, H * 3 * d, 3 * d)
    want = {x: expect_store(pool, x, f64(t), slots) for x, t in (("k", k), ("v", v))}
    assert store(pool, k, v, torch.from_numpy(slots).to(DEV), dims) == xkv.OK
    for x in "kv":
        assert same(O.e4m3_values(pool.dev[x].cpu().numpy()), want[x][0]), x
        assert same(pool.dev_s[x].cpu().numpy().astype(np.float64), want[x][1]), x


def test_store_rows_special_values():
    d, H, page = 64, 1, 16
    pool = Pool([[0, 0, 0, 0, 0, 3]], H, d, page, seed=4, spare_rows=16)
    vals = torch.zeros(6, H, d)
    vals[1] = 2.0 ** -130                                    # below the smallest scale's reach: rounds to zero codes
    vals[2, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 3.0])
    vals[3] = 3.38e38
    vals[4, 0, 0] = -7.0
    vals[5, 0, :2] = torch.tensor([float("nan"), 1e30])
    k = vals.to(torch.bfloat16).to(DEV)
    slots = np.array([pool.table[0, b, 0] * page + (3 if b == 5 else 0) for b in range(6)])
    want = expect_store(pool, "k", f64(k), slots)
    assert store(pool, k, k.clone(), torch.from_numpy(slots).to(DEV)) == xkv.OK
    assert same(O.e4m3_values(pool.dev["k"].cpu().numpy()), want[0])
    assert same(pool.dev_s["k"].cpu().numpy().astype(np.float64), want[1])
    row = O.e4m3_values(pool.dev["k"].cpu().numpy())[pool.table[0, 2, 0], 0, 0]
    assert row[0] == 448 and row[1] == -448 and np.isnan(row[2]) and row[3] == 384


def test_store_rows_refused_slots():
    pool = Pool([[0, 0]], 1, 64, 16, seed=4, spare_rows=32)
    k = torch.ones(4, 1, 64, dtype=torch.bfloat16, device=DEV)
    before = pool.dev["k"].clone()
    slots = torch.tensor([-1, pool.n_pages * 16, -5, 1 << 40], dtype=torch.int64, device=DEV)
    assert store(pool, k, k, slots) == xkv.ERR_CAPACITY
    assert torch.equal(pool.dev["k"], before)
    s = int(pool.table[0, 0, 0]) * 16
    # the second token repeats the first one's slot, the third and fourth go back within the block: only the first is stored
    assert store(pool, k, k, torch.tensor([s + 2, s + 2, s + 1, s], dtype=torch.int64, device=DEV)) == xkv.ERR_INVALID_ARG
    diff = (pool.dev["k"] != before).reshape(-1, 64).any(1).nonzero()[:, 0].tolist()
    assert s + 2 in diff and set(diff) <= {s, s + 1, s + 2}   # the rows before it are re-expressed, nothing behind it


@pytest.mark.parametrize("fmt", [xkv.KV_BF16, xkv.KV_INT8])
@pytest.mark.parametrize("d,H", [(64, 3), (128, 2)])
def test_store_rows_other_formats(fmt, d, H):
    page, n_pages, T = 32, 9, 70
    rng = np.random.default_rng(d)
    slots = rng.permutation(n_pages * page)[:T].astype(np.int64)
    slots[::9] = -1
    gen = torch.Generator().manual_seed(d)
    k, v = (torch.randn(T, H, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in "kv")
    dt = torch.bfloat16 if fmt == xkv.KV_BF16 else torch.uint8
    kp, vp = (torch.full((n_pages, H, page, d), 3, dtype=dt, device=DEV) for _ in "kv")
    ks, vs = (torch.full((n_pages, H, page), 5.0, device=DEV) for _ in "kv")
    cache = xkv.Cache(kp.data_ptr(), vp.data_ptr(), None, None, 1, page, 1, n_pages, ks.data_ptr(), vs.data_ptr(), fmt, 0)
    dims = xkv.Dims(1, H, H, d, 1, 1, 0, 0.0, H * d, d)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    xkv.store_rows(dims, cache, k, v, torch.from_numpy(slots).to(DEV), T, ws)
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) == xkv.OK
    for pages, scales, rows in ((kp, ks, k), (vp, vs, v)):
        want, want_s = np.full((n_pages, H, page, d), 3.0), np.full((n_pages, H, page), 5.0)
        for t, s in enumerate(slots):
            if s < 0:
                continue
            x = f64(rows[t])
            if fmt == xkv.KV_INT8:
                x, sc = O.quantize_rows_int8(x)
                want_s[s // page, :, s % page] = sc
            want[s // page, :, s % page] = x
        assert np.array_equal(f64(pages), want) and np.array_equal(f64(scales), want_s)


# ------------------------------------------------------------------ the plan of a step
def plan(lens, new, page, cols, n_pages, used, free=None, n_free=None, stride0=True, slots_stride=None, in_place=False,
         lens_null=False):
    L, B = np.shape(lens)
    rng = np.random.default_rng(3)
    table = rng.integers(0, n_pages, (L, B, cols))
    counts = np.asarray(new)
    per_layer = np.broadcast_to(counts, (L, B))
    free_list = list(range(n_pages if n_free is None else n_free)) if free is None else [int(x) for x in free]
    want = O.plan_append(per_layer, np.zeros((L, B), int) if lens_null else lens, table, page, free_list, used)
    dev = lambda a, t=torch.int32: torch.as_tensor(np.ascontiguousarray(a)).to(t).to(DEV)  # noqa: E731
    bt, ln, nn = dev(table), dev(lens), dev(counts)
    after = ln if in_place else torch.full((L, B), -7, dtype=torch.int32, device=DEV)
    stride = slots_stride if slots_stride is not None else int(per_layer.sum(1).max()) + 5
    slots = torch.full((L, max(1, stride)), -9, dtype=torch.int64, device=DEV)
    ub = torch.tensor([used], dtype=torch.int32, device=DEV)
    ua = ub if in_place else torch.full((1,), -7, dtype=torch.int32, device=DEV)
    fr = None if free is None else dev(np.asarray(free))
    cache = xkv.Cache(None, None, bt.data_ptr(), after.data_ptr(), L, page, cols, n_pages)
    dims = xkv.Dims(B, 1, 1, 64, 1, 1, 0, 0.0, 64, 64)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_PLAN_APPEND, dims, n_layers=L), dtype=torch.uint8, device=DEV)
    args = (cache, B, nn, B if counts.ndim == 2 else 0, None if lens_null else ln, fr, len(free_list), ub, ua, slots,
            slots.shape[1], ws)
    xkv.plan_append(*args)
    torch.cuda.synchronize()
    status = xkv.read_device_status(ws)
    if not in_place:                                         # the same call again on the same workspace: the same answer
        xkv.plan_append(*args)
        torch.cuda.synchronize()
        assert xkv.read_device_status(ws) == status
    return want, bt.cpu().numpy(), after.cpu().numpy(), slots.cpu().numpy(), int(ua.item()), status


def check_plan(want, bt, after, slots, used):
    table, lens, rows, end, _ = want
    assert np.array_equal(bt, table) and np.array_equal(after, lens) and used == end
    for l, row in enumerate(rows):
        n = min(len(row), slots.shape[1])
        assert np.array_equal(slots[l, :n], np.asarray(row[:n], dtype=np.int64)) and np.all(slots[l, n:] == -9)


@pytest.mark.parametrize("L,B,page,hi,new_hi", [(1, 1, 16, 0, 1), (4, 3, 16, 50, 1), (3, 7, 48, 200, 90), (2, 600, 32, 64, 33),
                                                (32, 64, 16, 700, 1), (5, 2, 256, 3000, 5000),
                                                (3, 1500, 16, 40, 3), (2, 2100, 48, 100, 60)])
@pytest.mark.parametrize("per_layer", [False, True])
def test_plan_append(L, B, page, hi, new_hi, per_layer):
    rng = np.random.default_rng(L * B + page)
    lens = rng.integers(0, hi + 1, (L, B))
    new = rng.integers(0, new_hi + 1, (L, B) if per_layer else (B,))
    cols = -(-(hi + new_hi) // page) + 1
    n_pages = L * B * cols + 11
    free = rng.permutation(n_pages)
    for kw in (dict(free=free), dict(free=None), dict(free=free, in_place=True), dict(free=free, lens_null=True)):
        want, *got, status = plan(lens, new, page, cols, n_pages, used=4, **kw)
        assert status == xkv.OK and want[4]
        check_plan(want, *got)


@pytest.mark.parametrize("page", [16, 48, 256])
@pytest.mark.parametrize("pad", [0, 1, 2, 7])
def test_plan_append_prompts(page, pad):
    """Long stretches of one sequence, from odd and even rows on, into slot maps whose layers begin at odd and even places."""
    lens = np.array([[0, 1, 15, 16, 33, 7], [2, 0, 31, 5, 16, 48], [1, 1, 1, 1, 1, 1]])
    new = np.array([[700, 1, 901, 64, 2000, 65], [63, 3001, 0, 130, 257, 511], [1000, 999, 129, 128, 127, 3]])
    cols = -(-(48 + 3001) // page) + 1
    n_pages = int((-(-(lens + new) // page)).sum()) + 3
    free = np.random.default_rng(page + pad).permutation(n_pages)
    for kw in (dict(free=free), dict(free=None), dict(free=free, slots_stride=int(new.sum(1).max()) + pad)):
        want, *got, status = plan(lens, new, page, cols, n_pages, used=0, **kw)
        assert status == xkv.OK and want[4]
        check_plan(want, *got)
    # an id outside the pool in the middle of a stretch: no slot for its rows, the others as they were
    free[20 if page == 16 else 2] = n_pages + 5
    want, *_, slots, used, status = plan(lens, new, page, cols, n_pages, used=0, free=free)
    assert status == xkv.ERR_INVALID_ARG
    for l, row in enumerate(np.asarray(r) for r in want[2]):
        assert np.array_equal(slots[l, :len(row)], np.where(row >= n_pages * page, -1, row))
    assert any(r >= n_pages * page for row in want[2] for r in row)


def test_plan_append_runs_out_of_pages():
    lens = np.array([[16, 10, 31, 0], [5, 16, 0, 64]])
    new = np.array([1, 6, 20, 16])
    for n_free in range(0, 9):
        want, *got, status = plan(lens, new, 16, 6, 40, used=0, n_free=n_free)
        assert status == (xkv.OK if want[4] else xkv.ERR_CAPACITY), n_free
        check_plan(want, *got)
    # a sequence that outgrows its table, and a slot map that is too short
    want, *got, status = plan(lens, np.array([1, 90, 20, 16]), 16, 6, 40, used=0)
    assert status == xkv.ERR_CAPACITY and not want[4]
    check_plan(want, *got)
    want, *got, status = plan(lens, new, 16, 6, 40, used=0, slots_stride=20)
    assert status == xkv.ERR_CAPACITY
    check_plan(want, *got)


def test_plan_append_bad_counts():
    lens, new = np.array([[16, -3, 31]]), np.array([1, 2, -4])
    got = plan(np.maximum(lens, 0), np.maximum(new, 0), 16, 4, 40, used=2)
    want = got[0]
    table, after, slots, used, status = plan(lens, new, 16, 4, 40, used=2)[1:]
    assert status == xkv.ERR_INVALID_ARG
    check_plan(want, table, after, slots, used)
    # page ids outside the pool, a list position outside the list
    *_, slots, used, status = plan(np.array([[0]]), np.array([20]), 16, 4, 40, used=0, free=[41, -1, 3])
    assert status == xkv.ERR_INVALID_ARG and np.all(slots[0, :20] == -1)
    *_, after, slots, used, status = plan(np.array([[0]]), np.array([20]), 16, 4, 40, used=99, free=[1, 2])
    assert status == xkv.ERR_INVALID_ARG and after.tolist() == [[0]] and np.all(slots[0, :20] == -1)


def test_plan_append_largest_batch():
    B = 16384
    rng = np.random.default_rng(0)
    lens, new = rng.integers(0, 90, (1, B)), rng.integers(0, 3, (B,))
    want, *got, status = plan(lens, new, 16, 6, 6 * B, used=1, free=rng.permutation(6 * B))
    assert status == xkv.OK
    check_plan(want, *got)


# ------------------------------------------------------------------ the three together
def test_serving_loop_in_one_graph():
    """Prompts planned and stored at once, then steps of plan, store and attention captured in one graph and replayed."""
    L, B, H, G, d, page = 2, 3, 2, 2, 128, 16
    prompts, cols, n_pages = np.array([40, 1, 18]), 6, 41
    rng = np.random.default_rng(0)
    free = torch.from_numpy(rng.permutation(n_pages).astype(np.int32)).to(DEV)
    bt = torch.full((L, B, cols), -1, dtype=torch.int32, device=DEV)
    lens = torch.zeros(L, B, dtype=torch.int32, device=DEV)
    used = torch.zeros(1, dtype=torch.int32, device=DEV)
    kp, vp = (torch.full((n_pages, H, page, d), 0x7F, dtype=torch.uint8, device=DEV) for _ in "kv")
    ks, vs = (torch.full((n_pages, H, 1), float("nan"), device=DEV) for _ in "kv")
    cache = xkv.Cache(kp.data_ptr(), vp.data_ptr(), bt.data_ptr(), lens.data_ptr(), L, page, cols, n_pages, ks.data_ptr(),
                      vs.data_ptr(), xkv.KV_E4M3, 0)
    dims = xkv.Dims(B, H * G, H, d, 1, 1, 0, 0.0, H * d, d)
    ws = torch.zeros(max(xkv.workspace_bytes(xkv.OP_DECODE_ATTN, dims, n_layers=L, max_cache_len=cols * page),
                         xkv.workspace_bytes(xkv.OP_PLAN_APPEND, dims, n_layers=L)), dtype=torch.uint8, device=DEV)
    gen = torch.Generator().manual_seed(1)
    ref = {(l, b, g, x): O.BlockCache(d) for l in range(L) for b in range(B) for g in range(H) for x in "kv"}

    def step(n_new, k, v, slots):
        T = k.shape[1]
        xkv.plan_append(cache, B, n_new, 0, lens, free, n_pages, used, used, slots, T, ws)
        xkv.store_rows(dims, cache, k, v, slots, L * T, ws)

    def note(n_new, k, v):
        at = 0
        for b, n in enumerate(n_new):
            for l in range(L):
                for g in range(H):
                    ref[l, b, g, "k"].append(f64(k[l, at:at + n, g]))
                    ref[l, b, g, "v"].append(f64(v[l, at:at + n, g]))
            at += n

    T = int(prompts.sum())
    k, v = (torch.randn(L, T, H, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in "kv")
    step(torch.from_numpy(prompts.astype(np.int32)).to(DEV), k, v, torch.empty(L, T, dtype=torch.int64, device=DEV))
    note(prompts, k, v)

    ones = torch.ones(B, dtype=torch.int32, device=DEV)
    k1, v1, q1 = (torch.zeros(L, B, n, d, dtype=torch.bfloat16, device=DEV) for n in (H, H, H * G))
    slots1 = torch.empty(L, B, dtype=torch.int64, device=DEV)
    out, lse = torch.empty(L, B, H * G, d, dtype=torch.bfloat16, device=DEV), torch.empty(L, B, H * G, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ones, k1, v1, slots1)
        xkv.decode_attn(dims, cache, 0, L, q1, None, None, out, lse, 0, ws)
    for i in range(20):
        for t, n in ((k1, 1.0 + i), (v1, 2.0 ** (i % 4)), (q1, 1.0)):
            t.copy_((torch.randn(t.shape, generator=gen) * n).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert xkv.read_device_status(ws) == xkv.OK
        note([1] * B, k1, v1)
        assert np.array_equal(lens.cpu().numpy(), np.broadcast_to(prompts + i + 1, (L, B)))
        qf, of, lf = f64(q1), f64(out), f64(lse)
        for l in range(L):
            for b in range(B):
                for h in range(H * G):
                    check_decode(qf[l, b, h], ref[l, b, h // G, "k"].values(), ref[l, b, h // G, "v"].values(),
                                 1 / math.sqrt(d), of[l, b, h], lf[l, b, h], f"step {i} {l} {b} {h}")
    assert int(used.item()) == L * int((-(-(prompts + 20) // page)).sum())


@pytest.mark.parametrize("head_level,on_demand", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("d", [64, 128])
def test_session(head_level, on_demand, d):
    """Prefill, eviction, further turns and generation through the session, caches in 8-bit floats."""
    from dataclasses import replace

    from paper_2412_05896_b200 import workloads as WL
    from paper_2412_05896_b200.pipeline import XkvSession
    w = replace(WL.CONFIGS["mistral_7b_gqa"], n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=d, batch=2, prompt=(120, 400),
                window=16, avg_budget=60, n_min=8, n_max=256, decode_steps=3)
    lengths = WL.prompt_lengths(w)
    L, B, H, Hq = w.n_layers, w.batch, w.n_kv_heads, w.n_q_heads
    tens = [WL.layer_tensors(w, l, DEV, lengths, stress=True) for l in range(L)]
    N = L * w.avg_budget * (H if head_level else 1)
    sess = XkvSession(L, Hq, H, d, w.window, w.pool_kernel, lengths, max_new_tokens=60, max_budget=w.n_max, total_budget=N,
                      curve_len=w.n_max, device=DEV, head_level=head_level, kv_format=xkv.KV_E4M3, pages_on_demand=on_demand)
    sess.score_layers([t[0] for t in tens], [t[1] for t in tens])
    budgets, _ = sess.solve_budgets(total=N, n_min=w.n_min, n_max=w.n_max)
    sess.assign_pages(budgets)
    planned = sess.seq_lens.cpu().numpy().copy()
    sel = torch.full((B, H, sess.max_seqlen), -1, dtype=torch.int32, device=DEV)
    ref = {}
    for l in range(L):
        sess.select_layer(l, budgets[l] if head_level else int(budgets[l]), tens[l][1], tens[l][2], sel=sel)
        torch.cuda.synchronize()
        assert sess.device_status("select") == xkv.OK
        lens = sess.seq_lens[l].cpu().numpy()
        if on_demand:
            assert np.array_equal(lens, planned[l])           # the tables were planned for what is then kept
        for b in range(B):
            lo = int(sess.cu_host[b])
            for g in range(H):
                kept = sel[b, g, : int(lens[b * H + g] if head_level else lens[b])].cpu().numpy()
                for x, t in (("k", tens[l][1]), ("v", tens[l][2])):
                    c = ref[l, b, g, x] = O.BlockCache(d)
                    c.append(O.evict_by_index(f64(t[lo: lo + lengths[b], g]), kept))

    def cached(l, b, g, x):
        ci, hp = (b * H + g, 0) if head_level else (b, g)
        n = int(sess.seq_lens[l, ci])
        s = np.arange(n)
        pg, off = sess.block_table[l, ci].cpu().numpy()[s // sess.page_size], s % sess.page_size
        codes, scales = ((sess.k_pages, sess.k_scales) if x == "k" else (sess.v_pages, sess.v_scales))
        return (O.e4m3_values(codes.cpu().numpy()[pg, hp, off]) *
                scales.cpu().numpy().astype(np.float64)[pg, hp, off // 16][:, None])

    if on_demand:                                             # a further turn of both conversations, then one of the second
        for n_new in ([5, 33], [0, 9]):
            T = sum(n_new)
            gen = torch.Generator().manual_seed(T)
            k, v = (torch.randn(L, T, H, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in "kv")
            sess.append(k, v, n_new)
            torch.cuda.synchronize()
            at = 0
            for b, n in enumerate(n_new):
                for l in range(L):
                    for g in range(H):
                        ref[l, b, g, "k"].append(f64(k[l, at:at + n, g]))
                        ref[l, b, g, "v"].append(f64(v[l, at:at + n, g]))
                at += n
        with pytest.raises(ValueError):
            sess.append(k, v, [1, 1])
    else:
        with pytest.raises(ValueError):
            sess.append(torch.zeros(L, 2, H, d, device=DEV), torch.zeros(L, 2, H, d, device=DEV), [1, 1])
    for step in range(w.decode_steps):
        q, kn, vn = WL.decode_tensors(w, step, DEV, stress=True)
        out = sess.decode(q, kn, vn)
        torch.cuda.synchronize()
        assert sess.device_status("decode") == xkv.OK and sess.device_status("append") == xkv.OK
        qf, of, lf = f64(q), f64(out), f64(sess.lse)
        for (l, b, g, x), c in ref.items():
            c.append(f64((kn if x == "k" else vn)[l, b, g])[None])
            assert np.array_equal(cached(l, b, g, x), c.values()), (step, l, b, g, x)
        for l in range(L):
            for b in range(B):
                for h in range(Hq):
                    check_decode(qf[l, b, h], ref[l, b, h // (Hq // H), "k"].values(),
                                 ref[l, b, h // (Hq // H), "v"].values(), 1 / math.sqrt(d), of[l, b, h], lf[l, b, h],
                                 f"step {step} {l} {b} {h}")
