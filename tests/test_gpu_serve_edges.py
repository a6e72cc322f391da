"""Serving on a reduced cache at the edges of what the entry points document."""
import math
import threading

import numpy as np
import pytest
import torch

from oracle import xkv_oracle as O
from paper_2412_05896_b200 import xkv

from gpu_util import f64, require_lib
from test_gpu_block_cache import BF16_HALF, DEV, Pool, check_plan, expect_store, plan, queries, run_decode, same, store

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    require_lib()


# ------------------------------------------------------------------ the plan of a step
HUGE = 2 ** 31 - 1


@pytest.mark.parametrize("L,B,stride", [(1, 5, 100), (3, 40, 1000), (3, 40, 9000), (2, 2500, 300), (40, 3, 64)])
@pytest.mark.parametrize("huge", [[HUGE], [2 ** 30, 2 ** 30], [HUGE, HUGE, HUGE]])
@pytest.mark.parametrize("per_layer", [False, True])
def test_plan_append_counts_that_no_cache_can_hold(monkeypatch, L, B, stride, huge, per_layer):
    """Counts up to 2^31 - 1: those caches keep their lengths, their tokens within the slot map get slot -1, every other
    cache gets its pages, also the ones whose tokens lie behind the map.  By one launch, by two, and by many blocks."""
    page, cols, clip = 16, 6, stride + 200                      # the definition walks its tokens: let it walk fewer
    define = O.plan_append
    monkeypatch.setattr(O, "plan_append", lambda new, *a: define(np.minimum(new, clip), *a))
    rng = np.random.default_rng(B + len(huge))
    lens = rng.integers(0, 40, (L, B))
    new = rng.integers(0, 4, (L, B) if per_layer else (B,))
    for i, n in enumerate(huge):
        new[..., B - len(huge) + i if B < 6 else B // 2 + 3 * i] = n
    n_pages = L * B * cols
    for kw in (dict(), dict(in_place=True), dict(free=rng.permutation(n_pages))):
        want, *got, status = plan(lens, new, page, cols, n_pages, used=2, slots_stride=stride, **kw)
        assert status == xkv.ERR_CAPACITY and not want[4]
        check_plan(want, *got)


@pytest.mark.parametrize("L,B", [(2, 30), (3, 1600)])
@pytest.mark.parametrize("stride", [1, 63, 64, 65, 700, 2500])
def test_plan_append_pages_of_tokens_behind_the_slot_map(L, B, stride):
    """Ragged prompts of which the slot map holds only the first tokens: all get their pages and lengths."""
    page, cols = 32, 12
    rng = np.random.default_rng(stride)
    lens = rng.integers(0, 70, (L, B))
    new = rng.integers(0, 300, (L, B))
    n_pages = L * B * cols
    want, *got, status = plan(lens, new, page, cols, n_pages, used=0, slots_stride=stride, free=rng.permutation(n_pages))
    assert status == xkv.ERR_CAPACITY and want[4]
    check_plan(want, *got)


@pytest.mark.parametrize("sizes", [((32, 128), (20, 130)), ((1, 16384), (1, 12000))])
def test_plan_append_from_two_host_threads(sizes):
    """Plans of different sizes from two threads, a stream and a workspace each: neither takes away the other's room."""
    page, cols, steps, errors = 16, 4, 1500, []

    def work(L, B):
        try:
            stream = torch.cuda.Stream(device=DEV)
            with torch.cuda.stream(stream):
                lens = torch.full((L, B), 15, dtype=torch.int32, device=DEV)
                after, table = torch.zeros_like(lens), torch.zeros(L, B, cols, dtype=torch.int32, device=DEV)
                new = torch.ones(B, dtype=torch.int32, device=DEV)
                dims = xkv.Dims(B, 1, 1, 64, 1, 1, 0, 0.0, 64, 64)
                ws = torch.zeros(xkv.workspace_bytes(xkv.OP_PLAN_APPEND, dims, n_layers=L), dtype=torch.uint8, device=DEV)
            cache = xkv.Cache(None, None, table.data_ptr(), after.data_ptr(), L, page, cols, L * B * cols)
            for _ in range(steps):
                xkv.plan_append(cache, B, new, 0, lens, None, L * B * cols, None, None, None, 0, ws, stream=stream)
            assert xkv.read_device_status(ws, stream=stream) == xkv.OK
            assert torch.all(after == 16)
        except Exception as e:                                  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=s) for s in sizes]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


# ------------------------------------------------------------------ V scales far apart
def check_products(q, K, codes, scales, out, lse, what):
    """One head's output where a cache's V scales differ: V = codes * scales[:, None].

    As check_decode, but the bound's floor goes by the weights times their rows' scales, not by the largest |V|: such a
    product enters as two codes, within 2^-8 of itself or, where it is small, within half a step of the smallest second
    code, 2^-10 / 32 in units of which 256 stand for the tile's largest product: 2^-23 of that."""
    z = K @ q / math.sqrt(len(q))
    m = z.max()
    p = np.exp(z - m)
    y = p * scales
    ref = (y @ codes) / p.sum()
    mag = (y @ np.abs(codes)) / p.sum()
    absqk = np.abs(K) @ np.abs(q) / math.sqrt(len(q))
    dz = (len(q) + 8) * 2.0 ** -23 * absqk.max() + 2.0 ** -21 * np.abs(q).max() * np.abs(K).sum(1).max() / math.sqrt(len(q))
    floor = 2.0 ** -23 * y.max() * np.abs(codes).sum(0) / p.sum()
    bound = (2 * dz + BF16_HALF + 2.0 ** -20) * mag + floor + BF16_HALF * np.abs(ref) + 1e-35
    assert np.all(np.isfinite(out)), what
    worst = (np.abs(out - ref) / bound).max()
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"
    want = m + math.log(p.sum())
    assert abs(lse - want) <= dz + 2.0 ** -21 * (1 + abs(want)), f"{what}: lse {lse} for {want}"


def check_scales(pool, Hq, q, out, lse, what, lens=None):
    G, qf, of, lf = Hq // pool.H, f64(q), f64(out), f64(lse)
    s = pool.dev_s["v"].cpu().numpy().astype(np.float64)
    for l in range(pool.L):
        for b in range(pool.B):
            n = np.arange(int((pool.lens if lens is None else lens)[l, b]))
            for g in range(pool.H):
                sv = s[pool.table[l, b, n // pool.page], g, n % pool.page // 16]
                K, V = pool.rows("k", l, b, g, len(n)), pool.rows("v", l, b, g, len(n))
                codes = V / np.where(sv > 0, sv, 1.0)[:, None]
                for h in range(g * G, (g + 1) * G):
                    check_products(qf[l, b, h], K, codes, sv, of[l, b, h], lf[l, b, h], f"{what} l{l} b{b} h{h}")


@pytest.mark.parametrize("d,G", [(128, 1), (128, 2), (128, 4), (128, 7), (64, 1), (64, 2), (64, 3), (64, 8)])
@pytest.mark.parametrize("logit", [-40.0, 0.0, 15.0])
def test_decode_scales_far_apart_in_a_tile(d, G, logit):
    """Blocks whose V scales are up to 2^60 times the others' and whose weights are e^-40, alike, or e^15 times theirs: what
    such rows do not weigh costs the others no bits."""
    H, page = 2, 32
    pool = Pool([[128, 33, 300], [600, 17, 200]], H, d, page, seed=G, spread=0)
    codes, ks, vs = (t.cpu().numpy() for t in (pool.dev["k"], pool.dev_s["k"], pool.dev_s["v"]))
    high = Pool._bytes(np.array([256.0]))[0]
    for l in range(2):
        for b in range(3):
            for i in range(0, int(pool.lens[l, b]), 16):
                pg, at = pool.table[l, b, i // page], i % page
                codes[pg, :, at:at + 16, 0] = 0
                if i // 16 % 5 == 1:                            # every fifth block: element 0 of its keys draws the logit
                    ks[pg, :, at // 16] = 1.0
                    codes[pg, :, at:at + 16] = 0
                    vs[pg, :, at // 16] *= 2.0 ** [4, 5, 8, 12, 16, 20, 24, 60][(i // 80 + b) % 8]
                    codes[pg, :, at:at + 16, 0] = high
                elif i // 16 % 5 == 3:
                    vs[pg, :, at // 16] *= 2.0 ** -6
    for t, x in ((pool.dev["k"], codes), (pool.dev_s["k"], ks), (pool.dev_s["v"], vs)):
        t.copy_(torch.from_numpy(x))
    q = queries(2, 3, H * G, d, G, size=0.25)
    q[..., 0] = math.sqrt(d) * logit / 256.0
    out, lse, st = run_decode(pool, H * G, q)
    assert st == xkv.OK
    check_scales(pool, H * G, q, out, lse, f"d{d} G{G} logit {logit}")


@pytest.mark.parametrize("d,G", [(128, 1), (128, 8), (64, 2), (64, 4)])
def test_decode_scales_of_zero_and_at_both_ends(d, G):
    """Blocks of scale 0, 2^-100 and 2^100 next to ordinary ones, and caches that hold nothing but blocks of scale 0."""
    pool = Pool([[128, 300, 40], [256, 16, 77]], 2, d, 16, seed=G)
    vs = pool.dev_s["v"].cpu().numpy()
    for b in range(3):
        for i in range(-(-int(pool.lens[0, b]) // 16)):
            vs[pool.table[0, b, i]] *= [1.0, 0.0, 2.0 ** -93, 1.0, 2.0 ** 100][i % (5 if b == 0 else 4)]
    vs[pool.table[1, 1]] = 0.0
    pool.dev_s["v"].copy_(torch.from_numpy(vs))
    q = queries(2, 3, 2 * G, d, G)
    out, lse, st = run_decode(pool, 2 * G, q)
    assert st == xkv.OK
    check_scales(pool, 2 * G, q, out, lse, f"d{d} G{G}")


# ------------------------------------------------------------------ NaN in cached rows
@pytest.mark.parametrize("d,G", [(128, 1), (128, 2), (128, 4), (128, 8), (64, 1), (64, 3)])
def test_decode_nan_in_cached_rows(d, G):
    """A NaN in a row of K makes that KV head's outputs and lse NaN, one in a row of V that column of its outputs; nothing
    else moves by a bit.  First, middle and last rows; caches of one tile, of several, and cut ones."""
    H, page = 2, 16
    pool = Pool([[5, 700, 6000], [130, 1, 259]], H, d, page, seed=G + d)
    q = queries(2, 3, H * G, d, G)
    want, want_lse, st = run_decode(pool, H * G, q)
    assert st == xkv.OK
    clean = {x: pool.dev[x].clone() for x in "kv"}
    for x, code in (("k", 0x7F), ("k", 0xFF), ("v", 0x7F), ("v", 0xFF)):
        nan, nan_lse = torch.zeros_like(want, dtype=torch.bool), torch.zeros_like(want_lse, dtype=torch.bool)
        for l, b, g, row, col in ((0, 0, 1, 4, 0), (0, 1, 0, 0, d - 1), (0, 2, 1, 3001, 17), (1, 0, 0, 129, 5), (1, 2, 1, 0, 31),
                                  (1, 2, 1, 258, 33)):
            pool.dev[x][pool.table[l, b, row // page], g, row % page, col] = code
            if x == "k":
                nan[l, b, g * G:(g + 1) * G] = nan_lse[l, b, g * G:(g + 1) * G] = True
            else:
                nan[l, b, g * G:(g + 1) * G, col] = True
        out, lse, st = run_decode(pool, H * G, q)
        assert st == xkv.OK
        assert torch.equal(torch.isnan(out), nan) and torch.equal(torch.isnan(lse), nan_lse), (x, code)
        assert torch.equal(out[~nan], want[~nan]) and torch.equal(lse[~nan_lse], want_lse[~nan_lse]), (x, code)
        pool.dev[x].copy_(clean[x])
    pool.dev["k"][pool.table[0, 2, 10:30]] = 0x7F            # whole tiles of them
    pool.dev["k"][pool.table[1, 0]] = 0x7F                   # a whole cache
    out, lse, st = run_decode(pool, H * G, q)
    assert st == xkv.OK and torch.isnan(out[0, 2]).all() and torch.isnan(lse[0, 2]).all() and torch.isnan(out[1, 0]).all()
    assert torch.equal(out[0, :2], want[0, :2]) and torch.equal(out[1, 1:], want[1, 1:])


# ------------------------------------------------------------------ rows stored by slot
@pytest.mark.parametrize("gap", [1, 2, 15, 31])
@pytest.mark.parametrize("d,H,many", [(64, 1, 0), (128, 8, 0), (128, 8, 600), (64, 16, 2400)])
def test_store_rows_padding_inside_a_block(gap, d, H, many):
    """Padding between two tokens of one block: the second is not stored, nor the rest of its run, and the status says so;
    padding between tokens of different blocks is nothing special.  A token, four and sixteen of them a warp."""
    page = 32
    pool = Pool([[7, 20] + [3] * 40], H, d, page, seed=gap, spare_rows=80, any_code=True)
    at = lambda b, i: int(pool.table[0, b, i // page]) * page + i % page         # noqa: E731
    slots = [at(0, 7), at(0, 8)] + [-1] * gap + [at(0, 9), at(0, 10)] + [-1] * gap + [at(1, 20)]
    slots += [at(2 + i % 40, 3 + j) for i in range(40) for j in range(many // 40)]
    kept = list(slots)
    kept[2 + gap] = kept[3 + gap] = -1
    slots, kept = (np.asarray(x, dtype=np.int64) for x in (slots, kept))
    gen = torch.Generator().manual_seed(gap)
    k, v = (torch.randn(len(slots), H, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in "kv")
    want = {x: expect_store(pool, x, f64(t), kept) for x, t in (("k", k), ("v", v))}
    assert store(pool, k, v, torch.from_numpy(slots).to(DEV)) == xkv.ERR_INVALID_ARG
    for x in "kv":
        assert same(O.e4m3_values(pool.dev[x].cpu().numpy()), want[x][0]), x
        assert same(pool.dev_s[x].cpu().numpy().astype(np.float64), want[x][1]), x


def test_store_rows_behind_padding():
    """Left-padded sequences: a run in the middle of a block behind padding is stored as ever."""
    d, H, page = 64, 2, 16
    pool = Pool([[5, 9, 33]], H, d, page, seed=1, spare_rows=20, any_code=True)
    slots = np.concatenate([np.concatenate([np.full(pad, -1), pool.table[0, b, (n + np.arange(6)) // page] * page +
                                            (n + np.arange(6)) % page])
                            for b, (n, pad) in enumerate(((5, 3), (9, 40), (33, 1)))]).astype(np.int64)
    gen = torch.Generator().manual_seed(2)
    k, v = (torch.randn(len(slots), H, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in "kv")
    want = {x: expect_store(pool, x, f64(t), slots) for x, t in (("k", k), ("v", v))}
    assert store(pool, k, v, torch.from_numpy(slots).to(DEV)) == xkv.OK
    for x in "kv":
        assert same(O.e4m3_values(pool.dev[x].cpu().numpy()), want[x][0]), x
        assert same(pool.dev_s[x].cpu().numpy().astype(np.float64), want[x][1]), x


# ------------------------------------------------------------------ sessions with pages on demand
def _session(head_level, fmt, steps=12, on_demand=True):
    from dataclasses import replace

    from paper_2412_05896_b200 import workloads as WL
    from paper_2412_05896_b200.pipeline import XkvSession
    w = replace(WL.CONFIGS["mistral_7b_gqa"], n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=64, batch=3, prompt=(90, 300),
                window=16, avg_budget=50, n_min=8, n_max=128, decode_steps=steps)
    lengths = WL.prompt_lengths(w)
    tens = [WL.layer_tensors(w, l, DEV, lengths, stress=True) for l in range(w.n_layers)]
    N = w.n_layers * w.avg_budget * (2 if head_level else 1)
    sess = XkvSession(2, 4, 2, 64, w.window, w.pool_kernel, lengths, max_new_tokens=80, max_budget=w.n_max, total_budget=N,
                      curve_len=w.n_max, device=DEV, head_level=head_level, kv_format=fmt, pages_on_demand=on_demand)
    sess.prefill(*(list(x) for x in zip(*tens)), total=N, n_min=w.n_min, n_max=w.n_max)
    torch.cuda.synchronize()
    return w, sess, [WL.decode_tensors(w, i, DEV, stress=True) for i in range(steps)]


def _counts_to_append(sess, w, seed):
    n_new = [3, 0, 21]
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(2, sum(n_new), 2, 64, generator=gen).to(torch.bfloat16).to(DEV) for _ in "kv"] + [n_new]


@pytest.mark.parametrize("fmt", [xkv.KV_E4M3, xkv.KV_BF16])
@pytest.mark.parametrize("head_level", [False, True])
def test_session_steps_in_a_graph(head_level, fmt):
    """A captured step of a session with pages on demand, replayed, against the same steps of a twin without a graph; every
    page of the caches grows on the way."""
    w, sess, steps = _session(head_level, fmt, steps=20)
    _, twin, _ = _session(head_level, fmt, steps=1)
    q, k, v = (x.clone() for x in steps[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sess.decode(q, k, v)
    torch.cuda.synchronize()
    assert torch.equal(sess.seq_lens, twin.seq_lens)            # nothing ran yet
    for step in steps:
        for t, x in zip((q, k, v), step):
            t.copy_(x)
        graph.replay()
        want = twin.decode(*step)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(sess.lse, twin.lse) and torch.equal(sess.seq_lens, twin.seq_lens)
    assert torch.equal(sess.block_table, twin.block_table) and torch.equal(sess.pages_used, twin.pages_used)
    assert sess.device_status("append") == xkv.OK and sess.device_status("decode") == xkv.OK


@pytest.mark.parametrize("head_level", [False, True])
def test_session_does_not_wait_for_the_device(head_level):
    w, sess, steps = _session(head_level, xkv.KV_E4M3)
    k, v, n_new = _counts_to_append(sess, w, 5)
    before = sess.seq_lens.clone()
    torch.cuda.synchronize()
    torch.cuda.set_sync_debug_mode("error")
    try:
        sess.append(k, v, n_new)
        sess.decode(*steps[0])
        sess.append(k[:, :3], v[:, :3], [0, 3, 0])
        sess.decode(*steps[1])
    finally:
        torch.cuda.set_sync_debug_mode("default")
    torch.cuda.synchronize()
    assert sess.device_status("append") == xkv.OK
    grown = torch.tensor([5, 5, 23], dtype=torch.int32, device=DEV)
    assert torch.equal(sess.seq_lens, before + (grown.repeat_interleave(2) if head_level else grown))


def test_session_refuses_rows_of_another_type_or_shape():
    w, sess, steps = _session(False, xkv.KV_E4M3, steps=1)
    q, k, v = steps[0]
    before = sess.seq_lens.clone()
    for bad in ((k.float(), v), (k, v.half()), (k, None), (k.cpu(), v), (k[:, :2], v[:, :2]), (k, v.view(torch.uint8))):
        with pytest.raises(ValueError):
            sess.decode(q, *bad)
        with pytest.raises(ValueError):
            sess.append(*bad, [1, 1, 1])
    for bad in ([1, 1], [1, -1, 3], [[1, 1, 1]]):
        with pytest.raises(ValueError):
            sess.append(k, v, bad)
    assert torch.equal(sess.seq_lens, before) and sess.device_status("append") == xkv.OK


def test_session_budgets_beyond_the_pool():
    """Refused on the host; the caches that live in the pool stay as they are."""
    w, sess, steps = _session(False, xkv.KV_E4M3, steps=1)
    pages, lens = sess.k_pages.clone(), sess.seq_lens.clone()
    sess.n_pages = int(sess.pages_used.item())                  # as many as the budgets so far took
    with pytest.raises(RuntimeError, match="page pool too small"):
        sess.assign_pages(np.asarray(sess.budgets) + 40)
    assert torch.equal(sess.k_pages, pages) and torch.equal(sess.seq_lens, lens)


@pytest.mark.parametrize("on_demand", [False, True])
def test_session_page_runs_of_two_requests_in_flight(on_demand):
    """Pages assigned for one request and then for the next while the device is still busy: each gets its own."""
    w, sess, _ = _session(False, xkv.KV_E4M3, steps=1, on_demand=on_demand)
    one, two = np.array([20, 70]), np.array([60, 9])
    seen = []
    for busy in (False, True):
        sess.block_table.fill_(-1)
        sess.seq_lens.fill_(-1)
        torch.cuda.synchronize()
        if busy:
            torch.cuda._sleep(200_000_000)                      # a tenth of a second of device time
        for budgets in (one, two):
            sess.assign_pages(budgets)
            seen.append((sess.block_table.clone(), sess.seq_lens.clone()))
            if not busy:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
    for a, b in zip(seen[:2], seen[2:]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ attention with the step's new rows in the call
@pytest.mark.parametrize("d,G", [(128, 4), (64, 1), (128, 7)])
def test_decode_with_new_rows_in_a_graph(d, G):
    """A captured call that appends, replayed right behind the kernels that write its inputs, against calls on a twin cache;
    one cache is full from the start, one becomes full on the way."""
    H, page = 2, 16
    lens = [[0, 15, 2500, 40], [300, 2505, 16, 2512]]           # 157 pages a table: 2512 rows
    pools = [Pool(lens, H, d, page, seed=d + G) for _ in range(2)]
    assert pools[0].cols * page == 2512
    dims = xkv.Dims(4, H * G, H, d, 1, 1, 0, 0.0, H * d, d)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DECODE_ATTN, dims, n_layers=2, max_cache_len=2512), dtype=torch.uint8,
                     device=DEV)
    q, kn, vn = (torch.zeros(2, 4, n, d, dtype=torch.bfloat16, device=DEV) for n in (H * G, H, H))
    out, lse = torch.zeros_like(q), torch.zeros(2, 4, H * G, device=DEV)
    handle = pools[0].handle()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xkv.decode_attn(dims, handle, 0, 2, q, kn, vn, out, lse, 0, ws)
    assert pools[0].seq_lens.tolist() == lens
    for step in range(10):
        gen = torch.Generator(device=DEV).manual_seed(step)
        for t in (q, kn, vn):
            t.copy_(torch.randn(t.shape, generator=gen, device=DEV).to(torch.bfloat16))
        graph.replay()
        got, got_lse = out.clone(), lse.clone()
        want, want_lse, status = run_decode(pools[1], H * G, q, kn=kn, vn=vn)
        assert status == xkv.ERR_CAPACITY and xkv.read_device_status(ws) == xkv.ERR_CAPACITY
        assert torch.equal(got, want) and torch.equal(got_lse, want_lse), step
        for x in "kv":
            assert torch.equal(pools[0].dev[x], pools[1].dev[x])
            assert torch.equal(pools[0].dev_s[x].view(torch.int32), pools[1].dev_s[x].view(torch.int32))
        grown = np.minimum(np.asarray(lens) + step + 1, 2512)
        assert np.array_equal(pools[0].seq_lens.cpu().numpy(), grown)
        check_scales(pools[0], H * G, q, got, got_lse, f"step {step}", grown)
