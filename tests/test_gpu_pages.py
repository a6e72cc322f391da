"""Pages copied, shared, given back and moved: state and bytes against the plain definitions, over random histories and at
the edges (empty caches, whole last pages, pages shared three ways, lists that end, ids outside the pool)."""
import numpy as np
import pytest
import torch

from oracle import xkv_oracle as O
from paper_2412_05896_b200 import xkv

from gpu_util import require_lib

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMATS = {"bf16": xkv.KV_BF16, "int8": xkv.KV_INT8, "e4m3": xkv.KV_E4M3}


class PagePool:
    """A pool of random pages with tables, a free list and counters on the device and their plain copies on the host."""

    def __init__(self, L, B, H, d, page, cols, n_pages, fmt="bf16", seed=0, lens=None):
        require_lib()
        g = torch.Generator().manual_seed(seed)
        self.L, self.B, self.H, self.d, self.page, self.cols, self.n_pages, self.fmt = L, B, H, d, page, cols, n_pages, fmt
        dtype = torch.int16 if fmt == "bf16" else torch.uint8
        self.pages = [torch.randint(0, 200, (n_pages, H, page, d), generator=g).to(dtype).to(DEV) for _ in range(2)]
        n_scales = {"bf16": 0, "int8": page, "e4m3": page // 16}[fmt]
        self.scales = [torch.rand(n_pages, H, n_scales, generator=g).to(DEV) if n_scales else None for _ in range(2)]
        rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens if lens is not None else rng.integers(0, cols * page + 1, (L, B)), dtype=np.int32)
        order = rng.permutation(n_pages).astype(np.int32)
        self.table, self.used = np.full((L, B, cols), -7, dtype=np.int32), 0
        for l in range(L):
            for b in range(B):
                n = -(-int(self.lens[l, b]) // page)
                self.table[l, b, :n] = order[self.used:self.used + n]
                self.used += n
        assert self.used <= n_pages
        self.free, self.shares = order, np.zeros(n_pages, dtype=np.int32)
        ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)        # noqa: E731
        self.d_table, self.d_lens, self.d_free, self.d_shares = map(ints, (self.table, self.lens, self.free, self.shares))
        self.d_used = ints(np.array([self.used], dtype=np.int32))
        self.dims = xkv.Dims(B, H, H, d, 1, 1, 0, 0.0, H * d, d)
        ptr = lambda t: None if t is None else t.data_ptr()                       # noqa: E731
        self.cache = xkv.Cache(ptr(self.pages[0]), ptr(self.pages[1]), self.d_table.data_ptr(), self.d_lens.data_ptr(), L, page,
                               cols, n_pages, ptr(self.scales[0]), ptr(self.scales[1]), FORMATS[fmt], 0)
        size = lambda op: xkv.workspace_bytes(op, self.dims, max_seqlen=cols, total_tokens=n_pages, n_layers=L)   # noqa: E731
        self.ws_fork = torch.zeros(size(xkv.OP_FORK_CACHES), dtype=torch.uint8, device=DEV)
        self.ws_compact = torch.zeros(size(xkv.OP_COMPACT_PAGES), dtype=torch.uint8, device=DEV)

    def expect_copies(self, copies):
        """What pages and scales hold after row copies [(from, to, rows)] that do not depend on each other."""
        want = [t.clone() for t in self.pages + [s for s in self.scales if s is not None]]
        now = self.pages + [s for s in self.scales if s is not None]
        for w, t in zip(want, now):
            per = self.page // t.shape[2]
            for a, b, rows in copies:
                n = -(-rows // per)
                w[b, :, :n] = t[a, :, :n]
        return want

    def check(self, want_pages, status=xkv.OK, ws=None):
        torch.cuda.synchronize()
        assert xkv.read_device_status(ws if ws is not None else self.ws_fork) == status
        for name in ("table", "lens", "shares", "free"):
            got = getattr(self, "d_" + name).cpu().numpy()
            assert np.array_equal(got, getattr(self, name)), name
        assert int(self.d_used) == self.used
        now = self.pages + [s for s in self.scales if s is not None]
        for w, t in zip(want_pages, now):
            assert torch.equal(w, t)

    def fork(self, parent, keep=None, stride=None, status=xkv.OK, n_free=None):
        par = torch.tensor(list(parent), dtype=torch.int32, device=DEV)
        k = None if keep is None else torch.tensor(np.asarray(keep), dtype=torch.int32, device=DEV).contiguous()
        full = None if keep is None else np.broadcast_to(np.asarray(keep), (self.L, self.B))
        n_free = len(self.free) if n_free is None else n_free
        self.table, self.lens, shares, free, self.used, copies, ok = O.fork_caches(
            parent, full, self.lens, self.table, self.page, self.shares, self.free[:n_free], self.used)
        self.shares = shares.astype(np.int32)
        self.free = np.concatenate([free, self.free[n_free:]]).astype(np.int32)
        want = self.expect_copies(copies)
        xkv.fork_caches(self.dims, self.cache, par, k, (0 if k is None or k.dim() == 1 else self.B) if stride is None else stride,
                        self.d_shares, self.d_free, n_free, self.d_used, self.ws_fork)
        self.check(want, status if status != xkv.OK else (xkv.OK if ok else xkv.ERR_CAPACITY))
        return copies

    def compact(self, in_place=True):
        before = self.d_table if in_place else self.d_table.clone()
        shares_before = self.d_shares if in_place else self.d_shares.clone()
        if not in_place:
            self.d_table.fill_(99)
            self.d_shares.fill_(99)
        self.table, self.shares, n_live, moves = O.compact_pages(self.table, self.lens, self.page, self.shares, self.n_pages)
        self.table, self.shares = self.table.astype(np.int32), self.shares.astype(np.int32)
        self.free = self.free.copy()
        self.free[n_live:] = np.arange(n_live, self.n_pages)
        self.used = n_live
        want = self.expect_copies([(a, b, self.page) for a, b in moves.items()])
        xkv.compact_pages(self.dims, self.cache, before, shares_before, self.d_shares, self.d_free, self.d_used, self.ws_compact)
        self.check(want, ws=self.ws_compact)
        return n_live, moves

    def grow(self, n_new):
        """n_new [B] more rows of every cache of every layer, by xkv_plan_append (bytes of the new rows do not matter here)."""
        new = torch.tensor(list(n_new), dtype=torch.int32, device=DEV)
        ws = torch.zeros(xkv.workspace_bytes(xkv.OP_PLAN_APPEND, self.dims, n_layers=self.L), dtype=torch.uint8, device=DEV)
        counts = np.broadcast_to(np.asarray(n_new), (self.L, self.B))
        self.table, self.lens, _, self.used, ok = O.plan_append(counts, self.lens, self.table, self.page, self.free, self.used)
        assert ok
        xkv.plan_append(self.cache, self.B, new, 0, self.d_lens, self.d_free, self.n_pages, self.d_used, self.d_used, None, 0, ws)
        self.check([t.clone() for t in self.pages], ws=ws)


SHAPES = [  # L, B, H, d, page, cols, format
    (1, 1, 1, 64, 16, 1, "bf16"),
    (2, 3, 2, 64, 16, 5, "int8"),
    (3, 8, 4, 128, 48, 4, "e4m3"),
    (5, 33, 1, 128, 256, 3, "bf16"),
    (32, 70, 1, 64, 16, 9, "int8"),
    (2, 300, 2, 64, 32, 2, "e4m3"),
]


@pytest.mark.parametrize("L,B,H,d,page,cols,fmt", SHAPES)
def test_random_histories(L, B, H, d, page, cols, fmt):
    rng = np.random.default_rng(L * 100 + B)
    lens = rng.integers(0, cols * page * 3 // 4 + 1, (L, B))
    pool = PagePool(L, B, H, d, page, cols, 2 * L * B * cols + 9, fmt, seed=B, lens=lens)
    for step in range(8):
        kind = step % 4
        me = np.arange(B)
        if kind == 0:                                       # forks of a few
            parent, keep = np.where(rng.random(B) < 0.6, rng.integers(0, B, B), me), None
        elif kind == 1:                                     # cut, some freed
            parent, keep = np.where(rng.random(B) < 0.2, -1, me), rng.integers(-1, cols * page + 2, (L, B))
        elif kind == 2:                                     # everything at once, the same counts for all layers
            parent, keep = rng.integers(-1, B, B), rng.integers(0, cols * page + 2, B)
        else:                                               # a beam step: forks only
            parent, keep = rng.integers(0, B, B), None
        pool.fork(parent.tolist(), keep)
        if step in (2, 5):
            n_live, _ = pool.compact(in_place=step == 2)
            assert n_live <= pool.n_pages
        room = cols * page - pool.lens.max(0)
        pool.grow(np.minimum(room, rng.integers(0, page + 1, B)))
    pool.fork([-1] * B)
    assert pool.used == 0 and not pool.shares.any() and sorted(pool.free.tolist()) == list(range(pool.n_pages))


def test_forks_share_whole_pages_and_copy_the_last_rows():
    lens = np.array([[37, 0, 0, 32], [16, 0, 0, 5]])
    pool = PagePool(2, 4, 2, 64, 16, 4, 40, lens=lens)
    copies = pool.fork([0, 0, 0, 3])
    assert [c[2] for c in copies] == [5, 5]                 # two forks of 37 rows; of 16 rows nothing is copied
    assert pool.shares.max() == 2 and pool.used == 3 + 2 + 1 + 1 + 2
    assert not pool.fork([0, 1, 2, 3])                      # nothing changes
    assert not pool.fork([0, -1, -1, 3]) and pool.used == 3 + 2 + 1 + 1 and not pool.shares.any()
    # a cut of a fork inside a page that its parent holds whole is copied, of the only holder not
    pool.fork([0, 0, 2, 3])
    assert [c[2] for c in pool.fork([0, 1, 2, 3], [-1, 20, 0, 20])] == [4]
    # parent and fork cut at different places of the same page: the one that stays keeps it
    pool.fork([0, 0, -1, 3])
    assert [c[2] for c in pool.fork([0, 1, 2, 3], [19, 23, -1, -1])] == [7]
    # a swap moves pages, copies nothing
    assert not pool.fork([1, 0, 3, 2])


def test_a_page_that_all_holders_leave_goes_to_one_of_them():
    pool = PagePool(1, 5, 1, 64, 16, 3, 30, lens=np.array([[20, 0, 0, 0, 0]]))
    assert len(pool.fork([-1, 0, 0, 0, 0])) == 3            # the parent is gone: cache 1 keeps its last page
    assert pool.table[0, 1, 1] == pool.table[0, 0, 1]


@pytest.mark.parametrize("room", [0, 1, 2])
def test_a_list_that_ends(room):
    pool = PagePool(2, 4, 1, 64, 16, 3, 30, lens=np.array([[20, 0, 0, 0], [33, 0, 0, 0]]))
    pool.fork([0, 0, 0, 0], n_free=pool.used + room, status=xkv.ERR_CAPACITY)
    assert (pool.lens[0] == 16).sum() == 3 - room and (pool.lens[1] == 32).sum() == 3    # whole pages only stay
    pool.fork([0, -1, -1, -1])
    assert not pool.shares.any()


def test_bad_parents_and_page_ids_are_reported():
    pool = PagePool(1, 3, 1, 64, 16, 3, 20, lens=np.array([[20, 7, 0]]))
    want = [t.clone() for t in pool.pages]
    par = torch.tensor([5, -3, 2], dtype=torch.int32, device=DEV)          # both are taken as the cache itself
    xkv.fork_caches(pool.dims, pool.cache, par, None, 0, pool.d_shares, pool.d_free, 20, pool.d_used, pool.ws_fork)
    pool.check(want, xkv.ERR_INVALID_ARG)
    bad = pool.d_table.clone()
    bad[0, 0, 0] = 20
    bad[0, 1, 0] = -1
    pool.d_table.copy_(bad)
    par = torch.tensor([0, 1, 0], dtype=torch.int32, device=DEV)
    xkv.fork_caches(pool.dims, pool.cache, par, None, 0, pool.d_shares, pool.d_free, 20, pool.d_used, pool.ws_fork)
    torch.cuda.synchronize()
    assert xkv.read_device_status(pool.ws_fork) == xkv.ERR_INVALID_ARG
    xkv.compact_pages(pool.dims, pool.cache, pool.d_table, pool.d_shares, pool.d_shares, None, pool.d_used, pool.ws_compact)
    torch.cuda.synchronize()
    assert xkv.read_device_status(pool.ws_compact) == xkv.ERR_INVALID_ARG
    assert int(pool.d_table[0, 0, 0]) == 20 and int(pool.d_table[0, 1, 0]) == -1


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("n", [1, 5, 300])
def test_copy_pages(fmt, n):
    H, d, page = (3, 64, 48) if n != 300 else (8, 128, 16)
    a = PagePool(1, 1, H, d, page, 1, n + 4, fmt, seed=1, lens=[[0]])
    b = PagePool(1, 1, H, d, page, 1, n + 2, fmt, seed=2, lens=[[0]])
    rng = np.random.default_rng(n)
    src, dst = rng.permutation(n + 4)[:n].astype(np.int32), rng.permutation(n + 2)[:n].astype(np.int32)
    live = np.ones(n, dtype=bool)
    if n > 1:                                               # ids outside their pools leave their pair out
        src[0], dst[1] = n + 4, -1
        live[:2] = False
    want = [t.clone() for t in b.pages + [s for s in b.scales if s is not None]]
    for w, t in zip(want, a.pages + [s for s in a.scales if s is not None]):
        w[torch.from_numpy(dst[live]).long().to(DEV)] = t[torch.from_numpy(src[live]).long().to(DEV)]
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_COPY_PAGES, a.dims), dtype=torch.uint8, device=DEV)
    xkv.copy_pages(a.dims, a.cache, torch.from_numpy(src).to(DEV), b.cache, torch.from_numpy(dst).to(DEV), n, ws)
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) == (xkv.OK if n == 1 else xkv.ERR_INVALID_ARG)
    for w, t in zip(want, b.pages + [s for s in b.scales if s is not None]):
        assert torch.equal(w, t)


def test_large_pool():
    """More pages than one CTA maps in shared memory, more table entries than one cluster handles."""
    rng = np.random.default_rng(5)
    L, B, page, cols = 6, 40, 16, 300
    pool = PagePool(L, B, 1, 64, page, cols, 60000, lens=rng.integers(0, cols * page // 2, (L, B)))
    pool.fork([int(b) for b in rng.integers(-1, B, B)])
    n_live, moves = pool.compact()
    assert moves and n_live < pool.n_pages
    pool.fork(list(range(B)), rng.integers(0, cols * page // 2, (L, B)))
    pool.compact(in_place=False)
    assert not pool.compact()[1]                            # nothing is left to move


def test_captured_and_replayed():
    pool = PagePool(4, 6, 2, 64, 16, 4, 200, lens=np.tile([[50, 0, 0, 33, 0, 0]], (4, 1)))
    fork = torch.tensor([0, 0, 0, 3, 3, 3], dtype=torch.int32, device=DEV)
    drop = torch.tensor([0, -1, -1, 3, -1, -1], dtype=torch.int32, device=DEV)

    def step():
        for par in (fork, drop):
            xkv.fork_caches(pool.dims, pool.cache, par, None, 0, pool.d_shares, pool.d_free, 200, pool.d_used, pool.ws_fork)

    step()                                                  # takes pages as the list has them, returns them in ascending order
    step()                                                  # takes and returns those: from here on a step repeats itself
    torch.cuda.synchronize()
    state = [t.clone() for t in (pool.d_table, pool.d_lens, pool.d_shares, pool.d_free, pool.d_used)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(20):
        graph.replay()
    torch.cuda.synchronize()
    assert xkv.read_device_status(pool.ws_fork) == xkv.OK
    for was, t in zip(state, (pool.d_table, pool.d_lens, pool.d_shares, pool.d_free, pool.d_used)):
        assert torch.equal(was, t)
