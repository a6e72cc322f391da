"""Workspaces of the page operators that have served something else before: only the header has to be as the last call left it."""
import numpy as np
import pytest
import torch

from paper_2412_05896_b200 import xkv

from gpu_util import require_lib
from test_gpu_pages import DEV, PagePool

pytestmark = pytest.mark.gpu
HEADER = 256


def shared_workspace(pools):
    size = max(max(p.ws_fork.numel(), p.ws_compact.numel()) for p in pools)
    ws = torch.zeros(size, dtype=torch.uint8, device=DEV)
    for p in pools:
        p.ws_fork = p.ws_compact = ws
    return ws


def steps(pool, rng, between):
    """Forks, cuts, frees and compactions, every state against its definition; between() before each call."""
    L, B, most = pool.L, pool.B, pool.cols * pool.page
    for parent, keep in ((rng.integers(-1, B, B), None), (np.arange(B), rng.integers(-1, most, (L, B))),
                         (np.where(rng.random(B) < 0.3, -1, np.arange(B)), None)):
        between()
        pool.fork([int(b) for b in parent], keep)
        between()
        pool.compact(in_place=keep is None)


# small pools are planned by one CTA; of the others one or both operators take several launches; pools that end inside a word of
# a bit a page
@pytest.mark.parametrize("L,B,cols,n_pages", [(2, 5, 4, 77), (3, 50, 8, 20011), (4, 40, 150, 33003), (4, 40, 150, 60000)])
@pytest.mark.parametrize("fill", [0xFF, 0x7F, 0x01])
def test_whatever_lies_behind_the_header(L, B, cols, n_pages, fill):
    rng = np.random.default_rng(n_pages)
    pool = PagePool(L, B, 1, 64, 16, cols, n_pages, "int8", seed=1, lens=rng.integers(0, cols * 16 * 2 // 3, (L, B)))
    ws = shared_workspace([pool])

    def between():
        ws[HEADER:] = fill

    steps(pool, rng, between)


def test_one_workspace_for_pools_of_any_size():
    """Pools in turn, smaller and larger, on both sides of what one CTA plans; step plans use the workspace as well."""
    sizes = [(2, 5, 4, 77), (4, 40, 150, 60000), (3, 50, 8, 40000), (3, 50, 8, 20011), (2, 70, 20, 9001), (4, 40, 150, 33003)]
    rng = np.random.default_rng(0)
    pools = [PagePool(L, B, 1, 64, 16, cols, n, "int8", seed=n, lens=rng.integers(0, cols * 16 * 2 // 3, (L, B)))
             for L, B, cols, n in sizes]
    ws = shared_workspace(pools)
    for at in (0, 1, 0, 2, 1, 3, 4, 1, 5, 2, 0, 1):
        pool = pools[at]

        def between():
            # a step of no new rows changes nothing but the workspace
            none = torch.zeros(pool.B, dtype=torch.int32, device=DEV)
            xkv.plan_append(pool.cache, pool.B, none, 0, pool.d_lens, pool.d_free, pool.n_pages, pool.d_used, pool.d_used, None,
                            0, ws)

        steps(pool, rng, between)


def test_captured_steps_over_a_shared_workspace():
    """A compaction and a fork captured over one workspace, replayed with other things written into it in between."""
    require_lib()
    pool = PagePool(4, 40, 1, 64, 16, 150, 60000, "int8", seed=3, lens=np.random.default_rng(3).integers(1, 1600, (4, 40)))
    ws = shared_workspace([pool])
    par = torch.arange(40, dtype=torch.int32, device=DEV)

    def step():
        xkv.fork_caches(pool.dims, pool.cache, par, None, 0, pool.d_shares, pool.d_free, pool.n_pages, pool.d_used, ws)
        xkv.compact_pages(pool.dims, pool.cache, pool.d_table, pool.d_shares, pool.d_shares, pool.d_free, pool.d_used, ws)

    step()
    torch.cuda.synchronize()
    state = [t.clone() for t in (pool.d_table, pool.d_lens, pool.d_shares, pool.d_free, pool.d_used, pool.pages[0])]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(10):
        ws[HEADER:] = (37 * i + 255) % 256
        graph.replay()
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) == xkv.OK
    for was, t in zip(state, (pool.d_table, pool.d_lens, pool.d_shares, pool.d_free, pool.d_used, pool.pages[0])):
        assert torch.equal(was, t)
