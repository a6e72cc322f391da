"""Pages behind the first 4 GB of a pool: attention, forks, copies and compaction reach the same bytes as in a small pool."""
import pytest
import torch

from paper_2412_05896_b200 import xkv

from diff_util import DEV, FORMATS, RowCache, weights
from test_gpu_diff_decode import attend, queries

pytestmark = pytest.mark.gpu


def far(c, at):
    """A cache over a pool that holds c's pages from page `at` on."""
    n = at + c.n_pages
    f = object.__new__(RowCache)
    f.__dict__.update(c.__dict__)
    f.pages, f.scales = [], []
    for x, s in zip(c.pages, c.scales):
        big = torch.empty(n, *x.shape[1:], dtype=x.dtype, device=DEV)
        big[at:] = x
        f.pages.append(big)
        f.scales.append(None if s is None else torch.empty(n, *s.shape[1:], device=DEV))
        if s is not None:
            f.scales[-1][at:] = s
    f.n_pages, f.d_table, f.d_lens = n, c.d_table + at, c.d_lens.clone()
    return f


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_far_pages(fmt):
    page, d = 256, 128
    c = RowCache(fmt, 2, 2, 1, d, [[700, 257], [100, 511]], page, seed=3)
    page_bytes = page * d * (2 if fmt == "bf16" else 1)
    at = (1 << 32) // page_bytes + 5
    f = far(c, at)
    assert f.pages[0].numel() * f.pages[0].element_size() > 1 << 32
    lam, gain = (t.to(DEV) for t in weights(2, 4, d, 5))
    q = queries(2, 2, 4, d, 6)
    for chunk in (0, 256):
        near, s0 = attend(c, 4, q, lam, gain, chunk=chunk)
        out, s1 = attend(f, 4, q, lam, gain, chunk=chunk)
        assert torch.equal(out, near) and torch.equal(s0, s1)
    # a fork whose open page is copied to the list's only pages, far ones
    dims = xkv.Dims(2, 1, 1, d, 1, 1, 0, 0.0, d, d)
    free = torch.arange(f.n_pages, dtype=torch.int32, device=DEV)
    held = sorted({int(p) for l in range(2) for b in range(2) for p in f.d_table[l, b, :-(-int(f.d_lens[l, b]) // page)].tolist()})
    spare = [p for p in range(at, f.n_pages) if p not in held]
    used = torch.tensor([f.n_pages - len(spare)], dtype=torch.int32, device=DEV)
    free[f.n_pages - len(spare):] = torch.tensor(spare, dtype=torch.int32, device=DEV)
    shares = torch.zeros(f.n_pages, dtype=torch.int32, device=DEV)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_FORK_CACHES, dims, max_seqlen=f.cols, total_tokens=f.n_pages, n_layers=2),
                     dtype=torch.uint8, device=DEV)
    parent = torch.tensor([0, 0], dtype=torch.int32, device=DEV)
    xkv.fork_caches(dims, f.handle(), parent, None, 0, shares, free, f.n_pages, used, ws)
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) == xkv.OK and f.d_lens.tolist() == [[700, 700], [100, 100]]
    assert int(f.d_table[0, 1, 2]) in spare and int(f.d_table[1, 1, 0]) in spare
    twin = q[:, :1].expand(-1, 2, -1, -1).contiguous()
    want, _ = attend(c, 4, twin, lam, gain)
    out, _ = attend(f, 4, twin, lam, gain)
    assert torch.equal(out[:, 0], want[:, 0]) and torch.equal(out[:, 1], want[:, 0])
    # down to the front of the pool, and a far page to another
    src = int(f.d_table[0, 0, 0])
    before = [x[src].clone() for x in f.pages]
    ids = [torch.tensor([i], dtype=torch.int32, device=DEV) for i in (src, f.n_pages - 1 if src != f.n_pages - 1 else 0)]
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_COMPACT_PAGES, dims, max_seqlen=f.cols, total_tokens=f.n_pages, n_layers=2),
                     dtype=torch.uint8, device=DEV)
    xkv.compact_pages(dims, f.handle(), f.d_table, shares, shares, free, used, ws)
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) == xkv.OK and int(used) == len(set(f.d_table[0, :, :3].flatten().tolist()) | set(
        f.d_table[1, :, 0].tolist())) and int(f.d_table[:, :, 0].max()) < int(used)
    out, _ = attend(f, 4, twin, lam, gain)
    assert torch.equal(out[:, 0], want[:, 0]) and torch.equal(out[:, 1], want[:, 0])
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_COPY_PAGES, dims), dtype=torch.uint8, device=DEV)
    xkv.copy_pages(dims, f.handle(), ids[0], f.handle(), ids[1], 1, ws)
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) == xkv.OK
    for x, b in zip(f.pages, before):
        assert torch.equal(x[int(ids[1])].view(torch.uint8), b.view(torch.uint8))
