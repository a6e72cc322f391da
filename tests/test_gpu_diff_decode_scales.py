"""8-bit cached rows that have a weight but no value: V all zero (which is stored with scale 1, far above the scales of ordinary
rows) or stored with scale 0.  They count in the denominators and nowhere else, however large their logits are."""
import numpy as np
import pytest
import torch

from diff_util import DEV, RowCache, weights
from gpu_util import f64, require_lib
from test_gpu_diff_decode import attend, check

pytestmark = pytest.mark.gpu
FAR = 3.5                              # of a key along the queries: its logits are about 14 above the others'


def queries(L, B, Hq, d, seed):
    """Halves whose elements are 1/2 in the mean, so that one key is far for all of them."""
    g = torch.Generator().manual_seed(seed)
    return (0.5 + 0.5 * torch.randn(L, B, Hq, d, generator=g)).to(torch.bfloat16).to(DEV)


def plant(c, l, b, rows, scale, code, key=None):
    """V of these rows becomes `code` in every column with this scale (code 128 or scale 0: no value), K `key` everywhere."""
    at = torch.as_tensor(rows)
    page, off = c.table[l, b, at // c.page].long(), at % c.page
    c.pages[1][page.to(DEV), :, off.to(DEV)] = code
    c.scales[1][page.to(DEV), :, off.to(DEV)] = scale
    c.values[1][page, :, off] = (code - 128) * scale
    if key is not None:
        s = float(np.float32(key / 127))
        c.pages[0][page.to(DEV), :, off.to(DEV)] = 255
        c.scales[0][page.to(DEV), :, off.to(DEV)] = s
        c.values[0][page, :, off] = 127 * s


def small_scales(c):
    """V's scales 2^-8 of what RowCache makes: the scales of rows of ordinary size beside the 1 of a row of zeros."""
    c.scales[1] *= 2.0 ** -3
    c.values[1] *= 2.0 ** -3


def check_lse(c, q, sums):
    """Logits of 8-bit rows: q times 1152 + integer, exact products below 1280 |q|, d/32 steps of 16 of them, and 1152 times q's sum off,
    formed alike.  A step adds 17 terms aligned to the largest, each short by at most 2^-23 of it, and no partial sum is above
    1280 sum |q|; queries here have a mean, so such sums come.  2e-5 for exponentials, their sum and the logarithm."""
    q64, s64, G, half = f64(q), sums.double().cpu().numpy(), q.shape[2] // c.H, c.d // 2
    for i in range(c.L):
        for b in range(0, c.B, max(1, c.B // 4)):
            at = torch.arange(int(c.lens[i, b]))
            page = c.table[i, b, at // c.page].long().to(DEV)
            ks = c.scales[0][page, :, (at % c.page).to(DEV)].double().cpu().numpy()
            for h in range(q.shape[2]):
                K, _ = c.rows(i, b, h // G)
                for m in range(2):
                    part = slice(m * half, (m + 1) * half)
                    z = half ** -0.5 * (K[:, part] @ q64[i, b, h, part])
                    want = z.max() + np.log(np.exp(z - z.max()).sum())
                    tol = 2e-5 + half ** -0.5 * ks[:, h // G].max() * 2 * 17 * (c.d // 32) * 2.0 ** -23 * 1280 * \
                        np.abs(q64[i, b, h, part]).sum()
                    assert abs(s64[i, b, h, m] - want) <= tol, (i, b, h, m)


def run(c, G, q, chunk=0):
    """With and without a norm.  Products of weight and scale are rounded to fp16: below 2^-14 of the largest of a row that has a
    value an absolute error would have to be counted; the ordinary rows' logits here lie within 2^9 of each other (0.7 standard
    deviations of the sum of 32 or 64 products, over up to 16 000 rows) and their scales within 2, so none comes there, and the bound
    is that of the roundings alone."""
    lam, gain = (t.to(DEV) for t in weights(c.L, c.H * G, c.d, 5))
    for g, eps in ((gain, 1e-5), (gain, 0.0), (None, 0.0)):
        out, sums = attend(c, c.H * G, q, lam, g, chunk=chunk, eps=eps)
        c.fmt = "bf16"                 # (no absolute error of a weight)
        check(c, c.H * G, q, lam, g, out, None, eps=eps, every=max(1, c.B // 4))
        c.fmt = "int8"
        check_lse(c, q, sums)
        if c.lens.max() * c.B < 5000:
            assert f64(out).any()


PLACES = [("one", [3]), ("last", [-1]), ("first forty", list(range(40))), ("every fifth", list(range(0, 90, 5)))]


@pytest.mark.parametrize("name,rows", PLACES, ids=[p[0] for p in PLACES])
@pytest.mark.parametrize("L,B,H,G,d,page,longest", [
    (1, 1, 1, 1, 64, 16, 97),           # eight warps a CTA, a tile or none each
    (1, 3, 2, 4, 128, 16, 400),         # several tiles a warp
    (1, 2, 1, 2, 128, 32, 16000),       # many chunks, joined
    (2, 160, 4, 3, 64, 16, 120),        # four warps a CTA
])
def test_far_rows_of_zeros(L, B, H, G, d, page, longest, name, rows):
    require_lib()
    lens = np.random.default_rng(1).integers(91, longest + 1, (L, B))
    lens.flat[0] = longest
    c = RowCache("int8", L, B, H, d, lens, page, seed=3)
    small_scales(c)
    for l in range(L):
        for b in range(B):
            plant(c, l, b, [r % int(c.lens[l, b]) for r in rows], 1.0, 128, FAR)
    run(c, G, queries(L, B, H * G, d, 6))


@pytest.mark.parametrize("chunk", [0, 64])
@pytest.mark.parametrize("far", [True, False])
@pytest.mark.parametrize("L,B,H,G,d,page,longest", [(1, 3, 2, 4, 128, 16, 400), (1, 2, 1, 2, 64, 32, 9000), (2, 160, 4, 3, 64, 16, 120)])
def test_scales_of_zero(L, B, H, G, d, page, longest, far, chunk):
    """A run of rows, whole tiles of a warp among them, whose V has scale 0."""
    require_lib()
    lens = np.random.default_rng(2).integers(91, longest + 1, (L, B))
    lens.flat[0] = longest
    c = RowCache("int8", L, B, H, d, lens, page, seed=3)
    for l in range(L):
        for b in range(B):
            plant(c, l, b, list(range(80)), 0.0, 200, 0.5 if far else None)
    run(c, G, queries(L, B, H * G, d, 6), chunk)


@pytest.mark.parametrize("scale,code", [(0.0, 255), (1.0, 128)])
@pytest.mark.parametrize("chunk", [0, 64])
@pytest.mark.parametrize("longest", [1, 70, 9000])
def test_no_row_has_a_value(longest, scale, code, chunk):
    """Outputs are zero, the statistics those of the logits."""
    require_lib()
    c = RowCache("int8", 1, 2, 2, 128, [[longest, max(1, longest // 3)]], 16, seed=4)
    for b in range(2):
        plant(c, 0, b, list(range(int(c.lens[0, b]))), scale, code)
    lam, gain = (t.to(DEV) for t in weights(1, 4, 128, 5))
    q = queries(1, 2, 4, 128, 6)
    for g in (gain, None):
        out, sums = attend(c, 4, q, lam, g, chunk=chunk)
        assert not out.float().any() and bool(torch.isfinite(sums).all())
        check(c, 4, q, lam, g, out, None)
        check_lse(c, q, sums)


@pytest.mark.parametrize("name,rows", PLACES, ids=[p[0] for p in PLACES])
@pytest.mark.parametrize("B,H,G,d,page,longest", [(3, 2, 4, 128, 16, 400), (2, 1, 2, 64, 32, 6000), (2, 2, 6, 128, 64, 300)])
def test_far_rows_of_zeros_with_chunks(B, H, G, d, page, longest, name, rows):
    """The streaming kernel, caches cut and joined."""
    require_lib()
    lens = np.random.default_rng(1).integers(91, longest + 1, (1, B))
    lens.flat[0] = longest
    c = RowCache("int8", 1, B, H, d, lens, page, seed=3)
    small_scales(c)
    for b in range(B):
        plant(c, 0, b, [r % int(c.lens[0, b]) for r in rows], 1.0, 128, FAR)
    run(c, G, queries(1, B, H * G, d, 6), 64)


def test_far_rows_of_zeros_in_pages_that_start_on_16_bytes():
    require_lib()
    c = RowCache("int8", 1, 2, 2, 128, [[333, 97]], 32, seed=3)
    small_scales(c)
    for b in range(2):
        plant(c, 0, b, [0, 50, 96], 1.0, 128, FAR)
    for i in range(2):
        x = c.pages[i]
        room = torch.empty(x.numel() + 32, dtype=torch.uint8, device=DEV)
        c.pages[i] = room[16:-16].view(x.shape).copy_(x)
        assert c.pages[i].data_ptr() % 32 == 16
    run(c, 4, queries(1, 2, 8, 128, 6))


@pytest.mark.parametrize("chunk", [0, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_a_far_new_row_of_zeros(d, chunk):
    """Stored by the call, with the scale that a row of zeros gets."""
    require_lib()
    L, B, H, G, page = 1, 3, 2, 3, 16
    c = RowCache("int8", L, B, H, d, [[100, 15, 320]], page, extra=1, seed=3)
    small_scales(c)
    q = queries(L, B, H * G, d, 6)
    lam, gain = (t.to(DEV) for t in weights(L, H * G, d, 5))
    kn, vn = (torch.full((L, B, H, d), x, dtype=torch.bfloat16, device=DEV) for x in (FAR, 0.0))
    out, sums = attend(c, H * G, q, lam, gain, kn, vn, chunk=chunk, eps=0.0)
    scale = float(np.float32(FAR) / np.float32(127))
    for b in range(B):
        n = int(c.lens[0, b])
        at = c.table[0, b, n // page].long()
        assert bool((c.scales[1][at, :, n % page] == 1.0).all()) and bool((c.pages[1][at, :, n % page] == 128).all())
        c.values[0][at, :, n % page], c.values[1][at, :, n % page] = 127 * scale, 0.0
    c.lens = c.lens + 1
    c.fmt = "bf16"                     # (no absolute error of a weight)
    check(c, H * G, q, lam, gain, out, None, eps=0.0)
    check_lse(c, q, sums)


@pytest.mark.parametrize("power", [-24, -14, 12, 30])
def test_row_scales_of_any_size_with_chunks(power):
    """V's scales far from 1, and a block of rows whose scales are far from the others', in the streaming kernel."""
    require_lib()
    c = RowCache("int8", 1, 3, 2, 128, [[400, 37, 1000]], 16, seed=3)
    c.scales[1] *= 2.0 ** power
    c.values[1] *= 2.0 ** power
    first = c.table[0, :, 0].long()
    c.scales[1][first] *= 2.0 ** -20
    c.values[1][first] *= 2.0 ** -20
    lam, gain = (t.to(DEV) for t in weights(1, 8, 128, 5))
    q = queries(1, 3, 8, 128, 6)
    for g in (gain, None):
        out, sums = attend(c, 8, q, lam, g, chunk=64, eps=0.0)
        c.fmt = "bf16"
        check(c, 8, q, lam, g, out, None, eps=0.0)
        c.fmt = "int8"
        check_lse(c, q, sums)
