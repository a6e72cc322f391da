"""Differential attention in 64 bits with bounds on what a kernel may be off, and caches of every format with known rows."""
import math

import numpy as np
import torch

from oracle import xkv_oracle as O
from paper_2412_05896_b200 import xkv

from gpu_util import require_lib

DEV = "cuda:0"
FORMATS = {"bf16": xkv.KV_BF16, "int8": xkv.KV_INT8, "e4m3": xkv.KV_E4M3}


def check_head(out, lse, q, K, V, lam, gain, eps, scale=None, what="", small=0.0):
    """out [d] and lse [2] of one head against the definition over rows K, V (64 bits).

    A weight is rounded to 8 significant bits (half a step: 2^-8 of it; 8-bit rows: of its product with the row's scale, never
    worse than that except for `small`, an absolute error of a weight relative to the largest), logits and sums are fp32, and
    the output rounds once: per element
      |dy| <= E = 2^-8 sum_c (a_1 + |lam| a_2) |V_c| (1 + 2^-4) + small sum_c |V_c| (1 + |lam|) / l
    where 2^-4 covers what fp32 logits change in a weight.  A norm r = 1/sqrt(mean y^2 + eps) moves by at most |E| / |y| of
    itself to first order."""
    half = q.shape[0] // 2
    s = half ** -0.5 if scale is None else scale
    ref, ref_lse = O.diff_attention(q, K, V, lam, gain, eps, scale)
    if K.shape[0] == 0:
        assert np.all(out == 0) and np.all(np.isneginf(lse)), what
        return 0.0
    y, _ = O.diff_attention(q, K, V, lam, None, 0.0, scale)
    size = 0.0
    for part, w in ((slice(0, half), 1.0), (slice(half, None), abs(lam))):
        z = s * (K[:, part] @ q[part])
        e = np.exp(z - z.max())
        size = size + w * (2.0 ** -8 * 1.0625 * (e @ np.abs(V)) + small * np.abs(V).sum(0)) / e.sum()
    bound = size
    if gain is not None:
        ms = np.mean(y * y)
        r = 1.0 / math.sqrt(ms + eps) if ms > 0 else 0.0
        rho = np.linalg.norm(size) / max(np.linalg.norm(y), 1e-300)
        assert rho < 0.5, f"{what}: the inputs cancel too far for the bound ({rho:.2g})"
        bound = np.abs(gain) * r * (size + np.abs(y) * rho) / (1 - rho)
    bound = bound + 2.0 ** -8 * np.abs(ref) + 1e-30
    worst = float((np.abs(out - ref) / bound).max())
    assert np.all(np.isfinite(out)) and worst <= 1.0, f"{what}: {worst:.3g} of the bound"
    if lse is not None:
        # fp32 sums of d/2 products, exponentials and a logarithm
        for i, part in enumerate((slice(0, half), slice(half, None))):
            tol = 2.0 ** -19 * s * float((np.abs(K[:, part]) @ np.abs(q[part])).max()) + 2e-5
            assert abs(lse[i] - ref_lse[i]) <= tol, f"{what}: lse {lse[i]} against {ref_lse[i]}"
    return worst


class RowCache:
    """Caches of random rows of any format in shuffled pages; rows behind the last one are NaN (8-bit: with NaN scales)."""

    def __init__(self, fmt, L, B, H, d, lens, page, extra=0, seed=0, layers_before=0):
        require_lib()
        g = torch.Generator().manual_seed(seed)
        self.fmt, self.L, self.B, self.H, self.d, self.page = fmt, L, B, H, d, page
        self.lens = np.asarray(lens, dtype=np.int64).reshape(L, B)
        self.cols = max(1, math.ceil((int(self.lens.max()) + extra) / page))
        self.n_pages = L * B * self.cols + 3
        self.table = torch.randperm(self.n_pages, generator=g)[: L * B * self.cols].to(torch.int32).reshape(L, B, self.cols)
        shape = (self.n_pages, H, page, d)
        live = torch.zeros(self.n_pages, page, dtype=torch.bool)
        for l in range(L):
            for b in range(B):
                n = int(self.lens[l, b])
                at = torch.arange(n)
                live[self.table[l, b, at // page].long(), at % page] = True
        self.pages, self.scales, self.values = [], [], []
        for kind in range(2):
            x = torch.randn(shape, generator=g) * (1.0 if kind == 0 else 0.7) + (0.0 if kind == 0 else 0.5)
            if fmt == "bf16":
                x = x.to(torch.bfloat16)
                val = x.double()
                x[~live[:, None].expand(-1, H, -1)] = float("nan")
                self.scales.append(None)
            elif fmt == "int8":
                q = (x * 40).round().clamp(-127, 127)
                s = 2.0 ** (torch.rand(self.n_pages, H, page, generator=g) - 5.5)
                val = q.double() * s.double()[..., None]
                x = (q + 128).to(torch.uint8)
                s[~live[:, None].expand(-1, H, -1)] = float("nan")
                self.scales.append(s.to(DEV))
            else:
                s = torch.exp2(torch.randint(-2, 2, (self.n_pages, H, page // 16), generator=g).float())
                c = x.to(torch.float8_e4m3fn)
                val = c.double() * s.double().repeat_interleave(16, -1)[..., None]
                x = c.view(torch.uint8)
                x[~live[:, None].expand(-1, H, -1)] = 0x7F
                s[~live[:, ::16][:, None].expand(-1, H, -1)] = float("nan")
                self.scales.append(s.to(DEV))
            self.pages.append(x.to(DEV))
            self.values.append(val)
        self.d_table = self.table.to(DEV)
        self.d_lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)

    def handle(self):
        ptr = lambda t: None if t is None else t.data_ptr()                       # noqa: E731
        return xkv.Cache(ptr(self.pages[0]), ptr(self.pages[1]), self.d_table.data_ptr(), self.d_lens.data_ptr(), self.L,
                         self.page, self.cols, self.n_pages, ptr(self.scales[0]), ptr(self.scales[1]), FORMATS[self.fmt], 0)

    def rows(self, l, b, g):
        """(K, V) [n, d] in 64 bits."""
        at = torch.arange(int(self.lens[l, b]))
        p = self.table[l, b, at // self.page].long()
        return tuple(v[p, g, at % self.page].numpy() for v in self.values)


def weights(L, Hq, d, seed, with_gain=True):
    g = torch.Generator().manual_seed(seed)
    lam = torch.rand(L, Hq, generator=g) * 0.7 + 0.1
    gain = torch.rand(L, d, generator=g) + 0.3 if with_gain else None
    return lam, gain


def small_weight(fmt, n):
    """What 8-bit rows may lose of a weight besides 2^-8 of it, relative to the largest."""
    # int8: fp16 products of weight and scale (2^-5.5 .. 2^-4.5 here), 2^-25 absolute below 2^-14; e4m3: 2^-23 of a tile's
    # largest product of weight and scale (scales within 2^3 of each other here)
    return {"bf16": 0.0, "int8": 2.0 ** -25 * 2.0 ** 5.5, "e4m3": 2.0 ** -23 * 8}[fmt]


def check_causal(out, lse, Q, K, V, lam, gain, eps, scale=None, what="", rows=None):
    """All rows of one head of one prompt, out [n, d] and lse [2, n], with check_head's bounds (16-bit rows)."""
    n, d = Q.shape
    rows = np.arange(n) if rows is None else rows
    half, s = d // 2, (d // 2) ** -0.5 if scale is None else scale
    dead = np.arange(n)[None, :] > rows[:, None]
    y, size = np.zeros((len(rows), d)), np.zeros((len(rows), d))
    for i, (part, sign) in enumerate(((slice(0, half), 1.0), (slice(half, None), -lam))):
        z = s * (Q[rows][:, part] @ K[:, part].T)
        z[dead] = -np.inf
        top = z.max(1, keepdims=True)
        e = np.exp(z - top)
        total = e.sum(1, keepdims=True)
        y += sign * (e @ V) / total
        size += abs(sign) * 2.0 ** -8 * 1.0625 * (e @ np.abs(V)) / total
        if lse is not None:
            tol = 2.0 ** -19 * s * np.where(dead, 0.0, np.abs(Q[rows][:, part]) @ np.abs(K[:, part]).T).max(1) + 2e-5
            err = np.abs(lse[i][rows] - (top + np.log(total))[:, 0])
            assert np.all(err <= tol), f"{what}: lse of map {i + 1} off by {(err / tol).max():.3g} of the bound"
    bound, ref = size, y
    if gain is not None:
        ms = (y * y).mean(1, keepdims=True)
        r = np.where(ms > 0, 1.0 / np.sqrt(np.maximum(ms, 1e-300) + eps), 0.0)
        ref = y * r * gain
        rho = np.linalg.norm(size, axis=1, keepdims=True) / np.maximum(np.linalg.norm(y, axis=1, keepdims=True), 1e-300)
        # rows whose maps cancel too far for the bound (y is then mostly rounding) are only asked to be finite
        fine = rho < 0.5
        assert fine.mean() > 0.9, what
        bound = np.where(fine, np.abs(gain) * r * (size + np.abs(y) * rho) / (1 - np.minimum(rho, 0.5)), np.inf)
    bound = bound + 2.0 ** -8 * np.abs(ref) + 1e-30
    assert np.all(np.isfinite(out[rows])), what
    worst = float((np.abs(out[rows] - ref) / bound).max())
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound"
