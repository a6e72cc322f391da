"""Bounded waits of the differential prompt kernel: one CTA's copies are withheld, its waits run out, the others' work is done."""
import pytest
import torch

from paper_2412_05896_b200 import xkv

from diff_util import DEV, weights
from test_gpu_diff_prefill import EPS, attend, prompts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_waits_that_run_out_are_reported(d):
    lens, Hq, H = [600, 600], 8, 2
    q, k, v = prompts(lens, Hq, H, d, 5)
    lam, gain = (t[0].to(DEV) for t in weights(1, Hq, d, 7))
    want, want_lse = attend(lens, q, k, v, H, lam, gain)
    dims = xkv.Dims(2, Hq, H, d, 1, 1, 0, 0.0, H * d, d)
    cu = torch.tensor([0, 600, 1200], dtype=torch.int32, device=DEV)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DIFF_PREFILL_ATTN, dims), dtype=torch.uint8, device=DEV)
    out, lse = torch.full_like(q, float("nan")), torch.full_like(want_lse, float("nan"))
    cta = 5                                                   # one item a CTA here: head 5 of the first sequence's last tile
    xkv.test_hooks(wait_limit_ns=1_000_000, withhold_decode_item=cta)
    try:
        xkv.diff_prefill_attn(dims, q, k, v, lam, gain, EPS, cu, 1200, 600, out, lse, ws)
        torch.cuda.synchronize()
    finally:
        xkv.test_hooks()
    assert xkv.read_device_status(ws) == xkv.ERR_TIMEOUT
    assert xkv.read_device_status(ws) == xkv.OK               # reading reset the word
    missing = torch.zeros(1200, Hq, dtype=torch.bool, device=DEV)
    missing[512:600, cta] = True
    assert bool(out[missing].isnan().all()) and torch.equal(out[~missing], want[~missing])
    rows = missing.t()[:, None].expand(-1, 2, -1)
    assert bool(lse[rows].isnan().all()) and torch.equal(lse[~rows], want_lse[~rows])
    xkv.diff_prefill_attn(dims, q, k, v, lam, gain, EPS, cu, 1200, 600, out, lse, ws)
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) == xkv.OK and torch.equal(out, want) and torch.equal(lse, want_lse)
