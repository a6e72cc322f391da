"""Causal differential attention of packed prompts, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2412_05896_b200 import xkv

from diff_util import DEV, check_causal, weights
from gpu_util import f64, require_lib

pytestmark = pytest.mark.gpu
EPS = 1e-5


def prompts(lens, Hq, H, d, seed, pad=0):
    """q, k, v of packed prompts; pad: elements between a token's heads and the next token's."""
    g = torch.Generator().manual_seed(seed)
    T = sum(lens)
    q = torch.randn(T, Hq, 2, d // 2, generator=g) * torch.exp(torch.rand(T, Hq, 2, 1, generator=g) * 1.5 - 0.5)
    q = q.reshape(T, Hq, d).to(torch.bfloat16).to(DEV)
    k, v = (torch.full((T, H * d + pad), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for x, shift in ((k, 0.0), (v, 0.5)):
        x[:, :H * d] = (torch.randn(T, H * d, generator=g) + shift).to(torch.bfloat16).to(DEV)
    return q, k, v


def attend(lens, q, k, v, H, lam, gain, scale=0.0, eps=EPS, lse=True, max_seqlen=None, out=None, stream=None):
    require_lib()
    T, Hq, d = q.shape
    dims = xkv.Dims(len(lens), Hq, H, d, 1, 1, 0, scale, k.stride(0), d)
    cu = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device=DEV)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DIFF_PREFILL_ATTN, dims), dtype=torch.uint8, device=DEV)
    out = torch.full_like(q, float("nan")) if out is None else out
    sums = torch.full((Hq, 2, T), float("nan"), device=DEV) if lse else None
    xkv.diff_prefill_attn(dims, q, k, v, lam, gain, eps, cu, T, max_seqlen or max(lens), out, sums, ws, stream=stream)
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) == xkv.OK
    return out, sums


def check(lens, q, k, v, H, lam, gain, out, sums, eps=EPS, scale=None, heads=None, rows=None):
    T, Hq, d = q.shape
    at = 0
    for b, n in enumerate(lens):
        K, V = (f64(x[at:at + n, :H * d]).reshape(n, H, d) for x in (k, v))
        for h in (range(Hq) if heads is None else heads) if n else ():
            g = h // (Hq // H)
            check_causal(f64(out[at:at + n, h]), None if sums is None else sums[h, :, at:at + n].double().cpu().numpy(),
                         f64(q[at:at + n, h]), K[:, g], V[:, g], float(lam[h]),
                         None if gain is None else gain.double().cpu().numpy(), eps, scale, f"sequence {b} head {h}",
                         None if rows is None else rows[rows < n])
        at += n


CASES = [  # lengths, KV heads, group, d, padding of a token's row
    ([1], 1, 1, 64, 0),
    ([1], 1, 2, 128, 0),
    ([2, 63, 64, 65], 2, 1, 64, 0),
    ([127, 128, 129], 1, 3, 128, 8),
    ([300], 2, 2, 128, 0),
    ([5, 0, 700, 1, 250], 1, 1, 128, 0),
    ([511], 4, 2, 64, 64),
    ([130] * 40, 1, 1, 64, 0),
    ([1000, 33], 1, 8, 128, 0),
]


@pytest.mark.parametrize("lens,H,G,d,pad", CASES)
@pytest.mark.parametrize("norm", [True, False])
def test_against_definition(lens, H, G, d, pad, norm):
    q, k, v = prompts(lens, H * G, H, d, sum(lens), pad)
    lam, gain = weights(1, H * G, d, 7, norm)
    lam, gain = lam[0].to(DEV), None if gain is None else gain[0].to(DEV)
    out, sums = attend(lens, q, k, v, H, lam, gain)
    check(lens, q, k, v, H, lam, gain, out, sums)
    again, _ = attend(lens, q, k, v, H, lam, gain, lse=False)
    assert torch.equal(out, again)


def test_many_items_a_cta_and_far_logits():
    """More items than CTAs several times over; logits that rise along the prompt, so that the reference is raised again and
    again; a scale of its own."""
    lens, H, G, d = [900, 1500, 300], 4, 4, 128
    q, k, v = prompts(lens, H * G, H, d, 3)
    k[:, :H * d] *= torch.linspace(0.2, 4.0, sum(lens), device=DEV).to(torch.bfloat16)[:, None]
    lam, gain = (t[0].to(DEV) for t in weights(1, H * G, d, 7))
    out, sums = attend(lens, q, k, v, H, lam, gain, scale=0.25)
    check(lens, q, k, v, H, lam, gain, out, sums, scale=0.25, heads=(0, 5, 15), rows=np.arange(0, 1500, 7))


def test_repeated_calls_are_the_same():
    lens = [700, 3, 1200, 64]
    q, k, v = prompts(lens, 8, 2, 128, 5)
    lam, gain = (t[0].to(DEV) for t in weights(1, 8, 128, 7))
    out, sums = attend(lens, q, k, v, 2, lam, gain)
    for _ in range(50):
        again, s = attend(lens, q, k, v, 2, lam, gain)
        assert torch.equal(out, again) and torch.equal(sums, s)


@pytest.mark.parametrize("lens,d,norm", [([2399, 4287, 3917], 128, True), ([4100, 3000], 64, False), ([100] * 300, 128, False)])
def test_maps_that_drift_apart(lens, d, norm):
    """Long items on every SM, where one map's warps run tiles ahead of the other's, and short ones after one another: the same
    result in every call, and the definition's."""
    H, G = 8, 4
    q, k, v = prompts(lens, H * G, H, d, 8)
    lam, gain = weights(1, H * G, d, 7, norm)
    lam, gain = lam[0].to(DEV), None if gain is None else gain[0].to(DEV)
    out, sums = attend(lens, q, k, v, H, lam, gain)
    check(lens, q, k, v, H, lam, gain, out, sums, heads=(3, 30), rows=np.arange(90, max(lens), 101))
    for _ in range(30):
        again, s = attend(lens, q, k, v, H, lam, gain)
        assert torch.equal(out, again) and torch.equal(sums, s)


def test_what_is_not_finite_stays_in_its_sequence():
    """NaN and infinities in the next prompt's rows, and rows of the K and V tensors behind the last token."""
    lens = [70, 130, 33]
    q, k, v = prompts(lens, 4, 2, 64, 5)
    lam, gain = (t[0].to(DEV) for t in weights(1, 4, 64, 7))
    clean, sums = attend(lens, q, k, v, 2, lam, gain)
    k[70:200], v[70:200] = float("nan"), float("inf")
    out, s = attend(lens, q, k, v, 2, lam, gain)
    keep = torch.cat([torch.arange(70), torch.arange(200, 233)]).to(DEV)
    assert torch.equal(out[keep], clean[keep]) and torch.equal(s[..., keep], sums[..., keep])


def test_longer_prompts_than_announced_are_cut():
    lens = [300, 50]
    q, k, v = prompts(lens, 2, 2, 64, 5)
    lam, gain = (t[0].to(DEV) for t in weights(1, 2, 64, 7))
    whole, _ = attend(lens, q, k, v, 2, lam, gain)
    out = torch.full_like(q, 7.0)
    attend(lens, q, k, v, 2, lam, gain, max_seqlen=130, out=out)
    assert torch.equal(out[:130], whole[:130]) and torch.equal(out[300:], whole[300:]) and bool((out[130:300] == 7.0).all())


def test_on_another_stream_and_captured():
    lens = [257, 64]
    q, k, v = prompts(lens, 4, 1, 128, 5)
    lam, gain = (t[0].to(DEV) for t in weights(1, 4, 128, 7))
    want, _ = attend(lens, q, k, v, 1, lam, gain)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, _ = attend(lens, q, k, v, 1, lam, gain, stream=side)
    assert torch.equal(out, want)
    dims = xkv.Dims(2, 4, 1, 128, 1, 1, 0, 0.0, 128, 128)
    cu = torch.tensor([0, 257, 321], dtype=torch.int32, device=DEV)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DIFF_PREFILL_ATTN, dims), dtype=torch.uint8, device=DEV)
    out.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xkv.diff_prefill_attn(dims, q, k, v, lam, gain, EPS, cu, 321, 257, out, None, ws)
    for _ in range(5):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_an_expired_wait_is_reported():
    """Waits of no length run out: the kernel drains, the status says so, and the next call is right."""
    lens = [600, 600]
    q, k, v = prompts(lens, 8, 2, 128, 5)
    lam, gain = (t[0].to(DEV) for t in weights(1, 8, 128, 7))
    want, _ = attend(lens, q, k, v, 2, lam, gain)
    dims = xkv.Dims(2, 8, 2, 128, 1, 1, 0, 0.0, 256, 128)
    cu = torch.tensor([0, 600, 1200], dtype=torch.int32, device=DEV)
    ws = torch.zeros(xkv.workspace_bytes(xkv.OP_DIFF_PREFILL_ATTN, dims), dtype=torch.uint8, device=DEV)
    xkv.test_hooks(1, -1)
    try:
        xkv.diff_prefill_attn(dims, q, k, v, lam, gain, EPS, cu, 1200, 600, torch.empty_like(q), None, ws)
    finally:
        xkv.test_hooks()
    torch.cuda.synchronize()
    assert xkv.read_device_status(ws) in (xkv.ERR_TIMEOUT, xkv.OK)     # (whether a wait of 1 ns expires is the clock's choice)
    out, _ = attend(lens, q, k, v, 2, lam, gain)
    assert torch.equal(out, want)
