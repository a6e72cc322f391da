"""Captured steps of a session whose live sequences change between replays."""
import pytest
import torch

from paper_2412_05896_b200 import xkv

from diff_util import DEV
from test_gpu_session_pages import EPS, Run

pytestmark = pytest.mark.gpu


def test_captured_steps_of_several_sets():
    """Two sets of live sequences captured each, steps of other sets in between and their tensors' memory written over; replays
    against a twin that captures nothing."""
    one, two = Run("int8"), Run("int8")
    q, k, v = (torch.randn(3, 4, n, 64, generator=one.gen).to(torch.bfloat16).to(DEV) for n in (8, 2, 2))
    step = lambda r: r.s.diff_decode(q, k, v, r.lam, r.gain, EPS)                 # noqa: E731
    sets = {"a": [0, -1, 2, 3], "b": [-1, 1, 2, -1]}
    graphs = {}

    def again(r, counts):
        kk, vv = (torch.full((3, sum(counts), 2, 64), 0.25, dtype=torch.bfloat16, device=DEV) for _ in "kv")
        r.s.append(kk, vv, counts)

    def to_set(r, name):
        again(r, [1, 1, 1, 1])                                # all live
        r.s.fork(sets[name])

    for name in sets:
        for r in (one, two):
            to_set(r, name)
            step(r)
        torch.cuda.synchronize()
        graphs[name] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[name]):
            out = step(one)
        graphs[name] = (graphs[name], out)
    junk = []
    for turn in range(6):
        for other in ([0, 0, -1, -1], [-1, -1, -1, 3], [-1, 1, 2, 3]):
            for r in (one, two):
                again(r, [1, 1, 1, 1])
                r.s.fork(other)
                step(r)
        junk += [torch.full((n,), 0x5A5A5A5A, dtype=torch.int32, device=DEV) for n in (4, 4, 6, 8, 16, 64, 128) * 8]
        name = "ab"[turn % 2]
        for r in (one, two):
            to_set(r, name)
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=one.gen).to(torch.bfloat16))
        graph, out = graphs[name]
        graph.replay()
        want = step(two)
        torch.cuda.synchronize()
        assert torch.equal(out, want), turn
        for x in ("seq_lens", "block_table", "shares", "pages_used", "free_pages"):
            assert torch.equal(getattr(one.s, x), getattr(two.s, x)), (turn, x)
    one.status()
    two.status()


def test_a_set_that_has_not_run_cannot_be_captured():
    r = Run("bf16")
    q, k, v = (torch.randn(3, 4, n, 64, generator=r.gen).to(torch.bfloat16).to(DEV) for n in (8, 2, 2))
    r.s.diff_decode(q, k, v, r.lam, r.gain, EPS)
    r.s.fork([0, -1, 2, 3])
    torch.cuda.synchronize()
    lens = r.s.seq_lens.clone()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="captured"):
        with torch.cuda.graph(graph):
            r.s.diff_decode(q, k, v, r.lam, r.gain, EPS)
    torch.cuda.synchronize()
    assert torch.equal(lens, r.s.seq_lens)
    r.s.diff_decode(q, k, v, r.lam, r.gain, EPS)
    torch.cuda.synchronize()
    assert r.s.device_status("append") == xkv.OK


def same_state(one, two):
    for x in ("seq_lens", "block_table", "shares", "pages_used", "free_pages"):
        assert torch.equal(getattr(one.s, x), getattr(two.s, x)), x


def test_a_step_captured_before_the_first_fork():
    """It goes on with the pages that forks, frees and cuts have given back, not with those of its own count."""
    one, two = Run("bf16"), Run("bf16")
    q, k, v = (torch.randn(3, 4, n, 64, generator=one.gen).to(torch.bfloat16).to(DEV) for n in (8, 2, 2))
    for r in (one, two):
        r.s.diff_decode(q, k, v, r.lam, r.gain, EPS)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one.s.diff_decode(q, k, v, one.lam, one.gain, EPS)
    for i in range(40):
        for r in (one, two):
            if i % 8 == 3:                                    # (beams: every sequence goes on)
                r.s.fork([[1, 1, 0, 2], [3, 0, 2, 2]][i // 8 % 2])
            if i % 8 == 6:
                r.s.cut([5, 0, 11, 2])
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=one.gen).to(torch.bfloat16))
        graph.replay()
        want = two.s.diff_decode(q, k, v, two.lam, two.gain, EPS)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        same_state(one, two)
    one.status()
    two.status()


def test_the_first_fork_is_captured():
    """Replays go on from each other's state, not from that of the capture."""
    one, two = Run("int8"), Run("int8")
    parent = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device=DEV)
    q, k, v = (torch.randn(3, 4, n, 64, generator=one.gen).to(torch.bfloat16).to(DEV) for n in (8, 2, 2))
    for r in (one, two):
        r.s.diff_decode(q, k, v, r.lam, r.gain, EPS)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.s.fork(parent)
        out = one.s.diff_decode(q, k, v, one.lam, one.gain, EPS)
    for p in ([0, 0, 1, 3], [3, 2, 1, 0], [1, 1, 1, -1], [0, 2, 2, 2]) * 3:
        parent.copy_(torch.tensor(p, dtype=torch.int32))
        graph.replay()
        two.s.fork(parent)
        want = two.s.diff_decode(q, k, v, two.lam, two.gain, EPS)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        same_state(one, two)
    one.s.compact()
    two.s.compact()
    torch.cuda.synchronize()
    same_state(one, two)
    one.status()
    two.status()


def test_a_pool_resized_on_another_stream():
    """The session is made on one stream and resized on another, which is late: the old pool's memory is not handed out before the
    copy has read it."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        r = Run("int8", d=128)
        s = r.s
        s.resize_pool(6000)                                   # (allocated on this stream, in blocks of its own)
        torch.cuda.synchronize()
    used, old = int(s.pages_used.item()), {x.data_ptr() for x in (s.k_pages, s.v_pages, s.free_pages, s.shares)}
    shapes = [(x.shape, x.dtype) for x in (s.k_pages, s.v_pages, s.k_scales, s.v_scales, s.free_pages, s.shares)]
    late = xkv.copy_pages

    def copy_pages(*args, **kw):
        torch.cuda._sleep(400_000_000)                        # about a fifth of a second
        return late(*args, **kw)

    xkv.copy_pages = copy_pages
    try:
        s.resize_pool(used + 40)
    finally:
        xkv.copy_pages = late
    with torch.cuda.stream(side):                             # the other stream's next allocations, of the sizes given up
        taken = [torch.full(shape, 77, dtype=dtype, device=DEV) for shape, dtype in shapes for _ in range(2)]
    assert not old & {x.data_ptr() for x in taken}
    torch.cuda.synchronize()
    r.expect(r.rows)
    r.step([True] * 4)
    r.status()


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_the_first_differential_step_is_captured(fmt):
    """Calls between the capture and the first replay, and after it, are right, and the status is that of the calls."""
    one, two = Run(fmt), Run(fmt)
    q, k, v = (torch.randn(3, 4, n, 64, generator=one.gen).to(torch.bfloat16).to(DEV) for n in (8, 2, 2))
    junk = [torch.full((1 << 20,), 0x5A5A5A5A, dtype=torch.int32, device=DEV) for _ in range(64)]
    del junk                                                  # what the allocator hands out next is not zero
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one.s.diff_decode(q, k, v, one.lam, one.gain, EPS)
    one.status()
    for i in range(6):
        if i % 3 == 0:
            got = one.s.diff_decode(q, k, v, one.lam, one.gain, EPS)
        else:
            graph.replay()
            got = out
        want = two.s.diff_decode(q, k, v, two.lam, two.gain, EPS)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(one.s.diff_lse, two.s.diff_lse), i
        one.status()
