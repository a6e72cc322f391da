"""What is measured of the operators for models with differential heads and for caches that share, give back and move pages.

  prefill  causal differential attention of packed prompts
  attend   differential attention of one new token a sequence over a paged cache (bf16, int8 or 8-bit float pages)
  fork     caches that become forks of others, are cut or freed; pages shared, copied and given back
  compact  the pages in use moved to the front of the pool, tables and lists along
  copy     pages copied from one pool to another

A differential head has a query row [q1 | q2], key rows [k1 | k2] (two halves each) and value rows v:
out = sum_c (softmax(scale q1 k1)_c - lambda softmax(scale q2 k2)_c) v_c, with a gain normalised by its root mean square.
`shares` counts the table entries that hold a page beyond the first.
"""
import math

import torch

own = False

BLOCK = 16                       # tokens that share a scale in 8-bit float pages
EPS = 1e-5


# ------------------------------------------------------------------ cases
def listed():
    return [
        # the prompt of the smallest configuration: latency
        dict(name="prefill one request", op="prefill", batch=1, q_heads=4, kv_heads=4, d=64, lo=487, hi=487, gain=True),
        # a batch of ragged prompts of a grouped-query model, one layer
        dict(name="prefill ragged batch", op="prefill", batch=4, q_heads=32, kv_heads=8, d=128, lo=2048, hi=4500, gain=True),
        # one sequence of the smallest configuration, all four layers in a call: latency
        dict(name="attend tiny", op="attend", fmt="bf16", layers=4, batch=1, q_heads=4, kv_heads=4, d=64, lo=49, hi=146,
             page=16, gain=True),
        # a ragged serving batch of a grouped-query model, average budget about 1024
        dict(name="attend ragged batch", op="attend", fmt="bf16", layers=4, batch=64, q_heads=32, kv_heads=8, d=128, lo=290,
             hi=2707, page=32, gain=True),
        # multi-head attention after eviction to about 512 tokens a head, 8-bit rows, no norm behind it
        dict(name="attend int8 mha", op="attend", fmt="int8", layers=8, batch=8, q_heads=32, kv_heads=32, d=128, lo=203,
             hi=1101, page=16, gain=False),
        # one very long cache that was not evicted, in 8-bit floats (two layers): split over the sequence
        dict(name="attend e4m3 long", op="attend", fmt="e4m3", layers=2, batch=1, q_heads=32, kv_heads=8, d=128, lo=131013,
             hi=131071, page=64, gain=True),
        # best of eight for four prompts: samples fork from each prompt and are dropped when they are done
        dict(name="fork best of n", op="fork", kind="sample", fmt="bf16", layers=32, groups=4, each=8, kv_heads=8, d=128,
             lo=1031, hi=4093, page=32),
        # a serving step with drafts: every sequence gets a few draft tokens, a few requests come in whole; then the drafts are
        # cut off again and those requests retire
        dict(name="fork draft step", op="fork", kind="draft", fmt="bf16", layers=4, groups=24, each=1, kv_heads=4, d=64,
             lo=97, hi=1231, page=16),
        # the pool of the smallest configuration: latency
        dict(name="compact tiny", op="compact", fmt="bf16", layers=4, batch=2, kv_heads=4, d=64, lo=49, hi=146, page=16,
             live=0.6),
        # a pool that requests of all lengths have come and gone from, six tenths full
        dict(name="compact pool", op="compact", fmt="bf16", layers=8, batch=32, kv_heads=8, d=128, lo=97, hi=1231, page=32,
             live=0.6),
        # a request's pages of 8-bit rows to another pool: latency
        dict(name="copy one request", op="copy", fmt="int8", kv_heads=8, d=128, page=16, pages=12),
        # the caches of a batch handed from one pool to another
        dict(name="copy batch", op="copy", fmt="bf16", kv_heads=8, d=128, page=32, pages=2011),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    op = rng.choice(["prefill", "prefill", "attend", "attend", "attend", "fork", "fork", "compact", "copy"])
    page = rng.choice([16, 16, 32, 48, 64, 128, 256])
    d = rng.choice([64, 128, 128])
    fmt = rng.choice(["bf16", "bf16", "int8", "e4m3"])
    if op == "prefill":
        kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8])
        kv = max(1, min(kv, 32 // group))
        batch = _log_int(rng, 1, 8)
        mean = _log_int(rng, 1, 6000 // batch if batch > 2 else 3000)
        spread = rng.choice([0.0, 0.5, 0.9])
        return dict(op=op, batch=batch, q_heads=kv * group, kv_heads=kv, d=d, lo=max(1, int(mean * (1 - spread))),
                    hi=max(1, int(mean * (1 + 0.5 * spread))), gain=rng.choice([True, True, False]))
    if op == "attend":
        kv, group = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 3, 4, 5, 8])
        rows = _log_int(rng, 2000, 2_000_000)                # over all layers, sequences and heads
        batch, layers = _log_int(rng, 1, 64), _log_int(rng, 1, 8)
        mean = max(2, min(131071, rows // (kv * batch * layers)))
        spread = rng.choice([0.0, 0.3, 0.9])
        return dict(op=op, fmt=fmt, layers=layers, batch=batch, q_heads=kv * group, kv_heads=kv, d=d,
                    lo=max(1, int(mean * (1 - spread))), hi=max(1, int(mean * (1 + spread))), page=page,
                    gain=rng.choice([True, True, False]))
    if op == "copy":
        kv = rng.choice([1, 4, 8, 32])
        return dict(op=op, fmt=fmt, kv_heads=kv, d=d, page=page, pages=max(1, _log_int(rng, 16, 500_000) // (kv * page)))
    kv = rng.choice([1, 4, 8])
    rows = _log_int(rng, 1000, 1_000_000) // kv              # over all layers and sequences
    if op == "fork":
        kind = rng.choice(["sample", "beam", "draft"])
        each = 1 if kind == "draft" else rng.choice([2, 3, 4, 8])
        layers, groups = _log_int(rng, 1, 32), _log_int(rng, 1, 64 if kind == "draft" else 12)
        mean = max(1, min(6000, rows // (layers * groups * (each if kind == "beam" else 1))))
        return dict(op=op, kind=kind, fmt=fmt, layers=layers, groups=groups, each=each, kv_heads=kv, d=d, lo=max(1, mean // 2),
                    hi=max(1, mean + mean // 2), page=page)
    layers, batch = _log_int(rng, 1, 32), _log_int(rng, 1, 64)
    mean = max(1, min(6000, rows // (layers * batch)))
    return dict(op=op, fmt=fmt, layers=layers, batch=batch, kv_heads=kv, d=d, lo=max(1, mean // 2),
                hi=max(1, mean + mean // 2), page=page, live=rng.choice([0.3, 0.6, 0.9]))


def _ints(lo, hi, shape, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(lo, max(lo, hi) + 1, shape, generator=g, dtype=torch.int64)


def _lengths(case):
    """The case's lengths.  The totals that work() goes by are those of the case's own numbers, not of the seed."""
    g = sum(ord(ch) for ch in repr(sorted((k, v) for k, v in case.items() if k != "name")))
    if case["op"] == "prefill":
        return _ints(case["lo"], case["hi"], (case["batch"],), g)
    if case["op"] == "fork":
        lens = _ints(case["lo"], case["hi"], (case["layers"], case["groups"], case["each"]), g)
        if case["kind"] == "sample":
            lens[:, :, 1:] = 0                               # the samples' places are empty
        if case["kind"] == "beam":
            lens = lens[:, :, :1].repeat(1, 1, case["each"])  # a prompt's beams are of one length
        if case["kind"] == "draft":
            lens[:, ::8] = 0                                 # requests that come in whole and retire
        return lens.reshape(case["layers"], -1)
    return _ints(case["lo"], case["hi"], (case["layers"], case["batch"]), g)


# ------------------------------------------------------------------ inputs
def _rows(shape, gen, kind):
    """Rows as a model's projections give them: K with channels of their own size, V with tokens of their own size."""
    x = torch.randn(shape, generator=gen, device="cuda")
    if kind == "k":
        return x * torch.exp(torch.rand(shape[-1], generator=gen, device="cuda") * 2.0 - 1.0)
    return x * torch.exp(torch.rand(shape[:-1], generator=gen, device="cuda").unsqueeze(-1) * 1.5)


def _power_scale(amax):
    """Smallest power of two s with amax <= 448 s; exact (frexp)."""
    m, e = torch.frexp(amax)                                 # amax = m 2^e, m in [0.5, 1);  448 = 0.875 2^9
    return torch.ldexp(torch.ones_like(amax), torch.where(m <= 0.875, e - 9, e - 8).clamp(-100, 120))


def _fill_pages(n_pages, heads, page, d, fmt, gen, kind):
    """Pages full of rows, as their format stores them, and the scales (bf16: None)."""
    dtype = torch.bfloat16 if fmt == "bf16" else torch.uint8
    pages = torch.empty(n_pages, heads, page, d, dtype=dtype, device="cuda")
    scales = None if fmt == "bf16" else torch.empty(n_pages, heads, page if fmt == "int8" else page // BLOCK, device="cuda")
    step = max(1, (1 << 26) // (heads * page * d))
    for at in range(0, n_pages, step):
        n = min(step, n_pages - at)
        x = _rows((n, heads, page, d), gen, kind).to(torch.bfloat16)
        if fmt == "bf16":
            pages[at:at + n] = x
        elif fmt == "int8":
            s = x.float().abs().amax(-1) / 127.0
            scales[at:at + n] = s
            pages[at:at + n] = (torch.round(x.float() / s[..., None]).clamp(-127, 127) + 128).to(torch.uint8)
        else:
            b = x.float().view(n, heads, page // BLOCK, BLOCK, d)
            s = _power_scale(b.abs().amax((-1, -2)))
            scales[at:at + n] = s
            pages[at:at + n] = (b / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(n, heads, page, d)
    return pages, scales


def _spread_pages(lens, page, cols, n_pages, seed):
    """Block tables [.., cols] of pages in shuffled order (-1 behind them), and the pages that are left, shuffled."""
    need = -(-lens // page)
    total = int(need.sum())
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
    have = torch.arange(cols) < need.reshape(-1, 1)
    table = torch.full(have.shape, -1, dtype=torch.int64)
    table[have] = order[:total]
    return table.reshape(*lens.shape, cols).to(torch.int32), order


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case, op=case["op"])
    {"prefill": _prepare_prefill, "attend": _prepare_attend, "fork": _prepare_fork, "compact": _prepare_compact,
     "copy": _prepare_copy}[case["op"]](st, case, seed, gen)
    if own:                                                  # the handle and the workspace that a program keeps
        _handles(st)
    return st


def _queries(shape, gen):
    """Query rows of two halves, flat and peaked maps among them."""
    q = torch.randn(*shape[:-1], 2, shape[-1] // 2, generator=gen, device="cuda")
    q = q * torch.exp(torch.rand(*shape[:-1], 2, 1, generator=gen, device="cuda") * 1.5 - 0.5)
    return q.view(shape).to(torch.bfloat16)


def _weights(st, lead, heads, d, gain, gen):
    st["lam"] = torch.rand(*lead, heads, generator=gen, device="cuda") * 0.7 + 0.1
    st["gain"] = torch.rand(*lead, d, generator=gen, device="cuda") + 0.2 if gain else None


def _prepare_prefill(st, case, seed, gen):
    lens = _lengths(case)
    T, Hq, H, d = int(lens.sum()), case["q_heads"], case["kv_heads"], case["d"]
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
    _weights(st, (), Hq, d, case["gain"], gen)
    st.update(T=T, Hq=Hq, H=H, d=d, lens=lens.tolist(), cu=cu.to(torch.int32).cuda(), q=_queries((T, Hq, d), gen),
              k=_rows((T, H, d), gen, "k").to(torch.bfloat16), v=_rows((T, H, d), gen, "v").to(torch.bfloat16),
              out=torch.empty(T, Hq, d, dtype=torch.bfloat16, device="cuda"), lse=torch.empty(Hq, 2, T, device="cuda"))


def _pool(st, case, n_pages, gen, suffix=""):
    for kind in ("k", "v"):
        st[kind + "_pages" + suffix], st[kind + "_scales" + suffix] = _fill_pages(
            n_pages, case["kv_heads"], case["page"], case["d"], case["fmt"], gen, kind)
    st["n_pages" + suffix] = n_pages


def _prepare_attend(st, case, seed, gen):
    lens = _lengths(case)
    L, B, Hq, H, d, page = (case[k] for k in ("layers", "batch", "q_heads", "kv_heads", "d", "page"))
    n_pages = int((-(-lens // page)).sum()) + 3
    table, _ = _spread_pages(lens, page, int(-(-lens.max() // page)) + 1, n_pages, seed)
    table = table.clamp(min=0)
    _pool(st, case, n_pages, gen)
    # what lies behind a cache's last row is whatever the page held before: here NaN, in the scales too
    last = ((lens.reshape(-1) - 1) // page).clamp(min=0)
    tail = table.reshape(L * B, -1).gather(1, last[:, None])[:, 0].long().cuda()
    behind = torch.arange(page, device="cuda") >= (lens.reshape(-1) - last * page).cuda()[:, None]        # [LB, page]
    for kind in ("k", "v"):
        pages, scales = st[kind + "_pages"], st[kind + "_scales"]
        nan = {"bf16": float("nan"), "int8": 255, "e4m3": 0x7F}[case["fmt"]]
        pages[tail] = torch.where(behind[:, None, :, None], torch.full((), nan, dtype=pages.dtype, device="cuda"), pages[tail])
        if scales is not None:
            b = behind[:, None, ::page // scales.shape[-1]]
            scales[tail] = torch.where(b, torch.full((), float("nan"), device="cuda"), scales[tail])
    _weights(st, (L,), Hq, d, case["gain"], gen)
    st.update(L=L, B=B, Hq=Hq, H=H, d=d, max_len=int(lens.max()), table=table.cuda(), lens=lens.to(torch.int32).cuda(),
              q=_queries((L, B, Hq, d), gen), out=torch.empty(L, B, Hq, d, dtype=torch.bfloat16, device="cuda"),
              lse=torch.empty(L, B, Hq, 2, device="cuda"))


def _prepare_fork(st, case, seed, gen):
    lens = _lengths(case)
    L, page, G, n = case["layers"], case["page"], case["groups"], case["each"]
    B = G * n
    more = torch.zeros(B, dtype=torch.int64)
    if case["kind"] == "draft":                              # draft tokens, and whole requests in the empty places
        more = torch.where(lens[0] == 0, case["hi"], 1 + torch.arange(B) % 8)
    need = -(-lens // page)
    # room for every last page's copy (and, of drafts, for the tokens to come)
    n_pages = int(need.sum() + (-(-(lens + more) // page) - need).sum()) + 2 * L * B + 5
    table, order = _spread_pages(lens, page, int(-(-(lens + more).max() // page)) + 1, n_pages, seed)
    _pool(st, case, n_pages, gen)
    me = torch.arange(B)
    if case["kind"] == "sample":
        steps = [me // n * n, torch.where(me % n == 0, me, -1)]
    elif case["kind"] == "beam":                             # two steps of a search: each beam goes on from one of its prompt's
        pick = torch.randint(0, n, (2, B), generator=torch.Generator().manual_seed(seed + 1))
        steps = [me // n * n + pick[0], me // n * n + pick[1]]
    else:
        steps = [torch.where(lens[0] == 0, -1, me)]
    ints = dict(dtype=torch.int32, device="cuda")
    st.update(L=L, B=B, H=case["kv_heads"], d=case["d"], table=table.cuda(), lens=lens.to(**ints), cols=table.shape[-1],
              shares=torch.zeros(n_pages, **ints), free=order.to(**ints), used=torch.tensor([int(need.sum())], **ints),
              steps=[s.to(**ints) for s in steps], keep=lens.to(**ints) if case["kind"] == "draft" else None,
              more=more.to(**ints) if case["kind"] == "draft" else None)


def _prepare_compact(st, case, seed, gen):
    lens = _lengths(case)
    L, B, page = case["layers"], case["batch"], case["page"]
    need = -(-lens // page)
    n_pages = int(int(need.sum()) / case["live"]) + 1
    table, _ = _spread_pages(lens, page, int(need.max()) + 1, n_pages, seed)
    if B > 1:                                                # the first half of the last cache's pages are the one's before it
        half = (torch.minimum(need[:, -1], need[:, -2]) // 2)[:, None]
        table[:, -1] = torch.where(torch.arange(table.shape[-1]) < half, table[:, -2], table[:, -1])
    _pool(st, case, n_pages, gen)
    shares = torch.zeros(n_pages, dtype=torch.int32)
    held = torch.arange(table.shape[-1]) < need[..., None]
    shares.index_add_(0, table[held].long(), torch.ones(int(held.sum()), dtype=torch.int32))
    st.update(L=L, B=B, H=case["kv_heads"], d=case["d"], before=table.cuda(), table=torch.empty_like(table, device="cuda"),
              lens=lens.to(torch.int32).cuda(), cols=table.shape[-1], shares_before=(shares - 1).clamp(min=0).cuda(),
              shares=torch.empty(n_pages, dtype=torch.int32, device="cuda"),
              free=torch.zeros(n_pages, dtype=torch.int32, device="cuda"), used=torch.zeros(1, dtype=torch.int32, device="cuda"))


def _prepare_copy(st, case, seed, gen):
    n = case["pages"]
    _pool(st, case, n + 7, gen)
    _pool(st, case, n + 5, gen, "_to")
    g = torch.Generator().manual_seed(seed)
    st.update(H=case["kv_heads"], d=case["d"], src=torch.randperm(n + 7, generator=g)[:n].to(torch.int32).cuda(),
              dst=torch.randperm(n + 5, generator=g)[:n].to(torch.int32).cuda())


def _handles(st):
    from paper_2412_05896_b200 import xkv
    case, op, d = st["case"], st["op"], st["d"]
    st["xkv"] = xkv
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    fmt = {"bf16": xkv.KV_BF16, "int8": xkv.KV_INT8, "e4m3": xkv.KV_E4M3}.get(case.get("fmt"))

    def cache(suffix="", table=None, lens=None, layers=1, cols=1):
        return xkv.Cache(ptr(st["k_pages" + suffix]), ptr(st["v_pages" + suffix]), ptr(table), ptr(lens), layers, case["page"],
                         cols, st["n_pages" + suffix], ptr(st["k_scales" + suffix]), ptr(st["v_scales" + suffix]), fmt, 0)

    H, batch, Hq = st["H"], st.get("B", 1), st.get("Hq", st["H"])
    if op == "prefill":
        batch = case["batch"]
    st["dims"] = xkv.Dims(batch, Hq, H, d, 1, 1, 0, 0.0, H * d, d)
    if op == "prefill":
        nbytes = xkv.workspace_bytes(xkv.OP_DIFF_PREFILL_ATTN, st["dims"])
    elif op == "attend":
        cols = st["table"].shape[-1]
        st["cache"] = cache(table=st["table"], lens=st["lens"], layers=st["L"], cols=cols)
        nbytes = xkv.workspace_bytes(xkv.OP_DIFF_DECODE_ATTN, st["dims"], n_layers=st["L"], max_cache_len=cols * case["page"])
    elif op == "copy":
        st["cache"], st["cache_to"] = cache(), cache("_to")
        nbytes = xkv.workspace_bytes(xkv.OP_COPY_PAGES, st["dims"])
    else:
        which = xkv.OP_FORK_CACHES if op == "fork" else xkv.OP_COMPACT_PAGES
        st["cache"] = cache(table=st["table"], lens=st["lens"], layers=st["L"], cols=st["cols"])
        nbytes = xkv.workspace_bytes(which, st["dims"], max_seqlen=st["cols"], total_tokens=st["n_pages"], n_layers=st["L"])
        if op == "fork" and st["more"] is not None:
            st["ws_plan"] = torch.zeros(xkv.workspace_bytes(xkv.OP_PLAN_APPEND, st["dims"], n_layers=st["L"]),
                                        dtype=torch.uint8, device="cuda")
    st["workspace"] = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ one pass
def run(st):
    return {"prefill": _run_prefill, "attend": _run_attend, "fork": _run_fork, "compact": _run_compact,
            "copy": _run_copy}[st["op"]](st)


def _run_prefill(st):
    if own:
        st["xkv"].diff_prefill_attn(st["dims"], st["q"], st["k"], st["v"], st["lam"], st["gain"], EPS, st["cu"], st["T"],
                                    max(st["lens"]), st["out"], st["lse"], st["workspace"])
        return {"out": st["out"], "lse": st["lse"]}
    return _prefill(st)


def _run_attend(st):
    if own:
        st["xkv"].diff_decode_attn(st["dims"], st["cache"], 0, st["L"], st["q"], None, None, st["lam"], st["gain"], EPS,
                                   st["out"], st["lse"], 0, st["workspace"])
        return {"out": st["out"], "lse": st["lse"]}
    return _attend(st)


def _bits(st, suffix=""):
    """Pages and scales as they are stored."""
    got = {n + suffix: st[n + suffix] for n in ("k_pages", "v_pages", "k_scales", "v_scales")}
    return {n: (t.view(torch.int16) if t.dtype == torch.bfloat16 else t) for n, t in got.items() if t is not None}


def _run_fork(st):
    if st["more"] is not None:
        if own:
            st["xkv"].plan_append(st["cache"], st["B"], st["more"], 0, st["lens"], st["free"], st["n_pages"], st["used"],
                                  st["used"], None, 0, st["ws_plan"])
        else:
            _grow(st)
    for parent in st["steps"]:
        if own:
            st["xkv"].fork_caches(st["dims"], st["cache"], parent, st["keep"], st["B"], st["shares"], st["free"],
                                  st["n_pages"], st["used"], st["workspace"])
        else:
            _fork(st, parent)
    return {"table": st["table"], "lens": st["lens"], "shares": st["shares"], "free": st["free"], "used": st["used"], **_bits(st)}


def _run_compact(st):
    if own:
        st["xkv"].compact_pages(st["dims"], st["cache"], st["before"], st["shares_before"], st["shares"], st["free"], st["used"],
                                st["workspace"])
    else:
        _compact(st)
    return {"table": st["table"], "shares": st["shares"], "free": st["free"], "used": st["used"], **_bits(st)}


def _run_copy(st):
    if own:
        st["xkv"].copy_pages(st["dims"], st["cache"], st["src"], st["cache_to"], st["dst"], st["case"]["pages"], st["workspace"])
    else:
        for name in ("k_pages", "v_pages", "k_scales", "v_scales"):
            if st[name] is not None:
                st[name + "_to"][st["dst"].long()] = st[name][st["src"].long()]
    return _bits(st, "_to")


# ------------------------------------------------------------------ plain forms
def _difference(z, v, lam, gain):
    """z [.., 2, rows, keys] logits (-inf where masked), v [.., keys, d], lam and gain shaped to go with [.., rows, d]."""
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    a = p / torch.where(total > 0, total, torch.ones_like(total))
    y = torch.matmul(a[..., 0, :, :], v) - lam * torch.matmul(a[..., 1, :, :], v)
    if gain is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS) * gain
    return y.to(torch.bfloat16), (top + torch.log(total))[..., 0]


def _prefill(st):
    Hq, H, d = st["Hq"], st["H"], st["d"]
    out, lse = torch.empty_like(st["out"]), torch.empty_like(st["lse"])
    at = 0
    for n in st["lens"]:
        rows = slice(at, at + n)
        q = st["q"][rows].float().view(n, Hq, 2, d // 2).permute(1, 2, 0, 3)
        k = st["k"][rows].float().view(n, H, 2, d // 2).permute(1, 2, 3, 0).repeat_interleave(Hq // H, 0)
        v = st["v"][rows].float().transpose(0, 1).repeat_interleave(Hq // H, 0)
        z = torch.matmul(q, k) / math.sqrt(d // 2)
        z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device=z.device).triu(1), float("-inf"))
        y, s = _difference(z, v, st["lam"][:, None, None], st["gain"])
        out[rows], lse[..., rows] = y.transpose(0, 1), s
        at += n
    return {"out": out, "lse": lse}


def _values(pages, scales, fmt):
    """What stored rows [.., page, d] stand for."""
    if fmt == "bf16":
        return pages.float()
    if fmt == "int8":
        return (pages.float() - 128.0) * scales[..., None]
    x = pages.view(torch.float8_e4m3fn).float()
    return (x.view(*x.shape[:-2], -1, BLOCK, x.shape[-1]) * scales[..., None, None]).view(x.shape)


def _attend(st):
    L, B, Hq, H, d, page = st["L"], st["B"], st["Hq"], st["H"], st["d"], st["case"]["page"]
    G, cols = Hq // H, -(-st["max_len"] // page)
    at = st["table"][..., :cols].reshape(-1).long()
    n = cols * page

    def rows(kind):
        s = st[kind + "_scales"]
        x = _values(st[kind + "_pages"][at], None if s is None else s[at], st["case"]["fmt"])
        return x.view(L * B, cols, H, page, d).transpose(1, 2).reshape(L * B, H, n, d)

    live = torch.arange(n, device=at.device) < st["lens"].reshape(-1, 1, 1, 1)                        # [LB, 1, 1, n]
    q = st["q"].float().view(L * B, H, G, 2, d // 2).transpose(2, 3)                                  # [LB, H, 2, G, d/2]
    k = rows("k").view(L * B, H, n, 2, d // 2).permute(0, 1, 3, 4, 2)                                 # [LB, H, 2, d/2, n]
    z = torch.matmul(q, k) / math.sqrt(d // 2)
    z = torch.where(live[:, :, None], z, torch.full_like(z, float("-inf")))
    v = rows("v")
    v = torch.where(live.transpose(-1, -2), v, torch.zeros_like(v))
    lam = st["lam"].view(L, 1, H, G, 1).expand(L, B, H, G, 1).reshape(L * B, H, G, 1)
    gain = None if st["gain"] is None else st["gain"].view(L, 1, 1, d).expand(L, B, 1, d).reshape(L * B, 1, 1, d)
    y, s = _difference(z, v, lam, gain)
    return {"out": y.view(L, B, Hq, d), "lse": s.transpose(2, 3).reshape(L, B, Hq, 2)}


def _grow(st):
    """Pages and lengths for more tokens of every cache, in the order of (layer, sequence)."""
    page, lens, more = st["case"]["page"], st["lens"].long(), st["more"].long().expand(st["L"], -1)
    have, need = -(-lens // page), -(-(lens + more) // page)
    ask = need - have
    start = (ask.reshape(-1).cumsum(0) - ask.reshape(-1)).view_as(ask) + st["used"].long()
    col = torch.arange(st["cols"], device=lens.device)
    take = (start[..., None] + col - have[..., None]).clamp(0, st["free"].numel() - 1)
    fresh = (col >= have[..., None]) & (col < need[..., None])
    st["table"].copy_(torch.where(fresh, st["free"][take], st["table"]))
    st["lens"].copy_(lens + more)
    st["used"].add_(ask.sum())


def _fork(st, parent):
    page, B, cols, n_pages = st["case"]["page"], st["B"], st["cols"], st["n_pages"]
    dev = parent.device
    parent, me = parent.long(), torch.arange(B, device=dev)
    src, lens, table = parent.clamp(min=0), st["lens"].long(), st["table"].long()
    new_lens = torch.where(parent >= 0, lens[:, src], torch.zeros_like(lens))
    if st["keep"] is not None:
        new_lens = torch.minimum(new_lens, st["keep"].long())
    col = torch.arange(cols, device=dev)
    old, new = col < (-(-lens // page))[..., None], col < (-(-new_lens // page))[..., None]
    fresh = torch.where(new, table[:, src], table)

    def count(entries, mask):                                # per page, how many of the masked entries hold it
        at = torch.where(mask, entries, torch.full_like(entries, n_pages)).reshape(-1)
        return torch.zeros(n_pages + 1, dtype=torch.int64, device=dev).index_add_(0, at, torch.ones_like(at))[:n_pages]

    was = count(table, old)
    holders = st["shares"].long() + 1 - was + count(fresh, new)
    gone = (was > 0) & (holders == 0)
    # last pages that are partly filled: all but one of those that share one get a copy, all of them if others hold it whole
    part = new_lens % page > 0
    last = fresh.gather(2, (-(-new_lens // page) - 1).clamp(min=0)[..., None])[..., 0]
    last = torch.where(part, last, torch.zeros_like(last))
    all_part = count(last, part)[last] == holders[last]
    key = (me + torch.where(parent == me, 0, B)).expand_as(last)
    first = torch.full((n_pages,), 2 * B, dtype=torch.int64, device=dev).scatter_reduce_(
        0, last[part], key[part], "amin")
    copy = part & (holders[last] > 1) & ~(all_part & (key == first[last]))
    l, b = torch.nonzero(copy, as_tuple=True)
    used = st["used"].long()
    to, frm = st["free"][used + torch.arange(l.numel(), device=dev)].long(), last[l, b]
    rows = (new_lens[l, b] % page)[:, None] > torch.arange(page, device=dev)                          # [copies, page]
    for name in ("k_pages", "v_pages"):
        st[name][to] = torch.where(rows[:, None, :, None], st[name][frm], st[name][to])
    for name in ("k_scales", "v_scales"):
        if st[name] is not None:
            per = page // st[name].shape[-1]                 # rows a scale stands for
            st[name][to] = torch.where(rows[:, None, ::per], st[name][frm], st[name][to])
    fresh[l, b, -(-new_lens[l, b] // page) - 1] = to
    holders.index_add_(0, frm, torch.full_like(frm, -1))
    back = torch.nonzero(gone)[:, 0]                         # ascending
    used = used + l.numel() - back.numel()
    st["free"][used + torch.arange(back.numel(), device=dev)] = back.to(torch.int32)
    st["used"].copy_(used)
    st["shares"].copy_((holders - 1).clamp(min=0))
    st["table"].copy_(fresh)
    st["lens"].copy_(new_lens)


def _compact(st):
    page, n_pages = st["case"]["page"], st["n_pages"]
    table = st["before"].long()
    dev = table.device
    held = torch.arange(st["cols"], device=dev) < (-(-st["lens"].long() // page))[..., None]
    live = torch.zeros(n_pages, dtype=torch.bool, device=dev)
    live[table[held]] = True
    n_live = live.sum()
    low = torch.arange(n_pages, device=dev) < n_live
    frm, to = torch.nonzero(live & ~low)[:, 0], torch.nonzero(~live & low)[:, 0]
    moved = torch.arange(n_pages, device=dev)
    moved[frm] = to
    for name in ("k_pages", "v_pages", "k_scales", "v_scales"):
        if st[name] is not None:
            st[name][to] = st[name][frm]
    st["table"].copy_(torch.where(held, moved[table.clamp(min=0)], table))
    shares = torch.where(low & live, st["shares_before"], torch.zeros_like(st["shares_before"]))
    shares[to] = st["shares_before"][frm]
    st["shares"].copy_(shares)
    at = torch.arange(n_pages, device=dev, dtype=torch.int32)
    st["free"].copy_(torch.where(low, st["free"], at))
    st["used"].copy_(n_live)


# ------------------------------------------------------------------ what a pass cannot do without
def _page_bytes(case, rows=None):
    """Bytes of K and V and their scales in `rows` rows (default: a page) of every KV head."""
    rows = case["page"] if rows is None else rows
    per_row = {"bf16": 2 * case["d"], "int8": case["d"] + 4, "e4m3": case["d"] + 4 / BLOCK}[case["fmt"]]
    return 2 * case["kv_heads"] * rows * per_row


def work(case):
    op, d, page = case["op"], case["d"], case.get("page")
    if op == "copy":
        return {"bytes": case["pages"] * (2 * _page_bytes(case) + 8), "flops": 0}
    lens = _lengths(case)
    if op == "prefill":
        T, pairs = int(lens.sum()), int((lens * (lens + 1) // 2).sum())
        return {"bytes": T * (4 * d * (case["q_heads"] + case["kv_heads"]) + 8 * case["q_heads"]),
                "flops": 6.0 * d * pairs * case["q_heads"]}
    pages = -(-lens // page)
    if op == "attend":
        heads = case["layers"] * case["batch"] * case["q_heads"]
        return {"bytes": _page_bytes(case, int(lens.sum())) + heads * (4 * d + 8) + int(pages.sum()) * 4 + lens.numel() * 4,
                "flops": 6.0 * d * int(lens.sum()) * case["q_heads"]}
    if op == "compact":
        n_live = int(pages.sum())
        if case["batch"] > 1:
            n_live -= int((torch.minimum(pages[:, -1], pages[:, -2]) // 2).sum())
        n_pages = int(int(pages.sum()) / case["live"]) + 1
        moved = n_live * (n_pages - n_live) / n_pages        # what pages spread at random give
        entries = lens.shape[0] * lens.shape[1] * (int(pages.max()) + 1)
        return {"bytes": 2 * moved * _page_bytes(case) + 8 * entries + 4 * lens.numel() + 8 * n_pages + 4 * (n_pages - n_live),
                "flops": 0}
    n = case["each"]
    if case["kind"] == "draft":                              # pages for the drafts and back again
        more = torch.where(lens[0] == 0, case["hi"], 1 + torch.arange(lens.shape[1]) % 8)
        fresh = int((-(-(lens + more) // page) - pages).sum())
        return {"bytes": 20 * lens.numel() + 20 * fresh, "flops": 0}
    lead = lens.view(case["layers"], case["groups"], n)[..., :1]
    part, whole = lead % page, -(-lead // page)
    if case["kind"] == "sample":
        # the samples' entries written, read again to be dropped; the pages' counters up and down; last pages read once and
        # written for each sample
        return {"bytes": int(whole.sum()) * (4 + 8 * (n - 1) + 16) + 20 * lens.numel() + _page_bytes(case, int(part.sum())) * n,
                "flops": 0}
    # two steps: tables read and written, lengths, counters; about n - 1 of a prompt's n last pages copied
    return {"bytes": 2 * (int(whole.sum()) * n * 16 + 8 * lens.numel() + 2 * _page_bytes(case, int(part.sum())) * (n - 1)), "flops": 0}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    if case["op"] not in ("prefill", "attend"):
        return None                                          # whole numbers and copies only
    st = prepare(case, seed)
    return _exact_prefill(st) if case["op"] == "prefill" else _exact_attend(st)


def _exact_head(q, k, v, lam, gain, visible=None):
    """q [rows, d], k and v [keys, d] in 64 bits -> (out [rows, d], the two maps' log sums [2, rows])."""
    half = q.shape[1] // 2
    y, sums = 0.0, []
    for at, sign in ((0, 1.0), (half, -lam)):
        z = q[:, at:at + half] @ k[:, at:at + half].T * half ** -0.5
        if visible is not None:
            z.masked_fill_(~visible, float("-inf"))
        s = torch.logsumexp(z, 1)
        y = y + sign * (torch.exp(z - s[:, None]) @ v)
        sums.append(s)
    if gain is not None:
        y = y * torch.rsqrt(y.square().sum(1, keepdim=True) / y.shape[1] + EPS) * gain
    return y, torch.stack(sums)


def _exact_prefill(st):
    Hq, G = st["Hq"], st["Hq"] // st["H"]
    out = torch.zeros(st["T"], Hq, st["d"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(Hq, 2, st["T"], dtype=torch.float64, device="cuda")
    gain = None if st["gain"] is None else st["gain"].double()
    at = 0
    for n in st["lens"]:
        i = torch.arange(n, device="cuda")
        for h in range(Hq):
            q, k, v = st["q"][at:at + n, h].double(), st["k"][at:at + n, h // G].double(), st["v"][at:at + n, h // G].double()
            out[at:at + n, h], lse[h, :, at:at + n] = _exact_head(q, k, v, st["lam"][h].double(), gain, i[None, :] <= i[:, None])
        at += n
    return {"out": out, "lse": lse}


def _exact_attend(st):
    L, B, Hq, H, d, page, fmt = st["L"], st["B"], st["Hq"], st["H"], st["d"], st["case"]["page"], st["case"]["fmt"]
    G = Hq // H
    out = torch.zeros(L, B, Hq, d, dtype=torch.float64)
    lse = torch.full((L, B, Hq, 2), float("-inf"), dtype=torch.float64)

    def rows(kind, pages, inside, g):
        x = st[kind + "_pages"][pages, g, inside]
        if fmt == "bf16":
            return x.double()
        s = st[kind + "_scales"][pages, g, inside if fmt == "int8" else inside // BLOCK].double()[:, None]
        return (x.double() - 128.0) * s if fmt == "int8" else x.view(torch.float8_e4m3fn).double() * s

    for l in range(L):
        gain = None if st["gain"] is None else st["gain"][l].double()
        for b in range(B):
            slot = torch.arange(int(st["lens"][l, b]), device="cuda")
            pages, inside = st["table"][l, b].long()[slot // page], slot % page
            for g in range(H):
                k, v = rows("k", pages, inside, g), rows("v", pages, inside, g)
                heads = slice(g * G, (g + 1) * G)
                y, s = _exact_head(st["q"][l, b, heads].double(), k, v, st["lam"][l, heads, None].double(), gain)
                out[l, b, heads], lse[l, b, heads] = y.cpu(), s.T.cpu()
    return {"out": out, "lse": lse}
