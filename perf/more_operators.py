"""Cases of attention that does not scan each request's whole cache by itself.

Two operators over the paged bf16 cache.  Attention with a sliding window and
sinks (`mx_paged_attn_window`): a token sees the last `window` positions up to its
own and the first `sinks` of its request; pages that no new token sees may have
been freed, and their table entries hold -1.  Attention over shared runs
(`mx_paged_attn_shared`): consecutive requests whose page tables agree in a run of
pages (a system prompt, a document, a branch of either) have the run's keys read
once for all of them.

A batch is `decodes` requests in the decode phase, then `prefill` prompt tokens in
`chunks` ragged chunks.  Of a "window" case the decodes' contexts are uniform in
[ctx_lo, ctx_hi] and the first chunk continues a prompt of `cached` tokens.  Of a
"shared" case all of these share the first `prefix` tokens, and each of `branches`
equal parts of them `branch` more; a decode has another ctx_lo .. ctx_hi tokens of
its own; `alone` decodes without a shared token, of ctx_lo + 1 .. ctx_hi + 1, follow.

`own` false computes the operators in plain torch operations in 32 bits, `own`
true through the library's entry points.
"""
import math

import numpy as np
import torch

own = False

# The benchmark's attention shapes: query heads, KV heads, head dim.
SHAPES = {
    "tiny": (4, 4, 64),
    "7b": (32, 32, 128),
    "13b": (40, 40, 128),
    "8b": (32, 8, 128),
    "70b": (64, 8, 128),
}
PAGE = 16
FAR = 1 << 30  # the position of padding keys: behind every token


def _case(kind, shape, decodes=0, ctx_lo=0, ctx_hi=0, prefill=0, chunks=0, cached=0, window=0,
          sinks=0, prefix=0, branches=0, branch=0, alone=0, name=None):
    c = dict(kind=kind, shape=shape, decodes=decodes, ctx_lo=ctx_lo, ctx_hi=ctx_hi,
             prefill=prefill, chunks=chunks, cached=cached, window=window, sinks=sinks,
             prefix=prefix, branches=branches, branch=branch, alone=alone)
    if name:
        c["name"] = name
    return c


def _window(shape, window, sinks, *batch, **kw):
    return _case("window", shape, *batch, window=window, sinks=sinks, **kw)


def _shared(shape, prefix, *batch, **kw):
    return _case("shared", shape, *batch, prefix=prefix, **kw)


def listed():
    return [
        # the smallest call: one decode of a 256-wide layer (head dim 64) past its window
        _window("tiny", 128, 4, 1, 250, 250, name="window tiny one decode"),
        # a decode batch on a layer with a short window
        _window("8b", 1024, 4, 64, 500, 16384, name="window 8b decode"),
        # a large decode batch with a long window: streams the cache
        _window("8b", 4096, 16, 128, 2000, 32000, name="window 8b many decodes"),
        # a whole prompt of odd length on an MHA layer, local attention only
        _window("7b", 1024, 0, 0, 0, 0, 8191, 1, 0, name="window 7b prompt"),
        # a late chunk of a long prompt
        _window("70b", 4096, 64, 0, 0, 0, 2048, 1, 14336, name="window 70b late chunk"),
        # a multiplexed iteration: decodes and ragged chunks, an odd window
        _window("70b", 1023, 5, 64, 32, 8192, 1024, 3, 5000, name="window 70b mixed"),
        # few requests of one short system prompt: bound by latency
        _shared("8b", 512, 4, 1, 60, name="shared 8b four decodes"),
        # an MHA decode batch of one system prompt
        _shared("7b", 2000, 32, 16, 700, name="shared 7b decode"),
        # a large batch that reads one long document
        _shared("70b", 16384, 128, 16, 512, name="shared 70b long document"),
        # a tree: a system prompt, four sets of examples below it, other requests beside it
        _shared("8b", 2048, 128, 30, 900, branches=4, branch=1008, alone=16, name="shared 8b tree"),
        # several samples of one prompt, far into their answers: little is shared
        _shared("13b", 1008, 16, 1000, 3000, name="shared 13b samples"),
        # short questions about one document as prompts, beside decodes of it
        _shared("8b", 8192, 24, 16, 400, 1500, 12, name="shared 8b questions"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        # at most what the largest listed cases read and compute
        if w["bytes"] <= 2.1e9 and w["flops"] <= 2.8e11:
            return c


def _draw(rng):
    shape = rng.choice(sorted(SHAPES))
    mix = rng.choice(["decode", "decode", "mixed", "prefill"])
    decodes = lo = hi = prefill = chunks = 0
    if rng.random() < 0.5:
        window, sinks = _log_int(rng, 16, 8192), rng.choice([0, 0, 1, 4, 16, _log_int(rng, 1, 300)])
        cached = 0
        if mix != "prefill":
            decodes = _log_int(rng, 1, 256)
            hi = _log_int(rng, 64, 32768)
            lo = rng.randint(max(1, hi // 16), hi)
        if mix != "decode":
            prefill, chunks = _log_int(rng, 16, 8192), rng.choice([1, 1, 2, 4])
            cached = rng.choice([0, _log_int(rng, 16, 16384)])
        return _window(shape, window, sinks, decodes, lo, hi, prefill, chunks, cached)
    prefix = PAGE * _log_int(rng, 1, 1024)
    branches = branch = alone = 0
    if mix != "prefill":
        decodes = _log_int(rng, 2, 256)
        hi = _log_int(rng, 2, 4096)
        lo = rng.randint(0, hi)
        alone = rng.choice([0, 0, _log_int(rng, 1, 16)])
    if mix != "decode":
        chunks = _log_int(rng, 2, 16)
        prefill = _log_int(rng, 2 * chunks, 2048)
    if rng.random() < 0.3:
        branches, branch = rng.randint(2, 5), PAGE * _log_int(rng, 1, 128)
        branches = min(branches, decodes + chunks)
    return _shared(shape, prefix, decodes, lo, hi, prefill, chunks, branches=branches, branch=branch,
                   alone=alone)


def _requests(case):
    """(phase, n_new, ctx_len) of the requests: the case alone decides them."""
    D, P, C = case["decodes"], case["prefill"], case["chunks"]
    rng = np.random.default_rng([D, case["ctx_lo"], case["ctx_hi"], P, C, case["cached"]])
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=D).tolist() if D else []
    phase, n_new = [1] * D, [1] * D
    if P:
        cuts = sorted(rng.choice(np.arange(1, P), size=C - 1, replace=False).tolist()) if C > 1 else []
        sizes = np.diff([0] + cuts + [P]).tolist()
        phase += [0] * len(sizes)
        n_new += sizes
        ctx += [case["cached"]] + [0] * (len(sizes) - 1)
    ctx = [c + case["prefix"] + (case["branch"] if case["branches"] else 0) for c in ctx]
    A = case["alone"]
    if A:
        phase, n_new = phase + [1] * A, n_new + [1] * A
        ctx += (1 + rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=A)).tolist()
    return phase, n_new, ctx


def _runs(case):
    """(first request, requests, pages) of the shared runs, outer ones first."""
    if case["kind"] != "shared":
        return []
    n, k = case["decodes"] + case["chunks"], case["branches"]
    runs = [(0, n, case["prefix"] // PAGE)]
    at = [n * i // k for i in range(k + 1)] if k else []
    return runs + [(a, b - a, case["branch"] // PAGE) for a, b in zip(at, at[1:])]


def _seen(case, n, c):
    """The positions that n new tokens after c cached ones see, as (first, end) ranges."""
    if case["kind"] != "window":
        return [(0, c + n)]
    lo = max(0, c - case["window"] + 1)
    s = min(case["sinks"], c + n)
    return [(0, c + n)] if lo <= s else [(0, s), (lo, c + n)]


def _pages_seen(case, n, c):
    return sorted({p for a, b in _seen(case, n, c) if b > a for p in range(a // PAGE, (b - 1) // PAGE + 1)})


def _cuda(a, dtype=torch.int64):
    return torch.as_tensor(np.asarray(a), dtype=dtype, device="cuda")


def _inputs(case, seed):
    """The case's data: batch in plain lists, page tables, the pools, the queries."""
    nq, nkv, d = SHAPES[case["shape"]]
    phase, n_new, ctx = _requests(case)
    R = len(n_new)
    own_of = [list(_pages_seen(case, n, c)) for n, c in zip(n_new, ctx)]
    pages = [np.full(-(-(c + n) // PAGE), -1, np.int32) for c, n in zip(ctx, n_new)]
    start = [0] * R  # a request's pages before this one are shared
    runs = []
    for first, n, k in _runs(case):
        runs.append((first, n, start[first], k))
        for r in range(first, first + n):
            start[r] += k
    total = sum(k for _, _, _, k in runs) + sum(sum(p >= s for p in o) for o, s in zip(own_of, start))
    pool_pages = total + total // 8 + 8
    order = iter(np.random.default_rng(seed).permutation(pool_pages).astype(np.int32)[:total])
    for first, n, at, k in runs:
        ids = np.fromiter(order, np.int32, k)
        for r in range(first, first + n):
            pages[r][at:at + k] = ids
    for r in range(R):
        mine = [p for p in own_of[r] if p >= start[r]]
        pages[r][mine] = np.fromiter(order, np.int32, len(mine))
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=g)

    T = sum(n_new)
    # key pages blocked by 32 dims, value pages transposed (the library's pool layout)
    s = dict(kind=case["kind"], case=case, heads=(nq, nkv, d), pages=pages, pool_pages=pool_pages,
             phase=phase, n_new=n_new, ctx=ctx, k_pool=normal(pool_pages, nkv, d // 32, PAGE, 32),
             v_pool=normal(pool_pages, nkv, d, PAGE), q=normal(T, nq, d),
             out=torch.zeros(T, nq, d, dtype=torch.bfloat16, device="cuda"))
    # the first page of a request takes a good part of the weight, as first tokens do
    towards = normal(d)
    s["q"] += (0.3 * towards).to(torch.bfloat16)
    firsts = torch.unique(_cuda([p[0] for p in pages if p[0] >= 0]))
    if len(firsts):
        s["k_pool"][firsts, :, :, :2] += (0.6 * towards).to(torch.bfloat16).reshape(1, 1, d // 32, 1, 32)
    return s


def _plan(s):
    """The plain form's plan: blocks of rows of one length, (row [B, n], their positions, which
    are real, the page tables [B, P] they see and the pages' first positions)."""
    case, (nq, nkv, d) = s["case"], s["heads"]
    start = np.concatenate([[0], np.cumsum(s["n_new"])])
    pieces = []  # (rows, pages) of up to 512 new tokens of a request
    for r, (n, c) in enumerate(zip(s["n_new"], s["ctx"])):
        for a in range(0, n, 512):
            m = min(512, n - a)
            pieces.append((start[r] + a, c + a, m, _pages_seen(case, m, c + a), r))
    pieces.sort(key=lambda p: (p[2], len(p[3])))
    blocks, at = [], 0
    while at < len(pieces):
        end = at
        while end < len(pieces) and pieces[end][2] == pieces[at][2] and (
                end == at or (end + 1 - at) * len(pieces[end][3]) * PAGE * nkv * d * 4 <= 1 << 30):
            end += 1
        part, n, P = pieces[at:end], pieces[at][2], len(pieces[end - 1][3])
        row = np.stack([p[0] + np.arange(n) for p in part])
        pos = np.stack([p[1] + np.arange(n) for p in part])
        table = np.stack([np.r_[s["pages"][p[4]][p[3]], np.full(P - len(p[3]), s["pages"][p[4]][p[3][0]])]
                          for p in part])
        first = np.stack([np.r_[np.array(p[3]) * PAGE, np.full(P - len(p[3]), FAR)] for p in part])
        blocks.append((_cuda(row), _cuda(pos), _cuda(table), _cuda(first)))
        at = end
    return blocks


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        s["blocks"] = _plan(s)
        return s
    import paper_2606_16264_amd as mx
    s["mx"], s["shape"] = mx, mx.attn_shape(*s["heads"], s["pool_pages"])
    s["batch"] = mx.Batch(s["phase"], s["n_new"], s["ctx"], s["pages"])
    if case["kind"] == "window":
        n = mx.mx_workspace_bytes_window_for(s["batch"], s["shape"], case["window"], case["sinks"])
    else:
        s["runs"] = mx.SharedRuns(_runs(case))
        n = mx.mx_workspace_bytes_shared_for(s["batch"], s["shape"], s["runs"])
    s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s


def _attend(s, row, pos, table, first):
    case, (nq, nkv, d) = s["case"], s["heads"]
    (B, n), P, group = row.shape, table.shape[1], nq // nkv
    # keys [B, nkv, d, 16 P] and values [B, nkv, 16 P, d] of the tables in 32 bits
    k = s["k_pool"][table].float().permute(0, 2, 3, 5, 1, 4).reshape(B, nkv, d, P * PAGE)
    v = s["v_pool"][table].float().permute(0, 2, 1, 4, 3).reshape(B, nkv, P * PAGE, d)
    q = s["q"][row].float().reshape(B, n, nkv, group, d).permute(0, 2, 3, 1, 4).reshape(B, nkv, group * n, d)
    sc = torch.matmul(q, k) / math.sqrt(d)
    key = (first[:, :, None] + torch.arange(PAGE, device="cuda")).reshape(B, 1, P * PAGE)
    hidden = key > pos[:, :, None]
    if case["kind"] == "window":
        hidden |= (key >= case["sinks"]) & (key <= pos[:, :, None] - case["window"])
    sc = sc.reshape(B, nkv, group, n, -1).masked_fill_(hidden[:, None, None], -math.inf)
    p = (sc - sc.amax(-1, keepdim=True)).exp_()
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(B, nkv, group * n, -1), v)
    o = o.reshape(B, nkv, group, n, d).permute(0, 3, 1, 2, 4).reshape(B, n, nq, d)
    s["out"][row] = o.to(torch.bfloat16)


def run(s):
    if own:
        mx, case = s["mx"], s["case"]
        if case["kind"] == "window":
            mx.mx_paged_attn_window(s["batch"], s["shape"], case["window"], case["sinks"], s["q"],
                                    s["k_pool"], s["v_pool"], s["out"], s["ws"])
        else:
            mx.mx_paged_attn_shared(s["batch"], s["shape"], s["runs"], s["q"], s["k_pool"],
                                    s["v_pool"], s["out"], s["ws"])
    else:
        for b in s["blocks"]:
            _attend(s, *b)
    return {"out": s["out"]}


def _pairs(case, n, c):
    """Query-key pairs of n new tokens after c cached ones."""
    if case["kind"] != "window":
        return n * c + n * (n + 1) // 2
    p = np.arange(c, c + n)
    low = np.maximum(0, p - case["window"] + 1)  # the window's first position
    return int((p - low + 1 + np.minimum(low, case["sinks"])).sum())


def work(case):
    nq, nkv, d = SHAPES[case["shape"]]
    _, n_new, ctx = _requests(case)
    keys = sum(b - a for n, c in zip(n_new, ctx) for a, b in _seen(case, n, c))
    # a run's keys are read once for all its requests
    keys -= sum((n - 1) * k * PAGE for _, n, k in _runs(case))
    pairs = sum(_pairs(case, n, c) for n, c in zip(n_new, ctx))
    return {"bytes": 4 * sum(n_new) * nq * d + 4 * keys * nkv * d, "flops": 4 * nq * d * pairs}


# ------------------------------------------------------------------ 64-bit reference
def exact(case, seed):
    s = _inputs(case, seed)
    nq, nkv, d = s["heads"]
    out = torch.zeros(sum(s["n_new"]), nq, d, dtype=torch.float64, device="cuda")
    t = 0
    for r, (n, c) in enumerate(zip(s["n_new"], s["ctx"])):
        j = torch.cat([torch.arange(a, b, device="cuda") for a, b in _seen(case, n, c)])
        page, slot = _cuda(s["pages"][r])[j // PAGE], j % PAGE
        K = s["k_pool"][page, :, :, slot].double().reshape(len(j), nkv, d)
        V = s["v_pool"][page, :, :, slot].double()
        for a in range(0, n, 2048):
            m = min(2048, n - a)
            p = torch.arange(c + a, c + a + m, device="cuda")[:, None]
            sees = j[None, :] <= p
            if case["kind"] == "window":
                sees &= (j[None, :] < case["sinks"]) | (p - j[None, :] < case["window"])
            for g in range(nkv):
                x = s["q"][t + a:t + a + m, g * (nq // nkv):(g + 1) * (nq // nkv)].double()
                w = torch.matmul(x.reshape(-1, d), K[:, g].t().contiguous()) * d ** -0.5
                w = w.reshape(m, -1, len(j)).masked_fill(~sees[:, None], -math.inf)
                w = torch.softmax(w, -1)
                out[t + a:t + a + m, g * (nq // nkv):(g + 1) * (nq // nkv)] = torch.matmul(
                    w.reshape(-1, len(j)), V[:, g].contiguous()).reshape(m, -1, d)
        t += n
    return {"out": out}
