"""GPU tests of attention over parts of the requests' keys (a sliding window with sinks;
shared runs of pages) against plain 64-bit references on the CPU.

With A = sum_j p_j |v_j|: every probability is rounded to bf16 (half a step, 2^-8) in the
product and in the row's sum, the output once more: |got - exact| <= 2^-8 |exact| +
2 * 2^-8 A, and 2^-10 A for the scores' fp32 arithmetic and the joining of partial sums."""
import math
import threading

import numpy as np
import pytest

import paper_2606_16264_amd as mx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ALL = 2 ** 31 - 1  # a window that holds everything


def bf16(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.float64).to(torch.bfloat16)


class Pools:
    """The pools on the device; their mirror [page][head][token][d] on the CPU.  Whatever is
    not written holds NaN."""

    def __init__(self, pages, nkv, d):
        self.pages, self.nkv, self.d = pages, nkv, d
        self.hk = torch.full((pages, nkv, 16, d), math.nan, dtype=torch.bfloat16)
        self.hv = self.hk.clone()

    def upload(self):
        P, g, d = self.pages, self.nkv, self.d
        self.k = self.hk.reshape(P, g, 16, d // 32, 32).permute(0, 1, 3, 2, 4).contiguous().cuda()
        self.v = self.hv.permute(0, 1, 3, 2).contiguous().cuda()

    def shape(self, nq, scale=0.0):
        return mx.attn_shape(nq, self.nkv, self.d, self.pages, scale)

    def fill(self, rng, table, j):
        """The positions j of a request with plausible values."""
        pg, sl = torch.as_tensor(np.asarray(table)[j // 16]), torch.as_tensor(j % 16)
        for pool in (self.hk, self.hv):
            pool[pg, :, sl] = bf16(rng.normal(0, 1, (len(j), self.nkv, self.d)))

    def dense(self, table, j):
        pg, sl = np.asarray(table)[j // 16], j % 16
        return (self.hk[pg, :, sl].double().numpy().transpose(1, 0, 2),
                self.hv[pg, :, sl].double().numpy().transpose(1, 0, 2))


def seen(n, ctx, window, sinks):
    """[n, ctx + n] which positions the new tokens see."""
    p, j = np.arange(ctx, ctx + n)[:, None], np.arange(ctx + n)[None]
    return (j <= p) & ((j > p - window) | (j < sinks))


def reference(pools, nq, reqs, q, window=ALL, sinks=0, scale=None):
    """(out, A) of requests (decode, n_new, ctx, table)."""
    group, scale = nq // pools.nkv, scale or 1 / math.sqrt(pools.d)
    out, mag, t = [], [], 0
    q = q.double().numpy()
    for _, n, ctx, table in reqs:
        see = seen(n, ctx, window, sinks)
        j = np.flatnonzero(see.any(0))
        K, V = pools.dense(table, j)
        see = see[:, j]
        o, a = np.zeros((n, nq, pools.d)), np.zeros((n, nq, pools.d))
        for h in range(nq):
            s = np.where(see, q[t:t + n, h] @ K[h // group].T * scale, -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[:, h], a[:, h] = p @ V[h // group], p @ np.abs(V[h // group])
        out.append(o), mag.append(a)
        t += n
    return np.concatenate(out), np.concatenate(mag)


def check(got, exp, mag, what=""):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    off = np.abs(got - exp) - (2.0 ** -8 * np.abs(exp) + (2.0 ** -7 + 2.0 ** -10) * mag)
    assert off.max() <= 0, f"{what}: {off.max():.3e} beyond the bound at {np.unravel_index(off.argmax(), off.shape)}"


def batch_of(reqs):
    return mx.Batch([int(r[0]) for r in reqs], [r[1] for r in reqs], [r[2] for r in reqs],
                    [r[3] for r in reqs])


def run_window(pools, nq, reqs, q, window, sinks, scale=0.0, stream=None, out=None):
    s, b = pools.shape(nq, scale), batch_of(reqs)
    n = mx.mx_workspace_bytes_window_for(b, s, window, sinks)
    assert n <= mx.mx_workspace_bytes_window(s, b.T, b.R, sum(len(r[3]) for r in reqs))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda") if out is None else out
    mx.mx_paged_attn_window(b, s, window, sinks, q, pools.k, pools.v, out, ws, stream=stream)
    return out, ws


def run_shared(pools, nq, reqs, runs, q, scale=0.0, stream=None, out=None):
    s, b, rs = pools.shape(nq, scale), batch_of(reqs), mx.SharedRuns(runs)
    n = mx.mx_workspace_bytes_shared_for(b, s, rs)
    depth = max([sum(a <= r < a + k for a, k, _ in runs) for r in range(b.R)], default=0)
    assert n <= mx.mx_workspace_bytes_shared(s, b.T, b.R, sum(len(r[3]) for r in reqs), depth)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda") if out is None else out
    mx.mx_paged_attn_shared(b, s, rs, q, pools.k, pools.v, out, ws, stream=stream)
    return out, ws


def window_case(nq, nkv, d, reqs, seed, window, sinks, spread=1.0):
    """Requests of (decode, n_new, ctx).  Only what some token sees is filled, pages that none
    sees are not in the tables."""
    rng = np.random.default_rng(seed)
    order = iter(rng.permutation(sum(-(-(n + c) // 16) for _, n, c in reqs) + 9).tolist())
    pools = Pools(sum(-(-(n + c) // 16) for _, n, c in reqs) + 9, nkv, d)
    full = []
    for decode, n, ctx in reqs:
        see = seen(n, ctx, window, sinks).any(0)
        table = [next(order) if see[16 * i:16 * i + 16].any() else -1 - i for i in range(-(-(n + ctx) // 16))]
        pools.fill(rng, table, np.flatnonzero(see))
        if spread != 1.0:
            pg = torch.as_tensor([p for p in table if p >= 0])
            pools.hk[pg] = (pools.hk[pg].double() * spread).to(torch.bfloat16)
        full.append((decode, n, ctx, table))
    pools.upload()
    return pools, full, bf16(rng.normal(0, 1, (sum(r[1] for r in reqs), nq, d)))


SHAPES = [(4, 4, 64), (8, 2, 64), (8, 1, 128), (5, 5, 128), (20, 1, 64), (36, 2, 128)]
DECODES = [1, 15, 16, 17, 63, 64, 65, 255, 300, 1023, 2500]
CHUNKS = [(1, 0), (2, 0), (17, 0), (128, 0), (129, 3), (200, 1000), (33, 64), (16, 15), (1, 31), (1, 400), (3, 700)]
WINDOWS = [(1, 0), (1, 1), (16, 0), (31, 3), (100, 16), (129, 40), (700, 33), (512, 0), (ALL, 0), (50, ALL)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("nq,nkv,d", SHAPES)
def test_window(nq, nkv, d, window, sinks):
    """Decodes and chunks in one batch, where NaN stands in all that no token sees."""
    reqs = [(1, 1, n) for n in DECODES] + [(0, n, x) for n, x in CHUNKS]
    pools, reqs, q = window_case(nq, nkv, d, reqs, nq + d, window, sinks)
    out, mag = reference(pools, nq, reqs, q, window, sinks)
    got, ws = run_window(pools, nq, reqs, q.cuda(), window, sinks)
    check(got, out, mag)
    ws.fill_(255)
    again, _ = run_window(pools, nq, reqs, q.cuda(), window, sinks)
    assert torch.equal(again.view(torch.uint16), got.view(torch.uint16))


@pytest.mark.parametrize("nq,nkv,d", [(150, 1, 64), (20, 10, 128), (19, 19, 64), (33, 11, 128)])
def test_odd_heads(nq, nkv, d):
    """A group of more rows than a tile has; numbers of KV heads that are no multiple of eight,
    above it: tiles alone, streams alone, both."""
    for reqs in ([(1, 1, 100), (1, 1, 17)], [(0, 70, 30), (0, 9, 200)], [(1, 1, 333), (0, 33, 0), (0, 1, 5)]):
        pools, full, q = window_case(nq, nkv, d, reqs, nq, 60, 7)
        got, _ = run_window(pools, nq, full, q.cuda(), 60, 7)
        check(got, *reference(pools, nq, full, q, 60, 7))
        n = len(reqs)
        pages = -(-(64 << 20) // (23 * 64 * d * nkv))
        more = [(1, 1, i) for i in range(24)]
        runs = [(0, n, 3), (n, 24, pages)]
        pools, full, q = shared_case(nq, nkv, d, reqs + more, runs, nq + 1)
        got, _ = run_shared(pools, nq, full, runs, q.cuda())
        check(got, *reference(pools, nq, full, q))


@pytest.mark.parametrize("kind", ["decode", "prefill"])
@pytest.mark.parametrize("nq,nkv,d,window,sinks", [
    (8, 2, 128, 4000, 100), (32, 32, 128, 1000, 4), (4, 4, 64, 3333, 0), (16, 1, 64, 5000, 600)])
def test_window_long(nq, nkv, d, window, sinks, kind):
    """Long contexts: keys split over workgroups, whole chunks between the edges."""
    reqs = [(1, 1, 9000), (1, 1, 4001)] if kind == "decode" else [(0, 300, 6001), (0, 700, 0), (0, 2, 9000)]
    pools, reqs, q = window_case(nq, nkv, d, reqs, 3, window, sinks)
    out, mag = reference(pools, nq, reqs, q, window, sinks)
    got, _ = run_window(pools, nq, reqs, q.cuda(), window, sinks)
    check(got, out, mag)


def test_window_scale_and_large_scores():
    """A scale of the caller's; scores of some hundreds, whose softmax is nearly one key."""
    pools, reqs, q = window_case(8, 2, 128, [(1, 1, 900), (0, 130, 70), (0, 40, 0)], 5, 90, 5, spread=12.0)
    out, mag = reference(pools, 8, reqs, q, 90, 5, scale=0.05)
    got, _ = run_window(pools, 8, reqs, q.cuda(), 90, 5, scale=0.05)
    check(got, out, mag)
    q = (q.double() * 30).to(torch.bfloat16)
    out, mag = reference(pools, 8, reqs, q, 90, 5)
    got, _ = run_window(pools, 8, reqs, q.cuda(), 90, 5)
    # (scores of up to 12 * 30 * 128 / 11: fp32 sums of products off by up to 128 * 2^-24 of
    # sum |q k|, which is up to 4 * 10^3, so 3 * 10^-2 of a probability)
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got - out) <= 2.0 ** -8 * np.abs(out) + (2.0 ** -7 + 2.0 ** -10 + 0.06) * mag).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("nq,nkv,d", [(4, 4, 64), (8, 2, 128)])
def test_window_not_finite(nq, nkv, d, what, bad):
    """A value that is no number reaches the rows that see its token and no other; a key
    likewise (minus infinity as a key may leave a row finite)."""
    window, sinks = 40, 6
    reqs = [(0, 150, 0), (0, 90, 333), (1, 1, 200), (0, 1, 300)]
    pools, reqs, q = window_case(nq, nkv, d, reqs, 9, window, sinks)
    q = q.abs()  # a key of minus infinity then has that score
    marks = [(0, 3), (0, 64), (0, 149), (0, 100), (1, 333), (1, 5), (1, 400), (2, 165), (3, 4)]
    target = pools.hk if what == "k" else pools.hv
    hit = torch.zeros(len(q), dtype=torch.bool)
    start = np.cumsum([0] + [r[1] for r in reqs])
    clean = [pools.hk.clone(), pools.hv.clone()]
    for r, j in marks:
        _, n, ctx, table = reqs[r]
        target[table[j // 16], :, j % 16, 7] = bad
        hit[start[r]:start[r + 1]] |= torch.from_numpy(seen(n, ctx, window, sinks)[:, j])
    pools.upload()
    got, _ = run_window(pools, nq, reqs, q.cuda(), window, sinks)
    got = got.cpu()
    pools.hk, pools.hv = clean
    out, mag = reference(pools, nq, reqs, q, window, sinks)
    check(got[~hit], out[~hit.numpy()], mag[~hit.numpy()])
    if what == "v":
        at = got[hit][..., 7].double()
        assert not torch.isfinite(at).any()
        if not math.isnan(bad):
            assert (at == bad).all()
        rest = torch.cat([got[..., :7], got[..., 8:]], -1)
        assert torch.isfinite(rest).all()
    elif bad > 0 or math.isnan(bad):
        assert torch.isnan(got[hit]).all()


# ----------------------------------------------------------------------- shared runs
@pytest.mark.parametrize("bad", [0.0, math.nan, math.inf])
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (5, 0), (40, 6), (700, 20), (ALL, 0)])
@pytest.mark.parametrize("nq,nkv,d", [(4, 4, 64), (8, 2, 128), (16, 2, 128)])
def test_few_tokens(nq, nkv, d, window, sinks, bad):
    """Chunks of a few tokens, whose rows see different keys of the same pages: values that are
    no numbers at both edges of the window, in the first token's sight and the last's."""
    reqs = [(0, n, c) for n, c in [(2, 0), (3, 62), (4, 300), (2, 1000), (16, 31), (9, 2000), (2, 47), (1, 90), (5, 3000)]]
    pools, reqs, q = window_case(nq, nkv, d, reqs, 10, window, sinks)
    start = np.cumsum([0] + [r[1] for r in reqs])
    clean = pools.hv.clone()
    hit = torch.zeros(len(q), dtype=torch.bool)
    for r, (_, n, ctx, table) in enumerate(reqs):
        see = seen(n, ctx, window, sinks)
        for j in {ctx + n - 1, max(0, ctx - window + 1), ctx} if bad else ():
            if see[:, j].any():
                pools.hv[table[j // 16], :, j % 16, 7] = bad
                hit[start[r]:start[r + 1]] |= torch.from_numpy(see[:, j])
    pools.upload()
    got, _ = run_window(pools, nq, reqs, q.cuda(), window, sinks)
    got, pools.hv = got.cpu(), clean
    out, mag = reference(pools, nq, reqs, q, window, sinks)
    if not hit.all():
        check(got[~hit], out[~hit.numpy()], mag[~hit.numpy()])
    rest = torch.arange(d) != 7
    check(got[..., rest], out[..., rest.numpy()], mag[..., rest.numpy()])
    at = got[hit][..., 7]
    assert torch.isnan(at).all() if math.isnan(bad) else (at == bad).all()


def shared_case(nq, nkv, d, reqs, runs, seed):
    """Requests of (decode, n_new, own cached tokens); runs of (first, requests, pages)."""
    rng = np.random.default_rng(seed)
    tables = [[] for _ in reqs]
    pages = sum(k for _, _, k in runs) + sum(-(-(n + c) // 16) + 1 for _, n, c in reqs) + 9
    order = iter(rng.permutation(pages).tolist())
    pools = Pools(pages, nkv, d)
    for first, n, k in runs:
        ids = [next(order) for _ in range(k)]
        pools.fill(rng, ids, np.arange(16 * k))
        for r in range(first, first + n):
            tables[r] += ids
    full = []
    for (decode, n, own), t in zip(reqs, tables):
        c = 16 * len(t)
        mine = [next(order) for _ in range(-(-(own + n) // 16))]
        pools.fill(rng, mine, np.arange(own + n))
        full.append((decode, n, c + own, t + mine))
    pools.upload()
    return pools, full, bf16(rng.normal(0, 1, (sum(r[1] for r in reqs), nq, d)))


D, P = 1, 0
# (runs are taken apart from their requests where that saves 64 MB of reads: `more` decodes
# of a run of their own, of as many pages as that takes, go with the requests that follow)
SHARED = [
    ([(D, 1, 0), (D, 1, 0)], [(0, 2, 1)]),
    ([(D, 1, c) for c in (0, 1, 15, 16, 17, 100, 333)], [(0, 7, 9)]),
    ([(D, 1, 5 * i) for i in range(40)], [(0, 40, 33)]),
    # a tree, an overlap of its branches, requests beside it
    ([(D, 1, 7 * i + 1) for i in range(20)], [(0, 16, 20), (0, 5, 3), (5, 6, 40), (12, 4, 1), (2, 3, 11)]),
    # prompts: short ones join the run, ones that fill their tiles do not
    ([(P, n, c) for n, c in ((1, 0), (2, 0), (17, 3), (128, 0), (130, 16), (300, 0))], [(0, 6, 30)]),
    ([(D, 1, 3), (P, 40, 0), (D, 1, 90), (P, 256, 2), (P, 1, 9), (D, 1, 16), (P, 9, 0)],
     [(0, 7, 17), (1, 4, 2), (5, 2, 60)]),
    # a run of one request alone, one that only one request of takes part in
    ([(D, 1, 30), (D, 1, 2), (P, 512, 0)], [(0, 1, 5), (1, 2, 10)]),
    ([(D, 1, 30), (P, 70, 2)], []),
]


@pytest.mark.parametrize("more", [0, 24])
@pytest.mark.parametrize("case", range(len(SHARED)))
@pytest.mark.parametrize("nq,nkv,d", SHAPES)
def test_shared(nq, nkv, d, case, more):
    reqs, runs = SHARED[case]
    if more:
        pages = -(-(64 << 20) // ((more - 1) * 64 * d * nkv))
        runs = runs + [(len(reqs), more, pages)]
        reqs = reqs + [(D, 1, i) for i in range(more)]
    pools, reqs, q = shared_case(nq, nkv, d, reqs, runs, 17 * case + nq)
    out, mag = reference(pools, nq, reqs, q)
    got, ws = run_shared(pools, nq, reqs, runs, q.cuda())
    check(got, out, mag)
    ws.fill_(255)
    again, _ = run_shared(pools, nq, reqs, runs, q.cuda())
    assert torch.equal(again.view(torch.uint16), got.view(torch.uint16))


@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 128), (32, 32, 128), (4, 4, 64), (64, 8, 128)])
def test_shared_long(nq, nkv, d):
    """A long document for many decodes: its tiles are split over their keys."""
    reqs = [(D, 1, 11 * i) for i in range(33)] + [(P, 20, 5)] * 3
    runs = [(0, 36, 300), (4, 20, 70)]
    pools, reqs, q = shared_case(nq, nkv, d, reqs, runs, 23)
    out, mag = reference(pools, nq, reqs, q, scale=0.11)
    got, _ = run_shared(pools, nq, reqs, runs, q.cuda(), scale=0.11)
    check(got, out, mag)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_shared_not_finite(bad):
    """A value that is no number in a run reaches all of the run's rows; in a chunk's own
    tokens those behind it."""
    reqs, runs = [(D, 1, 20), (P, 30, 0), (D, 1, 4), (D, 1, 9)], [(0, 3, 12), (1, 2, 4)]
    runs, reqs = runs + [(4, 24, 180)], reqs + [(D, 1, i) for i in range(24)]  # (enough to be taken apart)
    pools, reqs, q = shared_case(8, 2, 128, reqs, runs, 31)
    hk = pools.hv.clone()
    # of request 1: position 100 of the first run (rows of 0, 1, 2), 200 of the second (1, 2)
    for j, dim in ((100, 3), (200, 4), (16 * 16 + 12, 5)):
        pools.hv[reqs[1][3][j // 16], :, j % 16, dim] = bad
    pools.upload()
    got, _ = run_shared(pools, 8, reqs, runs, q.cuda())
    pools.hv = hk
    out, mag = reference(pools, 8, reqs, q)
    got = got.cpu()
    rows = {3: list(range(0, 32)), 4: list(range(1, 32)), 5: list(range(13, 31))}
    hit = torch.zeros(len(q), 128, dtype=torch.bool)
    for dim, r in rows.items():
        hit[r, dim] = True
    hit = hit[:, None].expand(-1, 8, -1)
    assert not torch.isfinite(got[hit].double()).any()
    assert torch.isfinite(got[~hit].double()).all()
    clean = torch.where(hit, torch.from_numpy(out).to(torch.bfloat16), got)
    check(clean, out, mag)


# ----------------------------------------------------------------------- both
def test_rows_behind_stay_and_output_in_place():
    """Rows of out behind the batch's last keep their bytes; out may be q."""
    reqs = [(1, 1, 700), (0, 45, 100), (1, 1, 20)]
    pools, reqs, q = window_case(8, 2, 64, reqs, 41, 64, 2)
    out, mag = reference(pools, 8, reqs, q, 64, 2)
    buf = torch.full((len(q) + 5, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    buf[:len(q)] = q.cuda()
    run_window(pools, 8, reqs, buf, 64, 2, out=buf)
    check(buf[:len(q)], out, mag)
    assert (buf[len(q):] == 3).all()
    reqs, runs = [(D, 1, 20), (P, 30, 0), (P, 400, 7)] + [(D, 1, 3)] * 40, [(0, 43, 200)]
    pools, reqs, q = shared_case(8, 2, 64, reqs, runs, 43)
    out, mag = reference(pools, 8, reqs, q)
    buf = torch.full((len(q) + 5, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    buf[:len(q)] = q.cuda()
    run_shared(pools, 8, reqs, runs, buf, out=buf)
    check(buf[:len(q)], out, mag)
    assert (buf[len(q):] == 3).all()


def test_matches_paged_attention():
    """With a window over everything, and with runs, the results of mx_paged_attn but for
    the rounding of probabilities and outputs: twice the bound of one against the exact."""
    reqs, runs = [(D, 1, 200), (P, 30, 64), (D, 1, 4), (P, 200, 0)], [(0, 3, 40)]
    pools, reqs, q = shared_case(8, 2, 128, reqs, runs, 51)
    s, b = pools.shape(8), batch_of(reqs)
    ws = torch.empty(mx.mx_workspace_bytes_for(b, s), dtype=torch.uint8, device="cuda")
    plain = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    mx.mx_paged_attn(b, s, q.cuda(), pools.k, pools.v, plain, ws)
    _, mag = reference(pools, 8, reqs, q)
    for got in (run_window(pools, 8, reqs, q.cuda(), ALL, 0)[0], run_shared(pools, 8, reqs, runs, q.cuda())[0]):
        check(got, plain.double().cpu().numpy(), 2 * mag + 2.0 ** -8 * np.abs(plain.double().cpu().numpy()))


def test_pools_beyond_4_gib():
    """Pages whose byte offsets pass 32 bits."""
    nq, nkv, d, pages = 8, 8, 128, 140000
    rng = np.random.default_rng(61)
    k = torch.empty((pages, nkv, d // 32, 16, 32), dtype=torch.bfloat16, device="cuda")
    v = torch.empty((pages, nkv, d, 16), dtype=torch.bfloat16, device="cuda")
    small = Pools(80, nkv, d)
    small.fill(rng, list(range(80)), np.arange(1280))
    small.upload()
    far = pages - 80
    k[far:], v[far:] = small.k, small.v
    shape = mx.attn_shape(nq, nkv, d, pages)
    near = [(D, 1, 300, list(range(20))), (P, 50, 200, list(range(20, 40))), (D, 1, 450, list(range(10)) + list(range(50, 70)))]
    q = bf16(rng.normal(0, 1, (52, nq, d)))
    b = mx.Batch([1, 0, 1], [1, 50, 1], [300, 200, 450], [[far + p for p in r[3]] for r in near])
    out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(mx.mx_workspace_bytes_window_for(b, shape, 77, 5), dtype=torch.uint8, device="cuda")
    mx.mx_paged_attn_window(b, shape, 77, 5, q.cuda(), k, v, out, ws)
    check(out, *reference(small, nq, near, q, 77, 5))
    near = [near[0], near[2], near[1]]
    b = mx.Batch([1, 1, 0], [1, 1, 50], [300, 450, 200], [[far + p for p in r[3]] for r in near])
    runs = mx.SharedRuns([(0, 2, 10)])
    ws = torch.empty(mx.mx_workspace_bytes_shared_for(b, shape, runs), dtype=torch.uint8, device="cuda")
    mx.mx_paged_attn_shared(b, shape, runs, q.cuda(), k, v, out, ws)
    check(out, *reference(small, nq, near, q))


def test_serving_loop():
    """As a decoder with alternating layers uses them: every step appends the new tokens to
    both layers' caches, then one layer attends through a window, the other over a shared
    system prompt; pages that leave the window are freed and given to other requests."""
    nq, nkv, d, window, sinks = 8, 2, 64, 40, 3
    rng = np.random.default_rng(71)
    R, prefix = 3, 4
    win, full = Pools(60, nkv, d), Pools(60, nkv, d)
    win.upload(), full.upload()
    free = list(range(60))
    wt, ft = [[] for _ in range(R)], [list(range(prefix)) for _ in range(R)]
    next_full = prefix
    ctx = [0] * R
    steps = [[16 * prefix + 5, 0, 0], [1, 16 * prefix + 40, 16 * prefix + 1]] + [[1, 1, 1]] * 45
    k_all, v_all = [[] for _ in range(R)], [[] for _ in range(R)]
    sys_k, sys_v = rng.normal(0, 1, (16 * prefix, nkv, d)), rng.normal(0, 1, (16 * prefix, nkv, d))
    for step, n_new in enumerate(steps):
        live = [r for r in range(R) if n_new[r]]
        T = sum(n_new)
        q = bf16(rng.normal(0, 1, (T, nq, d)))
        ks, vs = [], []
        for r in live:
            k, v = rng.normal(0, 1, (n_new[r], nkv, d)), rng.normal(0, 1, (n_new[r], nkv, d))
            if ctx[r] == 0:
                k[:16 * prefix], v[:16 * prefix] = sys_k, sys_v  # every prompt starts with it
            ks.append(bf16(k)), vs.append(bf16(v))
            k_all[r].append(ks[-1]), v_all[r].append(vs[-1])
            need = -(-(ctx[r] + n_new[r]) // 16)
            while len(wt[r]) < need:
                wt[r].append(free.pop(0))
            while len(ft[r]) < need:
                ft[r].append(next_full)
                next_full += 1
        k, v = torch.cat(ks).cuda(), torch.cat(vs).cuda()
        phase = [int(n_new[r] == 1 and ctx[r] > 0) for r in live]
        args = phase, [n_new[r] for r in live], [ctx[r] for r in live]
        shape = win.shape(nq)
        clean = mx.Batch(*args, [[max(p, 0) for p in wt[r]] for r in live])
        ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
        mx.mx_kv_append(clean, shape, k, v, win.k, win.v, ws)
        got_w, got_s = torch.empty_like(q, device="cuda"), torch.empty_like(q, device="cuda")
        mx.mx_paged_attn_window(mx.Batch(*args, [wt[r] for r in live]), shape, window, sinks, q.cuda(),
                                win.k, win.v, got_w, ws)
        for i, r in enumerate(live):  # the shared pages are written once per prompt: the same bytes
            t0 = sum(n_new[x] for x in live[:i])
            one = mx.Batch([phase[i]], [n_new[r]], [ctx[r]], [ft[r]])
            mx.mx_kv_append(one, shape, k[t0:t0 + n_new[r]].contiguous(), v[t0:t0 + n_new[r]].contiguous(), full.k, full.v, ws)
        joined = [i for i, r in enumerate(live) if ctx[r] >= 16 * prefix]
        runs = mx.SharedRuns([(joined[0], len(joined), prefix)] if len(joined) > 1 and joined == list(range(joined[0], joined[-1] + 1)) else [])
        if len(live) == 3 and step > 1:
            assert runs.n == 1
            b = mx.Batch(*args, [ft[r] for r in live])
            mx.mx_paged_attn_shared(b, shape, runs, q.cuda(), full.k, full.v, got_s, ws)
        t = 0
        for i, r in enumerate(live):
            n = n_new[r]
            kk, vv = torch.cat(k_all[r]).double().numpy(), torch.cat(v_all[r]).double().numpy()
            qq = q[t:t + n].double().numpy()
            for got, w, sk in ((got_w, window, sinks), (got_s, ALL, 0)):
                if got is got_s and not (len(live) == 3 and step > 1):
                    continue
                see = seen(n, ctx[r], w, sk)
                exp, mag = np.zeros((n, nq, d)), np.zeros((n, nq, d))
                for h in range(nq):
                    s = np.where(see, qq[:, h] @ kk[:, h // 4].T / math.sqrt(d), -np.inf)
                    p = np.exp(s - s.max(1, keepdims=True))
                    p /= p.sum(1, keepdims=True)
                    exp[:, h], mag[:, h] = p @ vv[:, h // 4], p @ np.abs(vv[:, h // 4])
                check(got[t:t + n], exp, mag, f"step {step} request {r}")
            t += n
            ctx[r] += n
            # pages that no later token sees go back
            for i in range(-(-sinks // 16), (ctx[r] - window + 1) // 16):
                if wt[r][i] >= 0:
                    free.append(wt[r][i])
                    wt[r][i] = -1


def test_streams_and_threads():
    """Calls from two threads on streams of their own, each with its workspace."""
    cases = []
    for i in range(2):
        reqs = [(1, 1, 300 + 100 * i), (0, 60, 40), (1, 1, 1500)]
        pools, reqs, q = window_case(8, 2, 64, reqs, 81 + i, 100, 4)
        sh, sreqs, sq = shared_case(8, 2, 64, [(D, 1, 9 * k) for k in range(33)], [(0, 33, 260 + i)], 91 + i)
        cases.append((pools, reqs, q.cuda(), reference(pools, 8, reqs, q, 100, 4), sh, sreqs, [(0, 33, 260 + i)],
                      sq.cuda(), reference(sh, 8, sreqs, sq)))
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            pools, reqs, q, exp, sh, sreqs, runs, sq, sexp = cases[i]
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for _ in range(20):
                    a, wa = run_window(pools, 8, reqs, q, 100, 4)
                    b, wb = run_shared(sh, 8, sreqs, runs, sq)
                st.synchronize()
                check(a, *exp)
                check(b, *sexp)
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors, errors


def test_captured_streams_are_refused():
    reqs = [(1, 1, 300), (0, 40, 20)]
    pools, reqs, q = window_case(8, 2, 64, reqs, 95, 64, 2)
    q = q.cuda()
    want, ws = run_window(pools, 8, reqs, q, 64, 2)
    b, s, out = batch_of([r[:3] + ([max(p, 0) for p in r[3]],) for r in reqs]), pools.shape(8), torch.zeros_like(want)
    big = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    y = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    graph, seen = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph):
        for call in (lambda: mx.mx_paged_attn_window(b, s, 64, 2, q, pools.k, pools.v, out, big),
                     lambda: mx.mx_paged_attn_shared(b, s, mx.SharedRuns([]), q, pools.k, pools.v, out, big)):
            try:
                call()
            except mx.MxError as x:
                seen.append(x.status)
        y += 1
    assert seen == [mx.MX_ERR_UNSUPPORTED] * 2
    graph.replay()
    torch.cuda.synchronize()
    assert y.tolist() == [1.0] * 4 and not out.any()
    assert torch.equal(run_window(pools, 8, reqs, q, 64, 2)[0], want)


def test_calls_in_a_row_on_one_workspace():
    """Calls of different batches on one stream and workspace, without a wait between them: small
    ones, whose metadata goes with the launch, and large ones, whose metadata is uploaded."""
    cases = []
    for i in range(6):
        n = [3, 40, 1, 90, 5, 60][i]
        reqs = [(1, 1, 17 * k + 200) for k in range(n)] + [(0, 20 * i + 1, 5 * i)]
        pools, reqs, q = window_case(8, 2, 64, reqs, 200 + i, 50 + 30 * i, i)
        cases.append((pools, reqs, q.cuda(), 50 + 30 * i, i, reference(pools, 8, reqs, q, 50 + 30 * i, i)))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    got = []
    for _ in range(5):
        for pools, reqs, q, w, sinks, _ in cases:
            out = torch.empty_like(q)
            mx.mx_paged_attn_window(batch_of(reqs), pools.shape(8), w, sinks, q, pools.k, pools.v, out, ws)
            got.append(out)
    for i, out in enumerate(got):
        check(out, *cases[i % 6][5], f"call {i}")


def test_binding_refuses_other_tensors():
    """Strided, of another type, too small, or not on the GPU: refused before anything runs."""
    reqs = [(1, 1, 90)]
    pools, reqs, q = window_case(4, 2, 64, reqs, 97, 64, 2)
    b, s, q = batch_of(reqs), pools.shape(4), q.cuda()
    out, ws = torch.zeros_like(q), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    good = dict(q=q, k_pool=pools.k, v_pool=pools.v, out=out, ws=ws)
    for name, t in (("q", q.float()), ("q", q.cpu()), ("q", q.transpose(1, 2)), ("out", out.half()),
                    ("out", out[:, :3].contiguous()), ("k_pool", pools.k[1:]), ("v_pool", pools.v.transpose(2, 3)),
                    ("v_pool", pools.v.cpu()), ("ws", ws.view(torch.float32)), ("ws", ws.cpu())):
        for call in (lambda a: mx.mx_paged_attn_window(b, s, 64, 2, **a),
                     lambda a: mx.mx_paged_attn_shared(b, s, mx.SharedRuns([]), **a)):
            with pytest.raises(ValueError, match=f"^{name} "):
                call(dict(good, **{name: t}))
    torch.cuda.synchronize()
    assert not out.any()
