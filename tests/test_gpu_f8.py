"""GPU tests of the 8-bit cache: append, attention, accumulated attention weights and
eviction against plain 64-bit references on the CPU.

Codes, scales and kept indices are compared exactly.  Attention outputs: with
A = sum_j p_j |v_j|, every probability is rounded to bf16 (half a step, 2^-8) in the
product and in the row's sum, the output once more: |got - exact| <= 2^-8 |exact| +
2 * 2^-8 A, and 2^-10 A for the scores' fp32 arithmetic.  Accumulated weights are fp32:
a score is a sum of d products whose fp32 summation is off by at most
d 2^-24 sum |q k|, the row's log-sum by as much, and a weight by their sum in the
exponent; 2^-20 is for the exponential and the sums."""
import math
import threading

import numpy as np
import pytest

import paper_2606_16264_amd as mx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
NAN = 0x7F


def bf16(x):
    return torch.as_tensor(x, dtype=torch.float64).to(torch.bfloat16)


class Cache:
    """The cache on the device, its mirror in plain arrays [page][head][token] on the CPU."""

    def __init__(self, pages, nkv, d, weight=True, poison=True):
        self.nkv, self.d, self.pages = nkv, d, pages
        fill = NAN if poison else 0
        nan = math.nan if poison else 0.0
        self.k = torch.full((pages, nkv, d // 64, 16, 64), fill, dtype=torch.uint8, device="cuda")
        self.v = torch.full((pages, nkv, d, 16), fill, dtype=torch.uint8, device="cuda")
        self.ks = torch.full((pages, nkv), nan, device="cuda")
        self.vs = torch.full((pages, nkv), nan, device="cuda")
        self.w = torch.full((pages, nkv, 16), nan, device="cuda") if weight else None
        self.mx = mx.CacheF8(self.k, self.v, self.ks, self.vs, self.w)
        # the mirror: codes as uint8 [page, head, token, d]
        self.hk = np.full((pages, nkv, 16, d), fill, np.uint8)
        self.hv = self.hk.copy()
        self.hks = np.full((pages, nkv), nan)
        self.hvs = self.hks.copy()
        self.hw = np.full((pages, nkv, 16), nan) if weight else None

    def shape(self, nq, scale=0.0):
        return mx.attn_shape(nq, self.nkv, self.d, self.pages, scale)

    def read(self):
        """(k, v) codes [page, head, token, d] as the device holds them."""
        P, g, d = self.pages, self.nkv, self.d
        k = self.k.cpu().numpy().transpose(0, 1, 3, 2, 4).reshape(P, g, 16, d)
        return k, self.v.cpu().numpy().transpose(0, 1, 3, 2)

    def upload(self):
        P, g, d = self.pages, self.nkv, self.d
        self.k.copy_(torch.from_numpy(np.ascontiguousarray(
            self.hk.reshape(P, g, 16, d // 64, 64).transpose(0, 1, 3, 2, 4))))
        self.v.copy_(torch.from_numpy(np.ascontiguousarray(self.hv.transpose(0, 1, 3, 2))))
        self.ks.copy_(torch.from_numpy(self.hks).float())
        self.vs.copy_(torch.from_numpy(self.hvs).float())
        if self.w is not None:
            self.w.copy_(torch.from_numpy(self.hw).float())

    def check(self, what=""):
        k, v = self.read()
        for name, got, exp in (("k", k, self.hk), ("v", v, self.hv)):
            bad = np.argwhere(got != exp)
            assert not len(bad), f"{what} {name} codes differ at {bad[:4].tolist()}"
        np.testing.assert_array_equal(self.ks.cpu().numpy(), self.hks.astype(np.float32), what)
        np.testing.assert_array_equal(self.vs.cpu().numpy(), self.hvs.astype(np.float32), what)


def decode8(codes):
    return torch.from_numpy(np.ascontiguousarray(codes)).view(F8).double().numpy()


def encode8(x):
    """The nearest e4m3 code of a value within +-448, ties to even; NaN as 0x7F."""
    c = torch.from_numpy(np.ascontiguousarray(x, np.float64)).float().to(F8).view(torch.uint8).numpy()
    return np.where(np.isnan(x), NAN, c).astype(np.uint8)


def fit_scale(amax):
    """Least 2^e >= amax / 448 with -100 <= e <= 119."""
    e = -100
    while e < 119 and amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append_ref(c, pages, ctx, k_new, v_new):
    """One request's append to the mirror; k_new, v_new [n, head, d] float64."""
    n, at = len(k_new), 0
    while at < n:
        page, s0 = pages[(ctx + at) // 16], (ctx + at) % 16
        m = min(16 - s0, n - at)
        for x, codes, scales in ((k_new, c.hk, c.hks), (v_new, c.hv, c.hvs)):
            for g in range(c.nkv):
                y = x[at:at + m, g]
                ok = np.isfinite(y)
                now = fit_scale(np.abs(y[ok]).max() if ok.any() else 0.0)
                if s0:
                    old = scales[page, g]
                    now = max(now, old)
                    codes[page, g, :s0] = encode8(decode8(codes[page, g, :s0]) * (old / now))
                codes[page, g, s0:s0 + m] = encode8(np.where(ok, np.clip(y / now, -448, 448), np.nan))
                scales[page, g] = now
        if c.hw is not None:
            c.hw[page, :, s0:s0 + m] = 0.0
        at += m


def batch_of(reqs):
    """reqs: (decode, n_new, ctx, pages)."""
    return mx.Batch([int(r[0]) for r in reqs], [r[1] for r in reqs], [r[2] for r in reqs],
                    [r[3] for r in reqs])


def tables(rng, pages, lens):
    order, out = rng.permutation(pages), []
    for n in lens:
        need = -(-n // 16)
        out.append(order[:need].tolist())
        order = order[need:]
    assert len(out[-1]) == -(-lens[-1] // 16)
    return out


def fill(c, rng, table, n, spread=2):
    """n cached tokens of plausible codes in the mirror, scales differing by page."""
    for i, page in enumerate(table):
        m = min(16, n - 16 * i)
        for codes, scales in ((c.hk, c.hks), (c.hv, c.hvs)):
            codes[page, :, :m] = encode8(np.clip(rng.normal(0, 80, (c.nkv, m, c.d)), -448, 448))
            scales[page] = 2.0 ** rng.integers(-7 - spread, -6 + spread, c.nkv)
        if c.hw is not None:
            c.hw[page, :, :m] = rng.exponential(0.01, (c.nkv, m)).astype(np.float32)


def dense(c, table, n, which):
    codes, scales = (c.hk, c.hks) if which == "k" else (c.hv, c.hvs)
    pos = np.arange(n)
    pg = np.asarray(table)[pos // 16]
    return (decode8(codes[pg, :, pos % 16]) * scales[pg][:, :, None]).transpose(1, 0, 2)  # [g, n, d]


def attend_ref(c, nq, reqs, q, scale=None):
    """(out, A, weights per request [g, kv_len], worst sum |q k| of a score)"""
    group = nq // c.nkv
    scale = scale or 1 / math.sqrt(c.d)
    out, mag, weights, worst, t = [], [], [], 0.0, 0
    for _, n, ctx, table in reqs:
        K, V = dense(c, table, ctx + n, "k"), dense(c, table, ctx + n, "v")
        w = np.zeros((c.nkv, ctx + n))
        o, a = np.zeros((n, nq, c.d)), np.zeros((n, nq, c.d))
        hidden = np.arange(ctx + n)[None] > np.arange(ctx, ctx + n)[:, None]
        for h in range(nq):
            g = h // group
            qh = q[t:t + n, h]
            s = np.where(hidden, -np.inf, qh @ K[g].T * scale)
            worst = max(worst, (np.abs(qh) @ np.abs(K[g]).T).max() * scale)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[:, h], a[:, h] = p @ V[g], p @ np.abs(V[g])
            w[g] += p.sum(0)
        out.append(o), mag.append(a), weights.append(w)
        t += n
    return np.concatenate(out), np.concatenate(mag), weights, worst


def check_out(got, exp, mag, what=""):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    off = np.abs(got - exp) - (2.0 ** -8 * np.abs(exp) + (2.0 ** -7 + 2.0 ** -10) * mag)
    assert off.max() <= 0, f"{what}: {off.max():.3e} beyond the bound at {np.unravel_index(off.argmax(), off.shape)}"


def weight_tol(d, worst):
    return 2 * d * 2.0 ** -24 * worst + 2.0 ** -20 * (1 + worst / 16)


def run_attn(c, nq, reqs, q, scale=0.0, stream=None):
    s = c.shape(nq, scale)
    b = batch_of(reqs)
    ws = torch.empty(mx.mx_workspace_bytes_f8_for(b, s, c.w is not None), dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda")
    mx.mx_paged_attn_f8(b, s, q, c.mx, out, ws, stream=stream)
    return out, ws


def check_weights(c, before, reqs, weights, worst):
    """The mirror's weights plus the call's; slots no request owns stay as they were."""
    exp = before.copy()
    for (_, n, ctx, table), w in zip(reqs, weights):
        pos = np.arange(ctx + n)
        np.add.at(exp, (np.asarray(table)[pos // 16][:, None], np.arange(c.nkv)[None], (pos % 16)[:, None]), w.T)
    got = c.w.double().cpu().numpy()
    assert (np.isnan(got) == np.isnan(exp)).all()
    ok = ~np.isnan(exp)
    off = np.abs(got[ok] - exp[ok]) - weight_tol(c.d, worst) * exp[ok]
    assert off.max() <= 0, f"{off.max():.3e} beyond the bound"
    return exp


# ----------------------------------------------------------------------- append
@pytest.mark.parametrize("nkv,d", [(1, 64), (3, 64), (8, 128), (5, 128)])
def test_append(nkv, d):
    """Ragged appends of 1 to 70 tokens at every kind of page boundary, three in a row:
    later ones find older tokens of smaller and of larger scale in their first page."""
    rng = np.random.default_rng(nkv * 1000 + d)
    c = Cache(80, nkv, d)
    c.upload()
    news = [[1, 16, 17, 5, 70, 3, 33], [1, 1, 15, 16, 2, 13, 1], [20, 1, 1, 31, 9, 1, 16]]
    total = [sum(n[r] for n in news) for r in range(7)]
    tabs = tables(rng, 80, total)
    ctx = [0] * 7
    for step, n_new in enumerate(news):
        T = sum(n_new)
        amp = 2.0 ** rng.integers(-4, 5, (T, nkv, 1)) * (10.0 if step == 1 else 1.0)
        k, v = bf16(rng.normal(0, 1, (T, nkv, d)) * amp), bf16(rng.normal(0, 1, (T, nkv, d)) / amp)
        reqs = [(n == 1 and ctx[r] > 0, n, ctx[r], tabs[r]) for r, n in enumerate(n_new)]
        mx.mx_kv_append_f8(batch_of(reqs), c.shape(nkv), k.cuda(), v.cuda(), c.mx)
        t = 0
        for r, n in enumerate(n_new):
            append_ref(c, tabs[r], ctx[r], k[t:t + n].double().numpy(), v[t:t + n].double().numpy())
            ctx[r] += n
            t += n
        c.check(f"step {step}")
        np.testing.assert_array_equal(c.w.cpu().numpy(), c.hw.astype(np.float32))


@pytest.mark.parametrize("d", [64, 128])
def test_append_extreme_values(d):
    """Zeros, values at code and scale borders, subnormals, the largest bf16, infinities, NaN."""
    big = float(torch.finfo(torch.bfloat16).max)
    rows = [np.zeros(d), np.full(d, big), np.full(d, -2.0 ** 127), np.full(d, 2.0 ** -133),
            np.full(d, 2.0 ** -100), np.full(d, 448.0), np.full(d, 450.0), np.full(d, 1.75 * 2.0 ** -30),
            np.r_[math.nan, np.linspace(-3, 3, d - 1)], np.r_[math.inf, -math.inf, np.linspace(-1, 1, d - 2)],
            np.full(d, math.nan), np.r_[464.0, np.geomspace(2.0 ** -12, 448, d - 1)],
            np.r_[big, np.geomspace(1e-30, 1e30, d - 1)]]
    n = len(rows)
    x = bf16(np.stack(rows))[:, None]
    c = Cache(40, 1, d)
    c.upload()
    # each value alone in its page, all in one page, and each behind a token of small scale
    reqs = [(0, 1, 0, [r]) for r in range(n)] + [(0, n, 0, [n])]
    k = torch.cat([x, x]).contiguous()
    mx.mx_kv_append_f8(batch_of(reqs), c.shape(1), k.cuda(), k.flip(0).contiguous().cuda(), c.mx)
    kd, vd = k.double().numpy(), k.flip(0).double().numpy()
    for r in range(n):
        append_ref(c, [r], 0, kd[r:r + 1], vd[r:r + 1])
    append_ref(c, [n], 0, kd[n:], vd[n:])
    c.check("fresh pages")
    reqs = [(1, 1, 1, [r]) for r in range(n)]
    k2 = bf16(np.full((n, 1, d), 1000.0))
    mx.mx_kv_append_f8(batch_of(reqs), c.shape(1), k2.cuda(), k2.cuda(), c.mx)
    for r in range(n):
        append_ref(c, [r], 1, k2[r:r + 1].double().numpy(), k2[r:r + 1].double().numpy())
    c.check("behind another token")


# ----------------------------------------------------------------------- attention
SHAPES = [(4, 4, 64), (8, 2, 64), (8, 1, 128), (5, 5, 128), (20, 1, 64), (36, 2, 128)]
DECODES = [1, 15, 16, 17, 47, 63, 64, 65, 255, 256, 300, 1023, 2500]
CHUNKS = [(1, 0), (2, 0), (17, 0), (128, 0), (129, 3), (200, 1000), (33, 64), (16, 15), (1, 31)]


def make_case(nq, nkv, d, reqs, seed, weight, **kw):
    rng = np.random.default_rng(seed)
    lens = [n + c for _, n, c in reqs]
    pages = sum(-(-n // 16) for n in lens) + 9
    c = Cache(pages, nkv, d, weight)
    tabs = tables(rng, pages, lens)
    for t, n in zip(tabs, lens):
        fill(c, rng, t, n, **kw)
    c.upload()
    reqs = [(a, n, x, t) for (a, n, x), t in zip(reqs, tabs)]
    q = bf16(rng.normal(0, 1, (sum(r[1] for r in reqs), nq, d)))
    return c, reqs, q


@pytest.mark.parametrize("weight", [False, True])
@pytest.mark.parametrize("kind", ["decode", "prefill", "mixed"])
@pytest.mark.parametrize("nq,nkv,d", SHAPES)
def test_attention(nq, nkv, d, kind, weight):
    """Unowned pages, slots behind each request and their scales hold NaN."""
    reqs = [(1, 1, n) for n in DECODES] * (kind != "prefill") + [(0, n, x) for n, x in CHUNKS] * (kind != "decode")
    c, reqs, q = make_case(nq, nkv, d, reqs, nq + d, weight)
    out, mag, weights, worst = attend_ref(c, nq, reqs, q.double().numpy())
    got, _ = run_attn(c, nq, reqs, q.cuda())
    check_out(got, out, mag, kind)
    if weight:
        before = check_weights(c, c.hw, reqs, weights, worst)
        again, _ = run_attn(c, nq, reqs, q.cuda())  # adds the same once more
        assert torch.equal(again, got)
        check_weights(c, before, reqs, weights, worst)


@pytest.mark.parametrize("nq,nkv,d,ctx", [(8, 1, 128, 40000), (32, 32, 128, 5000), (4, 4, 64, 33333)])
def test_attention_long_decodes(nq, nkv, d, ctx):
    """Contexts split over workgroups, with one key that takes most of the weight."""
    c, reqs, q = make_case(nq, nkv, d, [(1, 1, ctx), (1, 1, ctx // 3)], 3, True)
    for r, (_, _, x, table) in enumerate(reqs):  # the needle: a key along q
        j = x * (r + 1) // 3
        c.hk[table[j // 16], :, j % 16] = encode8(np.clip(q[r, ::nq // nkv].double().numpy() * 60, -448, 448))
    c.upload()
    out, mag, weights, worst = attend_ref(c, nq, reqs, q.double().numpy())
    got, _ = run_attn(c, nq, reqs, q.cuda())
    check_out(got, out, mag)
    check_weights(c, c.hw, reqs, weights, worst)


def test_attention_late_chunk():
    """A chunk over a long prefix, odd in every length, and a scale of the caller's."""
    c, reqs, q = make_case(8, 2, 128, [(0, 517, 3001), (0, 130, 0)], 4, True)
    out, mag, weights, worst = attend_ref(c, 8, reqs, q.double().numpy(), scale=0.2)
    got, _ = run_attn(c, 8, reqs, q.cuda(), scale=0.2)
    check_out(got, out, mag)
    check_weights(c, c.hw, reqs, weights, worst)


@pytest.mark.parametrize("weight", [False, True])
@pytest.mark.parametrize("nq,nkv,d,reqs", [
    (8, 2, 128, [(0, 5, 5000)]), (8, 2, 64, [(0, 1, 3000)]), (4, 1, 128, [(0, 33, 2047)]),
    (6, 2, 64, [(0, 50, 4100), (0, 9, 1500), (0, 3, 0)]), (5, 1, 128, [(0, 260, 2500)]),
    (3, 3, 64, [(0, 130, 1985)]), (16, 1, 128, [(0, 20, 6001), (1, 1, 2500), (1, 1, 33)]),
    (40, 2, 64, [(0, 7, 1030), (1, 1, 9000)]), (32, 8, 128, [(0, 140, 1100), (0, 65, 4095)]),
    (8, 8, 64, [(0, 300, 1900)]), (256, 2, 64, [(0, 4, 1500)])])
def test_attention_split_tiles(nq, nkv, d, reqs, weight):
    """Few prefill tiles over long contexts, which are split over their keys: groups that are a
    power of two, that hold one, that are odd; a first split that ends at a tile's positions."""
    c, reqs, q = make_case(nq, nkv, d, reqs, nq + d, weight)
    out, mag, weights, worst = attend_ref(c, nq, reqs, q.double().numpy())
    got, _ = run_attn(c, nq, reqs, q.cuda())
    check_out(got, out, mag)
    if weight:
        check_weights(c, c.hw, reqs, weights, worst)
    assert torch.equal(run_attn(c, nq, reqs, q.cuda())[0], got)


def test_chunk_weights_without_parts():
    """Keys and KV heads enough that a chunk's rows are not split, causal edges inside."""
    c, reqs, q = make_case(32, 32, 64, [(0, 300, 4001), (0, 33, 0)], 14, True)
    out, mag, weights, worst = attend_ref(c, 32, reqs, q.double().numpy())
    got, _ = run_attn(c, 32, reqs, q.cuda())
    check_out(got, out, mag)
    check_weights(c, c.hw, reqs, weights, worst)


def test_output_in_place_of_the_query():
    """Without weights the output may be the query itself: whole and split decodes and tiles."""
    for reqs in ([(1, 1, 70), (0, 150, 40), (1, 1, 5000), (0, 20, 3000)], [(0, 33, 10)], [(1, 1, 4000)],
                 [(0, 70, 64)] + [(1, 1, 9)] * 70):
        c, reqs, q = make_case(8, 2, 128, reqs, 41, False)
        q = q.cuda()
        want, ws = run_attn(c, 8, reqs, q)
        mx.mx_paged_attn_f8(batch_of(reqs), c.shape(8), q, c.mx, q, ws)
        assert torch.equal(q, want)


@pytest.mark.parametrize("weight", [False, True])
@pytest.mark.parametrize("nq,nkv,d,reqs", [
    # 8 heads of a tile, 408 and 440 tiles, whole ones of up to 70 chunks; beside decodes
    (64, 8, 128, [(0, 1 + r % 17, 40 * r % 900) for r in range(44)] + [(0, 70, 4400)]),
    (64, 8, 128, [(0, 33, 20 * r) for r in range(18)] + [(1, 1, 2100), (0, 9, 2950), (1, 1, 5)]),
    # one head a tile, 448 tiles; an odd group, 396 tiles
    (64, 64, 64, [(0, n, x) for n, x in ((3, 0), (1, 17), (16, 1500), (128, 1), (130, 1100), (2, 5))]),
    (36, 4, 64, [(0, 128, 3), (0, 1, 1700), (0, 4, 60)] + [(0, 5, 10 * r) for r in range(8)]),
    # 8 and 16 heads of a tile, split over keys
    (64, 8, 64, [(0, 5, 16500)]), (32, 2, 128, [(0, 200, 9000), (1, 1, 800), (0, 2, 1300)])])
def test_attention_many_and_wide_tiles(nq, nkv, d, reqs, weight):
    """More prefill tiles than are split over their keys, long ones among them, and tiles of 8 and
    more q heads."""
    c, reqs, q = make_case(nq, nkv, d, reqs, nq + nkv, weight)
    out, mag, weights, worst = attend_ref(c, nq, reqs, q.double().numpy())
    got, _ = run_attn(c, nq, reqs, q.cuda())
    check_out(got, out, mag)
    if weight:
        check_weights(c, c.hw, reqs, weights, worst)
    assert torch.equal(run_attn(c, nq, reqs, q.cuda())[0], got)


def test_small_calls_give_what_large_ones_give():
    """The same requests in one call, whose metadata is staged, and one by one, where it goes with
    the kernel's arguments: append, attention and eviction, bit for bit."""
    rng = np.random.default_rng(30)
    R, nq, nkv, d = 250, 8, 2, 128
    ctx = rng.integers(1, 300, R)
    pages = int((-(-(ctx + 1) // 16)).sum() + (-(-ctx // 2 // 16)).sum()) + 300
    tabs = tables(rng, pages, list(ctx + 1) + list(np.maximum(ctx // 2, 1)))
    kv = bf16(rng.normal(0, 1, (2, R, nkv, d))).cuda()
    q = bf16(rng.normal(0, 1, (R, nq, d))).cuda()
    reqs = [(1, 1, int(n), t) for n, t in zip(ctx, tabs)]
    ev = [(int(n), max(int(n) // 2, 1), min(3, max(int(n) // 2, 1)), tabs[r], tabs[R + r])
          for r, n in enumerate(ctx)]
    got = []
    for one_by_one in (False, True):
        c = Cache(pages, nkv, d, poison=False)
        r2 = np.random.default_rng(31)
        for t, n in zip(tabs, ctx):
            fill(c, r2, t, int(n))
        c.upload()
        s = c.shape(nq)
        plain = mx.CacheF8(c.k, c.v, c.ks, c.vs)
        out = torch.zeros(R, nq, d, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        kept = []
        for part in ([[r] for r in range(R)] if one_by_one else [list(range(R))]):
            lo, hi = part[0], part[-1] + 1
            b = batch_of([reqs[r] for r in part])
            k, v = kv[0, lo:hi].contiguous(), kv[1, lo:hi].contiguous()
            mx.mx_kv_append_f8(b, s, k, v, c.mx)
            mx.mx_paged_attn_f8(b, s, q[lo:hi], plain, out[lo:hi], ws)
            kept.append(run_evict(c, [ev[r] for r in part])[0][:-8])
        got.append((out, torch.cat(kept), c.k, c.v, c.ks, c.vs, c.w))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert got[0][0].float().abs().min(-1).values.max() > 0


def test_attention_scales_far_apart():
    """Pages whose scales differ by up to 2^40, values that no common scale could hold."""
    c, reqs, q = make_case(8, 2, 128, [(1, 1, 700), (0, 90, 200)], 5, False, spread=20)
    q = bf16(q.double() * 2.0 ** -14)
    out, mag, _, _ = attend_ref(c, 8, reqs, q.double().numpy())
    got, _ = run_attn(c, 8, reqs, q.cuda())
    check_out(got, out, mag)


def test_large_queries():
    """Query rows of very different size, and scores in the hundreds."""
    c, reqs, q = make_case(8, 2, 64, [(1, 1, 500), (0, 70, 33)], 15, False, spread=1)
    amp = 2.0 ** np.random.default_rng(1).integers(-30, 6, (q.shape[0], 8, 1))
    q = bf16(q.double() * torch.from_numpy(amp))
    q[3, 2] = 0
    out, mag, _, _ = attend_ref(c, 8, reqs, q.double().numpy())
    got, _ = run_attn(c, 8, reqs, q.cuda())
    check_out(got, out, mag)


@pytest.mark.parametrize("weight", [False, True])
@pytest.mark.parametrize("nq,nkv,d,reqs", [
    (8, 2, 128, [(0, 150, 301), (1, 1, 300)]), (4, 4, 64, [(0, 40, 0), (0, 3, 100)]),
    (8, 2, 64, [(0, 5, 3000)]), (2, 1, 128, [(1, 1, 77), (1, 1, 2000)])])
def test_cancelling_channels(nq, nkv, d, reqs, weight):
    """Channels whose products are hundreds and cancel: every key of a KV head has the same score,
    the part that differs cancels between two channels with the same query, one's codes the other's
    negated.  Codes are integers and queries multiples of 1 / 32, so with
    sum |q k| < 2^24 / 32 in units of a code every partial sum is an fp32 number: a score in 32 bits
    is exact in any order.  A row's probabilities are then equal, 1 before they are normalised (to
    2^-24 of the score in the exponent, which the rounding to bf16 takes away), and the output is
    the values' mean: one rounding to bf16, 2^-8, and the fp32 sums of n <= 3008 values,
    2 n 2^-24 A < 2^-11 A."""
    c, reqs, q = make_case(nq, nkv, d, reqs, d + nq, weight, spread=1)
    rng = np.random.default_rng(40)
    ch = rng.permutation(d)[:8].reshape(2, 4)
    same = rng.integers(8, 17, (nkv, d)) * rng.choice([-1, 1], (nkv, d))
    for _, n, ctx, table in reqs:
        for i, page in enumerate(table):
            m = min(16, n + ctx - 16 * i)
            k = np.repeat(same[:, None].astype(float), m, 1)
            k[:, :, ch[0]] = rng.choice([224, 240, 256, 288, 320, 352, 384], (nkv, m, 4))
            k[:, :, ch[1]] = -k[:, :, ch[0]]
            c.hk[page, :, :m] = encode8(k)
            c.hks[page] = 2.0 ** -6
    c.upload()
    q = np.clip(np.round(q.double().numpy() * 32), -96, 96) / 32
    big = rng.integers(96, 128, q.shape[:2] + (4,)).astype(float)
    q[:, :, ch[0]] = q[:, :, ch[1]] = big
    units = np.abs(q).sum(-1).max() * 16 + 8 * np.abs(big).max() * 384  # at least sum |q k| of any key
    assert (bf16(q).double().numpy() == q).all() and units < 2.0 ** 24 / 32
    out, mag, weights, worst = attend_ref(c, nq, reqs, q)
    assert worst > 250
    got = run_attn(c, nq, reqs, bf16(q).cuda())[0].double().cpu().numpy()
    off = np.abs(got - out) - (2.0 ** -8 * np.abs(out) + 2.0 ** -11 * mag)
    assert off.max() <= 0, f"{off.max():.3e} beyond the bound"
    if weight:
        check_weights(c, c.hw, reqs, weights, 16.0)  # exact scores; they and the log-sums are below 16


def test_nan_stays_in_its_rows():
    """A NaN key or value reaches the rows that attend to it, of its head, and no others; so does
    an infinite or NaN query."""
    c, reqs, q = make_case(8, 2, 128, [(1, 1, 100), (0, 40, 30)], 6, False)
    c.hk[reqs[1][3][3], 0, 2, 7] = NAN      # position 50: rows 20 .. of heads 0 .. 3
    c.hv[reqs[0][3][1], 1, 0, 9] = NAN      # the decode's heads 4 .. 7, dim 9
    q[5, 6, 3] = math.nan
    q[6, 5, 3] = math.inf
    c.upload()
    got = run_attn(c, 8, reqs, q.cuda())[0].double().cpu().numpy()
    bad = np.zeros_like(got, bool)
    bad[1 + 20:, :4] = True
    bad[0, 4:, 9] = True
    bad[5, 6] = bad[6, 5] = True
    assert (np.isnan(got) == bad).all()


@pytest.mark.parametrize("weight", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_nan_values_of_later_tokens(d, weight):
    """A NaN value of a chunk's token leaves the chunk's earlier rows as they are without it,
    and makes that dim of the token's own row and of all later ones NaN."""
    at = [(0, 0, 0, 3), (0, 37, 1, 0), (0, 130, 1, d - 1), (1, 63, 0, 17), (1, 64, 1, 40), (2, 2, 0, 1)]
    c, reqs, q = make_case(8, 2, d, [(False, 150, 0), (False, 65, 50), (False, 3, 8)], 23, weight)
    start = np.cumsum([0] + [r[1] for r in reqs])
    exp, mag, weights, worst = attend_ref(c, 8, reqs, q.double().numpy())
    bad = np.zeros(exp.shape, bool)
    for r, row, g, e in at:
        _, n, ctx, table = reqs[r]
        c.hv[table[(ctx + row) // 16], g, (ctx + row) % 16, e] = NAN if row % 2 else 0xFF
        bad[start[r] + row:start[r] + n, 4 * g:4 * g + 4, e] = True
    c.upload()
    got = run_attn(c, 8, reqs, q.cuda())[0].cpu()
    assert (got.isnan().numpy() == bad).all()
    check_out(got.masked_fill(torch.from_numpy(bad), 0), np.where(bad, 0, exp), mag)
    if weight:
        check_weights(c, c.hw, reqs, weights, worst)


@pytest.mark.parametrize("weight", [False, True])
def test_nan_in_split_tiles(weight):
    """A NaN key or value of any split reaches the rows that attend to it, of its heads and dim."""
    c, reqs, q = make_case(8, 2, 128, [(0, 40, 3000), (0, 3, 2000)], 24, weight)
    start = [0, 40]
    exp, mag, _, _ = attend_ref(c, 8, reqs, q.double().numpy())
    bad = np.zeros(exp.shape, bool)
    for r, pos, g, e in [(0, 700, 0, 5), (0, 3010, 1, 77), (1, 2001, 0, 3)]:
        table, first = reqs[r][3], max(0, pos - reqs[r][2])
        c.hv[table[pos // 16], g, pos % 16, e] = NAN
        bad[start[r] + first:start[r] + reqs[r][1], 4 * g:4 * g + 4, e] = True
    c.hk[reqs[1][3][60], 1, 2, 7] = NAN
    bad[40:, 4:] = True
    c.upload()
    got = run_attn(c, 8, reqs, q.cuda())[0].cpu()
    assert (got.isnan().numpy() == bad).all()
    check_out(got.masked_fill(torch.from_numpy(bad), 0), np.where(bad, 0, exp), mag)


@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 128), (4, 4, 64)])
def test_nan_weights(nq, nkv, d):
    """A NaN key or a query that is not finite makes the weight of every token that its rows attend
    to NaN, of that KV head, and no other; a NaN value changes no weight.  Chunks whole and split
    over their keys, decodes whole and split, more weights added in a second call."""
    c, reqs, q = make_case(nq, nkv, d, [(0, 40, 3000), (0, 150, 20), (0, 3, 8), (1, 1, 5000), (1, 1, 70),
                                        (1, 1, 90), (0, 20, 30)], 25, True)
    group = nq // nkv
    start = np.cumsum([0] + [r[1] for r in reqs])
    _, _, weights, worst = attend_ref(c, nq, reqs, q.double().numpy())
    for r, pos, g in [(0, 700, 1), (1, 100, 0), (3, 4321, 0), (4, 3, 1)]:  # keys
        table = reqs[r][3]
        c.hk[table[pos // 16], g, pos % 16, 7] = NAN
        weights[r][g] = math.nan  # the last row attends to the token, and to all others
    for r, row, h, x in [(0, 11, 0, math.nan), (2, 1, nq - 1, math.inf), (5, 0, 1, math.nan)]:  # queries
        q[start[r] + row, h, 5] = x
        weights[r][h // group, :reqs[r][2] + row + 1] = math.nan
    for r, pos, g in [(6, 35, 0), (4, 50, 0)]:  # values
        c.hv[reqs[r][3][pos // 16], g, pos % 16, 9] = 0xFF
    c.upload()
    run_attn(c, nq, reqs, q.cuda())
    before = check_weights(c, c.hw, reqs, weights, worst)
    run_attn(c, nq, reqs, q.cuda())
    check_weights(c, before, reqs, weights, worst)


def test_shared_prefix_weights_add_up():
    """Requests that read the same cached pages: each key receives the sum over all of them."""
    c, reqs, q = make_case(8, 2, 64, [(1, 1, 90), (0, 33, 64)], 7, True)
    shared = reqs[0][3][:4]
    for r in range(1, 2):
        reqs[r] = (*reqs[r][:3], shared + reqs[r][3][4:])
    reqs.append((1, 1, 63, shared))
    q = bf16(np.random.default_rng(8).normal(0, 1, (35, 8, 64)))
    out, mag, weights, worst = attend_ref(c, 8, reqs, q.double().numpy())
    got, _ = run_attn(c, 8, reqs, q.cuda())
    check_out(got, out, mag)
    check_weights(c, c.hw, reqs, weights, worst)


# ----------------------------------------------------------------------- eviction
def evict_ref(c, reqs):
    """reqs: (len, keep, recent, pages, dst).  Moves the mirror's tokens; the kept indices."""
    kept = []
    for n, keep, recent, src, dst in reqs:
        for g in range(c.nkv):
            pos = np.arange(n)
            w = c.hw[np.asarray(src, int)[pos // 16], g, pos % 16].astype(np.float32) if n else np.zeros(0)
            old = w[:n - recent]
            rank = np.where(np.isnan(old), np.inf, old)
            order = sorted(range(len(old)), key=lambda j: (not np.isnan(old[j]), -rank[j], j))
            idx = sorted(order[:keep - recent]) + list(range(n - recent, n))
            kept += idx
            for i0 in range(0, keep, 16):
                here = idx[i0:i0 + 16]
                page = dst[i0 // 16]
                at = [(src[j // 16], j % 16) for j in here]
                for codes, scales in ((c.hk, c.hks), (c.hv, c.hvs)):
                    now = max(scales[p, g] for p, _ in at)
                    for i, (p, s) in enumerate(at):
                        codes[page, g, i] = encode8(decode8(codes[p, g, s]) * (scales[p, g] / now))
                    scales[page, g] = now
                for i, (p, s) in enumerate(at):
                    c.hw[page, g, i] = c.hw[p, g, s]
    return np.array(kept, np.int32)


def run_evict(c, reqs, stream=None):
    e = mx.EvictBatch(*zip(*[(r[0], r[1], r[2]) for r in reqs]), [r[3] for r in reqs], [r[4] for r in reqs])
    s = c.shape(c.nkv)
    ws = torch.empty(mx.mx_kv_evict_f8_ws_bytes(e, s), dtype=torch.uint8, device="cuda")
    kept = torch.full((c.nkv * e.total_keep + 8,), -7, dtype=torch.int32, device="cuda")
    mx.mx_kv_evict_f8(e, s, c.mx, kept, ws, stream=stream)
    return kept, ws


def check_evict(c, reqs):
    exp = evict_ref(c, reqs)
    kept, _ = run_evict(c, reqs)
    kept = kept.cpu().numpy()
    np.testing.assert_array_equal(kept[:len(exp)], exp)
    assert (kept[len(exp):] == -7).all()
    c.check("evict")
    np.testing.assert_array_equal(c.w.cpu().numpy(), c.hw.astype(np.float32))


def evict_case(nkv, d, lens, keeps, recents, seed, weights=None):
    rng = np.random.default_rng(seed)
    pages = sum(-(-n // 16) for n in lens) + sum(-(-k // 16) for k in keeps) + 5
    c = Cache(pages, nkv, d)
    tabs = tables(rng, pages, list(lens) + list(keeps)) if keeps[-1] else None
    for r, n in enumerate(lens):
        fill(c, rng, tabs[r], n)
    R = len(lens)
    reqs = [(lens[r], keeps[r], recents[r], tabs[r], tabs[R + r]) for r in range(R)]
    if weights:
        for n, _, _, src, _ in reqs:
            for j in range(n):
                c.hw[src[j // 16], :, j % 16] = [weights(rng, j) for _ in range(nkv)]
    c.upload()
    return c, reqs


@pytest.mark.parametrize("nkv,d", [(1, 64), (3, 128), (8, 128)])
def test_evict(nkv, d):
    lens = [1, 2, 16, 17, 33, 100, 257, 1023, 1025, 2100, 40, 64, 5, 48]
    keeps = [1, 1, 8, 16, 32, 31, 256, 500, 1024, 2050, 40, 17, 5, 16]
    recents = [0, 1, 4, 0, 32, 1, 5, 100, 1024, 7, 3, 0, 5, 15]
    check_evict(*evict_case(nkv, d, lens, keeps, recents, nkv))


@pytest.mark.parametrize("name,weights", [
    ("all equal", lambda rng, j: 1.0),
    ("mostly zero", lambda rng, j: float(rng.random() < 0.1)),
    ("few values", lambda rng, j: float(rng.integers(0, 3)) * 2.0 ** -60),
    ("signed", lambda rng, j: float(np.float32(rng.normal()))),
    ("minus zero", lambda rng, j: -0.0 if rng.random() < 0.5 else 0.0),
    ("infinite and NaN", lambda rng, j: [math.inf, math.nan, 1.0, -math.inf][rng.integers(0, 4)]),
    ("denormal", lambda rng, j: float(np.float32(2.0 ** -149 * rng.integers(0, 1000)))),
])
def test_evict_ties_and_odd_weights(name, weights):
    check_evict(*evict_case(2, 64, [300, 1500, 2048], [100, 700, 1030], [10, 0, 1], 9, weights))


def test_evict_any_nan_counts_as_the_largest():
    """NaNs of either sign and any payload: above infinity, equal among themselves."""
    c, reqs = evict_case(2, 64, [300, 1500, 5000], [100, 700, 1030], [10, 0, 1], 13,
                         lambda rng, j: [math.inf, math.nan, 1.0, -math.inf][rng.integers(0, 4)])
    bits = torch.tensor([0x7FC00000, 0x7F800001, 0x7FFFFFFF, -0x00400000, -0x007FFFFF, -1],
                        dtype=torch.int32, device="cuda")
    w = c.w.view(torch.int32).flatten()
    w[:] = torch.where(c.w.flatten().isnan(), bits[torch.arange(w.numel(), device="cuda") % 6], w)
    assert (c.w.cpu().isnan() == torch.from_numpy(c.hw).isnan()).all()
    check_evict(c, reqs)


@pytest.mark.parametrize("n,keep,recent", [(40001, 12345, 300), (20000, 19999, 1), (4097, 5, 0),
                                           (32769, 1, 1)])
def test_evict_long(n, keep, recent):
    check_evict(*evict_case(1, 64, [n], [keep], [recent], 10))


def test_evict_keeps_nothing_or_everything():
    c, reqs = evict_case(2, 64, [50, 60, 33], [50, 0, 33], [0, 0, 33], 11)
    check_evict(c, reqs)


def test_evict_from_a_shared_prefix():
    """Two requests keep different parts of the same source pages."""
    c, reqs = evict_case(2, 64, [100, 80], [40, 30], [4, 9], 12)
    n, keep, recent, _, dst = reqs[1]
    reqs[1] = (n, keep, recent, reqs[0][3], dst)
    check_evict(c, reqs)


# ----------------------------------------------------------------------- together
def test_serving_loop():
    """A prompt in chunks, decodes that track their attention, an eviction in the middle, more
    decodes over what stayed: append, attention, eviction in turn, each step against the
    reference, which holds the same cache."""
    nq, nkv, d = 8, 2, 128
    rng = np.random.default_rng(20)
    c = Cache(200, nkv, d)
    c.upload()
    free = rng.permutation(200).tolist()
    ctx, tabs = [0, 0], [[], []]

    def step(n_new):
        reqs = []
        for r, n in enumerate(n_new):
            while len(tabs[r]) < -(-(ctx[r] + n) // 16):
                tabs[r].append(free.pop())
            reqs.append((n == 1 and ctx[r] > 0, n, ctx[r], list(tabs[r])))
        T = sum(n_new)
        k, v = bf16(rng.normal(0, 1, (T, nkv, d))), bf16(rng.normal(0, 1, (T, nkv, d)))
        q = bf16(rng.normal(0, 1.5, (T, nq, d)))
        mx.mx_kv_append_f8(batch_of(reqs), c.shape(nq), k.cuda(), v.cuda(), c.mx)
        t = 0
        for (_, n, x, table) in reqs:
            append_ref(c, table, x, k[t:t + n].double().numpy(), v[t:t + n].double().numpy())
            t += n
        out, mag, weights, worst = attend_ref(c, nq, reqs, q.double().numpy())
        got, _ = run_attn(c, nq, reqs, q.cuda())
        check_out(got, out, mag)
        check_weights(c, c.hw, reqs, weights, worst)
        c.hw[:] = c.w.cpu().numpy()  # go on from the device's sums
        for r, n in enumerate(n_new):
            ctx[r] += n

    step([200, 77])
    step([150, 1])
    for _ in range(3):
        step([1, 1])
    c.check("before the eviction")
    keeps = [120, 50]
    dst = [[free.pop() for _ in range(-(-k // 16))] for k in keeps]
    reqs = [(ctx[r], keeps[r], 20, tabs[r], dst[r]) for r in range(2)]
    check_evict(c, reqs)
    for r in range(2):
        free.extend(tabs[r])
        tabs[r], ctx[r] = dst[r], keeps[r]
    for _ in range(20):
        step([1, 1])
    step([40, 1])
    c.check("at the end")


def test_same_results_on_any_stream_and_thread():
    c, reqs, q = make_case(8, 2, 128, [(1, 1, 900), (0, 100, 50), (1, 1, 5000)], 21, False)
    q = q.cuda()
    want, _ = run_attn(c, 8, reqs, q)
    torch.cuda.synchronize()
    results = [None] * 4

    def work(i):
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            for _ in range(10):
                results[i], _ = run_attn(c, 8, reqs, q, stream=st)
        st.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert all(torch.equal(r, want) for r in results)


def test_streams_and_threads_of_all_calls():
    """Append, attention with weights and eviction in turn, in small calls and staged ones, by four
    threads at once, each on a stream and a cache of its own: bit for bit what they give alone."""
    nq, nkv, d, pages = 8, 2, 128, 1500

    def state(seed):
        rng = np.random.default_rng(seed)
        c = Cache(pages, nkv, d, poison=False)
        R = [3, 120, 5, 90][seed % 4]  # requests; the larger batches' metadata are staged
        ctx = rng.integers(1, 150, R)
        ctx[0] = 3000
        news = np.where(np.arange(R) % 2 == 0, 1, rng.integers(1, 20, R))
        tabs = tables(rng, pages, [int(n) for n in ctx + news] + [10] * R)
        for t, n in zip(tabs, ctx):
            fill(c, rng, t[:-(-int(n) // 16)], int(n))
        c.upload()
        reqs = [(i % 2 == 0, int(n), int(x), t) for i, (n, x, t) in enumerate(zip(news, ctx, tabs))]
        T = int(news.sum())
        kv = bf16(rng.normal(0, 1, (2, T, nkv, d))).cuda()
        q = bf16(rng.normal(0, 1, (T, nq, d))).cuda()
        ev = [(n + x, min(10, n + x), 1, t, tabs[R + i]) for i, (_, n, x, t) in enumerate(reqs)]
        return c, reqs, kv, q, ev

    def work(s, stream=None):
        c, reqs, kv, q, ev = s
        res = []
        for _ in range(6):
            mx.mx_kv_append_f8(batch_of(reqs), c.shape(nq), kv[0], kv[1], c.mx, stream=stream)
            out, ws = run_attn(c, nq, reqs, q, stream=stream)
            kept, ws2 = run_evict(c, ev, stream=stream)
            res += [out, kept, ws, ws2]  # (the workspaces stay until the stream is done)
        return res[0::4] + res[1::4] + [c.k, c.v, c.ks, c.vs, c.w], res

    want = [work(state(i))[0] for i in range(4)]
    states, got = [state(i) for i in range(4)], [None] * 4
    torch.cuda.synchronize()

    def thread(i):
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            got[i] = work(states[i], st)
        st.synchronize()

    threads = [threading.Thread(target=thread, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g[0], w))


def test_captured_streams_are_refused():
    c, reqs, q = make_case(4, 2, 64, [(1, 1, 90)], 22, True)
    s, b, q = c.shape(4), batch_of(reqs), q.cuda()
    out, ws = run_attn(c, 4, reqs, q)
    kv = bf16(np.ones((1, 2, 64))).cuda()
    e = mx.EvictBatch([90], [20], [1], [reqs[0][3]], [[p for p in range(c.pages) if p not in reqs[0][3]][:2]])
    kept = torch.zeros(40, dtype=torch.int32, device="cuda")
    big = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    y = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    graph, seen = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph):
        for call in (lambda: mx.mx_paged_attn_f8(b, s, q, c.mx, out, ws),
                     lambda: mx.mx_kv_append_f8(b, s, kv, kv, c.mx),
                     lambda: mx.mx_kv_evict_f8(e, s, c.mx, kept, big)):
            try:
                call()
            except mx.MxError as x:
                seen.append(x.status)
        y += 1
    assert seen == [mx.MX_ERR_UNSUPPORTED] * 3
    graph.replay()
    torch.cuda.synchronize()
    assert y.tolist() == [1.0] * 4
    assert torch.equal(run_attn(c, 4, reqs, q)[0], out)


def test_binding_refuses_other_tensors():
    """Strided, of another type, or not on the cache's device: refused before anything runs."""
    c, reqs, q = make_case(4, 2, 64, [(0, 5, 3)], 30, True)
    b, s, q = batch_of(reqs), c.shape(4), q.cuda()
    kv = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(mx.mx_workspace_bytes_f8_for(b, s, True), dtype=torch.uint8, device="cuda")
    e = mx.EvictBatch([8], [4], [1], [reqs[0][3]], [[p for p in range(c.pages) if p not in reqs[0][3]][:1]])
    kept = torch.zeros(2 * 4, dtype=torch.int32, device="cuda")
    for bad in (lambda t: torch.zeros(t.shape + (2,), dtype=t.dtype, device="cuda")[..., 0],
                lambda t: t.to(torch.float64), lambda t: t.cpu()):
        for args in ((bad(kv), kv), (kv, bad(kv))):
            with pytest.raises(ValueError):
                mx.mx_kv_append_f8(b, s, *args, c.mx)
        for i in range(3):
            t = [q, q.clone(), ws]
            t[i] = bad(t[i])
            with pytest.raises(ValueError):
                mx.mx_paged_attn_f8(b, s, t[0], c.mx, t[1], t[2])
        for args in ((bad(kept), ws), (kept, bad(ws))):
            with pytest.raises(ValueError):
                mx.mx_kv_evict_f8(e, s, c.mx, *args)
    c.check("refused")


def test_binding_refuses_other_types_of_the_same_size():
    """fp16 and int16 for bf16, fp32 for int32: refused before anything runs; the bits of bf16 as
    uint16 are taken."""
    c, reqs, q = make_case(4, 2, 64, [(0, 5, 3)], 31, False)
    b, s, q = batch_of(reqs), c.shape(4), q.cuda()
    kv = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    want, ws = run_attn(c, 4, reqs, q)
    for t in (torch.float16, torch.int16):
        for args in ((kv.view(t), kv), (kv, kv.view(t))):
            with pytest.raises(ValueError):
                mx.mx_kv_append_f8(b, s, *args, c.mx)
        for args in ((q.view(t), c.mx, q.clone()), (q, c.mx, q.clone().view(t))):
            with pytest.raises(ValueError):
                mx.mx_paged_attn_f8(b, s, *args, ws)
    e = mx.EvictBatch([8], [4], [1], [reqs[0][3]], [[p for p in range(c.pages) if p not in reqs[0][3]][:1]])
    with pytest.raises(ValueError):
        mx.mx_kv_evict_f8(e, s, c.mx, torch.zeros(8, device="cuda"), ws)
    c.check("refused")
    out = torch.zeros(q.shape, dtype=torch.uint16, device="cuda")
    mx.mx_paged_attn_f8(b, s, q.view(torch.uint16), c.mx, out, ws)
    assert torch.equal(out.view(torch.bfloat16), want)


def test_pages_beyond_4_gib():
    """Pages whose byte offsets pass 2^32 in every pool, against the same requests in low pages."""
    nq, nkv, d = 16, 8, 128
    pages = 300_000  # 16 KB of keys a page: 4.9 GB per pool; 128 B of weights a page
    c = Cache(pages, nkv, d, poison=False)
    rng = np.random.default_rng(23)
    lens, keep = [333, 40], [100, 17]
    k, v = (bf16(rng.normal(0, 1, (373, nkv, d))).cuda() for _ in range(2))
    q = bf16(rng.normal(0, 1, (2, nq, d))).cuda()
    got = []
    for base in (0, pages - 100):
        tabs = tables(np.random.default_rng(1), 50, lens + keep)
        tabs = [[base + p for p in t] for t in tabs]
        mx.mx_kv_append_f8(batch_of([(0, n, 0, t) for n, t in zip(lens, tabs)]), c.shape(nq), k, v, c.mx)
        out, _ = run_attn(c, nq, [(1, 1, n - 1, t) for n, t in zip(lens, tabs)], q)
        kept, _ = run_evict(c, [(lens[r], keep[r], 5, tabs[r], tabs[2 + r]) for r in range(2)])
        dst = torch.tensor(tabs[2] + tabs[3], device="cuda")
        got.append((out, kept, c.k[dst], c.v[dst], c.ks[dst], c.vs[dst], c.w[dst]))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert got[0][0].float().abs().max() > 0 and got[0][2].float().abs().max() > 0
