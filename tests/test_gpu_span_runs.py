"""GPU tests of attention over shared runs where the planner takes a batch apart (span_batches.py;
test_span_runs.py checks that it does), against the references and with the bounds of
test_gpu_span.py."""
import math

import numpy as np
import pytest

import paper_2606_16264_amd as mx
from span_batches import CASES, D, P
from test_gpu_span import Pools, bf16, check, reference, run_shared, run_window, shared_case, window_case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def case_of(name, seed):
    (nq, nkv, d), reqs, runs = CASES[name]
    return (nq, runs) + shared_case(nq, nkv, d, reqs, runs, seed)


def test_output_in_place():
    """Rows that several items read, as rows of a run and with their own keys, are written
    after all of them; rows of out behind the batch's last keep their bytes."""
    nq, runs, pools, reqs, q = case_of("in place", 143)
    out, mag = reference(pools, nq, reqs, q)
    buf = torch.full((len(q) + 5,) + q.shape[1:], 3.0, dtype=torch.bfloat16, device="cuda")
    buf[:len(q)] = q.cuda()
    run_shared(pools, nq, reqs, runs, buf, out=buf)
    check(buf[:len(q)], out, mag)
    assert (buf[len(q):] == 3).all()
    apart, _ = run_shared(pools, nq, reqs, runs, q.cuda())
    assert torch.equal(apart.view(torch.uint16), buf[:len(q)].view(torch.uint16))


@pytest.mark.parametrize("name", ["tree", "splits"])
def test_parts_join(name):
    """Rows of two runs and their own keys; a run of many splits, with a scale of the caller's."""
    nq, runs, pools, reqs, q = case_of(name, 144)
    out, mag = reference(pools, nq, reqs, q, scale=0.11)
    got, _ = run_shared(pools, nq, reqs, runs, q.cuda(), scale=0.11)
    check(got, out, mag)


def test_matches_paged_attention():
    """With runs that are read once for their requests, the results of mx_paged_attn but for the
    rounding of probabilities and outputs: twice the bound of one against the exact."""
    nq, runs, pools, reqs, q = case_of("paged", 145)
    s, b = pools.shape(nq), mx.Batch(*zip(*[(int(r[0]), r[1], r[2], r[3]) for r in reqs]))
    ws = torch.empty(mx.mx_workspace_bytes_for(b, s), dtype=torch.uint8, device="cuda")
    plain = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    mx.mx_paged_attn(b, s, q.cuda(), pools.k, pools.v, plain, ws)
    plain = plain.double().cpu().numpy()
    _, mag = reference(pools, nq, reqs, q)
    got, _ = run_shared(pools, nq, reqs, runs, q.cuda())
    check(got, plain, 2 * mag + 2.0 ** -8 * np.abs(plain))


def test_run_beyond_4_gib():
    """A run and own pages whose byte offsets pass 32 bits."""
    pages = 140000
    nq, runs, small, reqs, q = case_of("far pages", 146)
    _, nkv, d = CASES["far pages"][0]
    k = torch.empty((pages, nkv, d // 32, 16, 32), dtype=torch.bfloat16, device="cuda")
    v = torch.empty((pages, nkv, d, 16), dtype=torch.bfloat16, device="cuda")
    far = pages - small.pages
    k[far:], v[far:] = small.k, small.v
    s = mx.attn_shape(nq, nkv, d, pages)
    b = mx.Batch([int(r[0]) for r in reqs], [r[1] for r in reqs], [r[2] for r in reqs],
                 [[far + p for p in r[3]] for r in reqs])
    rs = mx.SharedRuns(runs)
    ws = torch.empty(mx.mx_workspace_bytes_shared_for(b, s, rs), dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda")
    mx.mx_paged_attn_shared(b, s, rs, q.cuda(), k, v, out, ws)
    check(out, *reference(small, nq, reqs, q))


def test_append_then_attention():
    """As a serving loop calls them: one request brings the shared prompt, the others only their
    questions behind its pages, then all decode; every step appends the new tokens and attends
    over the run and own pages."""
    nq, nkv, d, R, prefix = 16, 8, 128, 18, 64
    rng = np.random.default_rng(147)
    pools = Pools(prefix + 3 * R, nkv, d)
    pools.upload()
    s = pools.shape(nq)
    table = [list(range(prefix)) + [prefix + 3 * r + i for i in range(3)] for r in range(R)]
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    ctx = [0] * R
    steps = [[16 * prefix] + [0] * (R - 1), [5 + r % 7 for r in range(R)]] + [[1] * R] * 4
    for step, n_new in enumerate(steps):
        if step == 1:
            ctx = [16 * prefix] * R
        live = [r for r in range(R) if n_new[r]]
        reqs = [(D if step > 1 else P, n_new[r], ctx[r], table[r]) for r in live]
        T = sum(n_new)
        q, k, v = (bf16(rng.normal(0, 1, (T, h, d))) for h in (nq, nkv, nkv))
        t = 0
        for r in live:
            j = np.arange(ctx[r], ctx[r] + n_new[r])
            pg, sl = torch.as_tensor(np.asarray(table[r])[j // 16]), torch.as_tensor(j % 16)
            pools.hk[pg, :, sl], pools.hv[pg, :, sl] = k[t:t + len(j)], v[t:t + len(j)]
            t += len(j)
            ctx[r] += n_new[r]
        b = mx.Batch([r[0] for r in reqs], [r[1] for r in reqs], [r[2] for r in reqs], [r[3] for r in reqs])
        mx.mx_kv_append(b, s, k.cuda(), v.cuda(), pools.k, pools.v, ws)
        runs = [(0, R, prefix)] if step else []
        n = mx.mx_workspace_bytes_shared_for(b, s, mx.SharedRuns(runs))
        if step:  # the run is read for several requests: their rows have partials
            assert n > mx.mx_workspace_bytes_shared_for(b, s, mx.SharedRuns([]))
        out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda")
        mx.mx_paged_attn_shared(b, s, mx.SharedRuns(runs), q.cuda(), pools.k, pools.v, out, ws)
        check(out, *reference(pools, nq, reqs, q), f"step {step}")




def test_launch_timing():
    """Each call counts once under its tag, whichever way its metadata takes, and its results are
    those without timing."""
    window = [window_case(8, 2, 64, [(D, 1, 90 + i) for i in range(n)] + [(P, p, 9)] * (p > 0), 149, 33, 2)
              for n, p in ((3, 0), (300, 0), (2, 900))]
    nq, runs, pools, reqs, q = case_of("in place", 150)
    calls = [lambda c=c: run_window(c[0], 8, c[1], c[2].cuda(), 33, 2)[0] for c in window]
    calls.append(lambda: run_shared(pools, nq, reqs, runs, q.cuda())[0])
    plain = [f() for f in calls]
    mx.mx_profile_read()
    mx.mx_profile_enable(True)
    try:
        timed = [f() for f in calls]
        got = mx.mx_profile_read()
    finally:
        mx.mx_profile_enable(False)
    for a, b in zip(plain, timed):
        assert torch.equal(a.view(torch.uint16), b.view(torch.uint16))
    assert {k: v[1] for k, v in got.items()} == {"paged_attn_window": 3, "paged_attn_shared": 1}
    assert all(v[0] > 0 for v in got.values())
