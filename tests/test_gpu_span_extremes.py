"""GPU tests of values at the ends of bf16's range in attention over parts of the keys, with the
references and bounds of test_gpu_span.py."""
import math

import numpy as np
import pytest

from span_batches import CASES, D, P
from test_gpu_span import reference, check, run_shared, run_window, seen, shared_case, window_case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def low_key(pools, table, j):
    """Position j gets a key whose score, with queries of no negative element, underflows: -40 in
    every dim, times |q| of 0.8 on average, over sqrt(d): below -250."""
    pools.hk[table[j // 16], :, j % 16] = -40.0


def check_marked(pools, nq, reqs, q, got, clean, hit, window, sinks):
    """Rows of `hit` are not finite in dim 7, everything else is what it was without the value."""
    pools.hv = clean
    out, mag = reference(pools, nq, reqs, q, window, sinks)
    got, keep = got.cpu(), torch.ones(len(q), pools.d, dtype=torch.bool)
    keep[hit, 7] = False
    keep = keep[:, None].expand(-1, nq, -1)
    assert not torch.isfinite(got[~keep].double()).any()
    check(torch.where(keep, got, torch.from_numpy(out).to(torch.bfloat16)), out, mag)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("nq,nkv,d", [(4, 4, 64), (8, 2, 128), (16, 1, 128)])
@pytest.mark.parametrize("window,sinks", [(40, 6), (500, 0), (3000, 20)])
def test_values_whose_probability_underflows(nq, nkv, d, window, sinks, bad):
    """In whole chunks and at both edges of the window, of tiles, streams, splits: such a value
    makes the rows that see its token not finite in its dim, and no other row or dim."""
    reqs = [(P, 300, 0), (P, 140, 1000), (D, 1, 700), (P, 3, 2500), (D, 1, 2900), (P, 200, 2700)]
    pools, reqs, q = window_case(nq, nkv, d, reqs, 211, window, sinks)
    q = q.abs()
    clean, hit, start = pools.hv.clone(), torch.zeros(len(q), dtype=torch.bool), np.cumsum([0] + [r[1] for r in reqs])
    for r, (_, n, ctx, table) in enumerate(reqs):
        see = seen(n, ctx, window, sinks)
        low = max(1, ctx - window + 1)
        for j in {low, (low + ctx + n - 1) // 2, max(low, ctx - 1), ctx + n // 2}:
            # (not a row's only key: it would have a probability of 1)
            if see[:, j].any():
                low_key(pools, table, j)
                pools.hv[table[j // 16], :, j % 16, 7] = bad
                hit[start[r]:start[r + 1]] |= torch.from_numpy(see[:, j])
    pools.upload()
    got, _ = run_window(pools, nq, reqs, q.cuda(), window, sinks)
    check_marked(pools, nq, reqs, q, got, clean, hit, window, sinks)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("name", ["tree", "in place"])
def test_values_whose_probability_underflows_in_a_run(name, bad):
    """The same in a run that is read once for its requests, and behind it."""
    (nq, nkv, d), reqs, runs = CASES[name]
    pools, reqs, q = shared_case(nq, nkv, d, reqs, runs, 212)
    q = q.abs()
    clean, hit = pools.hv.clone(), torch.zeros(len(q), dtype=torch.bool)
    start = np.cumsum([0] + [r[1] for r in reqs])
    inner = runs[1] if len(runs) > 1 else (0, 0, 0)
    for first, n, r, j in ((inner[0], inner[1], inner[0], 16 * runs[0][2] + 37), (3, 1, 3, 16 * sum(k for a, n, k in runs if a <= 3 < a + n))):
        if n == 0:
            continue
        low_key(pools, reqs[r][3], j)
        pools.hv[reqs[r][3][j // 16], :, j % 16, 7] = bad
        for i in range(first, first + n):
            hit[start[i]:start[i + 1]] |= torch.from_numpy(seen(reqs[i][1], reqs[i][2], 2 ** 31 - 1, 0)[:, j])
    pools.upload()
    got, _ = run_shared(pools, nq, reqs, runs, q.cuda())
    check_marked(pools, nq, reqs, q, got, clean, hit, 2 ** 31 - 1, 0)


@pytest.mark.parametrize("window,n", [(64, 400), (4096, 4000)])
def test_values_up_to_the_documented_size(window, n):
    """Finite values up to 2^120 over the keys that a row sees: no overflow, the usual bound."""
    pools, reqs, q = window_case(8, 2, 128, [(P, 200, n), (D, 1, n)], 213, window, 0)
    keys = min(window, n + 200)
    top = 2.0 ** (119 - math.ceil(math.log2(keys)))
    pools.hv = (pools.hv.double().clamp(-4, 4) / 4 * top).to(torch.bfloat16)
    pools.upload()
    out, mag = reference(pools, 8, reqs, q, window, 0)
    got, _ = run_window(pools, 8, reqs, q.cuda(), window, 0)
    check(got, out, mag)
