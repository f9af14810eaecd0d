"""GPU tests of what attention over parts of the keys reads and writes of its workspace: nothing
that an earlier call left there, nothing behind the bytes that it asked for."""
import math

import pytest

import paper_2606_16264_amd as mx
from test_gpu_span import (ALL, CHUNKS, D, DECODES, P, SHARED, batch_of, check, reference, shared_case,
                           window_case)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

GUARD = 4096


def on_any_workspace(n, attend, q, exp, mag):
    """The call's result on a workspace of NaNs, of zeros, of its own leavings and of finite
    garbage: the reference's, each time the same bits; the bytes behind it stay."""
    buf = torch.empty(n + GUARD, dtype=torch.uint8, device="cuda")
    results = []
    for fill in (255, 0, None, 0x3F):
        if fill is not None:
            buf.fill_(fill)
        buf[n:] = 7
        out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda")
        attend(out, buf[:n])
        results.append(out)
        assert (buf[n:] == 7).all(), fill
        check(out, exp, mag, f"workspace of {fill}")
        assert torch.equal(out.view(torch.uint16), results[0].view(torch.uint16)), fill


@pytest.mark.parametrize("nq,nkv,d", [(4, 4, 64), (20, 1, 64), (36, 2, 128)])
@pytest.mark.parametrize("window,sinks", [(31, 3), (700, 33), (ALL, 0)])
def test_window(nq, nkv, d, window, sinks):
    reqs = [(1, 1, n) for n in DECODES] + [(0, n, x) for n, x in CHUNKS]
    pools, reqs, q = window_case(nq, nkv, d, reqs, nq + d, window, sinks)
    s, b, q_dev = pools.shape(nq), batch_of(reqs), q.cuda()
    n = mx.mx_workspace_bytes_window_for(b, s, window, sinks)
    on_any_workspace(n, lambda out, ws: mx.mx_paged_attn_window(b, s, window, sinks, q_dev, pools.k, pools.v, out, ws),
                     q, *reference(pools, nq, reqs, q, window, sinks))


@pytest.mark.parametrize("kind", ["decode", "prefill"])
@pytest.mark.parametrize("nq,nkv,d,window,sinks", [(8, 2, 128, 4000, 100), (16, 1, 64, 5000, 600)])
def test_window_splits(nq, nkv, d, window, sinks, kind):
    reqs = [(1, 1, 9000), (1, 1, 4001)] if kind == "decode" else [(0, 300, 6001), (0, 700, 0), (0, 2, 9000)]
    pools, reqs, q = window_case(nq, nkv, d, reqs, 3, window, sinks)
    s, b, q_dev = pools.shape(nq), batch_of(reqs), q.cuda()
    n = mx.mx_workspace_bytes_window_for(b, s, window, sinks)
    on_any_workspace(n, lambda out, ws: mx.mx_paged_attn_window(b, s, window, sinks, q_dev, pools.k, pools.v, out, ws),
                     q, *reference(pools, nq, reqs, q, window, sinks))


@pytest.mark.parametrize("more", [0, 24])
@pytest.mark.parametrize("case", range(len(SHARED)))
@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 64), (5, 5, 128), (36, 2, 128)])
def test_shared(nq, nkv, d, case, more):
    reqs, runs = SHARED[case]
    if more:  # decodes of a run that is long enough for all runs to be joined
        pages = -(-(64 << 20) // ((more - 1) * 64 * d * nkv))
        runs = runs + [(len(reqs), more, pages)]
        reqs = reqs + [(D, 1, i) for i in range(more)]
    pools, reqs, q = shared_case(nq, nkv, d, reqs, runs, 17 * case + nq)
    s, b, rs, q_dev = pools.shape(nq), batch_of(reqs), mx.SharedRuns(runs), q.cuda()
    n = mx.mx_workspace_bytes_shared_for(b, s, rs)
    on_any_workspace(n, lambda out, ws: mx.mx_paged_attn_shared(b, s, rs, q_dev, pools.k, pools.v, out, ws),
                     q, *reference(pools, nq, reqs, q))


@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 128), (4, 4, 64)])
def test_shared_splits(nq, nkv, d):
    reqs, runs = [(D, 1, 11 * i) for i in range(33)] + [(P, 20, 5)] * 3, [(0, 36, 300), (4, 20, 70)]
    pools, reqs, q = shared_case(nq, nkv, d, reqs, runs, 23)
    s, b, rs, q_dev = pools.shape(nq), batch_of(reqs), mx.SharedRuns(runs), q.cuda()
    n = mx.mx_workspace_bytes_shared_for(b, s, rs)
    on_any_workspace(n, lambda out, ws: mx.mx_paged_attn_shared(b, s, rs, q_dev, pools.k, pools.v, out, ws),
                     q, *reference(pools, nq, reqs, q))
