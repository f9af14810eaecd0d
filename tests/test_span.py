"""CPU checks of attention over parts of the requests' keys: the host's plans walked as the
kernels walk them; every malformed argument is refused on the host with the documented
status, before any device work; workspace sizes and their bounds; what the calls launch."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2606_16264_amd as mx
from test_host_runtime import fake_hip, run  # noqa: F401  (fake_hip is a fixture)

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
POOL = 64
ALL = 2 ** 31 - 1


def test_plans(tmp_path):
    """Every row meets each key that it sees exactly once, in random batches."""
    exe = str(tmp_path / "span_plan_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2606_16264_amd", "csrc"),
                    os.path.join(HERE, "span_plan_check.cpp"), "-o", exe], check=True)
    got = subprocess.run([exe, "60"], capture_output=True, text=True, timeout=240)
    assert got.returncode == 0, got.stdout


def shape(nq=4, nkv=2, d=64, pool=POOL):
    return mx.attn_shape(nq, nkv, d, pool)


def one(phase=mx.MX_PREFILL, n_new=4, ctx=0, pages=(1,)):
    return mx.Batch([phase], [n_new], [ctx], [pages])


def window(b, s, w=8, sinks=2, q=0x100000, k=0x200000, v=0x300000, out=0x110000, ws=0x120000, n=1 << 40):
    return mx.lib().mx_paged_attn_window(b.ptr, ctypes.byref(s), w, sinks, q, k, v, out, ws, n, None)


def shared(b, s, runs=(), q=0x100000, k=0x200000, v=0x300000, out=0x110000, ws=0x120000, n=1 << 40):
    r = mx.SharedRuns(runs)
    return mx.lib().mx_paged_attn_shared(b.ptr, ctypes.byref(s), r.n, r.ptr, q, k, v, out, ws, n, None)


def sizes(b, s, w=8, sinks=2, runs=()):
    r = mx.SharedRuns(runs)
    return (mx.lib().mx_workspace_bytes_window_for(b.ptr, ctypes.byref(s), w, sinks),
            mx.lib().mx_workspace_bytes_shared_for(b.ptr, ctypes.byref(s), r.n, r.ptr))


@pytest.mark.parametrize("b,status", [
    (mx.Batch([7], [1], [5], [[0]]), mx.MX_ERR_INVALID),
    (one(n_new=0), mx.MX_ERR_INVALID),
    (one(mx.MX_DECODE, 1, 0), mx.MX_ERR_INVALID),
    (one(n_new=2, ctx=15), mx.MX_ERR_NO_SPACE),
    (one(pages=[POOL]), mx.MX_ERR_INVALID),
    (one(pages=[-1]), mx.MX_ERR_INVALID),
    (mx.Batch([0, 1], [3, 1], [0, 2], [[5], [5]]), mx.MX_ERR_INVALID),
])
def test_bad_batches(b, status):
    for call in (window, shared):
        assert call(b, shape()) == status
        assert mx.last_error()
    assert sizes(b, shape()) == (0, 0)


@pytest.mark.parametrize("s,status", [
    (shape(4, 3), mx.MX_ERR_INVALID),
    (shape(d=96), mx.MX_ERR_UNSUPPORTED),
    (shape(pool=0), mx.MX_ERR_INVALID),
    (mx.attn_shape(4, 2, 64, POOL, page_size=32), mx.MX_ERR_UNSUPPORTED),
    (mx.attn_shape(4, 2, 64, POOL, scale=-1.0), mx.MX_ERR_INVALID),
])
def test_bad_shapes(s, status):
    assert window(one(), s) == shared(one(), s) == status
    assert sizes(one(), s) == (0, 0)
    assert mx.lib().mx_workspace_bytes_window(ctypes.byref(s), 10, 10, 10) == 0
    assert mx.lib().mx_workspace_bytes_shared(ctypes.byref(s), 10, 10, 10, 1) == 0


def test_bad_pointers():
    for call in (window, shared):
        for name in ("q", "k", "v", "out", "ws"):
            assert call(one(), shape(), **{name: None}) == mx.MX_ERR_NULL
            assert call(one(), shape(), **{name: 0x400008}) == mx.MX_ERR_INVALID
        assert call(one(), shape(), n=255) == mx.MX_ERR_TOO_LARGE
        # (these stop at a workspace too small where they are not refused before)
        n = 4 * 4 * 64 * 2
        for out in (0x100000 - n + 16, 0x100000 - 16, 0x100010, 0x100000 + n - 16):
            assert call(one(), shape(), out=out, n=255) == mx.MX_ERR_INVALID, hex(out)
            assert "overlaps" in mx.last_error()
        for out in (0x100000, 0x100000 - n, 0x100000 + n):
            assert call(one(), shape(), out=out, n=255) == mx.MX_ERR_TOO_LARGE
    for f in (mx.lib().mx_workspace_bytes_window, mx.lib().mx_workspace_bytes_shared):
        more = (0,) if f is mx.lib().mx_workspace_bytes_shared else ()
        for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, -1)):
            assert f(ctypes.byref(shape()), *bad, *more) == 0
    assert mx.lib().mx_workspace_bytes_shared(ctypes.byref(shape()), 1, 1, 1, -1) == 0


@pytest.mark.parametrize("w,sinks", [(0, 0), (-1, 0), (1, -1), (-2 ** 31, 0), (5, -2 ** 31)])
def test_bad_windows(w, sinks):
    assert window(one(), shape(), w, sinks) == mx.MX_ERR_INVALID
    assert mx.last_error()
    assert sizes(one(), shape(), w, sinks)[0] == 0


def test_window_looks_at_the_pages_it_sees():
    """Entries that no new token sees may hold anything, every other one is checked; with the
    numbers at the edges of their range."""
    s = shape()
    for ctx, n_new, w, sinks in ((100, 1, 20, 0), (100, 1, 20, 17), (95, 30, 33, 1), (64, 1, 1, 0), (79, 2, 17, 40),
                                 (100, 1, ALL, 0), (100, 1, 5, ALL), (100, 1, ALL, ALL), (47, 1, 32, 0), (48, 1, 32, 0)):
        n = -(-(ctx + n_new) // 16)
        p, j = np.arange(ctx, ctx + n_new)[:, None], np.arange(16 * n)[None]
        see = ((j <= p) & ((j > p - w) | (j < sinks))).any(0).reshape(n, 16).any(1)
        free = [3 + i if see[i] else -7 for i in range(n)]
        b = mx.Batch([0], [n_new], [ctx], [free])
        assert sizes(b, s, w, sinks)[0] > 0, (ctx, n_new, w, sinks, mx.last_error())
        assert (sizes(b, s, w, sinks)[1] > 0) == see.all()
        for i in range(n):
            bad = list(free)
            bad[i] = POOL
            got = window(mx.Batch([0], [n_new], [ctx], [bad]), s, w, sinks, n=255)
            assert got == (mx.MX_ERR_INVALID if see[i] else mx.MX_ERR_TOO_LARGE), (ctx, w, sinks, i)


PAGES = [[1, 2, 3, 10], [1, 2, 3, 11], [1, 2, 4, 12]]


@pytest.mark.parametrize("runs,ok", [
    ([], True),
    ([(0, 3, 2)], True),
    ([(0, 3, 2), (0, 2, 1)], True),       # a branch
    ([(0, 2, 2), (0, 2, 1)], True),
    ([(0, 1, 3), (2, 1, 3)], True),       # of one request each
    ([(1, 2, 1), (1, 2, 1)], True),
    ([(0, 3, 0)], False),                 # no pages
    ([(0, 0, 1)], False),                 # no requests
    ([(0, -1, 1)], False),
    ([(0, 1, -1)], False),
    ([(0, 4, 1)], False),                 # requests that are not there
    ([(-1, 2, 1)], False),
    ([(3, 1, 1)], False),
    ([(2 ** 31 - 1, 2 ** 31 - 1, 1)], False),
    ([(0, 3, 3)], False),                 # pages that differ
    ([(0, 3, 2), (0, 3, 1)], False),
    ([(0, 2, 4)], False),                 # the last page is not all cached
    ([(0, 2, 2 ** 31 - 1)], False),
    ([(0, 2, 1), (0, 3, 1)], False),      # starts that differ
    ([(0, 2, 3), (0, 1, 1)], False),
])
def test_runs(runs, ok):
    b = mx.Batch([1, 0, 1], [1, 5, 1], [50, 48, 60], PAGES)
    assert (sizes(b, shape(), runs=runs)[1] > 0) == ok
    assert shared(b, shape(), runs, n=255) == (mx.MX_ERR_TOO_LARGE if ok else mx.MX_ERR_INVALID)
    assert ok or mx.last_error()


def test_runs_as_null():
    b, s = mx.Batch([1, 0, 1], [1, 5, 1], [50, 48, 60], PAGES), shape()
    f = mx.lib().mx_paged_attn_shared
    args = (0x100000, 0x200000, 0x300000, 0x110000, 0x120000, 255, None)
    assert f(b.ptr, ctypes.byref(s), 1, None, *args) == mx.MX_ERR_NULL
    assert f(b.ptr, ctypes.byref(s), -1, None, *args) == mx.MX_ERR_INVALID
    assert f(b.ptr, ctypes.byref(s), 0, None, *args) == mx.MX_ERR_TOO_LARGE


def test_empty_calls_are_no_ops():
    empty = mx.Batch([], [], [], [])
    assert window(empty, shape()) == shared(empty, shape()) == mx.MX_OK
    assert all(n > 0 for n in sizes(empty, shape()))
    assert shared(empty, shape(), [(0, 1, 1)]) == mx.MX_ERR_INVALID


def test_rows_fit_32_bits():
    """New tokens times the q heads of a KV head are numbered in 32 bits, of a run's requests
    together."""
    s = shape(32767, 1, 64, 10000)
    b = mx.Batch([0], [65540], [0], [np.arange(4097)])
    assert sizes(b, s, 1000, 0) == (0, 0)
    assert window(b, s, out=1 << 50) == shared(b, s, out=1 << 50) == mx.MX_ERR_TOO_LARGE
    b = mx.Batch([0, 0], [33000, 33000], [0, 0], [np.arange(2063), np.arange(3000, 5063)])
    assert mx.lib().mx_workspace_bytes_shared_for(b.ptr, ctypes.byref(s), 0, None) == 0
    assert shared(b, s, out=1 << 50) == mx.MX_ERR_TOO_LARGE
    assert all(n > 0 for n in sizes(mx.Batch([0], [60], [0], [np.arange(4)]), s, 1000, 0))


@pytest.mark.parametrize("seed", range(4))
def test_workspace_bounds_cover_batches(seed):
    rng = np.random.default_rng(seed)
    for _ in range(40):
        nkv = int(rng.choice([1, 2, 8]))
        s = shape(nkv * int(rng.choice([1, 4, 20])), nkv, int(rng.choice([64, 128])), 1 << 20)
        R = int(rng.integers(1, 9))
        dec = rng.random(R) < 0.6
        depth, k = int(rng.integers(0, 4)), int(rng.choice([1, 30, 800]))
        ctx = rng.integers(1, rng.choice([20, 300, 40000]), R) + 16 * depth * k
        new = np.where(dec, 1, rng.integers(1, rng.choice([6, 400]), R))
        need = -(-(ctx + new) // 16)
        at = np.cumsum(np.concatenate([[depth * k], need - depth * k]))
        b = mx.Batch(dec.astype(int), new, ctx, [np.r_[np.arange(depth * k), np.arange(at[r], at[r + 1])] for r in range(R)])
        T, pages = int(new.sum()), int(need.sum())
        w = int(rng.choice([1, 50, 3000, ALL]))
        assert 0 < mx.mx_workspace_bytes_window_for(b, s, w, int(rng.integers(0, 50))) <= mx.mx_workspace_bytes_window(s, T, R, pages)
        runs = mx.SharedRuns([(0, R, k)] * depth)
        assert 0 < mx.mx_workspace_bytes_shared_for(b, s, runs) <= mx.mx_workspace_bytes_shared(s, T, R, pages, depth)


def test_workspace_bounds_of_large_numbers():
    """Bounds grow with what they bound, up to the largest numbers."""
    big = 2 ** 31 - 1
    for heads in ((32, 8, 128), (32767, 1, 64), (32767, 32767, 128)):
        s = shape(*heads, 1 << 40)
        last = 0
        for n in (1, 100, 10 ** 4, 10 ** 6, 10 ** 8, big):
            now = mx.mx_workspace_bytes_window(s, n, n, n * n)
            deep = mx.mx_workspace_bytes_shared(s, n, n, n * n, n)
            assert last <= now <= deep < 2 ** 42
            last = now


def test_binding_refuses_numbers_that_32_bits_do_not_hold():
    b, s = one(), shape()
    for n in (2 ** 31, 2 ** 32 + 1, -2 ** 31 - 1):
        for tokens, reqs, depth in ((n, 1, 1), (1, n, 1), (1, 1, n)):
            with pytest.raises(ValueError):
                mx.mx_workspace_bytes_shared(s, tokens, reqs, 1, depth)
            if depth == 1:
                with pytest.raises(ValueError):
                    mx.mx_workspace_bytes_window(s, tokens, reqs, 1)
    for w, sinks in ((2 ** 32 + 8, 0), (8, 2 ** 32 + 1), (2 ** 31, 0), (8, -2 ** 31 - 1)):
        with pytest.raises(ValueError):
            mx.mx_workspace_bytes_window_for(b, s, w, sinks)
    for run_ in ((2 ** 32, 1, 1), (0, 2 ** 32 + 1, 1), (0, 1, 2 ** 32 + 1)):
        with pytest.raises(ValueError):
            mx.SharedRuns([run_])


class OnGpu:
    """Stands for a tensor on a device."""

    def __init__(self, dtype=torch.bfloat16, n=1 << 40, device=0, contiguous=True):
        self.dtype, self.n, self.device, self.contiguous = dtype, n, device, contiguous

    def data_ptr(self):
        raise AssertionError("the call went past its checks")

    def numel(self):
        return self.n

    def get_device(self):
        return self.device

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return self.contiguous


def test_binding_refuses_tensors(monkeypatch):
    """Of another type, size, layout or device, each for each tensor.  No launch."""
    monkeypatch.setattr(mx, "_current_device", lambda: 0)
    b, s = one(), shape()
    rows, pool = 4 * 4 * 64, POOL * 2 * 16 * 64
    for name, n in (("q", rows), ("k_pool", pool), ("v_pool", pool), ("out", rows), ("ws", 0)):
        wrong = [OnGpu(t) for t in (torch.float16, torch.int16, torch.float32)]
        wrong += [OnGpu(torch.uint8, contiguous=False)] if name == "ws" else [
            OnGpu(torch.uint8), OnGpu(n=n - 1), OnGpu(contiguous=False)]
        wrong += [OnGpu(torch.uint8 if name == "ws" else torch.bfloat16, device=1)]
        wrong += [OnGpu(torch.uint8 if name == "ws" else torch.bfloat16, device=-1)]
        for t in wrong:
            args = {x: OnGpu(torch.uint8 if x == "ws" else torch.bfloat16) for x in ("q", "k_pool", "v_pool", "out", "ws")}
            args[name] = t
            with pytest.raises(ValueError, match=f"^{name} "):
                mx.mx_paged_attn_window(b, s, 8, 2, stream=0, **args)
            with pytest.raises(ValueError, match=f"^{name} "):
                mx.mx_paged_attn_shared(b, s, mx.SharedRuns([]), stream=0, **args)
    monkeypatch.setattr(mx, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="not the current one"):
        mx.mx_paged_attn_window(b, s, 8, 2, OnGpu(), OnGpu(), OnGpu(), OnGpu(), OnGpu(torch.uint8))
    bf = lambda *n: torch.zeros(n, dtype=torch.bfloat16)  # noqa: E731
    with pytest.raises(ValueError, match="GPU"):
        mx.mx_paged_attn_window(b, s, 8, 2, bf(4, 4, 64), bf(POOL, 2, 2, 16, 32), bf(POOL, 2, 64, 16),
                                bf(4, 4, 64), torch.zeros(1 << 16, dtype=torch.uint8))


def test_launches(fake_hip):  # noqa: F811
    """The kernels of each call, small ones (whose metadata goes with the kernels' arguments) and
    others, and staging buffers that outlive their readers."""
    r = run(fake_hip, """
        import ctypes
        s = mx.attn_shape(8, 2, 128, 1 << 20)
        L, S = mx.lib(), ctypes.byref(s)
        window = lambda b, w: lambda st: L.mx_paged_attn_window(b.ptr, S, w, 4, A(0), A(1), A(2), A(3), A(5), BIG, st)
        def shared(b, runs):
            r = mx.SharedRuns(runs)
            return lambda st: L.mx_paged_attn_shared(b.ptr, S, r.n, r.ptr, A(0), A(1), A(2), A(3), A(5), BIG, st)
        def group(n, pages, own=40):
            return mx.Batch([1] * n, [1] * n, [16 * pages + own] * n,
                            [np.r_[np.arange(pages), pages + 3 * i + np.arange(3)] for i in range(n)])
        long = mx.Batch([1], [1], [5000], [np.arange(400)])
        late = mx.Batch([0], [9], [5000], [np.arange(400)])
        prompt = mx.Batch([0], [3000], [0], [np.arange(400)])
        calls = dict(window=window(batch(3), 64), window_mixed=window(batch(3, 20), 64),
                     window_many=window(batch(300), 64), window_prompt=window(prompt, 500),
                     window_long=window(long, 1 << 20), window_late=window(late, 4000),
                     shared_few=shared(group(4, 20), [(0, 4, 20)]),
                     shared=shared(group(40, 400), [(0, 40, 400)]),
                     shared_none=shared(long, []))
        kernels, st = {}, []
        for name, f in calls.items():
            n = len(log())
            st.append(f(None))
            kernels[name] = [l[0] for l in log()[n:]]
        for i in range(40):
            st += [f([None, None, A(30), None, A(31)][i % 5]) for f in calls.values()]
        print(json.dumps(dict(kernels=kernels, st=st, bad=fake.fake_violations())))
        """)
    assert set(r["st"]) == {0} and r["bad"] == 0
    names = ("upload", "small_span_kernel", "small_span_merge", "span_attn", "span_merge")
    got = {k: [next(n for n in names if n in x) for x in v] for k, v in r["kernels"].items()}
    assert got == {
        "window": ["small_span_kernel"], "window_mixed": ["small_span_kernel"],
        "window_many": ["span_attn"], "window_prompt": ["upload", "span_attn"],
        "window_long": ["small_span_kernel", "small_span_merge"],
        "window_late": ["small_span_kernel", "small_span_merge"],
        "shared_few": ["small_span_kernel"], "shared": ["upload", "span_attn", "span_merge"],
        "shared_none": ["small_span_kernel", "small_span_merge"]}
