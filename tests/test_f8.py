"""CPU checks of the 8-bit cache's calls: every malformed argument is refused on the
host with the documented status, before any device work; workspace sizes and their
bounds; what the calls launch."""
import ctypes

import numpy as np
import pytest
import torch

import conftest
import paper_2606_16264_amd as mx
from test_host_runtime import fake_hip, run  # noqa: F401  (fake_hip is a fixture)

POOL = 64


def shape(nq=4, nkv=2, d=64, pool=POOL):
    return mx.attn_shape(nq, nkv, d, pool)


def cache(s, weight=True):
    P, g, d = s.pool_pages, s.n_kv_heads, s.head_dim
    z = lambda *n, t=torch.uint8: torch.zeros(n, dtype=t)  # noqa: E731
    return mx.CacheF8(z(P, g, d // 64, 16, 64), z(P, g, d, 16), z(P, g, t=torch.float32),
                      z(P, g, t=torch.float32), z(P, g, 16, t=torch.float32) if weight else None)


class Raw:
    """A made-up device tensor."""

    def __init__(self, ptr=0x100000, n=1 << 40):
        self.p, self.n = ptr, n

    def data_ptr(self):
        return self.p

    def numel(self):
        return self.n


def raw_cache(**changed):
    c = {n: 0x200000 for n in ("k_pool", "v_pool", "k_scale", "v_scale", "weight")}
    c.update(changed)
    return mx._CacheF8(*(c[n] for n in ("k_pool", "v_pool", "k_scale", "v_scale", "weight")))


def one(phase=mx.MX_PREFILL, n_new=4, ctx=0, pages=(1,)):
    return mx.Batch([phase], [n_new], [ctx], [pages])


def append(b, s, c, k=0x100000, v=0x100000):
    return mx.lib().mx_kv_append_f8(b.ptr, ctypes.byref(s), k, v, ctypes.byref(c) if c else None, None)


def attn(b, s, c, q=0x100000, out=0x110000, ws=0x120000, n=1 << 40):
    return mx.lib().mx_paged_attn_f8(b.ptr, ctypes.byref(s), q, ctypes.byref(c) if c else None, out,
                                     ws, n, None)


def evict(e, s, c, kept=0x100000, ws=0x120000, n=1 << 40):
    return mx.lib().mx_kv_evict_f8(e.R, e.ptr, ctypes.byref(s), ctypes.byref(c) if c else None, kept,
                                   ws, n, None)


BAD_BATCHES = [
    (mx.Batch([7], [1], [5], [[0]]), mx.MX_ERR_INVALID),
    (one(n_new=0), mx.MX_ERR_INVALID),
    (one(mx.MX_DECODE, 1, 0), mx.MX_ERR_INVALID),
    (one(n_new=2, ctx=15), mx.MX_ERR_NO_SPACE),
    (one(pages=[POOL]), mx.MX_ERR_INVALID),
    (one(pages=[-1]), mx.MX_ERR_INVALID),
    (mx.Batch([0, 1], [3, 1], [0, 2], [[5], [5]]), mx.MX_ERR_INVALID),
]


@pytest.mark.parametrize("b,status", BAD_BATCHES)
def test_bad_batches(b, status):
    for call in (append, attn):
        assert call(b, shape(), raw_cache()) == status
        assert mx.last_error()


@pytest.mark.parametrize("s,status", [
    (shape(4, 3), mx.MX_ERR_INVALID),
    (shape(d=96), mx.MX_ERR_UNSUPPORTED),
    (shape(pool=0), mx.MX_ERR_INVALID),
])
def test_bad_shapes(s, status):
    e = mx.EvictBatch([4], [2], [1], [[1]], [[2]])
    assert append(one(), s, raw_cache()) == status
    assert attn(one(), s, raw_cache()) == status
    assert evict(e, s, raw_cache()) == status
    assert mx.lib().mx_workspace_bytes_f8(ctypes.byref(s), 1, 10, 10, 10) == 0
    assert mx.lib().mx_kv_evict_f8_ws_bytes(e.R, e.ptr, ctypes.byref(s)) == 0


def test_bad_caches_and_pointers():
    e = mx.EvictBatch([4], [2], [1], [[1]], [[2]])
    for call in (lambda c: append(one(), shape(), c), lambda c: attn(one(), shape(), c),
                 lambda c: evict(e, shape(), c)):
        assert call(None) == mx.MX_ERR_NULL
        for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
            assert call(raw_cache(**{name: None})) == mx.MX_ERR_NULL
            assert call(raw_cache(**{name: 0x200008})) == mx.MX_ERR_INVALID
        assert call(raw_cache(weight=0x200004)) == mx.MX_ERR_INVALID
    c = raw_cache()
    assert append(one(), shape(), c, k=None) == mx.MX_ERR_NULL
    assert append(one(), shape(), c, v=0x100002) == mx.MX_ERR_INVALID
    for kw, status in ((dict(q=None), mx.MX_ERR_NULL), (dict(out=None), mx.MX_ERR_NULL),
                       (dict(ws=None), mx.MX_ERR_NULL), (dict(q=0x100008), mx.MX_ERR_INVALID),
                       (dict(ws=0x120004), mx.MX_ERR_INVALID), (dict(n=255), mx.MX_ERR_TOO_LARGE)):
        assert attn(one(), shape(), c, **kw) == status, kw
    for kw, status in ((dict(kept=None), mx.MX_ERR_NULL), (dict(ws=None), mx.MX_ERR_NULL),
                       (dict(kept=0x100004), mx.MX_ERR_INVALID), (dict(n=255), mx.MX_ERR_TOO_LARGE)):
        assert evict(e, shape(), c, **kw) == status, kw
    assert evict(e, shape(), raw_cache(weight=None)) == mx.MX_ERR_NULL


def test_append_refuses_a_page_of_two_requests():
    # distinct slots of one page: fine for a byte copy, not for a page with one scale
    b = mx.Batch([1, 1], [1, 1], [3, 4], [[5], [5]])
    assert mx.mx_batch_validate(b, shape()) == mx.MX_OK
    assert append(b, shape(), raw_cache()) == mx.MX_ERR_INVALID
    assert "page 5" in mx.last_error()
    # a shared prefix page that only one of them writes is fine as far as the host sees
    b = mx.Batch([1, 1], [1, 1], [16, 3], [[5, 6], [7]])
    assert append(b, shape(), raw_cache()) in (mx.MX_OK, mx.MX_ERR_HIP)


def test_append_takes_pages_of_one_request_each(fake_hip):  # noqa: F811
    """What the test above checks, on the stand-in runtime, where no kernel runs on the pointers."""
    r = run(fake_hip, """
        import ctypes
        s = mx.attn_shape(4, 2, 64, 64)
        c = mx._CacheF8(1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20)
        append = lambda b: mx.lib().mx_kv_append_f8(b.ptr, ctypes.byref(s), A(0), A(1), ctypes.byref(c), None)
        st = [append(mx.Batch([1, 1], [1, 1], [3, 4], [[5], [5]]))]
        refused = len(log())
        st.append(append(mx.Batch([1, 1], [1, 1], [16, 3], [[5, 6], [7]])))
        print(json.dumps(dict(st=st, refused=refused, launches=[l[0] for l in log()])))
        """)
    assert r["st"] == [mx.MX_ERR_INVALID, mx.MX_OK] and r["refused"] == 0
    assert len(r["launches"]) == 1 and "small_append_f8" in r["launches"][0]


def test_invented_pointers_are_kept_from_a_gpu():
    node = "tests/test_f8.py::test_append_refuses_a_page_of_two_requests"
    assert conftest.kept_from_a_gpu(node, True) and not conftest.kept_from_a_gpu(node, False)
    assert not conftest.kept_from_a_gpu("tests/test_f8.py::test_bad_batches[0]", True)
    assert test_append_refuses_a_page_of_two_requests.__name__ == node.split("::")[1]


@pytest.mark.parametrize("args,status", [
    (([4], [5], [0], [[1]], [[2]]), mx.MX_ERR_INVALID),          # keep > len
    (([4], [-1], [0], [[1]], [[2]]), mx.MX_ERR_INVALID),
    (([-1], [0], [0], [[1]], [[2]]), mx.MX_ERR_INVALID),
    (([4], [2], [3], [[1]], [[2]]), mx.MX_ERR_INVALID),          # recent > keep
    (([4], [2], [-1], [[1]], [[2]]), mx.MX_ERR_INVALID),
    (([17], [2], [1], [[1]], [[2]]), mx.MX_ERR_NO_SPACE),
    (([40], [17], [1], [[1, 3, 4]], [[2]]), mx.MX_ERR_NO_SPACE),
    (([4], [2], [1], [[]], [[2]]), mx.MX_ERR_NO_SPACE),
    (([4], [2], [1], [[POOL]], [[2]]), mx.MX_ERR_INVALID),
    (([4], [2], [1], [[1]], [[-2]]), mx.MX_ERR_INVALID),
    (([4], [2], [1], [[1]], [[1]]), mx.MX_ERR_INVALID),          # its own source
    (([4, 4], [2, 2], [1, 1], [[1], [2]], [[3], [3]]), mx.MX_ERR_INVALID),
    (([4, 4], [2, 2], [1, 1], [[1], [2]], [[3], [1]]), mx.MX_ERR_INVALID),  # another's source
    (([40], [20], [1], [[1, 3, 4]], [[2, 2]]), mx.MX_ERR_INVALID),
])
def test_bad_evictions(args, status):
    e = mx.EvictBatch(*args)
    assert evict(e, shape(), raw_cache()) == status
    assert mx.last_error()
    assert mx.lib().mx_kv_evict_f8_ws_bytes(e.R, e.ptr, ctypes.byref(shape())) == 0


def test_empty_calls_are_no_ops():
    s, c = shape(), raw_cache()
    empty = mx.Batch([], [], [], [])
    assert append(empty, s, c) == attn(empty, s, c) == mx.MX_OK
    assert evict(mx.EvictBatch([], [], [], [], []), s, c) == mx.MX_OK
    assert evict(mx.EvictBatch([20, 0], [0, 0], [0, 0], [[1, 2], []], [[], []]), s, c) == mx.MX_OK
    # a shared prefix is a source of two requests, only destinations are their own
    e = mx.EvictBatch([4, 4], [2, 2], [1, 1], [[1], [1]], [[3], [4]])
    assert mx.mx_kv_evict_f8_ws_bytes(e, s) > 0
    assert mx.mx_workspace_bytes_f8_for(empty, s) > 0


@pytest.mark.parametrize("weight", [0x200000, None])
def test_attention_refuses_an_output_over_the_query(weight):
    """A chunk's weights read the query again behind its output.  (The calls that are not refused
    here stop at a workspace too small.)"""
    c, n = raw_cache(weight=weight), 4 * 4 * 64 * 2
    for out in (0x100000 - n + 16, 0x100000 - 16, 0x100010, 0x100000 + n - 16):
        assert attn(one(), shape(), c, out=out, n=255) == mx.MX_ERR_INVALID, hex(out)
        assert "overlaps" in mx.last_error()
    assert attn(one(), shape(), c, out=0x100000, n=255) == (mx.MX_ERR_INVALID if weight else mx.MX_ERR_TOO_LARGE)
    for out in (0x100000 - n, 0x100000 + n):
        assert attn(one(), shape(), c, out=out, n=255) == mx.MX_ERR_TOO_LARGE


def test_rows_of_a_chunk_fit_32_bits():
    """New tokens times the q heads of a KV head are numbered in 32 bits."""
    s = shape(32767, 1, 64, 5000)
    for n_new, ok in ((65000, True), (65540, False)):
        b = mx.Batch([mx.MX_PREFILL], [n_new], [0], [np.arange(-(-n_new // 16))])
        need = mx.lib().mx_workspace_bytes_f8_for(b.ptr, ctypes.byref(s), 0)
        assert (need > 0) == ok
        if not ok:
            assert attn(b, s, raw_cache()) == mx.MX_ERR_TOO_LARGE


def test_binding_checks_the_cache():
    s = shape()
    c = cache(s)
    with pytest.raises(ValueError):  # heads of another shape
        mx.mx_kv_append_f8(one(), shape(4, 4), Raw(), Raw(), c, stream=0)
    with pytest.raises(ValueError):  # pages the tensors do not have
        mx.mx_paged_attn_f8(one(), shape(pool=POOL + 1), Raw(), c, Raw(), Raw(), stream=0)
    with pytest.raises(ValueError):
        mx.CacheF8(c.k_pool, c.v_pool, c.k_scale, c.v_scale.double())
    with pytest.raises(ValueError):
        mx.CacheF8(c.k_pool.transpose(3, 4), c.v_pool, c.k_scale, c.v_scale)
    with pytest.raises(ValueError):
        mx.CacheF8(c.k_pool, c.v_pool[1:], c.k_scale, c.v_scale)
    with pytest.raises(ValueError):
        mx.CacheF8(c.k_pool, c.v_pool, c.k_scale, c.v_scale, c.weight[:, :1].contiguous())


def test_binding_checks_sizes():
    s = shape()
    c, small, b = cache(s), Raw(n=4 * 2 * 64 - 1), one()
    with pytest.raises(ValueError, match="v_new"):
        mx.mx_kv_append_f8(b, s, Raw(), small, c, stream=0)
    with pytest.raises(ValueError, match="out"):
        mx.mx_paged_attn_f8(b, s, Raw(), c, Raw(n=4 * 4 * 64 - 1), Raw(), stream=0)
    with pytest.raises(ValueError, match="kept"):
        mx.mx_kv_evict_f8(mx.EvictBatch([4], [2], [1], [[1]], [[2]]), s, c, Raw(n=3), Raw(), stream=0)


def test_binding_refuses_a_cache_in_host_memory():
    """With valid arguments otherwise: the calls would hand host addresses to a kernel."""
    s = shape()
    c, e = cache(s), mx.EvictBatch([4], [2], [1], [[1]], [[2]])
    bf = lambda *n: torch.zeros(n, dtype=torch.bfloat16)  # noqa: E731
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for call in (lambda: mx.mx_kv_append_f8(one(), s, bf(4, 2, 64), bf(4, 2, 64), c, stream=0),
                 lambda: mx.mx_paged_attn_f8(one(), s, bf(4, 4, 64), c, bf(4, 4, 64), ws, stream=0),
                 lambda: mx.mx_kv_evict_f8(e, s, c, torch.zeros(4, dtype=torch.int32), ws, stream=0)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_binding_refuses_a_cache_of_other_types():
    """Types of the right size too, whose bytes would be read as something else."""
    c = cache(shape())
    names = ("k_pool", "v_pool", "k_scale", "v_scale", "weight")
    tensors = dict(zip(names, (c.k_pool, c.v_pool, c.k_scale, c.v_scale, c.weight)))
    mx.CacheF8(**dict(tensors, k_pool=c.k_pool.view(torch.float8_e4m3fn)))
    for name in names:
        wrong = ((torch.int8, torch.bool, torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz)
                 if "pool" in name else (torch.int32, torch.uint8, torch.float64))
        for t in wrong:
            with pytest.raises(ValueError, match=name):
                mx.CacheF8(**dict(tensors, **{name: torch.zeros(tensors[name].shape, dtype=t)}))


def test_binding_keeps_the_tensors_of_a_cache():
    """The calls use the addresses taken when the cache was made: a tensor put in the place of one
    would not be used, and the one it replaces might be freed."""
    c = cache(shape())
    for name in ("k_pool", "v_pool", "k_scale", "v_scale", "weight"):
        t = getattr(c, name)
        with pytest.raises(AttributeError):
            setattr(c, name, torch.zeros_like(t))
        assert getattr(c, name) is t
        assert t.data_ptr() == getattr(c._cache, name)
    assert cache(shape(), weight=False).weight is None


class OnGpu:
    """Stands for a tensor on device 0."""

    def __init__(self, dtype, n=1 << 40):
        self.dtype, self.n = dtype, n

    def data_ptr(self):
        raise AssertionError("the call went past its checks")

    def numel(self):
        return self.n

    def get_device(self):
        return 0

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True


def test_binding_refuses_tensors_of_other_types():
    """Types of the right size too.  No launch: each call has one wrong tensor."""
    s, e = shape(), mx.EvictBatch([4], [2], [1], [[1]], [[2]])
    c = cache(s)
    c._device, c._current_device = 0, lambda: 0
    calls = {
        "k_new": lambda t: mx.mx_kv_append_f8(one(), s, t, OnGpu(torch.bfloat16), c, stream=0),
        "v_new": lambda t: mx.mx_kv_append_f8(one(), s, OnGpu(torch.uint16), t, c, stream=0),
        "q": lambda t: mx.mx_paged_attn_f8(one(), s, t, c, OnGpu(torch.bfloat16), OnGpu(torch.uint8), stream=0),
        "out": lambda t: mx.mx_paged_attn_f8(one(), s, OnGpu(torch.bfloat16), c, t, OnGpu(torch.uint8), stream=0),
        "kept": lambda t: mx.mx_kv_evict_f8(e, s, c, t, OnGpu(torch.uint8), stream=0)}
    for name, call in calls.items():
        wrong = ((torch.float32, torch.uint32, torch.int64) if name == "kept"
                 else (torch.float16, torch.int16, torch.float32, torch.uint8))
        for t in wrong:
            with pytest.raises(ValueError, match=f"^{name} must"):
                call(OnGpu(t))


@pytest.mark.parametrize("track", [False, True])
def test_workspace_bound_covers_batches(track):
    rng = np.random.default_rng(5)
    for _ in range(60):
        nkv = int(rng.choice([1, 2, 8]))
        s = shape(nkv * int(rng.choice([1, 4, 20])), nkv, int(rng.choice([64, 128])), 1 << 20)
        R = int(rng.integers(1, 9))
        dec = rng.random(R) < 0.6
        ctx = rng.integers(1, rng.choice([20, 300, 40000]), R)
        new = np.where(dec, 1, rng.integers(1, 400, R))
        need = -(-(ctx + new) // 16)
        at = np.cumsum(np.concatenate([[0], need]))
        b = mx.Batch(dec.astype(int), new, ctx, [np.arange(at[r], at[r + 1]) for r in range(R)])
        exact = mx.mx_workspace_bytes_f8_for(b, s, track)
        assert exact <= mx.mx_workspace_bytes_f8(s, track, int(new.sum()), R, int(need.sum()))


def test_launches(fake_hip):  # noqa: F811
    """The kernels of each call, small ones (whose metadata goes with the kernel's arguments) and
    others, and staging buffers that outlive their readers."""
    r = run(fake_hip, """
        import ctypes
        s = mx.attn_shape(8, 2, 128, 1 << 20)
        c = lambda w: ctypes.byref(mx._CacheF8(1 << 20, 2 << 20, 3 << 20, 4 << 20, w))
        L, S = mx.lib(), ctypes.byref(s)
        append = lambda b: lambda st: L.mx_kv_append_f8(b.ptr, S, A(0), A(1), c(None), st)
        attn = lambda b, w: lambda st: L.mx_paged_attn_f8(b.ptr, S, A(0), c(w), A(1), A(2), BIG, st)
        def evict(n, keep):
            e = mx.EvictBatch([n, 3], [keep, 0], [4, 0], [np.arange(-(-n // 16)), [1 << 15]],
                              [np.arange(1 << 16, (1 << 16) + -(-keep // 16)), []])
            return lambda st: L.mx_kv_evict_f8(2, e.ptr, S, c(5 << 20), A(0), A(2), BIG, st)
        long = mx.Batch([1], [1], [5000], [np.arange(400)])  # split over keys
        late = mx.Batch([0], [9], [5000], [np.arange(400)])
        calls = dict(append=append(batch(3, 20)), append_many=append(batch(300, 20)),
                     attn=attn(batch(3, 20), None), attn_many=attn(batch(60, 20), None),
                     attn_split=attn(long, None), track=attn(batch(3, 20), 5 << 20),
                     track_decodes=attn(long, 5 << 20), attn_late=attn(late, None),
                     track_late=attn(late, 5 << 20),
                     evict=evict(40, 20), evict_long=evict(16000, 5000))
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
    names = ("upload", "small_append_f8", "kv_append_f8", "small_attn_f8", "paged_attn_f8", "finish",
             "decode_attn_f8", "weight_prefill", "weight_parts", "small_evict_select",
             "small_evict_move", "evict_select", "evict_move")
    got = {k: [next(n for n in names if n in x) for x in v] for k, v in r["kernels"].items()}
    assert got == {
        "append": ["small_append_f8"], "append_many": ["kv_append_f8"],
        "attn": ["small_attn_f8"], "attn_many": ["upload", "paged_attn_f8"],
        "attn_split": ["upload", "decode_attn_f8", "finish"],
        "track": ["upload", "paged_attn_f8", "finish", "weight_prefill", "weight_parts"],
        "track_decodes": ["upload", "decode_attn_f8", "finish"],
        "attn_late": ["upload", "paged_attn_f8", "finish"],
        "track_late": ["upload", "paged_attn_f8", "finish", "weight_prefill", "weight_parts"],
        "evict": ["small_evict_select", "small_evict_move"],
        "evict_long": ["upload", "evict_select", "evict_move"]}
