"""CPU checks of what the header says of calls beside each other."""
import ctypes

import numpy as np

import paper_2606_16264_amd as mx


def append(b, s, ws_bytes):
    return mx.lib().mx_kv_append(b.ptr, ctypes.byref(s), 0x100000, 0x110000, 0x200000, 0x300000, 0x120000,
                                 ws_bytes, None)


def test_tables_with_freed_pages():
    """Only the window's call takes a table whose entries out of sight are no pages; the append of
    the same tokens takes it with any ids in their place.  (Calls that pass every other check
    stop at a workspace of 0 bytes.)"""
    s = mx.attn_shape(4, 2, 64, 64)
    for decode, n_new, ctx in ((1, 1, 100), (0, 30, 200)):
        n = -(-(ctx + n_new) // 16)
        first = max(0, ctx - 20 + 1) // 16
        freed = [-1] * first + list(range(first, n))
        b = mx.Batch([decode], [n_new], [ctx], [freed])
        assert mx.mx_workspace_bytes_window_for(b, s, 20) > 0
        assert mx.mx_batch_validate(b, s) == mx.MX_ERR_INVALID
        assert append(b, s, 0) == mx.MX_ERR_INVALID
        assert mx.lib().mx_workspace_bytes_for(b.ptr, ctypes.byref(s), None) == 0
        for other in (np.zeros(first, int), np.full(first, 63), np.full(first, n - 1)):
            whole = mx.Batch([decode], [n_new], [ctx], [np.r_[other, np.arange(first, n)]])
            assert mx.mx_batch_validate(whole, s) == mx.MX_OK
            assert append(whole, s, 0) == mx.MX_ERR_TOO_LARGE
