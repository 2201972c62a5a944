"""Outputs whose heads lie over each other are refused, before anything is enqueued (no GPU)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def b():
    import os
    import paper_2502_08910_amd as pkg
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2502_08910_amd.build import build
        build(verbose=False)
    from paper_2502_08910_amd import binding
    return binding


@pytest.mark.parametrize("stride_h", [0, 64, 120, -64])
def test_overlapping_heads(b, stride_h):
    L, t, no = b.lib(), b.Tensor, b.NO_TENSOR
    row = t(4096, 64 * 128, 64 * 128, 128)
    store = b.StoreStruct(0, row, row, None, None, 1.0, 1.0, None)
    x, over = t(4096, 0, 128, 1024), t(4096, 1 << 20, stride_h, 1024)

    def append(q_out=no, k_out=no):
        p = b.PackedStruct(2, 8, 2, 128, 4096, 10, 10)
        return L.ihip_kv_append(ctypes.byref(p), x, x, x, 4096, 64, None, ctypes.byref(store), q_out, k_out, None)

    def gather(k, v):
        return L.ihip_kv_gather(ctypes.byref(store), 2, 2, 128, 4096, 64, k, v, None)

    assert append(q_out=over) == -1 and b"q_out overlap" in L.ihip_last_error()
    assert append(k_out=over) == -1 and b"k_out overlap" in L.ihip_last_error()
    assert gather(over, no) == -1 and b"k_out overlap" in L.ihip_last_error()
    assert gather(no, over) == -1 and b"v_out overlap" in L.ihip_last_error()


@pytest.mark.parametrize("fmt,stride_h", [(0, 0), (0, 64), (1, 64), (1, -112), (2, 0)])
def test_overlapping_heads_of_a_store(b, fmt, stride_h):
    """Refused where they are written; reading a cache whose heads are the same rows is another matter."""
    width = {0: 128, 1: 128, 2: 64}[fmt]
    row, x = b.Tensor(4096, 1 << 20, stride_h, width), b.Tensor(4096, 0, 128, 1024)
    scales = 4096 if fmt == 2 else None
    store = b.StoreStruct(fmt, row, row, scales, scales, 1.0, 1.0, None)
    p = b.PackedStruct(2, 8, 2, 128, 4096, 10, 10)
    assert b.lib().ihip_kv_append(ctypes.byref(p), x, x, x, 4096, 64, None, ctypes.byref(store), b.NO_TENSOR, b.NO_TENSOR, None) == -1
    assert b"store overlap" in b.lib().ihip_last_error()
