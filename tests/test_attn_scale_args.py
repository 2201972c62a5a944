"""sm_scale beyond what the scores' factor can be is refused, before anything is enqueued (no GPU)."""
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


@pytest.mark.parametrize("scale", [3.0e38, 3.4028234e38, float("inf"), -1e-45, float("nan")])
def test_scales_that_are_refused(b, scale):
    L, t = b.lib(), b.Tensor(4096, 0, 128, 1024)
    p = b.PackedStruct(1, 8, 2, 128, 4096, 10, 10)
    assert L.ihip_prompt_attn(ctypes.byref(p), t, t, t, None, 10, scale, 4096, None, None, 0, None) == -1
    assert b"sm_scale" in L.ihip_last_error()
    row, shape = b.Tensor(4096, 1 << 20, 1 << 16, 64), b.Shape(1, 8, 2, 128, 1, 1, 4096, 1000, 4, 64, 0)
    store = b.StoreStruct(2, row, row, 4096, 4096, 1.0, 1.0, None)
    assert L.ihip_sparse_attn_decode_mx4kv(ctypes.byref(shape), t, ctypes.byref(store), None, 0, 1, scale, 4096, None, 4096, 1 << 30, None) == -1
    assert b"sm_scale" in L.ihip_last_error()
