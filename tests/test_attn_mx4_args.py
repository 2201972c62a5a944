"""What the 4-bit decode attention refuses, before anything is enqueued (no GPU)."""
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


def test_decode_attention_over_4_bit_rows_refuses(b):
    t, L = b.Tensor, b.lib()
    row = t(4096, 1 << 20, 1 << 16, 64)

    def store(**kw):
        s = b.StoreStruct(2, row, row, 4096, 4096, 1.0, 1.0, None)
        for name, value in kw.items():
            setattr(s, name, value)
        return s

    def call(shape=b.Shape(2, 8, 2, 128, 1, 1, 4096, 1000, 4, 64, 0), q=t(4096, 1024, 128, 128), s=store(), starts=4096, n=4, block=16, out=4096,
             ws=4096, size=1 << 30, scale=0.1):
        return L.ihip_sparse_attn_decode_mx4kv(ctypes.byref(shape), q, ctypes.byref(s) if s else None, starts, n, block, scale, out, None, ws, size, None)

    Shape = b.Shape
    assert call(shape=Shape(2, 8, 2, 64, 1, 1, 4096, 1000, 4, 64, 0)) == -4
    assert call(shape=Shape(2, 6, 2, 128, 1, 1, 4096, 1000, 4, 64, 0)) == -4
    assert call(shape=Shape(2, 8, 2, 128, 16, 16, 4096, 1000, 4, 64, 0)) == -1
    assert call(q=t(None, 0, 0, 128)) == -1 and call(q=t(4100, 1024, 128, 128)) == -1
    assert call(s=None) == -1
    bf16 = b.StoreStruct(0, t(4096, 0, 0, 128), t(4096, 0, 0, 128), None, None, 1.0, 1.0, None)
    assert call(s=bf16) == -1 and b"4-bit" in L.ihip_last_error()
    assert call(s=store(k_scales=None)) == -1 and call(s=store(v=t(4096, 1 << 20, 1 << 16, 128))) == -1
    back = t(4096, 1 << 20, -64, 64)
    assert call(s=store(k=back, v=back)) == -4 and b"strides" in L.ihip_last_error()
    pg = b.PagedStruct(4096, 10, 64)                                     # 640 of 1,000 tokens
    assert call(s=store(paged=ctypes.cast(ctypes.pointer(pg), ctypes.c_void_p))) == -1
    for scale in (-0.1, float("nan"), float("inf")):
        assert call(scale=scale) == -1 and b"sm_scale" in L.ihip_last_error()
    assert call(n=-1) == -1 and call(block=12) == -1 and call(starts=None) == -1 and call(out=None) == -1
    assert call(n=1 << 20, block=4096) == -4 and b"slots" in L.ihip_last_error()
    assert call(ws=None) == -2 and call(ws=4100) == -2 and call(size=100) == -2 and b"workspace" in L.ihip_last_error()
    one = ctypes.c_int32 * 1
    need = L.ihip_workspace_bytes(b.OP_ATTN_DECODE_MX4, ctypes.byref(Shape(2, 8, 2, 128, 1, 1, 4096, 1000, 4, 64, 0)), 1, one(16), one(4))
    assert call(size=need - 1) == -2
    assert call(shape=Shape(0, 8, 2, 128, 1, 1, None, 1000, 4, 64, 0), s=None) == 0


def test_scratch_serves_fewer_blocks(b):
    """With more blocks, or longer ones, no less scratch: what was asked for with one block serves a call without any."""
    L, one = b.lib(), ctypes.c_int32 * 1
    for B in (1, 3, 8, 27, 96):
        for Hkv in (1, 4, 8):
            for length in (100, 1000, 1921, 4099, 16384, 250007):
                shape = b.Shape(B, 4 * Hkv, Hkv, 128, 1, 1, 4096, length, 0, length, 0)
                need = [L.ihip_workspace_bytes(b.OP_ATTN_DECODE_MX4, ctypes.byref(shape), 1, one(block), one(n))
                        for block, n in ((1, 1), (16, 1), (16, 2), (64, 5), (64, 40), (64, 400))]
                assert need == sorted(need) and need[0] > 0, (B, Hkv, length, need)
