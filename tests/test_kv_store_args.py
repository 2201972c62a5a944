"""What cache filling and reading back refuse, before anything is enqueued (no GPU)."""
import ctypes

import pytest

BAD, UNSUPPORTED = -1, -4


@pytest.fixture(scope="module")
def b():
    import os
    import paper_2502_08910_amd as pkg
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2502_08910_amd.build import build
        build(verbose=False)
    from paper_2502_08910_amd import binding
    return binding


def store_of(b, fmt, **kw):
    row = {0: 128, 1: 128, 2: 64}[fmt]
    t = b.Tensor(4096, 1024 * row, 64 * row, row)
    s = b.StoreStruct(fmt, t, t, 4096 if fmt == 2 else None, 4096 if fmt == 2 else None, 1.0, 1.0, None)
    for name, value in kw.items():
        setattr(s, name, value)
    return s


def append(b, packed=None, q=None, k=None, v=None, lens=4096, max_len=64, rope=None, store=None, q_out=None, k_out=None):
    t = b.Tensor(4096, 0, 128, 1024)
    p = b.PackedStruct(2, 8, 2, 128, 4096, 10, 10) if packed is None else packed
    s = store_of(b, 0) if store is None else store
    return b.lib().ihip_kv_append(ctypes.byref(p), q or t, k or t, v or t, lens, max_len, rope, ctypes.byref(s) if s else None,
                                  q_out or b.NO_TENSOR, k_out or b.NO_TENSOR, None)


def test_append_refuses(b):
    t, P = b.Tensor, b.PackedStruct
    L = b.lib()
    assert L.ihip_kv_append(None, t(), t(), t(), 1, 1, None, None, t(), t(), None) == BAD and b"packed" in L.ihip_last_error()
    assert append(b, packed=P(2, 8, 3, 128, 4096, 10, 10)) == BAD
    assert append(b, packed=P(2, 8, 2, 64, 4096, 10, 10)) == UNSUPPORTED and b"128" in L.ihip_last_error()
    assert append(b, packed=P(-1, 8, 2, 128, 4096, 10, 10)) == BAD
    assert append(b, packed=P(2, 8, 2, 128, 4096, -1, 10)) == BAD
    assert append(b, packed=P(2, 8, 2, 128, None, 10, 10)) == BAD and b"cu_q" in L.ihip_last_error()
    assert append(b, k=t(None, 0, 128, 1024)) == BAD and b"k.ptr" in L.ihip_last_error()
    assert append(b, v=t(4096 + 8, 0, 128, 1024)) == BAD and b"aligned" in L.ihip_last_error()
    assert append(b, q=t(4096, 0, 100, 1024), q_out=t(4096, 0, 128, 1024)) == BAD
    assert append(b, q_out=t(4096, 0, 128, 0)) == BAD                     # an output's rows must be rows of their own
    assert append(b, k_out=t(4096, 0, 128, 64)) == BAD
    assert append(b, lens=None) == BAD and append(b, max_len=0) == BAD
    assert append(b, rope=ctypes.byref(b.RopeStruct(4096, 4096, 63, 0, 0))) == BAD and b"63 positions" in L.ihip_last_error()
    assert append(b, rope=ctypes.byref(b.RopeStruct(4096, None, 64, 0, 0))) == BAD
    assert append(b, rope=ctypes.byref(b.RopeStruct(4096, 4100, 64, 0, 0))) == BAD
    # an empty batch and no rows at all: nothing is enqueued, no pointer is looked at
    assert append(b, packed=P(0, 8, 2, 128, None, 10, 10), k=t(None, 0, 0, 0)) == 0
    assert append(b, packed=P(2, 8, 2, 128, 4096, 0, 0), k=t(None, 0, 0, 0)) == 0


def test_stores_that_are_refused(b):
    L, t = b.lib(), b.Tensor
    inf = float("inf")
    bad = [dict(fmt=0, k=t(None, 0, 0, 128)), dict(fmt=0, v=t(4096, 0, 0, 0)), dict(fmt=0, k=t(4096, 4, 0, 128)),
           dict(fmt=1, k_scale=0.0), dict(fmt=1, v_scale=inf), dict(fmt=1, k=t(4096, 0, 0, 136)), dict(fmt=1, v=t(4096, 0, 0, 64)),
           dict(fmt=2, k=t(4096, 0, 0, 32)), dict(fmt=2, v=t(4096, 1024 * 64, 64 * 64, 128)), dict(fmt=2, k_scales=None),
           dict(fmt=2, v_scales=4098), dict(fmt=2, k=t(4104, 1024 * 64, 64 * 64, 64)), dict(fmt=2, k=t(4096, 1024 * 64 + 32, 64 * 64, 64))]
    for kw in bad:
        s = store_of(b, **kw)
        assert append(b, store=s) == BAD, kw
        assert L.ihip_kv_gather(ctypes.byref(s), 2, 2, 128, 4096, 64, t(4096, 0, 0, 128), b.NO_TENSOR, None) == BAD, kw
    s = store_of(b, 0)
    s.format = 3
    assert append(b, store=s) == BAD and b"format" in L.ihip_last_error()
    for pg in (b.PagedStruct(None, 4, 16), b.PagedStruct(4096, 4, 24), b.PagedStruct(4096, 3, 16)):       # the last covers 48 of 64 tokens
        s = store_of(b, 2, paged=ctypes.cast(ctypes.pointer(pg), ctypes.c_void_p))
        assert append(b, store=s) == BAD


def test_gather_refuses(b):
    L, t = b.lib(), b.Tensor
    s, o = store_of(b, 2), t(4096, 0, 0, 128)
    call = lambda B=2, Hkv=2, d=128, lens=4096, m=64, k=o, v=o, st=s: L.ihip_kv_gather(ctypes.byref(st) if st else None, B, Hkv, d, lens, m, k, v, None)  # noqa: E731
    assert call(B=-1) == BAD and call(Hkv=0) == BAD and call(m=-1) == BAD and call(lens=None) == BAD
    assert call(d=64) == UNSUPPORTED
    assert call(k=t(4096, 0, 0, 0)) == BAD and call(v=t(4100, 0, 0, 128)) == BAD and call(st=None) == BAD
    assert call(B=0, lens=None) == 0 and call(m=0, lens=None) == 0 and call(k=b.NO_TENSOR, v=b.NO_TENSOR) == 0
