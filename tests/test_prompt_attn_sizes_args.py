"""Numbers of heads and rows whose offsets the prompt attention could not hold in 32 bits are refused, before anything is enqueued (no GPU)."""
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


@pytest.mark.parametrize("Hq,Hkv,rows", [(70000, 70000, 100), (140000, 70000, 300), (131000, 131000, 7), (131000, 1, 1 << 15), (120000, 2, 40000)])
def test_more_heads_than_offsets_reach(b, Hq, Hkv, rows):
    stride = min(Hq * 128, (1 << 24) - 8)
    q, k = b.Tensor(4096, 0, 128, stride), b.Tensor(4096, 0, 128, Hkv * 128)
    p = b.PackedStruct(1, Hq, Hkv, 128, 4096, rows, rows)
    for ws, size in ((None, 0), (4096, 1 << 40)):
        assert b.lib().ihip_prompt_attn(ctypes.byref(p), q, k, k, None, rows, 0.1, 4096, None, ws, size, None) == -4
        assert b"are too many" in b.lib().ihip_last_error()
