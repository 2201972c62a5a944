"""What the prompt attention refuses, before anything is enqueued (no GPU)."""
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


def test_prompt_attention_refuses(b):
    t, P, L = b.Tensor, b.PackedStruct, b.lib()
    ok = t(4096, 0, 128, 1024)

    def call(packed=P(2, 8, 2, 128, 4096, 10, 10), q=ok, k=ok, v=ok, cu_k=4096, rows_k=20, out=4096, scale=0.1):
        return L.ihip_prompt_attn(ctypes.byref(packed) if packed else None, q, k, v, cu_k, rows_k, scale, out, None, None, 0, None)

    assert call(packed=None) == -1
    assert call(packed=P(2, 8, 3, 128, 4096, 10, 10)) == -1
    assert call(packed=P(2, 8, 2, 256, 4096, 10, 10)) == -4
    assert call(packed=P(2, 8, 2, 128, None, 10, 10)) == -1
    assert call(packed=P(2, 8, 2, 128, 4096, 10, -1)) == -1
    assert call(q=t(None, 0, 128, 1024)) == -1 and call(k=t(4100, 0, 128, 1024)) == -1 and call(v=t(4096, 0, 4, 1024)) == -1
    assert call(k=t(4096, 0, 128, 64)) == -1
    assert call(out=None) == -1 and call(out=4100) == -1
    assert call(rows_k=-1) == -1
    for scale in (-0.1, float("nan"), float("inf")):
        assert call(scale=scale) == -1 and b"sm_scale" in L.ihip_last_error()
    assert call(cu_k=None, rows_k=20) == -1 and b"rows_k" in L.ihip_last_error()      # whole prompts: as many keys as queries
    assert call(packed=P(1, 1 << 20, 1 << 20, 128, 4096, 1 << 30, 1 << 30)) == -4 and b"workgroups" in L.ihip_last_error()
    # nothing to do
    assert call(packed=P(0, 8, 2, 128, None, 10, 10), q=t()) == 0
    assert call(packed=P(2, 8, 2, 128, 4096, 0, 0), q=t()) == 0
    assert call(packed=P(2, 8, 2, 128, 4096, 10, 0), q=t()) == 0
