"""Reading a cache back where sequences x heads x max_seq_len, a bound, ask for more threads than one dimension of a grid has."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ihip():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_08910_amd as pkg
    pkg.lib()
    return pkg


@pytest.mark.parametrize("B,max_len", [(1 << 14, 1 << 13), ((1 << 13) + 77, (1 << 14) - 5)])
def test_more_threads_than_a_dimension_of_the_grid(ihip, B, max_len):
    """All sequences are empty but one, at the far end, and all lie on the same memory: 2^30 rows of bounds, one sequence of rows."""
    from paper_2502_08910_amd import binding as b
    Hkv, T = 8, max_len
    k, v = (torch.randn((Hkv, T, 128), device="cuda").bfloat16() for _ in range(2))
    for b0, n in ((B - 1, T), (0, 5), (B // 2 + 1, T - 31)):
        lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        lens[b0] = n
        k_out, v_out = (torch.zeros_like(k) for _ in range(2))
        as_tensor = lambda t: b.Tensor(t.data_ptr(), 0, t.stride(0), t.stride(1))  # noqa: E731
        store = b.StoreStruct(b.KV_BF16, as_tensor(k), as_tensor(v), None, None, 1.0, 1.0, None)
        rc = b.lib().ihip_kv_gather(ctypes.byref(store), B, Hkv, 128, lens.data_ptr(), max_len, as_tensor(k_out), as_tensor(v_out),
                                    torch.cuda.current_stream().cuda_stream)
        assert rc == 0, b.lib().ihip_last_error()
        torch.cuda.synchronize()
        for got, want in ((k_out, k), (v_out, v)):
            assert torch.equal(got[:, :n], want[:, :n]) and bool((got[:, n:] == 0).all())
