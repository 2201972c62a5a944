"""How the scratch of ihip_attn_decode_tracked is laid out, as far as its size tells (no GPU)."""
import ctypes

from tests.test_kv_store_args import b  # noqa: F401


def test_arrays_of_whole_16_bytes(b):  # noqa: F811
    """Scores, pairs of numbers for each part, partial results: all are read 16 bytes at a time, odd numbers of heads and parts too."""
    odd = 0
    for B, heads in ((1, 1), (3, 1), (1, 3), (5, 7), (2, 1)):
        for T in range(100, 9000, 317):
            need = b.lib().ihip_attn_decode_tracked_workspace_bytes(ctypes.byref(b.Shape(B, heads, heads, 128, 1, 1, 4096, T, 0, 1, 0)))
            stride = -(-T // 32) * 32
            parts, left = divmod(need // 4 - B * heads * stride, B * heads * 130)
            assert need % 16 == 0 and left in (0, 2)
            odd += left == 2
    assert odd > 20
