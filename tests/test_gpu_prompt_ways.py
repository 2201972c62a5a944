"""Which of its two ways the prompt attention takes for calls that other tests make because of it (blocks by themselves, or equal shares), and
rows that are NaN among others whose block is done again."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D  # noqa: E402
from tests.test_gpu_prompt_attn import check, ihip, normal, offsets  # noqa: E402, F401

FAR = (1 << 32) // (2 * D * 2) + 13          # keys in front of test_rows_beyond_four_gigabytes'


@pytest.mark.parametrize("B,Hq,Hkv,rows,max_q,rows_k,shares", [
    (2, 4, 2, 300, 300, FAR + 30300, True),                                                     # rows beyond 4 GiB
    (1, 8, 2, 300, 300, 20300, True), (1, 16, 2, 512, 512, 16512, True), (1, 96, 2, 700, 700, 700, False),    # what is not finite
    (1, 4, 2, 200, 200, 6200, True),                                                            # scores that leave the first tile's range
    (2, 8, 2, 500, 500, 9000, True),                                                            # a graph whose lengths change
    (1, 32, 8, 1200, 1200, 1200, False), (2, 32, 8, 1200, 1000, 21200, True),                   # two calls at once
])
def test_ways(ihip, B, Hq, Hkv, rows, max_q, rows_k, shares):  # noqa: F811
    from paper_2502_08910_amd.binding import PackedStruct
    p = PackedStruct(B, Hq, Hkv, D, 4096, rows, max_q)
    assert (ihip.lib().ihip_prompt_attn_workspace_bytes(ctypes.byref(p), rows_k) > 256) == shares


@pytest.mark.parametrize("n,ahead", [(300, 0), (300, 20000)])
@pytest.mark.parametrize("grow", [False, True])
def test_queries_that_are_nan(ihip, n, ahead, grow):  # noqa: F811
    """They make their own results NaN and nobody else's; grow: their blocks are done again for a key that dwarfs the others."""
    t = n + ahead
    q, k, v = normal(1, n, 8, D), normal(2, t, 2, D), normal(3, t, 2, D)
    if grow:
        k[ahead + 10] *= 60
    nan = torch.zeros((n, 8), dtype=torch.bool, device="cuda")
    nan[::7, 1] = nan[50:60] = nan[n - 1, 5] = True
    bad = q.clone()
    bad[..., 77][nan] = float("nan")
    cu, cu_k = offsets([n]), offsets([t])
    out, lse = ihip.prompt_attn(bad, k, v, cu, n, cu_k=cu_k, want_lse=True)
    assert bool(torch.isnan(out[nan]).all()) and bool(torch.isnan(lse[nan]).all())
    clean, clean_lse = ihip.prompt_attn(q, k, v, cu, n, cu_k=cu_k, want_lse=True)
    out[nan], lse[nan] = clean[nan], clean_lse[nan]
    check(q, k, v, [n], [t], out, lse)
