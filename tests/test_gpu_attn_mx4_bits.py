"""The bits that 4-bit decode attention keeps of a probability: 16 or more, so that its results are as good as their last rounding.

Tolerance: a probability goes into the second product in two bf16 parts (half a step of the second: 2^-8 of 2^-8); scores, sums and
the result's own rounding as in test_gpu_attn_mx4."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import attention, f64  # noqa: E402
from tests.test_gpu_attn_mx4 import SCALE, Cache, ihip, queries  # noqa: E402, F401


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("page,lens", [(0, [40, 333]), (16, [5000])])
def test_results_are_as_good_as_their_last_rounding(ihip, G, page, lens):  # noqa: F811
    Hkv = 2
    c = Cache(ihip, lens, Hkv, page, seed=60 + G)
    q = queries(len(lens), G * Hkv, 61)
    sl = torch.tensor(lens, dtype=torch.int32).cuda()
    out, _ = ihip.sparse_attn_decode_mx4(ihip.Layer(q, c.store, sl, 1, 0, c.T, max_seq_len=c.T), q, c.store)
    Q, got = f64(q), f64(out)
    for b, t in enumerate(lens):
        for g in range(Hkv):
            heads = slice(g * G, (g + 1) * G)
            k, v = c.rows(b, g, np.arange(t))
            seen = np.ones((G, t), dtype=bool)
            want, _ = attention(Q[b, heads, 0], k, v, SCALE, seen)
            mag, _ = attention(Q[b, heads, 0], k, np.abs(v), SCALE, seen)
            off = 2.0 ** -17 * SCALE * (np.abs(Q[b, heads, 0]) @ np.abs(k).T).max(axis=1)
            tol = mag * (2.0 ** -16 + 2 * off + 2.0 ** -20)[:, None] + np.abs(want) * 2.0 ** -8
            assert (np.abs(got[b, heads, 0] - want) <= tol).all(), (b, g)
