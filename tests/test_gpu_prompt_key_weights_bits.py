"""The log-sum-exp of ihip_prompt_key_weights is taken to base 2 with one rounding."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, f64  # noqa: E402
from tests.test_gpu_prompt_key_weights import ihip  # noqa: E402, F401

LN2, LOG2_E = np.log(2.0), 1 / np.log(2.0)


def chosen_lse(n):
    """n log-sum-exps whose product with log2 e ends, if that is rounded to fp32 first, 0.62 of a last place and more from the true one."""
    x = np.random.default_rng(1).uniform(60, 84, 100000).astype(np.float32)
    once = (x * np.float32(LOG2_E)).astype(np.float64)
    off = np.abs(once - x.astype(np.float64) * LOG2_E) * 2.0 ** 17
    x = x[(off > 0.62) & (once > 64) & (once < 128)]
    assert len(x) >= n
    return x[:n]


@pytest.mark.parametrize("max_q", [1, 1000])         # a window's kernel; that of many queries
def test_log_sum_exp_is_rounded_once(ihip, max_q):  # noqa: F811
    """64 sequences of one query of zeros: every key's weight is exp(-lse).  Tolerance: half a last place of lse log2 e (64 .. 128: 2^-18), a hundredth of it
    for the two products that it is made of, and exp2, 2^-23, with the result's rounding."""
    B, H, keys = 64, 4, 3
    lse = torch.from_numpy(chosen_lse(B * H)).view(B, H)
    k = torch.randn((B * keys, H, D), generator=torch.Generator().manual_seed(1)).bfloat16()
    at = torch.arange(B + 1, dtype=torch.int32)
    track = ihip.KVTrack(torch.zeros((B, H, keys)).cuda())
    ihip.prompt_key_weights(torch.zeros((B, H, D), dtype=torch.bfloat16).cuda(), k.cuda(), at.cuda(), max_q, lse.cuda(), track, cu_k=(at * keys).cuda(), fresh=True)
    off = f64(track.weights) * np.exp(f64(lse))[:, :, None] - 1
    assert np.abs(off).max() <= LN2 * 1.01 * 2.0 ** -18 + 2.0 ** -22, np.abs(off).max() / (LN2 * 2.0 ** -18)


@pytest.mark.parametrize("lse,weight", [(float("inf"), 0.0), (-float("inf"), float("inf")), (float("nan"), float("nan")), (0.0, 1.0), (3e38, 0.0), (1e-42, 1.0)])
def test_log_sum_exps_at_the_ends(ihip, lse, weight):  # noqa: F811
    """What is not finite or very large comes out as the formula has it."""
    for max_q in (1, 1000):
        track = ihip.KVTrack(torch.zeros((1, 1, 2)).cuda())
        ihip.prompt_key_weights(torch.zeros((1, 1, D), dtype=torch.bfloat16).cuda(), torch.ones((2, 1, D), dtype=torch.bfloat16).cuda(),
                                torch.tensor([0, 1], dtype=torch.int32).cuda(), max_q, torch.full((1, 1), lse).cuda(), track,
                                cu_k=torch.tensor([0, 2], dtype=torch.int32).cuda(), fresh=True)
        want = torch.full((1, 1, 2), weight)
        assert torch.equal(track.weights.cpu(), want) or (np.isnan(weight) and bool(track.weights.isnan().all()))
