"""Sums over many keys of the same small probability, where fp32 rounds every addition the same way."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D  # noqa: E402
from tests.test_gpu_prompt_attn import SCALE, ihip, normal, offsets  # noqa: E402, F401


@pytest.mark.parametrize("t", [30000, 120000, 600000])
@pytest.mark.parametrize("part", [0.3, 0.013, 0.77])
@pytest.mark.parametrize("grow", [False, True])
def test_the_sum_of_many_equal_probabilities(ihip, t, part, grow):  # noqa: F811
    """One key, then all others with a part of its probability (grow: another one far above it in between, so that the block is done again).
    The kernel adds up 16 of them before it adds them to a row's sum, in two lanes: t / 32 additions off by at most 2^-24 of what the sum has
    then, half of its end on the mean, which makes t * 2^-30; 16 within; 2^-18 for the exponentials, their scores and the logarithm."""
    n = 64
    q = torch.ones((n, 2, D), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((t, 1, D), dtype=torch.bfloat16, device="cuda")
    k[1:] = math.log(part) / (SCALE * D)
    if grow:
        k[t // 3] = 6.0
    v = normal(1, t, 1, D)
    _, lse = ihip.prompt_attn(q, k, v, offsets([n]), n, cu_k=offsets([t]), want_lse=True, ws=torch.empty(0, dtype=torch.uint8, device="cuda"))
    scores = k[:, 0, 0].double() * D * SCALE
    want = torch.logcumsumexp(scores, 0)[t - n:].view(-1, 1)
    assert bool(((lse.double() - want).abs() <= t * 2.0 ** -30 + 2.0 ** -18 + 2.0 ** -22 * want.abs()).all()), float((lse.double() - want).abs().max())
