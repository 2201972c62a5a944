"""The ends of sm_scale in the prompt attention and in the 4-bit decode attention: 0, smallest numbers, under products near the end of fp32."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests import test_gpu_attn_mx4_range as decode  # noqa: E402
from tests import test_gpu_prompt_range as prompt  # noqa: E402
from tests.test_gpu_attn_mx4 import ihip  # noqa: E402, F401


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -149, 2.0 ** -148])
def test_decode_attention(ihip, scale):  # noqa: F811
    """Products of 2^107 to 2^126, times next to nothing: all the same."""
    sizes = torch.randint(100, 114, (300,), generator=torch.Generator().manual_seed(56)).tolist()
    c, q = decode.one_direction(ihip, [127 + s for s in sizes], True)
    out, lse = decode.run(ihip, c, q * 48, scale=scale)
    decode.check_mean(c, 0, 0.0, out, lse)


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -149, 2.0 ** -148])
@pytest.mark.parametrize("n,ahead,shares", prompt.WAYS)
def test_prompt_attention(ihip, n, ahead, shares, scale):  # noqa: F811
    sizes = np.random.default_rng(n).integers(100, 114, n + ahead)
    q, k, v = prompt.one_direction(n, ahead, sizes, True)
    out, lse = prompt.run(ihip, q * 48, k, v, ahead, shares, scale=scale)
    prompt.check_mean(v, torch.zeros(n, dtype=torch.int64, device="cuda"), n, ahead, 0.0, out, lse)
