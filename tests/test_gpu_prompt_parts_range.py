"""Prompt attention in shares: parts of a block whose sums are finite, and whose sum over all parts is not, though the mean is."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D  # noqa: E402
from tests.test_gpu_prompt_attn import check, ihip, normal  # noqa: E402, F401
from tests.test_gpu_prompt_range import run  # noqa: E402


@pytest.mark.parametrize("power", [-90, 112, 114, 116, 118, 120, 122, 124])
@pytest.mark.parametrize("n,ahead", [(64, 60000), (300, 20000)])
def test_the_mean_over_many_parts(ihip, n, ahead, power):  # noqa: F811
    q, k, v = normal(1, n, 8, D), torch.ones((n + ahead, 2, D), dtype=torch.bfloat16, device="cuda"), normal(2, n + ahead, 2, D)
    v = (v.float().abs().clamp(1, 3.9) * 2.0 ** power).bfloat16()
    out, lse = run(ihip, q, k, v, ahead, True)
    assert bool(torch.isfinite(out).all())
    check(q, k, v, [n], [n + ahead], out, lse)
