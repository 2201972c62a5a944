"""Prompt attention at the ends of what bf16 holds: scores far from 0 in either direction, values near the largest and far below 1 under scores
that grow along the keys; blocks by themselves and dealt out in shares.  Results against float64."""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D  # noqa: E402
from tests.test_gpu_prompt_attn import SCALE, check, ihip, normal, offsets  # noqa: E402, F401

WAYS = [(1, 0, False), (300, 0, False), (300, 20000, True)]       # queries, keys in front of them, whether the call is dealt out


def run(ihip, q, k, v, ahead, shares, scale=SCALE):  # noqa: F811
    from paper_2502_08910_amd.binding import PackedStruct
    n = q.shape[0]
    cu, cu_k = offsets([n]), offsets([n + ahead])
    p = PackedStruct(1, q.shape[1], k.shape[1], D, cu.data_ptr(), n, n)
    assert (ihip.lib().ihip_prompt_attn_workspace_bytes(ctypes.byref(p), n + ahead) > 256) == shares
    return ihip.prompt_attn(q, k, v, cu, n, cu_k=cu_k, want_lse=True, sm_scale=scale)


def one_direction(n, ahead, sizes, up):
    """Keys that are multiples, by powers of two, of one direction, and queries along it (against it: up False).  Products are exact in fp32,
    so that equal keys have equal scores."""
    k = (2.0 ** torch.tensor(sizes, dtype=torch.float64, device="cuda")).view(-1, 1, 1).expand(n + ahead, 2, D).bfloat16()
    q = torch.full((n, 8, D), 1.296875 if up else -1.296875, dtype=torch.bfloat16, device="cuda")
    return q, k, normal(1, n + ahead, 2, D)


def check_mean(v, first, n, ahead, score, out, lse):
    """Query i sees keys 0 .. i + ahead, of which those from first(i) on share everything equally: sums in fp32 (2^-16 of the largest), the
    result's own rounding; score: that of the last key of a query."""
    v = v.double().repeat_interleave(4, dim=1)
    total = torch.cat((torch.zeros_like(v[:1]), v.cumsum(0)))
    end = torch.arange(n, device="cuda") + ahead + 1
    count = (end - first).double()
    want = (total[end] - total[first]) / count.view(-1, 1, 1)
    assert bool(((out.double() - want).abs() <= want.abs() * 2.0 ** -8 + v.abs().max() * 2.0 ** -16).all())
    want_lse = (score + count.log()).view(-1, 1)
    assert bool(((lse.double() - want_lse).abs() <= 2.0 ** -22 * want_lse.abs() + 2.0 ** -18 * (1 + count.log().view(-1, 1))).all())


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("size", [40, 105])
@pytest.mark.parametrize("n,ahead,shares", WAYS)
def test_equal_scores_far_from_zero(ihip, n, ahead, shares, size, up):  # noqa: F811
    q, k, v = one_direction(n, ahead, [size] * (n + ahead), up)
    out, lse = run(ihip, q, k, v, ahead, shares)
    zero = torch.zeros(n, dtype=torch.int64, device="cuda")
    check_mean(v, zero, n, ahead, float(q[0, 0, 0]) * D * 2.0 ** size * SCALE, out, lse)


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("n,ahead,shares", WAYS)
def test_scores_far_from_zero_and_from_each_other(ihip, n, ahead, shares, up):  # noqa: F811
    """Ever larger scores: the last key of 5 and those of its size that are seen share everything."""
    t = n + ahead
    step = -(-t // 80)
    sizes = np.arange(t) // step
    first = torch.tensor(np.arange(ahead, t) // step * step, device="cuda")
    sizes = 20 + sizes if up else 100 - sizes
    q, k, v = one_direction(n, ahead, sizes, up)
    out, lse = run(ihip, q, k, v, ahead, shares)
    score = float(q[0, 0, 0]) * D * SCALE * 2.0 ** torch.tensor(sizes[ahead:], dtype=torch.float64, device="cuda")
    check_mean(v, first, n, ahead, score, out, lse)


@pytest.mark.parametrize("power", [120, 126, -90])
@pytest.mark.parametrize("n,ahead,shares", WAYS)
def test_values_at_the_ends_under_growing_scores(ihip, n, ahead, shares, power):  # noqa: F811
    t = n + ahead
    q, k, v = normal(2, n, 8, D, scale=2.0), normal(3, t, 2, D), normal(4, t, 2, D)
    grow = 2.0 ** torch.linspace(-5, 2, t, device="cuda")
    k = (k.float() * grow.view(-1, 1, 1)).bfloat16()
    v = (v.float().clamp(-3.9, 3.9) * 2.0 ** power).bfloat16()
    out, lse = run(ihip, q, k, v, ahead, shares)
    assert bool(torch.isfinite(out).all())
    check(q, k, v, [n], [t], out, lse)


@pytest.mark.parametrize("n,ahead,shares", WAYS)
def test_the_mean_of_large_values(ihip, n, ahead, shares):  # noqa: F811
    """Equal keys and values of 2^125 to 2^127, whose sum is beyond fp32."""
    q, k, v = normal(5, n, 8, D), torch.ones((n + ahead, 2, D), dtype=torch.bfloat16, device="cuda"), normal(6, n + ahead, 2, D)
    v = (v.float().abs().clamp(1, 3.9) * 2.0 ** 125).bfloat16()
    out, lse = run(ihip, q, k, v, ahead, shares)
    assert bool(torch.isfinite(out).all())
    check(q, k, v, [n], [n + ahead], out, lse)
