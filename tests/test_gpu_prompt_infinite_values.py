"""Prompt attention over infinite values: a result is +infinity where the query sees +infinity in that dimension, -infinity where it sees
that, NaN where it sees both or a NaN, wherever tiles and parts end and however small the probability is; all others are as they would be
without (test_gpu_prompt_attn's tolerances)."""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D  # noqa: E402
from tests.test_gpu_prompt_attn import SCALE, ihip, normal, offsets  # noqa: E402, F401


@pytest.mark.parametrize("Hq,n,ahead,shares", [(4, 1, 0, False), (4, 200, 0, False), (6, 517, 77, False), (2, 300, -150, False), (8, 300, 20000, True)])
@pytest.mark.parametrize("spread", [1, 60])
def test_infinite_values(ihip, Hq, n, ahead, shares, spread):  # noqa: F811
    """spread: of the scores, in nats and more; 60: most keys have a probability of 0 in fp32."""
    from paper_2502_08910_amd.binding import PackedStruct
    t = n + ahead
    q, k, v = normal(1, n, Hq, D, scale=float(spread)), normal(2, t, 2, D), normal(3, t, 2, D)
    rng = np.random.default_rng(n + spread)
    for i in range(40):                                  # four dims each with +, with -, with both, with NaN, in some rows
        kind = i % 4
        for value in [(np.inf,), (-np.inf,), (np.inf, -np.inf), (np.nan,)][kind]:
            v[int(rng.integers(t)), int(rng.integers(2)), 4 * kind + int(rng.integers(4))] = value
    cu, cu_k = offsets([n]), offsets([t])
    p = PackedStruct(1, Hq, 2, D, cu.data_ptr(), n, n)
    assert (ihip.lib().ihip_prompt_attn_workspace_bytes(ctypes.byref(p), t) > 256) == shares
    out, _ = ihip.prompt_attn(q, k, v, cu, n, cu_k=cu_k)

    Q, K, V = (x.double().transpose(0, 1) for x in (q, k, v))
    K, V = (x.repeat_interleave(Hq // 2, dim=0) for x in (K, V))
    sees = (torch.arange(t, device="cuda") <= torch.arange(n, device="cuda").view(-1, 1) + (t - n)).double().expand(Hq, n, t)
    up, down, nan = (sees @ x.double() > 0 for x in (V == np.inf, V == -np.inf, torch.isnan(V)))
    Kt = K.transpose(1, 2).contiguous()
    prob = torch.nan_to_num((Q @ Kt * SCALE).masked_fill(sees == 0, -np.inf).softmax(dim=2))
    finite = torch.where(torch.isfinite(V), V, torch.zeros_like(V))
    want = prob @ finite
    off = 2.0 ** -17 * SCALE * (Q.abs() @ Kt.abs()).amax(dim=2)
    tol = (prob @ finite.abs()) * (2.0 ** -8 + 2 * off + 2.0 ** -20).unsqueeze(2) + want.abs() * 2.0 ** -8
    got = out.double().transpose(0, 1)
    clean = ~(up | down | nan)
    assert bool(((got - want).abs() <= tol)[clean].all())
    assert bool((got[up & ~down & ~nan] == np.inf).all())
    assert bool((got[down & ~up & ~nan] == -np.inf).all())
    assert bool(torch.isnan(got[nan | (up & down)]).all())
    assert bool(up.any() or n == 1) and bool(clean.any())
