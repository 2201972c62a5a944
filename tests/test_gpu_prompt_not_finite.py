"""Prompt attention over keys and values that are not finite: only the queries that see one get a result that is not finite, in the
dimensions that have it (a value) or in all (a key); all others are as they would be without it (test_gpu_prompt_attn's tolerances)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D  # noqa: E402
from tests.test_gpu_prompt_attn import SCALE, ihip, normal, offsets  # noqa: E402, F401


def reference(q, k, v):
    """[n, Hq, D] in float64 from what is finite, its tolerance, and where a query sees what is not."""
    n, t, G = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    Q, K, V = (x.double().transpose(0, 1) for x in (q, k, v))
    K, V = (x.repeat_interleave(G, dim=0) for x in (K, V))
    bad_k, bad_v = ~torch.isfinite(K).all(dim=2, keepdim=True), ~torch.isfinite(V)
    K, V = (torch.where(torch.isfinite(x), x, torch.zeros_like(x)) for x in (K, V))
    sees = torch.arange(t, device="cuda") <= torch.arange(n, device="cuda").view(-1, 1) + (t - n)
    Kt = K.transpose(1, 2).contiguous()
    s = (Q @ Kt * SCALE).masked_fill(~sees, -np.inf)
    p = torch.nan_to_num(s.softmax(dim=2))
    bad = sees.double().expand(Q.shape[0], n, t) @ (bad_v | bad_k).double() > 0
    want = p @ V
    off = 2.0 ** -17 * SCALE * (Q.abs() @ Kt.abs()).amax(dim=2)
    tol = (p @ V.abs()) * (2.0 ** -8 + 2 * off + 2.0 ** -20).unsqueeze(2) + want.abs() * 2.0 ** -8
    return (x.transpose(0, 1) for x in (want, tol, bad))


@pytest.mark.parametrize("Hq,n,ahead", [
    (4, 1, 0), (4, 200, 0), (8, 517, 77), (2, 300, -150),
    (96, 700, 0),                                        # more blocks than the chip holds at a time
    (8, 300, 20000), (16, 512, 16000),                   # equal shares
])
@pytest.mark.parametrize("what", ["values", "keys", "both"])
def test_what_is_not_finite_stays_with_those_who_see_it(ihip, Hq, n, ahead, what):  # noqa: F811
    t = n + ahead
    q, k, v = normal(1, n, Hq, D, scale=2.0), normal(2, t, 2, D), normal(3, t, 2, D)
    rng = np.random.default_rng(n)
    if what != "keys":
        for row in rng.integers(max(0, ahead), t, 12):
            v[row, int(rng.integers(2)), int(rng.integers(D))] = float(rng.choice([np.nan, np.inf, -np.inf]))
        v[t - 1] = float("nan")
    if what != "values":
        for row in rng.integers(max(0, t - n // 2 - 1), t, 3):
            k[row, 0, int(rng.integers(D))] = float(rng.choice([np.nan, np.inf]))
    out, _ = ihip.prompt_attn(q, k, v, offsets([n]), n, cu_k=offsets([t]))
    want, tol, bad = reference(q, k, v)
    finite = torch.isfinite(out)
    # (an infinite key gives some queries a score of -inf, whose probability is 0 like that of a key they do not see)
    assert bool(finite[~bad].all())
    if what == "values":
        assert not bool(finite[bad].any())
    assert bool(((out.double() - want).abs() <= tol)[~bad].all())
    if what != "values":
        k0 = torch.where(torch.isinf(k), torch.full_like(k, float("nan")), k)
        assert not bool(torch.isfinite(ihip.prompt_attn(q, k0, v, offsets([n]), n, cu_k=offsets([t]))[0])[bad].any())
