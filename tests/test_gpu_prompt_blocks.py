"""Prompt attention with more work than the chip holds at a time, in blocks that end inside and outside of tiles: the same
corners and tolerances as for those (test_gpu_prompt_attn)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D  # noqa: E402
from tests.test_gpu_prompt_attn import check, ihip, normal, offsets  # noqa: E402, F401


@pytest.mark.parametrize("Hq,Hkv,new,ctx", [
    (128, 32, [300] * 3, None),
    (64, 16, [255, 257, 64, 513, 33, 1, 0, 770], None),
    (96, 3, [260, 3, 300, 7, 600, 900], [-100, -3, 0, -7, 77, -300]),
    (128, 128, [257, 2, 600, 0, 512], [1000, 77, 1, 5, 95]),
    (8, 2, [290 + i % 7 for i in range(70)], [(37 * i) % 300 for i in range(70)]),
])
def test_large_calls(ihip, Hq, Hkv, new, ctx):  # noqa: F811
    total = new if ctx is None else [a + b for a, b in zip(new, ctx)]
    N, K = sum(new), sum(total)
    q, k, v = (torch.full((r + 40, h, D), float("nan"), dtype=torch.bfloat16, device="cuda") for r, h in ((N, Hq), (K, Hkv), (K, Hkv)))
    q[:N], k[:K], v[:K] = normal(1, N, Hq, D, scale=2.0), normal(2, K, Hkv, D), normal(3, K, Hkv, D)
    out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    ihip.prompt_attn(q, k, v, offsets(new), max(new), cu_k=None if ctx is None else offsets(total), out=out, lse=lse)
    check(q, k, v, new, total, out, lse)
    assert bool((out[N:] == 5).all()) and bool((lse[N:] == 5).all())


def test_scores_that_grow_and_shrink_along_the_keys(ihip):  # noqa: F811
    """As in small calls: a running reference that has to follow upwards, by little and by much."""
    n, Hq = 700, 128
    q, k, v = normal(8, n, Hq, D), normal(9, n, Hq, D), normal(10, n, Hq, D)
    grow = torch.ones(n, device="cuda")
    grow[100:] = 6
    grow[300:] = 40
    grow[500:] = 0.01
    k = (k.float() * grow.view(-1, 1, 1)).bfloat16()
    k[50] = q[600] * 4
    out, lse = ihip.prompt_attn(q, k, v, offsets([n]), n, want_lse=True)
    check(q, k, v, [n], [n], out, lse)


@pytest.mark.parametrize("new", [
    [1] * 4200,
    [(i * 7919) % 131 for i in range(700)],
    [0] * 100 + [300] + [0] * 200 + [128, 129, 1] + [0] * 90,
    [0] * 65,
    [256] + [0] * 64,
])
def test_many_sequences(ihip, new):  # noqa: F811
    N = sum(new)
    q, k, v = normal(1, N + 5, 4, D), normal(2, N + 5, 2, D), normal(3, N + 5, 2, D)
    out, lse = torch.full_like(q, 5.0), torch.full((N + 5, 4), 5.0, device="cuda")
    ihip.prompt_attn(q, k, v, offsets(new), max(new + [1]), out=out, lse=lse)
    check(q, k, v, new, new, out, lse)
    assert bool((out[N:] == 5).all()) and bool((lse[N:] == 5).all())
