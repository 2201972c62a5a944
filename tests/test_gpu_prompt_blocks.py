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


@pytest.mark.parametrize("Hq,Hkv,lists", [
    (8, 2, [[300, 1, 99], [100, 200, 100], [0, 0, 400], [398, 1, 1]]),                            # all at once
    (128, 16, [[300, 500, 99], [500, 399, 0], [1, 400, 498]]),                                    # in the order of their keys
    (6, 2, [[(i * 7) % 40 for i in range(70)], [(i * 11) % 40 for i in range(70)], [0] * 69 + [40]]),        # found by their rows
])
def test_lengths_that_change_under_a_graph(ihip, Hq, Hkv, lists):  # noqa: F811
    N, most = max(sum(x) for x in lists), max(max(x) for x in lists)
    q, k, v = normal(21, N, Hq, D), normal(22, N, Hkv, D), normal(23, N, Hkv, D)
    cu = offsets(lists[0])
    out, lse = torch.empty_like(q), torch.empty((N, Hq), device="cuda")

    def step():
        ihip.prompt_attn(q, k, v, cu, most, out=out, lse=lse)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for new in lists:
        cu.copy_(offsets(new))
        out.fill_(5), lse.fill_(5)
        g.replay()
        torch.cuda.synchronize()
        check(q, k, v, new, new, out, lse)
        n = sum(new)
        assert bool((out[n:] == 5).all()) and bool((lse[n:] == 5).all())


def test_two_calls_at_once(ihip):  # noqa: F811
    """Two streams, each with calls in shares and by themselves, whose workgroups share the chip."""
    sets = []
    for i in range(2):
        q, k, v = normal(40 + i, 1200, 32, D), normal(50 + i, 21200, 8, D), normal(60 + i, 21200, 8, D)
        sets.append((q, k, v, [(offsets([1200]), 1200, None, 1200), (offsets([200, 1000]), 1000, offsets([15000, 6200]), 21200)]))
    want = [[ihip.prompt_attn(q, k[:rows], v[:rows], cu, n, cu_k=cu_k)[0] for cu, n, cu_k, rows in calls] for q, k, v, calls in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        got = [[], []]
        for i, (q, k, v, calls) in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                for cu, n, cu_k, rows in calls:
                    got[i].append(ihip.prompt_attn(q, k[:rows], v[:rows], cu, n, cu_k=cu_k)[0])
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
