"""Dense causal attention of packed prompts (ihip_prompt_attn) against float64.

Tolerances.  The probabilities are rounded to bf16 (half a step, 2^-8 of each), the result once more (2^-8 of it); the rest is
fp32: scores off by at most 2^-17 of sum |q_i k_i| (128 terms, each sum off by 2^-24 of what it has so far), which moves a
probability by as much, relative."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D  # noqa: E402

SCALE = 1 / np.sqrt(D)


@pytest.fixture(scope="module")
def ihip():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_08910_amd as pkg
    pkg.lib()
    return pkg


def normal(seed, *shape, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).bfloat16()


def offsets(new):
    return torch.tensor(np.concatenate(([0], np.cumsum(new))), dtype=torch.int32).cuda()


def check(q, k, v, new, total, out, lse, scale=SCALE):
    """All heads of all sequences, in float64 on the GPU."""
    G = q.shape[1] // k.shape[1]
    q0 = k0 = 0
    for n, t in zip(new, total):
        if n:
            Q = q[q0:q0 + n].double().transpose(0, 1)                                          # [Hq, n, D]
            K, V = (x[k0:k0 + t].double().transpose(0, 1).repeat_interleave(G, dim=0) for x in (k, v))
            Kt = K.transpose(1, 2).contiguous()
            s = Q @ Kt * scale
            s = s.masked_fill(torch.arange(t, device="cuda") > torch.arange(n, device="cuda").view(-1, 1) + (t - n), -np.inf)
            want_lse = torch.logsumexp(s, dim=2) if t else torch.full((q.shape[1], n), -np.inf, device="cuda", dtype=torch.float64)
            p = torch.nan_to_num((s - want_lse.unsqueeze(2)).exp())
            want = p @ V
            off = 2.0 ** -17 * scale * ((Q.abs() @ Kt.abs()).amax(dim=2) if t else torch.zeros_like(want_lse))
            got, got_lse = out[q0:q0 + n].double().transpose(0, 1), lse[q0:q0 + n].double().t()
            tol = (p @ V.abs()) * (2.0 ** -8 + 2 * off + 2.0 ** -20).unsqueeze(2) + want.abs() * 2.0 ** -8
            assert bool(((got - want).abs() <= tol).all()), (n, t, float(((got - want).abs() - tol).max()))
            empty = torch.isinf(want_lse)
            assert torch.equal(torch.isinf(got_lse), empty) and bool((got_lse[empty] < 0).all()) and bool((got[empty] == 0).all())
            lse_off = (got_lse - want_lse).abs()[~empty]
            assert bool((lse_off <= (off + 2.0 ** -20 * (1 + want_lse.abs()))[~empty]).all()), (n, t)
        q0, k0 = q0 + n, k0 + t


CASES = [
    # Hq, Hkv, new tokens, context
    (4, 4, [1], [0]),
    (8, 2, [33, 0, 1, 32, 31], None),
    (8, 1, [255, 257, 64], None),
    (6, 2, [513, 5], None),
    (7, 7, [100], None),
    (32, 8, [700, 1, 129], None),
    (5, 1, [1, 1, 1], [0, 31, 2047]),
    (16, 2, [300, 64], [1000, 77]),
    (4, 2, [260, 3, 40, 7], [-100, -3, 0, -7]),       # fewer keys than queries: the first queries see none
    (2, 1, [(i * 7) % 5 for i in range(150)], None),
    (2, 2, [5] * 65, [i for i in range(65)]),
]


@pytest.mark.parametrize("Hq,Hkv,new,ctx", CASES)
def test_prompt_attention(ihip, Hq, Hkv, new, ctx):
    total = new if ctx is None else [a + b for a, b in zip(new, ctx)]
    N, K = sum(new), sum(total)
    # rows behind the last sequence hold NaN in the inputs, and are left as they are in the outputs
    q, k, v = (torch.full((r + 40, h, D), float("nan"), dtype=torch.bfloat16, device="cuda") for r, h in ((N, Hq), (K, Hkv), (K, Hkv)))
    q[:N], k[:K], v[:K] = normal(1, N, Hq, D, scale=2.0), normal(2, K, Hkv, D), normal(3, K, Hkv, D)
    out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    ihip.prompt_attn(q, k, v, offsets(new), max(new), cu_k=None if ctx is None else offsets(total), out=out, lse=lse)
    check(q, k, v, new, total, out, lse)
    assert bool((out[N:] == 5).all()) and bool((lse[N:] == 5).all())


@pytest.mark.parametrize("n", [1500, 4099])
def test_longer_prompts(ihip, n):
    q, k, v = normal(4, n + 37, 8, D), normal(5, n + 37, 2, D), normal(6, n + 37, 2, D)
    out, lse = ihip.prompt_attn(q, k, v, offsets([37, n]), n, want_lse=True)
    check(q, k, v, [37, n], [37, n], out, lse)


def test_parts_of_a_fused_projection_and_another_scale(ihip):
    x = normal(7, 333, 12, D)
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
    out, lse = ihip.prompt_attn(q, k, v, offsets([133, 200]), 200, sm_scale=0.3, want_lse=True)
    check(q, k, v, [133, 200], [133, 200], out, lse, scale=0.3)


def test_scores_that_grow_and_shrink_along_the_keys(ihip):
    """The running reference of the exponentials has to follow upwards, by little and by much, and large scores must not overflow."""
    n, Hq = 700, 4
    q, k, v = normal(8, n, Hq, D), normal(9, n, Hq, D), normal(10, n, Hq, D)
    grow = torch.ones(n, device="cuda")
    grow[100:] = 6
    grow[300:] = 40
    grow[500:] = 0.01
    k = (k.float() * grow.view(-1, 1, 1)).bfloat16()
    k[50] = q[600] * 4                                # one key far above the others for one query
    out, lse = ihip.prompt_attn(q, k, v, offsets([n]), n, want_lse=True)
    check(q, k, v, [n], [n], out, lse)


def test_one_key_each_and_equal_scores(ihip):
    """Keys that are all the same: the mean of the values; a first token: its value, up to two roundings."""
    n = 97
    q, k, v = normal(11, n, 2, D), normal(12, 1, 2, D).expand(n, 2, D).contiguous(), normal(13, n, 2, D)
    out, lse = ihip.prompt_attn(q, k, v, offsets([n]), n, want_lse=True)
    check(q, k, v, [n], [n], out, lse)
    assert bool(((out[0].double() - v[0].double()).abs() <= v[0].double().abs() * 2.0 ** -7).all())


def test_offsets_beyond_the_rows_stay_inside(ihip):
    """cu_q and cu_k that promise more rows than there are: what is there is used, nothing else is touched."""
    q, k, v = normal(14, 100, 2, D), normal(15, 100, 2, D), normal(16, 100, 2, D)
    cu = torch.tensor([0, 60, 150], dtype=torch.int32).cuda()
    out, lse = ihip.prompt_attn(q, k, v, cu, 90, want_lse=True)
    check(q, k, v, [60, 40], [60, 40], out, lse)


def test_a_scale_of_zero_gives_the_mean(ihip):
    q, k, v = normal(17, 300, 4, D), normal(18, 300, 2, D), normal(19, 300, 2, D)
    out, lse = ihip.prompt_attn(q, k, v, offsets([33, 267]), 267, sm_scale=0.0, want_lse=True)
    check(q, k, v, [33, 267], [33, 267], out, lse, scale=0.0)


@pytest.mark.parametrize("ctx,shares", [(0, False), (30000, True)])
def test_rows_beyond_four_gigabytes(ihip, ctx, shares):
    """Keys behind 2^32 bytes of other sequences' keys, queries 2^32 bytes apart from first to last."""
    n, far, step = 300, (1 << 32) // (2 * D * 2) + 13, (1 << 23)
    total = n + ctx
    k, v = (torch.empty((far + total, 2, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[far:], v[far:] = normal(20, total, 2, D), normal(21, total, 2, D)
    wide = torch.empty((n * step,), dtype=torch.bfloat16, device="cuda").view(n, step)
    q = wide[:, :4 * D].unflatten(1, (4, D))
    q.copy_(normal(22, n, 4, D))
    cu, cu_k = offsets([0, n]), offsets([far, total])
    out, lse = ihip.prompt_attn(q, k, v, cu, n, cu_k=cu_k, want_lse=True, ws=None if shares else torch.empty(0, dtype=torch.uint8, device="cuda"))
    check(q, k[far:], v[far:], [n], [total], out, lse)


def test_on_another_stream_and_in_a_graph(ihip):
    q, k, v = (torch.empty((400, h, D), dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2))
    cu = offsets([130, 270])
    out, lse = torch.empty_like(q), torch.empty((400, 8), device="cuda")

    def step():
        ihip.prompt_attn(q, k, v, cu, 270, out=out, lse=lse)

    def fill(i):
        for j, t in enumerate((q, k, v)):
            t.copy_(normal(50 + 10 * i + j, *t.shape))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    check(q, k, v, [130, 270], [130, 270], out, lse)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(1, 4):
        fill(i)
        step()
        want = out.clone(), lse.clone()
        out.zero_(), lse.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
