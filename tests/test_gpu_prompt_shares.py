"""Prompt attention whose tiles are dealt out to the chip in equal shares: few queries on many keys, sequences that bring keys and
others that do not, blocks without keys, more sequences than lanes.  The same tolerances as without shares (test_gpu_prompt_attn)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D  # noqa: E402
from tests.test_gpu_prompt_attn import check, normal, offsets  # noqa: E402


@pytest.fixture(scope="module")
def ihip():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_08910_amd as pkg
    pkg.lib()
    return pkg


def workspace_bytes(ihip, q, k, cu, max_q):
    import ctypes
    from paper_2502_08910_amd.binding import PackedStruct
    p = PackedStruct(cu.numel() - 1, q.shape[1], k.shape[1], D, cu.data_ptr(), q.shape[0], max_q)
    return ihip.lib().ihip_prompt_attn_workspace_bytes(ctypes.byref(p), k.shape[0])


@pytest.mark.parametrize("Hq,Hkv,new,ctx,shares", [
    (8, 8, [1], [5000], True),
    (8, 2, [300, 1, 0, 64], [9000, 3, 0, 1200], True),
    (8, 2, [300, 1, 0, 64], [29000, 3, 0, 1200], True),
    (16, 2, [700], [20011], True),
    (3, 1, [257, 255], [4096, 31], True),
    (3, 1, [257, 255], [9096, 31], True),
    (4, 2, [2500], [0], False),
    (4, 2, [4500], [0], True),
    (1, 1, [1000, 300, 900], [-700, 4000, -900], False),
    (1, 1, [1000, 300, 900], [-700, 40000, -900], True),      # blocks whose queries see nothing
    (2, 1, [17] * 70, [(i * 37) % 300 for i in range(70)], False),
    (2, 1, [17] * 70, [(i * 373) % 17000 for i in range(70)], True),
    (1, 1, [40000], [0], True),
    (7, 1, [40, 0, 333], [9000, 10, 1200], True),
    (16, 8, [600, 300, 1100, 0, 260], [32000, 29000, -200, 50, 16001], True)
])
def test_shares(ihip, Hq, Hkv, new, ctx, shares):
    total = [a + b for a, b in zip(new, ctx)]
    N, K = sum(new), sum(total)
    q, k, v = (torch.full((r + 9, h, D), float("nan"), dtype=torch.bfloat16, device="cuda") for r, h in ((N, Hq), (K, Hkv), (K, Hkv)))
    q[:N], k[:K], v[:K] = normal(1, N, Hq, D, scale=2.0), normal(2, K, Hkv, D), normal(3, K, Hkv, D)
    cu, cu_k = offsets(new), offsets(total)
    assert (workspace_bytes(ihip, q, k, cu, max(new)) > 256) == shares
    out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    ihip.prompt_attn(q, k, v, cu, max(new), cu_k=cu_k, out=out, lse=lse)
    check(q, k, v, new, total, out, lse)
    assert bool((out[N:] == 5).all()) and bool((lse[N:] == 5).all())
    again = ihip.prompt_attn(q, k, v, cu, max(new), cu_k=cu_k, want_lse=True)
    assert torch.equal(again[0][:N], out[:N]) and torch.equal(again[1][:N], lse[:N])
    # without scratch: not dealt out
    alone = ihip.prompt_attn(q, k, v, cu, max(new), cu_k=cu_k, want_lse=True, ws=torch.empty(0, dtype=torch.uint8, device="cuda"))
    check(q, k, v, new, total, alone[0], alone[1])


@pytest.mark.parametrize("n,ctx,Hq", [(200, 6000, 4), (512, 16000, 16)])
def test_scores_that_leave_the_first_tiles_range(ihip, n, ctx, Hq):
    """Parts whose later scores are far above their first ones', in one part and not in others."""
    q, k, v = normal(4, n, Hq, D), normal(5, ctx + n, 2, D), normal(6, ctx + n, 2, D)
    k[3000:3100] *= 50
    k[4000:] *= 0.01
    k[5990] = 30 * q[100, 0]
    cu, cu_k = offsets([n]), offsets([ctx + n])
    out, lse = ihip.prompt_attn(q, k, v, cu, n, cu_k=cu_k, want_lse=True)
    check(q, k, v, [n], [ctx + n], out, lse)


def test_shares_in_a_graph_whose_lengths_change(ihip):
    """The shares follow the offsets in device memory: one captured call serves other lengths of the same totals."""
    q, k, v = normal(7, 500, 8, D), normal(8, 9000, 2, D), normal(9, 9000, 2, D)
    cu, cu_k = offsets([100, 400]), offsets([4000, 5000])
    p_bytes = workspace_bytes(ihip, q, k, cu, 500)
    ws = torch.empty(p_bytes, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((500, 8), device="cuda")

    def step():
        ihip.prompt_attn(q, k, v, cu, 500, cu_k=cu_k, out=out, lse=lse, ws=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for new, total in (([100, 400], [4000, 5000]), ([499, 1], [600, 8000]), ([0, 500], [100, 8900]), ([250, 250], [250, 8000])):
        cu.copy_(offsets(new)), cu_k.copy_(offsets(total))
        step()
        torch.cuda.synchronize()
        check(q, k, v, new, total, out, lse)
        want = out.clone(), lse.clone()
        out.zero_(), lse.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
