"""ihip_kv_evict where many rows move, in a launch of their own: K and V of every format, pages that are missing, token-major caches, lengths cut in
place, a captured call.  Everything is compared bit for bit (test_gpu_kv_evict)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_kv_evict import check, ihip, make_track  # noqa: E402, F401
from tests.tracked_reference import FORMATS, Cache, evicted  # noqa: E402


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,Hkv,lens,keep,token_major,missing", [
    (16, 2, [3000, 2100, 1200, 5], 1200, False, [(0, 2), (0, 100), (0, 187), (1, 80)]),          # one workgroup a (sequence, KV head)
    (0, 3, [2500], 600, True, []),
    (64, 2, [20000, 17001, 0], 3001, True, [(0, 1), (0, 200), (1, 46), (1, 265)]),               # rows in chunks
    (0, 1, [18000, 2999], 3000, False, []),
])
def test_rows_that_move(ihip, fmt, page, Hkv, lens, keep, token_major, missing):  # noqa: F811
    for in_place in (True, False):
        c = Cache(ihip, fmt, lens, Hkv, page, seed=keep + in_place, token_major=token_major, missing=missing)
        check(ihip, c, make_track(ihip, c, c.T + 5, seed=3, extra=10), keep, 4, 100, in_place, lens_in_place=in_place)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("most,keep,steps", [([120, 80], 40, ([120, 80], [41, 40])), ([2000, 1500], 700, ([2000, 1500], [699, 1001])),
                                             ([20000, 17000], 3000, ([20000, 17000], [2999, 16500]))])
def test_captured_rows(ihip, fmt, most, keep, steps):  # noqa: F811
    """Each replay moves what the eager call of the same lengths moves."""
    caches = [Cache(ihip, fmt, most, 2, 16, seed=1) for _ in range(2)]
    tracks = [make_track(ihip, c, c.T, seed=3) for c in caches]
    def memory(i):                                   # noqa: E306
        return [x for x in (caches[i].k, caches[i].v, caches[i].ks, caches[i].vs, tracks[i].weights, tracks[i].positions) if x is not None]
    fresh = [x.clone() for x in memory(0)]
    for x, y in zip(memory(1), fresh):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        new, kept = torch.zeros(2, dtype=torch.int32).cuda(), torch.zeros((2, 2, keep), dtype=torch.int32).cuda()
        ws = ihip.kv_evict_workspace(caches[0].store, 2, caches[0].T, keep)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ihip.kv_evict(caches[0].store, tracks[0], caches[0].seq_lens, caches[0].T, keep, n_sink=2, n_recent=8, new_lens=new, kept=kept, ws=ws)
        for lens in (*steps, steps[0]):
            for i in range(2):
                for x, y in zip(memory(i), fresh):
                    x.copy_(y)
                caches[i].seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            n, k = ihip.kv_evict(caches[1].store, tracks[1], caches[1].seq_lens, caches[1].T, keep, n_sink=2, n_recent=8)
            assert torch.equal(n, new) and torch.equal(k, kept)
            for x, y in zip(memory(0), memory(1)):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
            w, p = (fresh[-2][0, 0].cpu().numpy(), fresh[-1][0, 0].cpu().numpy())
            assert (kept[0, 0].cpu().numpy() == evicted(w, p, lens[0], keep, 2, int(tracks[0].seen[0]) - 8)).all()
            # K and V at the kept rows of the first KV head
            at = kept[0, 0].cpu().long()
            row, at, t = (at >= 0).nonzero()[:, 0], at[at >= 0], caches[0].table.cpu().long()[0]
            for x, y in zip(memory(0)[:-2], fresh[:-2]):
                x, y = x.view(torch.uint8).cpu(), y.view(torch.uint8).cpu()
                assert torch.equal(x[t[row // 16], 0, row % 16], y[t[at // 16], 0, at % 16])
