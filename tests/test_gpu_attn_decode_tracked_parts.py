"""ihip_attn_decode_tracked where sequences are several parts, which a second launch joins: every number of heads and format, sequences of no rows,
of one part and of many, missing pages, extreme scores and scales, lengths that change under a captured graph.  Tolerances: test_gpu_attn_decode_tracked."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, f64  # noqa: E402
from tests.test_gpu_attn_decode_tracked import check, ihip, queries, run  # noqa: E402, F401
from tests.tracked_reference import FORMATS, Cache  # noqa: E402


def in_parts(ihip, q, c):  # noqa: F811
    """Scratch for more than one part of each sequence."""
    ws, heads = ihip.attn_decode_tracked_workspace(q, c.store, c.T), q.shape[0] * q.shape[1]
    assert ws.numel() > heads * 4 * (-(-c.T // 32) * 32 + 130) + 16
    return ws


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("page,Hkv,lens,token_major,missing", [
    (16, 2, [1500, 0, 1, 129, 1025], True, [(0, 3), (0, 93), (3, 0), (3, 8), (4, 20)]),
    (0, 1, [2600], False, []),                       # (21 parts of one head: odd numbers of both)
])
def test_all_rows(ihip, fmt, G, page, Hkv, lens, token_major, missing):  # noqa: F811
    c = Cache(ihip, fmt, lens, Hkv, page, seed=G, token_major=token_major, missing=missing)
    q = queries(len(lens), G * Hkv, 10 + G, scale=2.0)
    ws = in_parts(ihip, q, c)
    for before in (False, True):
        out, lse, w, old = run(ihip, c, q, before=before, decay=0.5, ws=ws)
        check(c, q, out, lse, w, old, 0.5)


@pytest.mark.parametrize("G", [1, 8])
def test_sequences_without_any_page(ihip, G):  # noqa: F811
    """Parts whose rows are all left out, alone and beside others."""
    c = Cache(ihip, "e4m3", [1200, 300, 1100], 1, 64, seed=3, missing=[(0, i) for i in range(19)] + [(2, i) for i in range(3, 15)])
    q = queries(3, G, 4)
    out, lse, w, old = run(ihip, c, q, before=True, ws=in_parts(ihip, q, c))
    check(c, q, out, lse, w, old)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("scale", [0.0, 1e-30, 3.0])
def test_scales(ihip, fmt, scale):  # noqa: F811
    c = Cache(ihip, fmt, [1300, 77], 2, 16, seed=8)
    q = queries(2, 16, 9)
    out, lse, w, old = run(ihip, c, q, scale=scale, ws=in_parts(ihip, q, c))
    check(c, q, out, lse, w, old, scale=scale)


@pytest.mark.parametrize("G", [1, 2, 8])
def test_large_scores_and_values(ihip, G):  # noqa: F811
    """Scores far beyond what an exponential holds in every part, values close to the largest number: one row takes all of each head."""
    c = Cache(ihip, "bf16", [1400], 1, 0, seed=10)
    c.k.mul_(2.0 ** 20)
    c.v.mul_(2.0 ** 124).clamp_(-3e38, 3e38)
    q = queries(1, G, 11, scale=100.0)
    track = ihip.KVTrack(torch.zeros((1, 1, 1400)).cuda())
    out, lse = ihip.attn_decode_tracked(q, c.store, track, c.seq_lens, 1400, fresh=True, want_lse=True, ws=in_parts(ihip, q, c))
    k, v = c.rows(0, 0, np.arange(1400))
    best = (f64(q)[0, :, 0] @ k.T).argmax(axis=1)
    assert (f64(track.weights)[0, 0] == np.bincount(best, minlength=1400)).all()
    assert (np.abs(f64(out)[0, :, 0] - v[best]) <= np.abs(v[best]) * 2.0 ** -8).all()


@pytest.mark.parametrize("G", [1, 4, 8])
def test_captured_and_replayed(ihip, G):  # noqa: F811
    """Lengths that change between replays, from no part to all of them: the bits of the eager call, which are right."""
    T = 1500
    c = Cache(ihip, "bf16", [T, T], 2, 16, seed=13)
    q = queries(2, 2 * G, 14)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        track, ws = ihip.KVTrack(torch.zeros((2, 2, T)).cuda()), in_parts(ihip, q, c)
        out, lse = torch.zeros((2, 2 * G, 1, D), dtype=torch.bfloat16).cuda(), torch.zeros((2, 2 * G, 1)).cuda()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ihip.attn_decode_tracked(q, c.store, track, c.seq_lens, T, out=out, lse=lse, ws=ws)
        for lens in ([1500, 0], [1, 1100], [0, 0], [128, 129], [1500, 1499]):
            c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
            c.lens = lens
            track.weights.fill_(1.0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            other = ihip.KVTrack(torch.ones((2, 2, T)).cuda())
            o, l = ihip.attn_decode_tracked(q, c.store, other, c.seq_lens, T, want_lse=True)
            assert torch.equal(o, out) and torch.equal(l, lse) and torch.equal(other.weights, track.weights)
            check(c, q, o, l, other.weights, torch.ones((2, 2, T)))
            for b, n in enumerate(lens):
                assert bool((track.weights[b, :, n:] == 1).all())
