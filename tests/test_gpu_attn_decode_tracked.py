"""Decode attention over all rows of a cache of any format, with the rows' weights (ihip_attn_decode_tracked), against float64 on the values
that the rows stand for.

Tolerances.  Rows are widened exactly; scores are off by at most 2^-17 of sum |q_i k_i| (128 products and sums of fp32), which moves a probability and
the sum that it is divided by by as much, relative.  The probabilities go into the output with 16 bits, the result is rounded to bf16; into the
weights they go as they are: exp2 and its argument, at most 64 in magnitude where it counts, 2^-17."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, attention, f64  # noqa: E402
from tests.tracked_reference import FORMATS, Cache  # noqa: E402

SCALE = 1 / np.sqrt(D)


@pytest.fixture(scope="module")
def ihip():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_08910_amd as pkg
    pkg.lib()
    return pkg


def queries(B, Hq, seed, scale=1.0):
    return (torch.randn((B, Hq, 1, D), generator=torch.Generator().manual_seed(seed)) * scale).bfloat16().cuda()


def check(c, q, out, lse, weights, before, decay=1.0, scale=SCALE):
    B, Hq = q.shape[:2]
    G = Hq // c.Hkv
    q, out, lse, weights = f64(q), f64(out), f64(lse), f64(weights)
    before = f64(before) if before is not None else None
    for b in range(B):
        r = np.arange(c.lens[b])
        on = c.there(b, r)
        for g in range(c.Hkv):
            Q = q[b, g * G:(g + 1) * G, 0]
            k, v = c.rows(b, g, r[on]) if on.any() else (np.zeros((0, D)), np.zeros((0, D)))
            seen = np.ones((G, len(k)), dtype=bool)
            want, want_lse = attention(Q, k, v, scale, seen)
            mag, _ = attention(Q, k, np.abs(v), scale, seen)
            off = 2.0 ** -17 * scale * (np.abs(Q) @ np.abs(k).T).max(axis=1, initial=0)
            got, got_lse = out[b, g * G:(g + 1) * G, 0], lse[b, g * G:(g + 1) * G, 0]
            lost = 2.0 ** -99 * np.abs(v).sum(axis=0)            # (exponentials below 2^-126, of 2^-26 for the largest)
            assert (np.abs(got - want) <= mag * (2.0 ** -15 + 2 * off)[:, None] + np.abs(want) * 2.0 ** -8 + lost).all(), (b, g, np.abs(got - want).max())
            w = np.zeros(len(r))
            tol = np.zeros(len(r))
            if len(k):
                assert (np.abs(got_lse - want_lse) <= off + 2.0 ** -20 * (1 + np.abs(want_lse))).all(), (b, g)
                p = np.exp(Q @ k.T * scale - want_lse[:, None])
                w[on], tol[on] = p.sum(axis=0), (p * (2 * off + 2.0 ** -17)[:, None]).sum(axis=0) + 2.0 ** -120
            else:
                assert (got_lse == -np.inf).all() and (got == 0).all()
            old = 0.0 if before is None else decay * before[b, g, :len(r)]
            assert (np.abs(weights[b, g, :len(r)] - (w + old)) <= tol + 2.0 ** -23 * (np.abs(old) + w)).all(), (b, g)


def run(ihip, c, q, rows=None, before=False, decay=1.0, scale=None, **kw):
    """-> out, lse, weights, what they were added to; rows behind the sequences are looked at here."""
    rows = rows or c.T + 3
    old = torch.rand((c.B, c.Hkv, rows), generator=torch.Generator().manual_seed(5)) * 3
    track = ihip.KVTrack(old.clone().cuda())
    out, lse = ihip.attn_decode_tracked(q, c.store, track, c.seq_lens, c.T, sm_scale=scale, fresh=not before, decay=decay, want_lse=True, **kw)
    for b, t in enumerate(c.lens):
        assert (track.weights[b, :, t:].cpu() == old[b, :, t:]).all()
    return out, lse, track.weights, old if before else None


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("page,Hkv,lens,token_major", [(0, 2, [1, 0, 31, 32, 33], True), (16, 8, [500, 129, 15], False), (1, 1, [70], False), (64, 3, [1000, 128, 64, 63], True)])
def test_all_rows(ihip, fmt, G, page, Hkv, lens, token_major):
    c = Cache(ihip, fmt, lens, Hkv, page, seed=G, token_major=token_major)
    q = queries(len(lens), G * Hkv, 10 + G, scale=2.0)
    for before in (False, True):
        out, lse, w, old = run(ihip, c, q, before=before, decay=0.5)
        check(c, q, out, lse, w, old, 0.5)


@pytest.mark.parametrize("fmt", FORMATS)
def test_long_and_ragged(ihip, fmt):
    """Parts of many rows, sequences shorter than a part among them."""
    lens = [20011, 3, 9000] if fmt != "mx4" else [20011] + [50] * 19         # (the latter: parts of as many rows as there may be)
    c = Cache(ihip, fmt, lens, 1, 32, seed=2)
    q = queries(len(lens), 4, 3, scale=2.0)
    out, lse, w, old = run(ihip, c, q, before=True)
    check(c, q, out, lse, w, old)


def test_many_sequences(ihip):
    """More problems than places: one part each, nothing to join."""
    lens = [(i * 37) % 200 for i in range(60)]
    c = Cache(ihip, "e4m3", lens, 8, 16, seed=4)
    q = queries(60, 8, 5)
    out, lse, w, old = run(ihip, c, q)
    check(c, q, out, lse, w, old)


def test_more_problems_than_a_grid_has_rows(ihip):
    """8,200 sequences of 8 KV heads: the same bits as in calls of fewer of them."""
    B, Hkv, Hq, T = 8200, 8, 16, 4
    g = torch.Generator().manual_seed(31)
    k, v = (torch.randn((B, Hkv, T, D), generator=g).bfloat16().cuda() for _ in range(2))
    lens = torch.randint(0, T + 1, (B,), generator=g).to(torch.int32).cuda()
    q = queries(B, Hq, 32)
    old = torch.rand((B, Hkv, T), generator=g).cuda()
    track = ihip.KVTrack(old.clone())
    out, lse = ihip.attn_decode_tracked(q, ihip.KVStore.bf16(k, v), track, lens, T, want_lse=True)
    for b0 in range(0, B, 2050):
        b1 = b0 + 2050
        part = ihip.KVTrack(old[b0:b1].clone())
        o, l = ihip.attn_decode_tracked(q[b0:b1], ihip.KVStore.bf16(k[b0:b1], v[b0:b1]), part, lens[b0:b1].clone(), T, want_lse=True)
        assert torch.equal(o, out[b0:b1]) and torch.equal(l, lse[b0:b1]) and torch.equal(part.weights, track.weights[b0:b1])


def test_heads_that_are_one_in_memory(ihip):
    """K and V heads that stand for all of them, a query that is that of all sequences: what copies of them give."""
    lens = torch.tensor([777, 64], dtype=torch.int32).cuda()
    k, v = (queries(2, 800, s).view(2, 1, 800, D) for s in (33, 34))
    q = queries(1, 8, 35)
    got = []
    for copies in (False, True):
        a, b, x = k.expand(-1, 4, -1, -1), v.expand(-1, 4, -1, -1), q.expand(2, -1, -1, -1)
        if copies:
            a, b, x = a.contiguous(), b.contiguous(), x.contiguous()
        track = ihip.KVTrack(torch.zeros((2, 4, 800)).cuda())
        got.append((*ihip.attn_decode_tracked(x, ihip.KVStore.bf16(a, b), track, lens, 800, want_lse=True), track.weights))
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_on_no_page(ihip, fmt):
    c = Cache(ihip, fmt, [100, 40, 33], 2, 16, seed=6, missing=[(0, 2), (1, 0), (1, 1), (1, 2), (2, 2)])
    q = queries(3, 8, 7)
    out, lse, w, old = run(ihip, c, q, before=True, decay=0.25)
    check(c, q, out, lse, w, old, 0.25)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("scale", [0.0, 1e-30, 0.5, 3.0])
def test_scales(ihip, fmt, scale):
    """From the mean of all rows to one row that takes everything."""
    c = Cache(ihip, fmt, [300, 77], 2, 16, seed=8)
    q = queries(2, 4, 9)
    out, lse, w, old = run(ihip, c, q, scale=scale)
    check(c, q, out, lse, w, old, scale=scale)


def test_large_scores_and_values(ihip):
    """Scores far beyond what an exponential holds, values close to the largest number."""
    c = Cache(ihip, "bf16", [400], 1, 0, seed=10)
    c.k.mul_(2.0 ** 20)
    c.v.mul_(2.0 ** 124).clamp_(-3e38, 3e38)
    q = queries(1, 2, 11, scale=100.0)
    track = ihip.KVTrack(torch.zeros((1, 1, 400)).cuda())
    out, lse = ihip.attn_decode_tracked(q, c.store, track, c.seq_lens, 400, fresh=True, want_lse=True)
    # differences between scores are 2^20 and more: one row takes all of each head
    k, v = c.rows(0, 0, np.arange(400))
    best = (f64(q)[0, :, 0] @ k.T).argmax(axis=1)
    w = np.bincount(best, minlength=400).astype(float)
    assert (f64(track.weights)[0, 0] == w).all()
    assert (np.abs(f64(out)[0, :, 0] - v[best]) <= np.abs(v[best]) * 2.0 ** -8).all()


def test_probabilities_add_up(ihip):
    """Over steps whose old weights stay: each adds 1 a query head."""
    c = Cache(ihip, "mx4", [2000, 321], 2, 16, seed=12)
    track = ihip.KVTrack.empty(2, 2, 2000)
    for step in range(5):
        ihip.attn_decode_tracked(queries(2, 8, step), c.store, track, c.seq_lens, 2000)
    sums = f64(track.weights).sum(axis=2)
    assert (np.abs(sums - 20.0) <= 20 * 2.0 ** -16).all()


def test_captured_and_replayed(ihip):
    """Lengths that change under the graph, two graphs with scratch of their own, on a stream of its own; the same bits as the eager call."""
    caches = [Cache(ihip, fmt, [700, 300], 2, 16, seed=13) for fmt in ("bf16", "e4m3")]
    q = queries(2, 8, 14)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        made = []
        for c in caches:
            track, ws = ihip.KVTrack(torch.zeros((2, 2, 700)).cuda()), ihip.attn_decode_tracked_workspace(q, c.store, 700)
            out, lse = torch.zeros((2, 8, 1, D), dtype=torch.bfloat16).cuda(), torch.zeros((2, 8, 1)).cuda()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                ihip.attn_decode_tracked(q, c.store, track, c.seq_lens, 700, out=out, lse=lse, ws=ws)
            made.append((track, out, lse, graph))
        for lens in ([700, 300], [1, 0], [333, 129], [700, 300]):
            for c, (track, out, lse, graph) in zip(caches, made):
                c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
                track.weights.fill_(1.0)
                torch.cuda.synchronize()
                graph.replay()
                torch.cuda.synchronize()
                other = ihip.KVTrack(torch.ones((2, 2, 700)).cuda())
                o, l = ihip.attn_decode_tracked(q, c.store, other, c.seq_lens, 700, want_lse=True)
                assert torch.equal(o, out) and torch.equal(l, lse) and torch.equal(other.weights, track.weights)
