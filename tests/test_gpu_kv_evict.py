"""Cutting a cache down (ihip_kv_evict) against a plain form: everything it writes is a copy or a number, so all of it is equal, and all
other memory is as it was."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.tracked_reference import FORMATS, Cache, evicted  # noqa: E402


@pytest.fixture(scope="module")
def ihip():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_08910_amd as pkg
    pkg.lib()
    return pkg


def make_track(ihip, c, rows, seed, kind="normal", extra=0):
    """Weights of a kind, positions in any order below the tokens seen."""
    g = torch.Generator().manual_seed(seed)
    shape = (c.B, c.Hkv, rows)
    if kind == "normal":
        w = torch.randn(shape, generator=g).mul(2).exp()
    elif kind == "few":                              # few values: ties everywhere
        w = torch.randint(0, 3, shape, generator=g).float()
    elif kind == "zero":
        w = torch.zeros(shape)
    elif kind == "close":                            # one bin of a histogram
        w = 1.0 + torch.randint(0, 1 << 19, shape, generator=g).float() * 2.0 ** -23
    else:                                            # odd ones
        odd = torch.tensor([0.0, -0.0, 1.0, -1.0, float("nan"), float("inf"), -float("inf"), 1e-42, -1e-42, 3e38, -float("nan")])
        w = odd[torch.randint(0, len(odd), shape, generator=g)]
    seen = torch.tensor([t + extra + 7 * b for b, t in enumerate(c.lens)], dtype=torch.int32)
    pos = torch.zeros(shape, dtype=torch.int32)
    for b, t in enumerate(c.lens):
        for h in range(c.Hkv):
            pos[b, h, :t] = torch.randperm(int(seen[b]), generator=g)[:t].to(torch.int32)
    return ihip.KVTrack(w.cuda(), pos.cuda(), seen.cuda())


def check(ihip, c, track, keep, n_sink, n_recent, in_place, lens_in_place=False):
    raw = c.raw()
    w0, p0 = track.weights.cpu().numpy().copy(), track.positions.cpu().numpy().copy()
    seen = track.seen.cpu().numpy()
    to = None if in_place else ihip.KVTrack(torch.full((c.B, c.Hkv, min(keep, c.T) + 3), 5.0).cuda(), torch.full((c.B, c.Hkv, min(keep, c.T) + 3), -5, dtype=torch.int32).cuda())
    lens = c.seq_lens.clone()
    new, kept = ihip.kv_evict(c.store, track, lens, c.T, keep, n_sink=n_sink, n_recent=n_recent, to=to, new_lens=lens if lens_in_place else None)
    assert new.cpu().tolist() == [min(t, keep) for t in c.lens]
    if not lens_in_place:
        assert lens.cpu().tolist() == list(c.lens)
    to = to or track
    w1, p1, kept = to.weights.cpu().numpy(), to.positions.cpu().numpy(), kept.cpu().numpy()
    want_w, want_p = (w0.copy(), p0.copy()) if in_place else (np.full_like(w1, 5.0), np.full_like(p1, -5))
    want = [x.copy() for x in raw]
    table = None if c.table is None else c.table.cpu().numpy()
    for b, t in enumerate(c.lens):
        for g in range(c.Hkv):
            m = evicted(w0[b, g], p0[b, g], t, keep, n_sink, int(seen[b]) - n_recent)
            assert (kept[b, g] == m).all(), (b, g)
            n = min(t, keep)
            want_w[b, g, :n], want_p[b, g, :n] = w0[b, g, m[:n]], p0[b, g, m[:n]]
            for dst in np.flatnonzero(m[:n] != np.arange(n)):
                src = int(m[dst])
                (ps, js), (pd, jd) = (((b, r) if table is None else (int(table[b, r // c.page]), r % c.page)) for r in (src, int(dst)))
                if ps >= 0 and pd >= 0:
                    for x, y in zip(want, raw):
                        x[pd, g, jd] = y[ps, g, js]
    assert w1.tobytes() == want_w.tobytes() and p1.tobytes() == want_p.tobytes()
    if not in_place:
        assert track.weights.cpu().numpy().tobytes() == w0.tobytes() and track.positions.cpu().numpy().tobytes() == p0.tobytes()
    for x, y in zip(c.raw(), want):
        assert x.tobytes() == y.tobytes()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,Hkv,lens,keep,n_sink,n_recent,token_major", [
    (16, 2, [100, 64, 65, 3, 0], 64, 4, 16, False),
    (0, 3, [257, 1, 2], 1, 0, 0, True),
    (64, 1, [1000], 999, 1, 998, False),
    (1, 2, [130, 90], 70, 0, 10, False),
    (128, 8, [700, 500], 100, 50, 50, True),
    (8, 1, [70, 33], 5000, 4, 4, False),             # nothing to evict
])
def test_evict(ihip, fmt, page, Hkv, lens, keep, n_sink, n_recent, token_major):
    for in_place in (True, False):
        c = Cache(ihip, fmt, lens, Hkv, page, seed=keep + in_place, token_major=token_major)
        check(ihip, c, make_track(ihip, c, c.T + 5, seed=3, extra=10), keep, n_sink, n_recent, in_place, lens_in_place=in_place)


@pytest.mark.parametrize("kind", ["few", "zero", "close", "odd"])
@pytest.mark.parametrize("n,keep", [(90, 20), (4500, 1100), (4500, 4400), (9000, 17), (12345, 5000), (20001, 7000), (33000, 100), (33000, 32990)])
def test_weights_that_tie(ihip, kind, n, keep):
    """Equal weights, all in one bin of the histogram (more than are listed at once too), not finite, negative, tiny."""
    c = Cache(ihip, "mx4", [n, n - 1], 1, 0, seed=n)
    check(ihip, c, make_track(ihip, c, c.T, seed=keep, kind=kind), keep, min(3, keep), min(10, keep - 3), in_place=True)


def test_first_and_last_positions_are_kept(ihip):
    """Whatever they weigh, and wherever they stand."""
    c = Cache(ihip, "bf16", [300], 2, 16, seed=1)
    track = make_track(ihip, c, c.T, seed=2, kind="normal")
    pos = torch.randperm(300, generator=torch.Generator().manual_seed(4)).to(torch.int32).cuda()
    track.positions[:] = pos
    track.seen[:] = 300
    track.weights[:, :, (pos < 8) | (pos >= 290)] = -1.0
    track.weights[:, 0, int((pos == 295).nonzero())] = float("nan")
    new, kept = ihip.kv_evict(c.store, track, c.seq_lens, c.T, 32, n_sink=8, n_recent=10)
    for g in range(2):
        left = set(track.positions[0, g, :32].cpu().tolist())
        assert len(left) == 32 and set(range(8)) | set(range(290, 300)) <= left


@pytest.mark.parametrize("n,keep", [(300, 250), (2000, 700), (20000, 900)])
@pytest.mark.parametrize("shared", ["weights", "positions"])
def test_a_cut_track_that_shares_an_array(ihip, n, keep, shared):
    """One of the two arrays of `to` is that of the track itself, the other one apart."""
    c = Cache(ihip, "e4m3", [n, n // 2], 2, 16, seed=21)
    track = make_track(ihip, c, c.T, seed=22)
    w, p, seen = (x.clone() for x in (track.weights, track.positions, track.seen))
    other = torch.full(w.shape, 7.0 if shared == "positions" else 7, dtype=torch.float32 if shared == "positions" else torch.int32).cuda()
    to = ihip.KVTrack(other, track.positions) if shared == "positions" else ihip.KVTrack(track.weights, other)
    ihip.kv_evict(c.store, track, c.seq_lens, c.T, keep, n_sink=2, n_recent=9, to=to)
    for b, t in enumerate(c.lens):
        for g in range(2):
            m = evicted(w[b, g].cpu().numpy(), p[b, g].cpu().numpy(), t, keep, 2, int(seen[b]) - 9)
            m = torch.from_numpy(m[:min(t, keep)]).long().cuda()
            assert torch.equal(to.weights[b, g, :len(m)], w[b, g, m]) and torch.equal(to.positions[b, g, :len(m)], p[b, g, m])
            assert bool((other[b, g, len(m):] == 7).all())
    assert torch.equal(track.positions if shared == "weights" else track.weights, p if shared == "weights" else w)


def test_more_protected_rows_than_are_kept(ihip):
    """Positions that are not distinct: no more than `keep` rows, the lower ones."""
    c = Cache(ihip, "bf16", [200], 1, 0, seed=1)
    track = make_track(ihip, c, c.T, seed=2)
    track.positions[:] = 0
    check(ihip, c, track, 50, 1, 0, in_place=True)


def test_rows_on_no_page(ihip):
    """A page with id -1 among those that are left, one among those that are evicted from: K and V do not move there."""
    c = Cache(ihip, "e4m3", [200, 150], 2, 16, seed=7, missing=[(0, 1), (0, 9), (1, 8)])
    check(ihip, c, make_track(ihip, c, c.T, seed=8), 64, 2, 20, in_place=True)


def test_lengths_beyond_the_bound(ihip):
    """Of a sequence that says it is longer than max_seq_len, max_seq_len rows count; a negative length is none."""
    c = Cache(ihip, "bf16", [100, 100], 1, 0, seed=1)
    track = make_track(ihip, c, c.T, seed=2)
    w, p, seen = (x.clone() for x in (track.weights, track.positions, track.seen))
    lens = torch.tensor([250, -7], dtype=torch.int32).cuda()
    new, kept = ihip.kv_evict(c.store, track, lens, 90, 40, n_recent=5)
    assert new.cpu().tolist() == [40, 0]
    m = evicted(w[0, 0].cpu().numpy(), p[0, 0].cpu().numpy(), 90, 40, 0, int(seen[0]) - 5)
    assert (kept[0, 0].cpu().numpy() == m).all() and (kept[1] == -1).all()


@pytest.mark.parametrize("Hkv,lens,keep,equal", [(2, [70001, 66000], 20000, False), (1, [262144 + 77], 1000, False), (1, [200003, 4], 50000, True), (1, [140000], 139000, False)])
def test_long(ihip, Hkv, lens, keep, equal):
    """equal: a tenth of the rows has the weight at which the kept ones end."""
    c = Cache(ihip, "mx4", lens, Hkv, 64, seed=5)
    g = torch.Generator().manual_seed(9)
    w = torch.randn((len(lens), Hkv, c.T), generator=g).mul(2).exp()
    if equal:
        w[torch.rand(w.shape, generator=g) < 0.1] = float(w[0, 0].sort(descending=True).values[keep])
    pos = torch.arange(c.T, dtype=torch.int32).repeat(len(lens), Hkv, 1)
    check(ihip, c, ihip.KVTrack(w.cuda(), pos.cuda(), c.seq_lens.clone()), keep, 4, 64, in_place=False)


@pytest.mark.parametrize("most,keep,steps", [([120, 80], 40, ([120, 80], [41, 40], [0, 77])), ([2000, 1500], 700, ([2000, 1500], [699, 1001])),
                                             ([20000, 17000], 3000, ([20000, 17000], [2999, 16500], [20000, 1]))])
def test_captured_and_replayed(ihip, most, keep, steps):
    """A captured call, replayed on lengths and weights that change under it, on a stream of its own; two graphs with scratch of their own.  Few moves,
    many, and rows in chunks."""
    caches = [Cache(ihip, "bf16", most, 2, 16, seed=s) for s in (1, 2)]
    tracks = [make_track(ihip, c, c.T, seed=3) for c in caches]
    fresh = [[x.clone() for x in (c.k, c.v, t.weights, t.positions)] for c, t in zip(caches, tracks)]
    out, graphs = [], []
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for c, t in zip(caches, tracks):
            ws, new, kept = ihip.kv_evict_workspace(c.store, 2, c.T, keep), torch.zeros(2, dtype=torch.int32).cuda(), torch.zeros((2, 2, keep), dtype=torch.int32).cuda()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                ihip.kv_evict(c.store, t, c.seq_lens, c.T, keep, n_sink=2, n_recent=8, new_lens=new, kept=kept, ws=ws)
            graphs.append(graph)
            out.append((new, kept))
        for lens in steps:
            for i in (0, 1, 0):
                c, t = caches[i], tracks[i]
                for x, y in zip((c.k, c.v, t.weights, t.positions), fresh[i]):
                    x.copy_(y)
                c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
                torch.cuda.synchronize()
                graphs[i].replay()
                torch.cuda.synchronize()
                new, kept = out[i]
                assert new.cpu().tolist() == [min(x, keep) for x in lens]
                for b, n in enumerate(lens):
                    for g in range(2):
                        m = evicted(fresh[i][2][b, g].cpu().numpy(), fresh[i][3][b, g].cpu().numpy(), n, keep, 2, int(t.seen[b]) - 8)
                        assert (kept[b, g].cpu().numpy() == m).all()
