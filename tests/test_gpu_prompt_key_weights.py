"""What a prompt's queries attend to (ihip_prompt_key_weights) against float64; the tolerances are those of tracked_reference.key_weights."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, attention, f64  # noqa: E402
from tests.tracked_reference import key_weights  # noqa: E402

SCALE = 1 / np.sqrt(D)


@pytest.fixture(scope="module")
def ihip():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_08910_amd as pkg
    pkg.lib()
    return pkg


def offsets(lens):
    return torch.tensor(np.concatenate(([0], np.cumsum(lens))), dtype=torch.int32)


def inputs(new, total, Hq, Hkv, seed, extra=3):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((sum(new) + extra, Hq, D), generator=g).bfloat16()
    k = torch.randn((sum(total) + extra, Hkv, D), generator=g).bfloat16()
    lse = torch.full((q.shape[0], Hq), 3.0)
    G, q0, k0 = Hq // Hkv, 0, 0
    for n, t in zip(new, total):
        seen = np.arange(t)[None, :] <= (np.arange(n) + t - n)[:, None]
        for h in range(Hq):
            kk = f64(k[k0:k0 + t, h // G])
            lse[q0:q0 + n, h] = torch.from_numpy(attention(f64(q[q0:q0 + n, h]), kk, kk, SCALE, seen)[1]) if t else -float("inf")
        q0, k0 = q0 + n, k0 + t
    return q, k, lse


def check(got, before, decay, q, k, lse, new, total, Hkv, window, rows, scale=SCALE):
    """got [B, Hkv, rows]; before: what it was added to, or 5 where nothing was."""
    G, q0, k0 = q.shape[1] // Hkv, 0, 0
    got, q, k, lse = f64(got), f64(q), f64(k), f64(lse)
    for b, (n, t) in enumerate(zip(new, total)):
        m = min(t, rows)
        for g in range(Hkv):
            w, tol = key_weights(q[q0:q0 + n, g * G:(g + 1) * G], k[k0:k0 + t, g], lse[q0:q0 + n, g * G:(g + 1) * G], scale, G, window)
            old = decay * f64(before)[b, g, :m] if before is not None else 0.0
            assert (np.abs(got[b, g, :m] - (w[:m] + old)) <= tol[:m] + 2.0 ** -23 * (np.abs(old) + w[:m])).all(), (b, g)
        q0, k0 = q0 + n, k0 + t


@pytest.mark.parametrize("Hq,Hkv,new,ctx,window", [
    (8, 2, [5, 0, 1, 33], [0, 0, 0, 0], None),
    (4, 4, [300, 64, 65], [0, 0, 0], None),
    (16, 2, [200, 31, 257], [0, 0, 0], 32),
    (7, 1, [130, 1, 66], [10, 300, 0], None),
    (12, 4, [1, 1, 1], [0, 255, 256], None),
    (8, 8, [513], [0], 1),
    (10, 2, [100, 0], [200, 77], 64),                # (a sequence without new tokens: its keys get nothing)
    (32, 8, [700], [0], 100),
])
def test_against_float64(ihip, Hq, Hkv, new, ctx, window):
    total = [a + b for a, b in zip(new, ctx)]
    q, k, lse = inputs(new, total, Hq, Hkv, seed=Hq)
    rows = max(total) + 2
    own = any(ctx)
    if not own:
        k = k[:q.shape[0]]
    for fresh in (True, False):
        old = torch.rand((len(new), Hkv, rows), generator=torch.Generator().manual_seed(1)) * 10
        track = ihip.KVTrack(old.clone().cuda())
        ihip.prompt_key_weights(q.cuda(), k.cuda(), offsets(new).cuda(), max(new), lse.cuda(), track, cu_k=offsets(total).cuda() if own else None,
                                window=window, fresh=fresh, decay=0.75)
        check(track.weights, None if fresh else old, 0.75, q, k, lse, new, total, Hkv, window or 10 ** 9, rows)
        for b, t in enumerate(total):                # rows behind a sequence's keys
            assert (track.weights[b, :, t:].cpu() == old[b, :, t:]).all()


@pytest.mark.parametrize("Hq,Hkv,window", [(8, 1, None), (6, 2, None), (16, 2, 100)])
def test_wide_blocks_of_keys(ihip, Hq, Hkv, window):
    """What calls of much work take: packed tensors of many rows, bounds to match, and a few short sequences in them."""
    new, rows = [600, 1, 77, 300], 40000
    q, k, lse = inputs(new, new, Hq, Hkv, seed=2, extra=0)
    wide = [torch.full((rows, *x.shape[1:]), float("nan"), dtype=x.dtype).cuda() for x in (q, k, lse)]
    for x, y in zip(wide, (q, k, lse)):
        x[:sum(new)] = y.cuda()
    track = ihip.KVTrack(torch.full((4, Hkv, 610), 5.0).cuda())
    ihip.prompt_key_weights(wide[0], wide[1], offsets(new).cuda(), rows, wide[2], track, window=window, fresh=True)
    check(track.weights, None, 1.0, q, k, lse, new, new, Hkv, window or 10 ** 9, 610)
    for b, n in enumerate(new):
        assert bool((track.weights[b, :, n:] == 5).all())


def test_windows_of_many_keys(ihip):
    """Workgroups that go through several blocks of keys: a call of many rows, with a few short sequences in them."""
    new, rows, Hq = [700, 1, 260], 200000, 8
    q, k, lse = inputs(new, new, Hq, 1, seed=3, extra=0)
    wide = [torch.full((rows, *x.shape[1:]), float("nan"), dtype=x.dtype).cuda() for x in (q, k, lse)]
    for x, y in zip(wide, (q, k, lse)):
        x[:sum(new)] = y.cuda()
    track = ihip.KVTrack(torch.full((3, 1, 710), 5.0).cuda())
    ihip.prompt_key_weights(wide[0], wide[1], offsets(new).cuda(), rows, wide[2], track, window=30, fresh=True)
    check(track.weights, None, 1.0, q, k, lse, new, new, 1, 30, 710)
    for b, n in enumerate(new):
        assert bool((track.weights[b, :, n:] == 5).all())


@pytest.mark.parametrize("max_q,window", [(9, None), (100, None), (9, 2)])
def test_many_sequences(ihip, max_q, window):
    """More sequences than a wave has lanes, empty ones among them; a bound that is loose by much."""
    new, total = [i * 7 % 10 for i in range(150)], [i * 7 % 10 + i * i % 23 for i in range(150)]
    q, k, lse = inputs(new, total, 8, 1, seed=11)
    track = ihip.KVTrack(torch.full((150, 1, 40), 5.0).cuda())
    ihip.prompt_key_weights(q.cuda(), k.cuda(), offsets(new).cuda(), max_q, lse.cuda(), track, cu_k=offsets(total).cuda(), window=window, fresh=True)
    check(track.weights, None, 1.0, q, k, lse, new, total, 1, window or 10 ** 9, 40)
    for b, t in enumerate(total):
        assert bool((track.weights[b, :, t:] == 5).all())


@pytest.mark.parametrize("window", [None, 16])
def test_heads_that_are_one_in_memory(ihip, window):
    """A key head that stands for all of them, a query's heads that are the same."""
    new, Hq, Hkv = [140, 33], 8, 4
    q, k, lse = inputs(new, new, 1, 1, seed=12, extra=0)
    q, k, lse = q.expand(-1, Hq, -1), k.expand(-1, Hkv, -1), lse.expand(-1, Hq).contiguous()
    track = ihip.KVTrack(torch.zeros((2, Hkv, 140)).cuda())
    ihip.prompt_key_weights(q[:, :1].cuda().expand(-1, Hq, -1), k[:, :1].cuda().expand(-1, Hkv, -1), offsets(new).cuda(), 140, lse.cuda(), track, window=window,
                            fresh=True)
    check(track.weights, None, 1.0, q, k, lse, new, new, Hkv, window or 10 ** 9, 140)


@pytest.mark.parametrize("window", [None, 40])
def test_sequences_longer_than_max_q(ihip, window):
    """They may be done in part; the others are not."""
    new, Hq, Hkv = [30, 500, 40], 8, 2
    q, k, lse = inputs(new, new, Hq, Hkv, seed=9)
    k = k[:q.shape[0]]
    track = ihip.KVTrack(torch.full((3, Hkv, 510), 5.0).cuda())
    ihip.prompt_key_weights(q.cuda(), k.cuda(), offsets(new).cuda(), 40, lse.cuda(), track, window=window, fresh=True)
    whole = ihip.KVTrack(torch.full((3, Hkv, 510), 5.0).cuda())
    ihip.prompt_key_weights(q.cuda(), k.cuda(), offsets(new).cuda(), 500, lse.cuda(), whole, window=window, fresh=True)
    for b in (0, 2):
        assert (track.weights[b] - whole.weights[b]).abs().max() <= 2.0 ** -12          # (sums in another order)
    assert bool((track.weights[1, :, :500] <= whole.weights[1, :, :500] + 2.0 ** -12).all()) and bool((track.weights[1, :, 500:] == 5).all())


def test_chunks_of_queries(ihip):
    """Many queries on few keys, in chunks whose sums are added up, and without scratch: equal up to rounding, and the same bits each time."""
    new, Hq, Hkv = [2500, 1200], 8, 1
    q, k, lse = inputs(new, new, Hq, Hkv, seed=1)
    k = k[:q.shape[0]]
    args = (q.cuda(), k.cuda(), offsets(new).cuda(), max(new), lse.cuda())
    got = []
    for ws in (None, None, torch.empty(0, dtype=torch.uint8).cuda()):
        track = ihip.KVTrack(torch.zeros((2, Hkv, 2500)).cuda())
        ihip.prompt_key_weights(*args, track, fresh=True, ws=ws)
        check(track.weights, None, 1.0, q, k, lse, new, new, Hkv, 10 ** 9, 2500)
        got.append(track.weights.cpu())
    assert torch.equal(got[0], got[1])
    assert not torch.equal(got[0], got[2])           # (the two ways were taken)


def test_the_attention_s_own_sums(ihip):
    """With the log-sum-exp of ihip_prompt_attn every query's probabilities add up to 1 for each head."""
    new, Hq, Hkv = [333, 64, 1], 16, 4
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn((sum(new), h, D), generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    cu = offsets(new).cuda()
    _, lse = ihip.prompt_attn(q, k, v, cu, max(new), want_lse=True)
    track = ihip.KVTrack(torch.zeros((3, Hkv, 333)).cuda())
    ihip.prompt_key_weights(q, k, cu, max(new), lse, track, fresh=True)
    for b, n in enumerate(new):
        sums = track.weights[b].double().sum(dim=1).cpu()
        # log-sum-exp and scores in fp32, as in key_weights: a probability is off by 2^-17 of sum |q k| / sqrt(d) (about 7.2 here, 20 at most)
        assert (sums / (n * Hq / Hkv) - 1).abs().max() <= 2 * 20 * 2.0 ** -17


def test_masked_keys_and_unused_rows(ihip):
    """NaN in rows behind the sequences, and in keys that only later queries see."""
    new, Hq, Hkv = [100, 50], 4, 2
    q, k, lse = inputs(new, new, Hq, Hkv, seed=3)
    k = k[:q.shape[0]]
    q[150:], k[150:], lse[150:] = float("nan"), float("nan"), float("nan")
    k[99] = float("nan")                             # the first sequence's last key: seen by its last query alone
    track = ihip.KVTrack(torch.zeros((2, Hkv, 100)).cuda())
    ihip.prompt_key_weights(q.cuda(), k.cuda(), offsets(new).cuda(), 100, lse.cuda(), track, fresh=True)
    w = track.weights.cpu()
    assert bool(w[0, :, 99].isnan().all())
    # the other keys as without any of that (the last query's log-sum-exp is given as it was)
    track2 = ihip.KVTrack(torch.zeros((2, Hkv, 100)).cuda())
    q3, k3, l3 = inputs(new, new, Hq, Hkv, seed=3)
    ihip.prompt_key_weights(q3.cuda(), k3[:q3.shape[0]].cuda(), offsets(new).cuda(), 100, l3.cuda(), track2, fresh=True)
    assert torch.equal(w[0, :, :99], track2.weights.cpu()[0, :, :99]) and torch.equal(w[1], track2.weights.cpu()[1])


def test_queries_without_keys(ihip):
    """More queries than keys: the first ones see none and have a log-sum-exp of -infinity."""
    new, total, Hq, Hkv = [40], [10], 4, 1
    q, k, lse = inputs(new, total, Hq, Hkv, seed=4)
    assert bool((lse[:30] == -float("inf")).all())
    track = ihip.KVTrack(torch.zeros((1, 1, 12)).cuda())
    ihip.prompt_key_weights(q.cuda(), k.cuda(), offsets(new).cuda(), 40, lse.cuda(), track, cu_k=offsets(total).cuda(), fresh=True)
    check(track.weights, None, 1.0, q, k, lse, new, total, Hkv, 10 ** 9, 12)


def test_no_queries_at_all(ihip):
    """Keys, and no new tokens in any sequence: what was there fades."""
    k = torch.randn((50, 2, D), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    old = torch.rand((2, 2, 40), generator=torch.Generator().manual_seed(2))
    track = ihip.KVTrack(old.clone().cuda())
    ihip.prompt_key_weights(torch.zeros((0, 8, D), dtype=torch.bfloat16).cuda(), k, offsets([0, 0]).cuda(), 0, torch.zeros((0, 8)).cuda(), track,
                            cu_k=offsets([30, 20]).cuda(), decay=0.5)
    want = old.clone()
    want[0, :, :30] *= 0.5
    want[1, :, :20] *= 0.5
    assert torch.equal(track.weights.cpu(), want)


def test_strides_and_fewer_rows_than_keys(ihip):
    """Queries and keys inside wider tensors; a track of fewer rows than a sequence has keys."""
    new, Hq, Hkv = [130, 70], 8, 2
    q, k, lse = inputs(new, new, Hq, Hkv, seed=5)
    k = k[:q.shape[0]]
    wide = torch.full((q.shape[0], Hq + 2 * Hkv + 1, D + 8), float("nan"), dtype=torch.bfloat16).cuda()
    wide[:, :Hq, :D], wide[:, Hq:Hq + Hkv, :D] = q.cuda(), k.cuda()
    old = torch.full((2, Hkv, 100), 5.0)
    track = ihip.KVTrack(old.clone().cuda())
    ihip.prompt_key_weights(wide[:, :Hq, :D], wide[:, Hq:Hq + Hkv, :D], offsets(new).cuda(), 130, lse.cuda(), track)
    check(track.weights, old, 1.0, q, k, lse, new, new, Hkv, 10 ** 9, 100)


def test_captured_and_replayed(ihip):
    """On a stream of its own, with lengths that change under the graph, and a loose bound of them."""
    Hq, Hkv = 8, 2
    q, k, lse = inputs([90, 60], [90, 60], Hq, Hkv, seed=6, extra=0)
    q2, k2, lse2 = inputs([20, 130], [20, 130], Hq, Hkv, seed=7, extra=0)
    dev = [x.clone().cuda() for x in (q, k, lse)]
    cu = offsets([90, 60]).cuda()
    track = ihip.KVTrack(torch.zeros((2, Hkv, 150)).cuda())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        ws = torch.empty(1 << 20, dtype=torch.uint8).cuda()
        with torch.cuda.graph(graph, stream=stream):
            ihip.prompt_key_weights(dev[0], dev[1], cu, 150, dev[2], track, fresh=True, ws=ws)
        for new, src in (([90, 60], (q, k, lse)), ([20, 130], (q2, k2, lse2)), ([90, 60], (q, k, lse))):
            for x, y in zip(dev, src):
                x.copy_(y)
            cu.copy_(offsets(new))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            check(track.weights, None, 1.0, *src, new, new, Hkv, 10 ** 9, 150)
