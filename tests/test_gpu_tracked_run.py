"""Appending into caches whose rows are evicted (ihip_kv_append_tracked), and all of it together as a serving program runs it."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, attention, f64, fp32_turned  # noqa: E402
from tests.tracked_reference import evicted  # noqa: E402
from workloads import gen  # noqa: E402

SCALE = 1 / np.sqrt(D)


@pytest.fixture(scope="module")
def ihip():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_08910_amd as pkg
    pkg.lib()
    return pkg


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).bfloat16()


def offsets(new):
    return torch.tensor(np.concatenate(([0], np.cumsum(new))), dtype=torch.int32)


def junk_store(ihip, fmt, B, Hkv, T, page, seed=0):
    g = torch.Generator().manual_seed(seed)
    table, n = None, B
    if page:
        per = -(-T // page)
        n = B * per + 1
        table = torch.randperm(n, generator=g)[:B * per].to(torch.int32).view(B, per).contiguous().cuda()
    shape = (n, Hkv, page or T)
    if fmt == "bf16":
        k, v = (torch.randn((*shape, D), generator=g).bfloat16().cuda() for _ in range(2))
        return ihip.KVStore.bf16(k, v, table), (k, v)
    if fmt == "e4m3":
        k, v = (torch.randint(0, 120, (*shape, D), generator=g, dtype=torch.uint8).cuda() for _ in range(2))
        return ihip.KVStore.e4m3(k, v, (1 / 64, 0.0131), table), (k, v)
    k, v = (torch.randint(0, 256, (*shape, D // 2), generator=g, dtype=torch.uint8).cuda() for _ in range(2))
    ks, vs = (torch.randint(100, 140, (*shape, 4), generator=g, dtype=torch.uint8).cuda() for _ in range(2))
    return ihip.KVStore.mx4(k, v, ks, vs, table), (k, v, ks, vs)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "mx4"])
@pytest.mark.parametrize("page,Hq,Hkv,new,ctx,gone", [
    (0, 8, 2, [5, 0, 1, 33], [0, 7, 40, 3], [0, 11, 500, 60]),
    (16, 8, 8, [1, 1, 1, 1], [0, 15, 16, 31], [9, 0, 100, 900]),
    (64, 7, 1, [130, 1], [0, 63], [1, 2]),
])
@pytest.mark.parametrize("rope", [True, False])
def test_append_goes_on_from_the_tokens_seen(ihip, fmt, page, Hq, Hkv, new, ctx, gone, rope):
    """Rows as ihip_kv_append writes them for tokens that it is given turned already; a rotated token's bits are those of the rotation to its
    position (fp32, each product and sum rounded)."""
    B, N, total = len(new), sum(new), [a + b for a, b in zip(new, ctx)]
    T = max(total)
    q, k, v = normal(1, N + 3, Hq, D), normal(2, N + 3, Hkv, D), normal(3, N + 3, Hkv, D)
    cos, sin = gen.rope_table(T + max(gone), D)
    tables = (cos.cuda(), sin.cuda())
    lens, seen = torch.tensor(total, dtype=torch.int32).cuda(), torch.tensor([t + x for t, x in zip(total, gone)], dtype=torch.int32).cuda()
    w0, p0 = torch.full((B, Hkv, T + 2), 3.5), torch.full((B, Hkv, T + 2), -9, dtype=torch.int32)
    track = ihip.KVTrack(w0.clone().cuda(), p0.clone().cuda(), seen)
    store, mem = junk_store(ihip, fmt, B, Hkv, T, page)
    q_out, k_out = (torch.full((N + 3, h, D), 5.0, dtype=torch.bfloat16).cuda() for h in (Hq, Hkv))
    ihip.kv_append(store, k.cuda(), v.cuda(), offsets(new).cuda(), lens, T, q=q.cuda(), rope=tables if rope else None, q_out=q_out, k_out=k_out, track=track)
    # the same through sequences that hold everything: a table whose row r is that of position r + gone
    for b in range(B):
        t0 = int(offsets(new)[b])
        for i in range(new[b]):
            row, pos = ctx[b] + i, ctx[b] + i + gone[b]
            w0[b, :, row], p0[b, :, row] = 0.0, pos
            if rope:
                for x, y in ((q[t0 + i], q_out[t0 + i]), (k[t0 + i], k_out[t0 + i])):
                    want = torch.from_numpy(fp32_turned(f64(x), f64(cos[pos]), f64(sin[pos]))).float().bfloat16()
                    assert torch.equal(y.cpu(), want)
    assert torch.equal(track.weights.cpu(), w0) and torch.equal(track.positions.cpu(), p0)
    assert bool((q_out[N:] == 5).all()) and bool((k_out[N:] == 5).all())
    other, mem2 = junk_store(ihip, fmt, B, Hkv, T, page)
    for b in range(B):                               # sequence by sequence, with its own part of the table
        if new[b] == 0:
            continue
        t0 = int(offsets(new)[b])
        cu = torch.zeros(B + 1, dtype=torch.int32)
        cu[b + 1:] = new[b]
        part = tuple(x[gone[b]:gone[b] + T].contiguous() for x in tables) if rope else None
        ihip.kv_append(other, k[t0:t0 + new[b]].cuda(), v[t0:t0 + new[b]].cuda(), cu.cuda(), lens, T, rope=part)
    for x, y in zip(mem, mem2):
        assert torch.equal(x, y)


def test_tokens_that_are_dropped(ihip):
    """Rows or positions out of range, pages that are not there: nothing is written."""
    store, mem = junk_store(ihip, "bf16", 4, 2, 32, 16)
    store.block_table[2, 0] = -1
    before = [m.clone() for m in mem]
    lens = torch.tensor([33, 5, 4, 3], dtype=torch.int32).cuda()             # the first one's second token is row 32
    seen = torch.tensor([40, 1, 9, 65], dtype=torch.int32).cuda()            # the second one's first token is at -1, the last one's second at 64
    track = ihip.KVTrack(torch.full((4, 2, 32), 7.0).cuda(), torch.full((4, 2, 32), -3, dtype=torch.int32).cuda(), seen)
    cos, sin = (t.cuda() for t in gen.rope_table(64, D))
    k, v = normal(1, 8, 2, D).cuda(), normal(2, 8, 2, D).cuda()
    q_out = torch.full((8, 4, D), 5.0, dtype=torch.bfloat16).cuda()
    ihip.kv_append(store, k, v, offsets([2, 2, 2, 2]).cuda(), lens, 32, q=normal(3, 8, 4, D).cuda(), rope=(cos, sin), q_out=q_out, track=track)
    w, p = torch.full((4, 2, 32), 7.0), torch.full((4, 2, 32), -3, dtype=torch.int32)
    for b, row, pos in ((0, 31, 38), (1, 4, 0), (3, 1, 63)):
        w[b, :, row], p[b, :, row] = 0.0, pos
    assert torch.equal(track.weights.cpu(), w) and torch.equal(track.positions.cpu(), p)
    written = [i for i in range(8) if not bool((q_out[i] == 5).all())]
    assert written == [0, 3, 4, 5, 6]                # (tokens 4 and 5 have a place and no page)
    for m, m0 in zip(mem, before):
        rows = {(int(store.block_table[b, r // 16]), r % 16) for b, r in ((0, 31), (1, 4), (3, 1))}
        changed = {(int(i), int(j)) for i, _, j in (m != m0).any(dim=3).nonzero().cpu().tolist()}
        assert changed == rows


def test_prompts_then_steps_with_evictions(ihip):
    """Prompts into pages, their weights, a first cut; then steps that append, attend and, now and then, cut again.  Beside it a float64 program that
    keeps a list of (position, key, value, weight) a head: what is kept is compared through the positions, outputs and weights within the
    tolerances of the single calls (weights add up: so do theirs)."""
    B, Hq, Hkv, page, keep, n_sink, n_recent, slack, window = 2, 4, 2, 16, 48, 2, 8, 8, 16
    G, prompts, steps = Hq // Hkv, [100, 71], 30
    T = max(prompts)
    store, _ = junk_store(ihip, "bf16", B, Hkv, T, page, seed=3)
    cos, sin = gen.rope_table(max(prompts) + steps, D)
    tables = (cos.cuda(), sin.cuda())
    track = ihip.KVTrack.empty(B, Hkv, T)
    lens = torch.tensor(prompts, dtype=torch.int32).cuda()
    track.seen.copy_(lens)
    N, cu = sum(prompts), offsets(prompts).cuda()
    q, k, v = normal(1, N, Hq, D).cuda(), normal(2, N, Hkv, D).cuda(), normal(3, N, Hkv, D).cuda()
    q, k_turned = ihip.kv_append(store, k, v, cu, lens, T, q=q, rope=tables, k_out=torch.empty_like(k), track=track)
    _, lse = ihip.prompt_attn(q, k_turned, v, cu, T, want_lse=True)
    ihip.prompt_key_weights(q, k_turned, cu, T, lse, track, window=window, fresh=True)

    rows = [[[] for _ in range(Hkv)] for _ in range(B)]              # (position, key, value, weight), in the cache's order
    for b in range(B):
        t0 = sum(prompts[:b])
        seen = np.arange(prompts[b])[None, :] <= np.arange(prompts[b])[:, None]
        for g in range(Hkv):
            K, V = f64(k_turned[t0:t0 + prompts[b], g]), f64(v[t0:t0 + prompts[b], g])
            W = np.zeros(prompts[b])
            for h in range(g * G, (g + 1) * G):
                Q = f64(q[t0:t0 + prompts[b], h])
                _, l = attention(Q, K, V, SCALE, seen)
                W += np.where(seen, np.exp(Q @ K.T * SCALE - l[:, None]), 0.0)[-window:].sum(axis=0)
            rows[b][g] = [[i, K[i], V[i], W[i]] for i in range(prompts[b])]

    def cut():
        n = [len(rows[b][0]) for b in range(B)]
        w, p = track.weights.cpu().numpy().copy(), track.positions.cpu().numpy().copy()
        ihip.kv_evict(store, track, lens, T, keep, n_sink=n_sink, n_recent=n_recent, new_lens=lens)
        for b in range(B):
            for g in range(Hkv):
                # the kernel's own weights choose (a near tie may fall either way in float64), and they are close to the program's
                assert np.abs(w[b, g, :n[b]] - [r[3] for r in rows[b][g]]).max() <= 1e-3
                assert p[b, g, :n[b]].tolist() == [r[0] for r in rows[b][g]]
                m = evicted(w[b, g], p[b, g], n[b], keep, n_sink, int(track.seen[b]) - n_recent)
                rows[b][g] = [rows[b][g][i] for i in m[m >= 0]]

    cut()
    for step in range(steps):
        lens += 1
        track.seen += 1
        q, k, v = normal(10 + step, B, Hq, D).cuda(), normal(100 + step, B, Hkv, D).cuda(), normal(200 + step, B, Hkv, D).cuda()
        q, k = ihip.kv_append(store, k, v, offsets([1] * B).cuda(), lens, T, q=q, rope=tables, k_out=torch.empty_like(k), track=track)
        out, lse = ihip.attn_decode_tracked(q.view(B, Hq, 1, D), store, track, lens, T, want_lse=True)
        for b in range(B):
            for g in range(Hkv):
                rows[b][g].append([prompts[b] + step, f64(k[b, g]), f64(v[b, g]), 0.0])
                K, V = np.stack([r[1] for r in rows[b][g]]), np.stack([r[2] for r in rows[b][g]])
                Q, seen = f64(q[b, g * G:(g + 1) * G]), np.ones((G, len(K)), dtype=bool)
                want, l = attention(Q, K, V, SCALE, seen)
                mag, _ = attention(Q, K, np.abs(V), SCALE, seen)
                off = 2.0 ** -17 * SCALE * (np.abs(Q) @ np.abs(K).T).max()
                assert (np.abs(f64(out)[b, g * G:(g + 1) * G, 0] - want) <= mag * (2.0 ** -15 + 2 * off) + np.abs(want) * 2.0 ** -8).all()
                for r, w in zip(rows[b][g], np.exp(Q @ K.T * SCALE - l[:, None]).sum(axis=0)):
                    r[3] += w
        if (step + 1) % slack == 0:
            cut()
    assert track.seen.cpu().tolist() == [p + steps for p in prompts]
    assert lens.cpu().tolist() == [keep + steps % slack] * B


def test_two_streams_at_once(ihip):
    """Two caches in the hands of two streams, step by step without a wait between them, and the same one after the other: the same bits."""
    B, Hq, Hkv, T, keep = 2, 8, 2, 400, 300
    lens0, results = [400, 333], []
    for streams in (1, 2):
        runs = []
        pool = [torch.cuda.Stream() for _ in range(streams)]
        for i in range(2):
            store, mem = junk_store(ihip, "e4m3", B, Hkv, T, 16, seed=i)
            g = torch.Generator().manual_seed(20 + i)
            track = ihip.KVTrack(torch.rand((B, Hkv, T), generator=g).cuda(), torch.arange(T, dtype=torch.int32).repeat(B, Hkv, 1).cuda(),
                                 torch.tensor(lens0, dtype=torch.int32).cuda())
            runs.append([store, mem, track, torch.tensor(lens0, dtype=torch.int32).cuda(), None])
        qs = [normal(30 + s, B, Hq, 1, D).cuda() for s in range(4)]
        torch.cuda.synchronize()
        for q in qs:
            for i, run in enumerate(runs):
                store, mem, track, lens, _ = run
                with torch.cuda.stream(pool[i % streams]):
                    run[4] = ihip.attn_decode_tracked(q, store, track, lens, T, want_lse=True)
                    ihip.kv_evict(store, track, lens, T, keep, n_sink=2, n_recent=20, new_lens=lens)
        torch.cuda.synchronize()
        results.append([[x.cpu() for x in (*run[1], run[2].weights, run[2].positions, run[3], *run[4])] for run in runs])
    for a, b in zip(*results):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
