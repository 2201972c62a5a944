"""A second prompt behind a cache that has been cut: its tokens are appended at rows that are not their positions, attend to what is left and to each
other, and add to the weights of both; then the cache is cut again."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, attention, f64, fp32_turned  # noqa: E402
from tests.test_gpu_tracked_run import SCALE, ihip, junk_store, normal, offsets  # noqa: E402, F401
from tests.tracked_reference import evicted, key_weights  # noqa: E402
from workloads import gen  # noqa: E402


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "mx4"])
@pytest.mark.parametrize("window", [None, 8])
def test_second_prompt(ihip, fmt, window):  # noqa: F811
    """The rows that stand in the cache are read back and compared with what went in (bit for bit in bf16); weights with float64 on them, within the
    tolerances of tracked_reference.key_weights, the old ones with one product and sum more."""
    B, Hq, Hkv, page, keep, n_sink, n_recent = 3, 8, 2, 16, 40, 2, 6
    G, first, second = Hq // Hkv, [90, 33, 64], [50, 1, 29]
    T = keep + max(second) + 60
    store, _ = junk_store(ihip, fmt, B, Hkv, T, page, seed=3)
    cos, sin = gen.rope_table(max(first) + max(second), D)
    tables = (cos.cuda(), sin.cuda())
    track = ihip.KVTrack.empty(B, Hkv, T)
    lens = torch.tensor(first, dtype=torch.int32).cuda()
    track.seen.copy_(lens)
    q, k, v = normal(1, sum(first), Hq, D), normal(2, sum(first), Hkv, D), normal(3, sum(first), Hkv, D)
    q, k = ihip.kv_append(store, k.cuda(), v.cuda(), offsets(first).cuda(), lens, T, q=q.cuda(), rope=tables, k_out=torch.empty_like(k).cuda(), track=track)
    _, lse = ihip.prompt_attn(q, k, v.cuda(), offsets(first).cuda(), max(first), want_lse=True)
    ihip.prompt_key_weights(q, k, offsets(first).cuda(), max(first), lse, track, window=window, fresh=True)
    ihip.kv_evict(store, track, lens, T, keep, n_sink=n_sink, n_recent=n_recent, new_lens=lens)
    cut = [min(t, keep) for t in first]
    assert lens.cpu().tolist() == cut
    left, _ = (x.clone() for x in ihip.kv_gather(store, lens, T))

    # the second prompt
    lens += torch.tensor(second, dtype=torch.int32).cuda()
    track.seen += torch.tensor(second, dtype=torch.int32).cuda()
    total = [a + n for a, n in zip(cut, second)]
    q2, k2, v2 = normal(4, sum(second), Hq, D), normal(5, sum(second), Hkv, D), normal(6, sum(second), Hkv, D)
    q2_out, k2_out = ihip.kv_append(store, k2.cuda(), v2.cuda(), offsets(second).cuda(), lens, T, q=q2.cuda(), rope=tables, k_out=torch.empty_like(k2).cuda(),
                                    track=track)
    rows_k, rows_v = ihip.kv_gather(store, lens, T)                  # [B, Hkv, T, D], as the cache has them
    at = 0
    for b, (n, c) in enumerate(zip(second, cut)):
        assert torch.equal(rows_k[b, :, :c], left[b, :, :c])
        assert torch.equal(track.positions[b, :, c:c + n].cpu(), torch.arange(first[b], first[b] + n, dtype=torch.int32).expand(Hkv, n))
        assert bool((track.weights[b, :, c:c + n] == 0).all())
        for i in range(n):
            for x, y in ((q2, q2_out), (k2, k2_out)):
                want = torch.from_numpy(fp32_turned(f64(x[at + i]), f64(cos[first[b] + i]), f64(sin[first[b] + i]))).float().bfloat16()
                assert torch.equal(y[at + i].cpu(), want)
        if fmt == "bf16":
            assert torch.equal(rows_k[b, :, c:c + n].transpose(0, 1), k2_out[at:at + n])
        at += n
    packed = [torch.cat([x[b, :, :t].transpose(0, 1) for b, t in enumerate(total)]).contiguous() for x in (rows_k, rows_v)]
    cu_q, cu_k = offsets(second).cuda(), offsets(total).cuda()
    out, lse = ihip.prompt_attn(q2_out, *packed, cu_q, max(second), cu_k=cu_k, want_lse=True)
    old = track.weights.clone()
    ihip.prompt_key_weights(q2_out, packed[0], cu_q, max(second), lse, track, cu_k=cu_k, window=window, decay=0.5)
    at, kt = 0, 0
    for b, (n, t) in enumerate(zip(second, total)):
        seen = np.arange(t)[None, :] <= (np.arange(n) + t - n)[:, None]
        for g in range(Hkv):
            Q, K, V = f64(q2_out[at:at + n, g * G:(g + 1) * G]), f64(packed[0][kt:kt + t, g]), f64(packed[1][kt:kt + t, g])
            exact = np.stack([attention(Q[:, h], K, V, SCALE, seen)[1] for h in range(G)], axis=1)
            off = 2.0 ** -17 * SCALE * (np.abs(Q.reshape(-1, D)) @ np.abs(K).T).max()
            given = f64(lse[at:at + n, g * G:(g + 1) * G])
            assert (np.abs(given - exact) <= off + 2.0 ** -20 * (1 + np.abs(exact))).all()
            w, tol = key_weights(Q, K, given, SCALE, G, window or 10 ** 9)
            before = f64(old)[b, g, :t]
            assert (before[cut[b]:] == 0).all()
            assert (np.abs(f64(track.weights)[b, g, :t] - (w + 0.5 * before)) <= tol + 2.0 ** -23 * (w + before)).all()
        assert torch.equal(track.weights[b, :, t:], old[b, :, t:])
        at, kt = at + n, kt + t

    # cut again, by the kernel's own weights
    w, p = track.weights.cpu().numpy().copy(), track.positions.cpu().numpy().copy()
    new, kept = ihip.kv_evict(store, track, lens, T, keep, n_sink=n_sink, n_recent=n_recent)
    again, _ = ihip.kv_gather(store, new, T)
    for b, t in enumerate(total):
        for g in range(Hkv):
            m = evicted(w[b, g], p[b, g], t, keep, n_sink, int(track.seen[b]) - n_recent)
            assert (kept[b, g].cpu().numpy() == m).all()
            m = torch.from_numpy(m[m >= 0]).cuda()
            assert torch.equal(again[b, g, :len(m)], rows_k[b, g, m])
