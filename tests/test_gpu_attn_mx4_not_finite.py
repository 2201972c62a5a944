"""4-bit decode attention over groups that are NaN (scale byte 255), whatever codes stand there: a key with one makes all results of its
KV head's queries NaN, a value with one the 32 dimensions of the group; everything else is as it would be without
(test_gpu_attn_mx4's tolerances)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, attention, f64  # noqa: E402
from tests.test_gpu_attn_mx4 import SCALE, Cache, ihip, positions, queries  # noqa: E402, F401


def check_nan(c, q, out, lse, n_sink, n_stream, starts=None, block=1):
    """As test_gpu_attn_mx4.check, with NaN where something that is attended to is NaN."""
    Hkv = c.k.shape[1]
    G = q.shape[1] // Hkv
    q, out, lse = f64(q), f64(out), f64(lse)
    found = 0
    for b in range(q.shape[0]):
        for g in range(Hkv):
            pos = positions(c.lens[b], n_sink, n_stream, [] if starts is None else starts[b * Hkv + g].tolist(), block)
            k, v = c.rows(b, g, pos)
            got, got_lse = out[b, g * G:(g + 1) * G, 0], lse[b, g * G:(g + 1) * G, 0]
            if np.isnan(k).any():
                assert np.isnan(got).all() and np.isnan(got_lse).all(), (b, g)
                found += 1
                continue
            bad = np.isnan(v).any(axis=0)
            found += bad.any()
            v = np.nan_to_num(v)
            Q = q[b, g * G:(g + 1) * G, 0]
            seen = np.ones((G, len(pos)), dtype=bool)
            want, want_lse = attention(Q, k, v, SCALE, seen)
            mag, _ = attention(Q, k, np.abs(v), SCALE, seen)
            off = 2.0 ** -17 * SCALE * (np.abs(Q) @ np.abs(k).T).max(axis=1, initial=0)
            tol = mag * (2.0 ** -8 + 2 * off + 2.0 ** -20)[:, None] + np.abs(want) * 2.0 ** -8
            assert np.isnan(got[:, bad]).all(), (b, g)
            assert (np.abs(got - want) <= tol)[:, ~bad].all(), (b, g)
            assert (np.abs(got_lse - want_lse) <= off + 2.0 ** -20 * (1 + np.abs(want_lse))).all(), (b, g)
    assert found


@pytest.mark.parametrize("G", [1, 4, 8])
@pytest.mark.parametrize("codes", ["zero", "any"])
@pytest.mark.parametrize("page,lens", [(0, [200, 33, 1]), (16, [4500, 700])])
def test_groups_that_are_nan(ihip, G, codes, page, lens):  # noqa: F811
    Hkv = 3
    c = Cache(ihip, lens, Hkv, page, seed=40 + G)
    rng = np.random.default_rng(G)

    def poison(rows, scales, b, g, pos, group):
        p, j = (b, pos) if c.table is None else (int(c.table[b, pos // page]), pos % page)
        scales[p, g, j, group] = 255
        if codes == "zero":
            rows[p, g, j, 16 * group:16 * group + 16] = 0

    for b, t in enumerate(lens):                         # head 0: a key; head 1: values; head 2: nothing
        poison(c.k, c.ks, b, 0, int(rng.integers(t)), int(rng.integers(4)))
        for _ in range(2):
            poison(c.v, c.vs, b, 1, int(rng.integers(t)), int(rng.integers(4)))
    q = queries(len(lens), G * Hkv, 41, scale=2.0)
    sl = torch.tensor(lens, dtype=torch.int32).cuda()
    out, lse = ihip.sparse_attn_decode_mx4(ihip.Layer(q, c.store, sl, 1, 0, c.T, max_seq_len=c.T), q, c.store, want_lse=True)
    check_nan(c, q, out, lse, 0, c.T)


def test_only_what_is_attended_to_counts(ihip):  # noqa: F811
    """Sink, kept blocks and window: a NaN key in a kept block, NaN values in the window, NaN everywhere between them."""
    lens, Hkv, Hq, n_sink, n_stream, block = [900, 417], 2, 8, 20, 70, 16
    c = Cache(ihip, lens, Hkv, 0, seed=43)
    q = queries(2, Hq, 44)
    starts = torch.tensor([[20, 132], [36, -1], [52, 100], [-1, -1]], dtype=torch.int32)
    for b, t in enumerate(lens):
        c.ks[b, :, 200:t - n_stream] = 255
        c.vs[b, :, 200:t - n_stream] = 255
    c.ks[0, 0, 135, 2] = 255
    c.vs[0, 1, 900 - 5, 1] = 255
    c.vs[1, 0, 100 + 15, 3] = 255
    sl = torch.tensor(lens, dtype=torch.int32).cuda()
    L = ihip.Layer(q, c.store, sl, 1, n_sink, n_stream, max_seq_len=c.T)
    out, lse = ihip.sparse_attn_decode_mx4(L, q, c.store, starts.cuda(), block, want_lse=True)
    check_nan(c, q, out, lse, n_sink, n_stream, starts, block)


def test_what_is_appended_not_finite_is_answered_with_nan(ihip):  # noqa: F811
    """NaN and infinite keys and values through kv_append: the decode attention and the cache read back say the same."""
    T, Hkv, Hq = 100, 2, 8
    x = torch.randn((T, 2 * Hkv, D), generator=torch.Generator().manual_seed(45)).bfloat16()
    x[30, 0, 77] = float("inf")                          # a key of head 0
    x[99, Hkv + 1, 5] = float("nan")                     # a value of head 1: dims 0 .. 31
    x[3, Hkv + 1, 127] = -float("inf")                   # and dims 96 .. 127
    x = x.cuda()
    k, v = (torch.zeros((1, Hkv, T, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((1, Hkv, T, 4), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    store = ihip.KVStore.mx4(k, v, ks, vs)
    sl = torch.tensor([T], dtype=torch.int32).cuda()
    ihip.kv_append(store, x[:, :Hkv], x[:, Hkv:], torch.tensor([0, T], dtype=torch.int32).cuda(), sl, T)
    q = queries(1, Hq, 46)
    out, lse = ihip.sparse_attn_decode_mx4(ihip.Layer(q, store, sl, 1, 0, T, max_seq_len=T), q, store, want_lse=True)
    k16, v16 = ihip.kv_gather(store, sl, T)
    key, value = (torch.isnan(t[0]).any(dim=1).cpu() for t in (k16, v16))          # [Hkv, D]
    want = (key.any(dim=1, keepdim=True) | value).repeat_interleave(Hq // Hkv, dim=0)
    assert torch.equal(torch.isnan(out[0, :, 0]).cpu(), want) and bool(want.any()) and not bool(want.all())
    assert torch.equal(torch.isnan(lse[0, :, 0]).cpu(), key.any(dim=1).repeat_interleave(Hq // Hkv))
