"""What the calls around an evicting cache refuse, before anything is enqueued (no GPU)."""
import ctypes

import pytest

from tests.test_kv_store_args import b, store_of  # noqa: F401

BAD, WORKSPACE, UNSUPPORTED = -1, -2, -4
NAN, INF = float("nan"), float("inf")


def track_of(b, rows=64, weights=4096, positions=4096, seen=4096):  # noqa: F811
    return b.TrackStruct(weights, positions, rows, seen)


def by(x):
    return ctypes.byref(x) if x is not None else None


def append(b, packed=None, track=0, rope=None, max_len=64, store=None):  # noqa: F811
    t = b.Tensor(4096, 0, 128, 1024)
    p = b.PackedStruct(2, 8, 2, 128, 4096, 10, 10) if packed is None else packed
    return b.lib().ihip_kv_append_tracked(by(p), t, t, t, 4096, max_len, rope, by(store or store_of(b, 0)), by(track_of(b) if track == 0 else track),
                                          b.NO_TENSOR, b.NO_TENSOR, None)


def test_append_refuses(b):  # noqa: F811
    L = b.lib()
    assert append(b, track=None) == BAD and b"track is NULL" in L.ihip_last_error()
    assert append(b, track=track_of(b, rows=63)) == BAD and b"63 rows, 64" in L.ihip_last_error()
    assert append(b, track=track_of(b, weights=None)) == BAD and append(b, track=track_of(b, positions=None)) == BAD
    assert append(b, track=track_of(b, seen=None)) == BAD
    assert append(b, packed=b.PackedStruct(2, 8, 3, 128, 4096, 10, 10)) == BAD
    assert append(b, rope=ctypes.byref(b.RopeStruct(4096, None, 64, 0, 0))) == BAD
    assert append(b, max_len=0) == BAD
    t = b.Tensor(4096, 8192, 64, 128)
    assert append(b, store=store_of(b, 0, k=t, v=t)) == BAD and b"heads of the store overlap" in L.ihip_last_error()
    assert append(b, packed=b.PackedStruct(0, 8, 2, 128, None, 10, 10), track=None) == 0
    assert append(b, packed=b.PackedStruct(2, 8, 2, 128, 4096, 0, 0), track=None) == 0


def weights(b, packed=None, q=None, k=None, cu_k=None, rows_k=10, scale=0.1, lse=4096, window=5, before=None, decay=1.0, track=0):  # noqa: F811
    t = b.Tensor(4096, 0, 128, 1024)
    p = b.PackedStruct(2, 8, 2, 128, 4096, 10, 10) if packed is None else packed
    return b.lib().ihip_prompt_key_weights(by(p), q or t, k or t, cu_k, rows_k, scale, lse, window, before, decay,
                                           by(track_of(b, positions=None, seen=None) if track == 0 else track), None, 0, None)


def test_key_weights_refuses(b):  # noqa: F811
    L = b.lib()
    none = b.Tensor(None, 0, 0, 0)
    assert weights(b, packed=b.PackedStruct(2, 8, 3, 128, 4096, 10, 10)) == BAD
    assert weights(b, packed=b.PackedStruct(2, 8, 2, 64, 4096, 10, 10)) == UNSUPPORTED
    assert weights(b, rows_k=11) == BAD and weights(b, rows_k=-1, cu_k=4096) == BAD
    assert weights(b, window=0) == BAD and b"window" in L.ihip_last_error()
    assert weights(b, q=none) == BAD and weights(b, k=none) == BAD
    assert weights(b, q=b.Tensor(4096, 0, 132, 1024)) == BAD
    assert weights(b, lse=None) == BAD and b"lse" in L.ihip_last_error()
    for decay in (-1.0, NAN, INF):
        assert weights(b, decay=decay) == BAD and b"decay" in L.ihip_last_error()
    for scale in (-0.1, NAN, INF, 3e38):
        assert weights(b, scale=scale) == BAD and b"sm_scale" in L.ihip_last_error()
    assert weights(b, track=None) == BAD and weights(b, track=track_of(b, weights=None)) == BAD and weights(b, track=track_of(b, rows=-1)) == BAD
    assert weights(b, packed=b.PackedStruct(2, 8, 1, 128, 4096, 1 << 29, 10), rows_k=1 << 29) == UNSUPPORTED
    # nothing to do
    assert weights(b, packed=b.PackedStruct(0, 8, 2, 128, None, 10, 10), track=None) == 0
    assert weights(b, packed=b.PackedStruct(2, 8, 2, 128, 4096, 0, 0), rows_k=0, k=none, track=None) == 0


def test_key_weights_scratch(b):  # noqa: F811
    L = b.lib()
    need = lambda p, rows_k, window: L.ihip_prompt_key_weights_workspace_bytes(by(p), rows_k, window)  # noqa: E731
    assert need(b.PackedStruct(2, 8, 3, 128, 4096, 10, 10), 10, 5) == 0
    assert need(b.PackedStruct(2, 8, 2, 128, 4096, 10, 10), 10, 0) == 0 and need(b.PackedStruct(2, 8, 2, 128, 4096, 10, 10), -1, 5) == 0
    assert need(b.PackedStruct(1, 8, 2, 128, 4096, 20, 20), 20, 100) == 256
    many = b.PackedStruct(1, 32, 8, 128, 4096, 4000, 4000)
    assert need(many, 4000, 4000) >= 2 * 8 * 4000 * 4                       # two chunks and more
    assert need(many, 4000, 16) == 256


def decode(b, shape=None, q=None, store=None, scale=0.1, before=None, decay=1.0, track=0, out=4096, ws=4096, ws_bytes=1 << 30):  # noqa: F811
    s = b.Shape(2, 8, 2, 128, 1, 1, 4096, 64, 0, 1, 0) if shape is None else shape
    return b.lib().ihip_attn_decode_tracked(by(s), q or b.Tensor(4096, 1024, 128, 128), by(store or store_of(b, 0)), scale, before, decay,
                                            by(track_of(b, positions=None, seen=None) if track == 0 else track), out, None, ws, ws_bytes, None)


def test_decode_refuses(b):  # noqa: F811
    L, S = b.lib(), b.Shape
    assert decode(b, shape=S(2, 6, 2, 128, 1, 1, 4096, 64, 0, 1, 0)) == UNSUPPORTED         # 3 heads a KV head
    assert decode(b, shape=S(2, 8, 2, 64, 1, 1, 4096, 64, 0, 1, 0)) == UNSUPPORTED
    assert decode(b, shape=S(2, 8, 2, 128, 4, 1, 4096, 64, 0, 4, 0)) == BAD and b"Tq" in L.ihip_last_error()
    assert decode(b, shape=S(2, 8, 2, 128, 1, 1, None, 64, 0, 1, 0)) == BAD
    assert decode(b, shape=S(2, 8, 2, 128, 1, 1, 4096, 0, 0, 1, 0)) == BAD
    assert decode(b, shape=S(40000, 8, 2, 128, 1, 1, 4096, 1, 0, 1, 0), ws_bytes=1 << 60) == UNSUPPORTED
    assert decode(b, shape=S(1, 8, 2, 128, 1, 1, 4096, 1 << 28, 0, 1, 0), track=track_of(b, rows=1 << 28), ws_bytes=1 << 60) == UNSUPPORTED
    assert decode(b, q=b.Tensor(None, 0, 0, 0)) == BAD and decode(b, out=None) == BAD
    assert decode(b, store=store_of(b, 0, format=7)) == BAD
    assert decode(b, store=store_of(b, 1, k_scale=0.0)) == BAD
    assert decode(b, store=store_of(b, 1, k_scale=1e30), scale=1e30) == BAD and b"sm_scale" in L.ihip_last_error()
    for decay in (-1.0, NAN, INF):
        assert decode(b, decay=decay) == BAD
    for scale in (-0.1, NAN, INF):
        assert decode(b, scale=scale) == BAD
    assert decode(b, track=None) == BAD and decode(b, track=track_of(b, rows=63)) == BAD and decode(b, track=track_of(b, weights=None)) == BAD
    s = S(2, 8, 2, 128, 1, 1, 4096, 64, 0, 1, 0)
    need = L.ihip_attn_decode_tracked_workspace_bytes(by(s))
    assert need >= 2 * 8 * 64 * 4
    assert decode(b, ws_bytes=need - 1) == WORKSPACE and decode(b, ws=None) == WORKSPACE and decode(b, ws=4104) == WORKSPACE
    assert L.ihip_attn_decode_tracked_workspace_bytes(by(S(2, 6, 2, 128, 1, 1, 4096, 64, 0, 1, 0))) == 0
    assert decode(b, shape=S(0, 8, 2, 128, 1, 1, None, 64, 0, 1, 0), track=None) == 0


def evict(b, store=None, track=0, B=2, Hkv=2, d=128, lens=4096, max_len=64, keep=16, n_sink=2, n_recent=4, to=None, new=4096, kept=4096,  # noqa: F811
          ws=4096, ws_bytes=1 << 30):
    return b.lib().ihip_kv_evict(by(store or store_of(b, 0)), by(track_of(b) if track == 0 else track), B, Hkv, d, lens, max_len, keep, n_sink, n_recent,
                                 by(to), new, kept, ws, ws_bytes, None)


def test_evict_refuses(b):  # noqa: F811
    L = b.lib()
    assert evict(b, B=-1) == BAD and evict(b, Hkv=0) == BAD and evict(b, d=64) == UNSUPPORTED
    assert evict(b, keep=0) == BAD and evict(b, max_len=-1) == BAD
    assert evict(b, n_sink=-1) == BAD and evict(b, n_recent=-1) == BAD
    assert evict(b, n_sink=10, n_recent=7) == BAD and b"keep = 16" in L.ihip_last_error()
    assert evict(b, keep=2 ** 31 - 1, n_sink=2 ** 31 - 1, n_recent=1) == BAD
    assert evict(b, lens=None) == BAD and evict(b, new=None) == BAD and evict(b, kept=None) == BAD
    assert evict(b, new=4100) == BAD and evict(b, new=4092) == BAD and b"overlaps" in L.ihip_last_error()
    assert evict(b, track=None) == BAD and evict(b, track=track_of(b, rows=63)) == BAD
    for name in ("weights", "positions", "seen"):
        assert evict(b, track=track_of(b, **{name: None})) == BAD
    assert evict(b, to=track_of(b, rows=15, weights=8192, positions=8192)) == BAD
    assert evict(b, to=track_of(b, rows=32, weights=8192)) == BAD and b"share" in L.ihip_last_error()
    assert evict(b, to=track_of(b, weights=8192, positions=None)) == BAD
    t = b.Tensor(4096, 8192, 64, 128)
    assert evict(b, store=store_of(b, 0, k=t, v=t)) == BAD and b"heads of the store overlap" in L.ihip_last_error()
    assert evict(b, store=store_of(b, 2, k_scales=None)) == BAD
    for rows in (4096, 50000):                        # many rows that move; rows in chunks
        need = L.ihip_kv_evict_workspace_bytes(2, 2, rows, 1024)
        big = dict(max_len=rows, keep=1024, track=track_of(b, rows=rows))
        assert need > 256 and evict(b, ws_bytes=need - 1, **big) == WORKSPACE
        assert evict(b, ws=None, **big) == WORKSPACE and evict(b, ws=4104, **big) == WORKSPACE and evict(b, ws_bytes=0, **big) == WORKSPACE
    assert evict(b, keep=1 << 30, max_len=64, B=1) == UNSUPPORTED
    assert L.ihip_kv_evict_workspace_bytes(2, 2, 64, 0) == 0 and L.ihip_kv_evict_workspace_bytes(2, 0, 64, 1) == 0
    assert evict(b, B=0, track=None, lens=None, kept=None) == 0


def test_arrays_that_overlap_in_part(b):  # noqa: F811
    """The same array or one apart is taken, a shifted one is not: rows of it would be read behind their change."""
    L, at = b.lib(), 1 << 20
    bytes_ = 2 * 2 * 64 * 4
    track = track_of(b, weights=at, positions=at + 8 * bytes_)
    for shift in (4, -4, bytes_ - 4, 4 - bytes_):
        assert weights(b, before=at + shift, track=track) == BAD and b"before" in L.ihip_last_error()
        assert decode(b, before=at + shift, track=track) == BAD and b"before" in L.ihip_last_error()
        assert evict(b, track=track, to=track_of(b, weights=at + shift, positions=4096)) == BAD and b"overlap" in L.ihip_last_error()
        assert evict(b, track=track, to=track_of(b, weights=4096, positions=at + 8 * bytes_ + shift)) == BAD and b"overlap" in L.ihip_last_error()
    for shift in (0, bytes_, -bytes_):                # (refused for what is looked at later)
        assert decode(b, before=at + shift, track=track, ws=None) == WORKSPACE
    big = dict(max_len=4096, keep=1024)
    at, rows = 1 << 30, 2 * 2 * 4096 * 4
    track = track_of(b, rows=4096, weights=at, positions=at)
    for shift in (0, rows, -rows):
        assert evict(b, track=track, to=track_of(b, rows=4096, weights=at + shift, positions=at), ws=None, **big) == WORKSPACE


def test_tensors_that_are_refused(b):  # noqa: F811
    import torch
    import paper_2502_08910_amd as ih
    for w in (torch.zeros((2, 2, 8)), torch.zeros((2, 8)), torch.zeros((2, 2, 8), dtype=torch.float64)):
        with pytest.raises(ih.IhipError, match="weights"):
            ih.KVTrack(w)
