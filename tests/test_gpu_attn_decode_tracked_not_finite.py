"""What is not finite in K, and rows that are left out beside it (ihip_attn_decode_tracked)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_attn_decode_tracked import ihip, queries  # noqa: E402, F401
from tests.tracked_reference import Cache  # noqa: E402

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("T", [200, 3000])           # one part, and many
@pytest.mark.parametrize("value", [NAN, INF])
def test_rows_that_are_left_out_beside_rows_that_are_not_finite(ihip, T, value):  # noqa: F811
    """The results of the KV head are NaN; rows on no page keep decay * before."""
    c = Cache(ihip, "bf16", [200], 2, 16, seed=1, T=T, missing=[(0, 3), (0, 12)])
    c.k[int(c.table[0, 5]), 0, 4] = value            # row 84 of the first KV head
    q = queries(1, 8, 2).abs()
    old = torch.rand((1, 2, T), generator=torch.Generator().manual_seed(3))
    track = ihip.KVTrack(old.clone().cuda())
    out, lse = ihip.attn_decode_tracked(q, c.store, track, c.seq_lens, T, decay=0.5, want_lse=True)
    w, out, lse = track.weights.cpu(), out.cpu(), lse.cpu()
    assert bool(out[0, :4].isnan().all()) and bool(lse[0, :4].isnan().all())
    assert bool(out[0, 4:].isfinite().all()) and bool(lse[0, 4:].isfinite().all()) and bool(w[0, 1, :200].isfinite().all())
    gone = torch.zeros(T, dtype=torch.bool)
    gone[48:64] = gone[192:200] = True
    assert torch.equal(w[:, :, gone], old[:, :, gone] * 0.5)
    there = ~gone
    there[200:] = False
    assert bool(w[0, 0, there].isnan().all()) and torch.equal(w[:, :, 200:], old[:, :, 200:])


@pytest.mark.parametrize("T", [200, 3000])
def test_scores_of_minus_infinity(ihip, T):  # noqa: F811
    """A row with such a score has no part in anything: the others' results are the bits that they have beside a row on no page."""
    c = Cache(ihip, "bf16", [200], 2, 1, seed=4, T=T)
    q = queries(1, 8, 5).abs()
    page = int(c.table[0, 84])
    c.k[page], c.v[page] = 1.0, 0.0
    c.k[page, :, 0, 7] = -INF
    got = []
    for on in (True, False):
        c.table[0, 84] = page if on else -1
        track = ihip.KVTrack(torch.zeros((1, 2, T)).cuda())
        out, lse = ihip.attn_decode_tracked(q, c.store, track, c.seq_lens, T, fresh=True, want_lse=True)
        assert bool(track.weights.isfinite().all()) and bool((track.weights[:, :, 84] == 0).all())
        got.append((out, lse, track.weights))
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("T", [70, 3000])
@pytest.mark.parametrize("scale", [0.0, 0.1])
def test_scores_of_minus_infinity_alone(ihip, T, scale):  # noqa: F811
    """A sequence of such scores: as one without pages."""
    c = Cache(ihip, "bf16", [70], 1, 0, seed=6, T=T)
    c.k[:, :, :70] = 1.0
    c.k[:, :, :70, 9] = -INF
    old = torch.rand((1, 1, T), generator=torch.Generator().manual_seed(7))
    track = ihip.KVTrack(old.clone().cuda())
    out, lse = ihip.attn_decode_tracked(queries(1, 2, 8).abs() + 0.5, c.store, track, c.seq_lens, T, sm_scale=scale, want_lse=True)
    assert bool((out == 0).all()) and bool((lse == -INF).all()) and torch.equal(track.weights.cpu(), old)
