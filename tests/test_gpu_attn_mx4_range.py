"""4-bit decode attention at the ends of what the formats hold: values up to 6 * 2^125 and down to 2^-101 under scores that grow along
the keys, scores far from 0 in either direction.  Results against float64, test_gpu_attn_mx4's tolerances."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, attention, f64  # noqa: E402
from tests.test_gpu_attn_mx4 import SCALE, Cache, ihip, queries  # noqa: E402, F401


def run(ihip, c, q, scale=None):  # noqa: F811
    sl = torch.tensor(c.lens, dtype=torch.int32).cuda()
    L = ihip.Layer(q, c.store, sl, 1, 0, c.T, max_seq_len=c.T)
    return ihip.sparse_attn_decode_mx4(L, q, c.store, want_lse=True, **({} if scale is None else {"sm_scale": scale}))


def check_all_keys(c, q, out, lse):
    """test_gpu_attn_mx4.check for one sequence, one KV head and all keys, and for values near fp32's smallest numbers: a product of a
    probability, which is 2^-26 or more of what it is in the end, and a value is a multiple of 2^-149 in fp32, and so is what a sum loses when its
    reference moves.  A step for each key covers both: 2^-123 a key."""
    Q, G = f64(q)[0, :, 0], q.shape[1]
    k, v = c.rows(0, 0, np.arange(c.lens[0]))
    seen = np.ones((G, c.lens[0]), dtype=bool)
    want, want_lse = attention(Q, k, v, SCALE, seen)
    mag, _ = attention(Q, k, np.abs(v), SCALE, seen)
    off = 2.0 ** -17 * SCALE * (np.abs(Q) @ np.abs(k).T).max(axis=1)
    tol = mag * (2.0 ** -8 + 2 * off + 2.0 ** -20)[:, None] + np.abs(want) * 2.0 ** -8 + c.lens[0] * 2.0 ** -123
    assert (np.abs(f64(out)[0, :, 0] - want) <= tol).all()
    assert (np.abs(f64(lse)[0, :, 0] - want_lse) <= off + 2.0 ** -20 * (1 + np.abs(want_lse))).all()


@pytest.mark.parametrize("G", [1, 8])
@pytest.mark.parametrize("byte", [100 + 127, 252, 27], ids=["2^100", "2^125", "2^-100"])
@pytest.mark.parametrize("length", [700, 6000])
def test_values_at_the_ends_under_growing_scores(ihip, G, byte, length):  # noqa: F811
    """Scores from about 0 to some fifty nats: what is the largest probability so far is a vanishing part later."""
    c = Cache(ihip, [length], 1, 0, seed=50)
    c.vs[0, 0, :length] = byte
    for i in range(10):
        c.ks[0, 0, 20 + i * length // 10:] = 120 + i
    q = queries(1, G, 51, scale=2.0)
    out, lse = run(ihip, c, q)
    assert bool(torch.isfinite(out).all())
    check_all_keys(c, q, out, lse)


@pytest.mark.parametrize("byte", [252, 27])
def test_many_equal_keys_with_the_largest_and_smallest_values(ihip, byte):  # noqa: F811
    """The mean of 3,000 values, whose sum would be beyond fp32 (or far below 1)."""
    c = Cache(ihip, [3000], 1, 16, seed=52)
    c.ks[:] = 120
    c.k[:] = c.k[0, 0, 0]
    c.vs[:] = byte
    c.v[:] = c.v % 8 + 16 * (c.v // 16 % 8)              # no sign bits: what is added up does not cancel
    q = queries(1, 4, 53)
    out, lse = run(ihip, c, q)
    check_all_keys(c, q, out, lse)


def one_direction(ihip, sizes, up):  # noqa: F811
    """Keys that are multiples, by powers of two, of one direction, and a query along it (against it: up False).  Products are exact in fp32,
    so that equal keys have equal scores and others are whole powers of two apart, at 2^23 and more."""
    c = Cache(ihip, [len(sizes)], 1, 0, seed=54)
    c.k[:] = 0x22                                        # all ones
    c.ks[0, 0, :, :] = torch.tensor(sizes, dtype=torch.uint8).view(-1, 1).cuda()
    q = torch.full((1, 2, 1, D), 1.296875 if up else -1.296875).bfloat16().cuda()
    return c, q


def check_mean(c, first, score, out, lse):
    """Keys first .. share everything: equal probabilities, sums in fp32 (2^-16 of the largest), the result's own rounding; lse 2^-22."""
    n = c.lens[0] - first
    _, v = c.rows(0, 0, np.arange(first, c.lens[0]))
    want = v.mean(axis=0)
    assert (np.abs(f64(out)[0, :, 0] - want) <= np.abs(want) * 2.0 ** -8 + np.abs(v).max() * 2.0 ** -16).all()
    assert (np.abs(f64(lse)[0, :, 0] - (score + np.log(n))) <= 2.0 ** -22 * abs(score) + 2.0 ** -20 * np.log(n)).all()


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("length", [200, 5000])
@pytest.mark.parametrize("size", [40, 105])
def test_equal_scores_far_from_zero(ihip, up, length, size):  # noqa: F811
    c, q = one_direction(ihip, [127 + size] * length, up)
    out, lse = run(ihip, c, q)
    check_mean(c, 0, float(q[0, 0, 0, 0]) * D * 2.0 ** size * SCALE, out, lse)


@pytest.mark.parametrize("up", [True, False])
def test_scores_far_from_zero_and_from_each_other(ihip, up):  # noqa: F811
    """The last five keys share everything."""
    sizes = [20 + i // 5 for i in range(400)]
    sizes = sizes if up else sizes[::-1]
    c, q = one_direction(ihip, [127 + s for s in sizes], up)
    out, lse = run(ihip, c, q)
    check_mean(c, 395, float(q[0, 0, 0, 0]) * D * 2.0 ** sizes[-1] * SCALE, out, lse)
