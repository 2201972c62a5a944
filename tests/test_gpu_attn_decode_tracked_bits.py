"""How many bits of a probability reach the output of ihip_attn_decode_tracked: a value is taken away from its own probability times 1, in pieces
that the rows hold, so that what is left is what the probability was off by."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, E2M1, f64  # noqa: E402
from tests.test_gpu_attn_decode_tracked import ihip  # noqa: E402, F401

PIECES = 9


def bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).bfloat16().double().numpy()


def chosen_queries():
    """Four numbers x (bf16) for which exp(-x) is far from a sum of two bf16 numbers."""
    x = np.unique(bf16(np.arange(0.25, 4, 1 / 64)))
    p = np.exp(-x).astype(np.float32).astype(np.float64)
    off = np.abs(p - bf16(p) - bf16(p - bf16(p))) / p
    best = np.argsort(-off)[:4]
    assert off[best].min() > 2.0 ** -17.7
    return x[best]


def grid(fmt):
    """Positive numbers that a row of 32 equal values can hold, scale and code of 4-bit ones."""
    if fmt == "bf16":
        return None
    if fmt == "e4m3":
        v = torch.arange(1, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
        return [(x, i + 1, 0) for i, x in enumerate(v)]
    return [(E2M1[c] * 2.0 ** (s - 127), c, s) for c in (2, 3) for s in range(90, 140)]


def pieces_of(t, fmt):
    """[(value, code, scale)] whose sum is t up to 2^-13 of it, and to 2^-17 where the format has numbers as small (multiples of 2^-22 t: what is added
    up in fp32 is exact)."""
    out, left = [], t
    for _ in range(PIECES):
        if abs(left) < 2.0 ** -17 * t:
            break
        if fmt == "bf16":
            v, c, s = float(bf16(abs(left))), 0, 0
        else:
            v, c, s = min(grid(fmt), key=lambda g: abs(g[0] - abs(left)))
        if v > 2 * abs(left):                        # the smallest number, and too large
            break
        out.append((np.sign(left) * v, c, s))
        left -= np.sign(left) * v
    return out


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "mx4"])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("T", [64, 5000])            # one part, and many of which one has rows
def test_bits_of_a_probability(ihip, fmt, G, T):  # noqa: F811
    """Row 0 has probability p = exp(-x) (times the largest) and the value 1 (448 in E4M3), the others 1 and pieces of -p.  Tolerance, relative to p: exponent
    x log2 e with three roundings of 2^-24 (the product, sm_scale log2 e, log2 e), x at most 4: 4 * 3 * 2^-24; exp2 2^-23; three parts of a probability
    that keep 2^-24; the output's own rounding.  Two bf16 parts of p alone are off by 2^-17.7 and more for these x."""
    x = chosen_queries()
    unit = 448.0 if fmt == "e4m3" else 1.0
    n = PIECES + 1
    k, v = np.zeros((n, D)), np.zeros((n, D))
    code, scale = np.zeros((n, D), dtype=np.uint8), np.full((n, 4), 127, dtype=np.uint8)
    k[1:, 0] = 1.0
    for j in range(4):                               # dims 32 j .. are for head j, 4 + j
        cols = slice(32 * j, 32 * j + 32)
        v[0, cols] = unit
        code[0, cols] = 2
        for i, (val, c, s) in enumerate(pieces_of(unit * np.exp(-x[j % min(G, 4)]), fmt)):
            v[1 + i, cols] = -val
            code[1 + i, cols] = c | (8 if val > 0 else 0)
            scale[1 + i, j] = s
    k_code = (k != 0).astype(np.uint8) * 2
    def place(t, fill=0):                            # noqa: E306
        whole = torch.full((1, 2, T, t.shape[1]), fill, dtype=t.dtype)
        whole[0, :, :n] = t
        return whole.cuda()
    def packed(c):                                   # noqa: E306
        return torch.from_numpy(c[:, 0::2] | (c[:, 1::2] << 4))
    if fmt == "bf16":
        store = ihip.KVStore.bf16(place(torch.from_numpy(k).bfloat16()), place(torch.from_numpy(v).bfloat16()))
    elif fmt == "e4m3":
        store = ihip.KVStore.e4m3(*(place(torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8)) for y in (k, v)), (1.0, 1.0))
    else:
        store = ihip.KVStore.mx4(place(packed(k_code)), place(packed(code)), place(torch.full((n, 4), 127, dtype=torch.uint8)), place(torch.from_numpy(scale)))
    q = torch.zeros((1, 2 * G, 1, D))
    for h in range(2 * G):
        q[0, h, 0, 0] = x[(h % G) % 4]
    track = ihip.KVTrack(torch.zeros((1, 2, T)).cuda())
    out, _ = ihip.attn_decode_tracked(q.bfloat16().cuda(), store, track, torch.tensor([n], dtype=torch.int32).cuda(), T, sm_scale=1.0, fresh=True)
    for h in range(2 * G):
        y = x[(h % G) % 4]
        p = np.concatenate(([np.exp(-y)], np.ones(PIECES)))
        for j in range(4):
            if j % min(G, 4) != (h % G) % 4:
                continue
            want = (p @ v[:, 32 * j]) / p.sum()
            got = f64(out)[0, h, 0, 32 * j:32 * j + 32]
            assert abs(want) <= 2.0 ** -13 * unit * p[0]
            tol = unit * p[0] / p.sum() * (y * 3 * 2.0 ** -24 + 2.0 ** -23 + 2.0 ** -24) + abs(want) * 2.0 ** -8
            assert (np.abs(got - want) <= tol).all(), (h, j, np.abs(got - want).max() / (unit * p[0] / p.sum()) * 2 ** 20)
