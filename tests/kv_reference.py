"""Plain float64 forms of the KV storages, the position rotation, cache filling and dense attention (CPU, numpy): what the
tests of ihip_kv_append, ihip_kv_gather, ihip_prompt_attn and ihip_sparse_attn_decode_mx4kv compare with."""
import numpy as np
import torch

D = 128
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx4_values(codes, scales):
    """uint8 codes [..., 64], scales [..., 4] -> float64 [..., 128]."""
    codes, scales = codes.cpu().numpy(), scales.cpu().numpy()
    c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(*codes.shape[:-1], D)
    v = np.where(c & 8, -1.0, 1.0) * E2M1[c & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=-1)


def mx4_rounded(x):
    """float64 rows [..., 128] -> (nearest 4-bit values, ties to the even code; scale bytes)."""
    g = x.reshape(*x.shape[:-1], 4, 32)
    top = np.abs(g).max(axis=-1)
    e = np.full(top.shape, -100.0)
    nz = top > 0
    e[nz] = np.ceil(np.log2(top[nz] / 7))
    e = np.where(top > 7 * 2.0 ** e, e + 1, e)
    e = np.where((top <= 7 * 2.0 ** (e - 1)) & nz, e - 1, e)
    e = np.clip(e, -100, 125)                        # 4 * 2^126 would be no bf16 number any more
    a = np.abs(g) / 2.0 ** e[..., None]
    dist = np.abs(a[..., None] - E2M1)
    best = dist.min(axis=-1, keepdims=True)
    near = dist == best                              # two of them at a tie: the even code
    code = np.where(near & (np.arange(8) % 2 == 0), np.arange(8), -1).max(axis=-1)
    code = np.where(code < 0, np.where(near, np.arange(8), -1).max(axis=-1), code)
    v = np.sign(g) * E2M1[code] * 2.0 ** e[..., None]
    return v.reshape(x.shape), (e + 127).astype(np.uint8)


def turned(x, cos, sin):
    """float64 rows [..., 128] turned by rows of the tables [..., 64], pairs (2j, 2j+1)."""
    y = np.empty_like(x)
    y[..., 0::2] = x[..., 0::2] * cos - x[..., 1::2] * sin
    y[..., 1::2] = x[..., 0::2] * sin + x[..., 1::2] * cos
    return y


def fp32_turned(x, cos, sin):
    """The same in float32, every product and sum rounded: numpy rounds each of them."""
    x, cos, sin = (t.astype(np.float32) for t in (x, cos, sin))
    return turned(x, cos, sin).astype(np.float64)


def attention(q, k, v, scale, seen):
    """One head in float64: q [n, D], k, v [t, D], seen bool [n, t] -> (out [n, D], lse [n]); rows that see nothing: 0, -inf."""
    s = np.where(seen, (q @ k.T) * scale, -np.inf)
    m = s.max(axis=1, keepdims=True, initial=-np.inf)
    p = np.exp(s - np.where(np.isfinite(m), m, 0.0))
    l = p.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = np.where(l > 0, m + np.log(np.where(l > 0, l, 1.0)), -np.inf)[:, 0]
    return np.where(l > 0, p @ np.where(seen.any(axis=0)[:, None], v, 0.0) / np.where(l > 0, l, 1.0), 0.0), lse


def f64(t: torch.Tensor):
    return t.detach().to("cpu").double().numpy()
