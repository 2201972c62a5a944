"""Caches with what stands beside their rows, and plain forms (float64, numpy) of what is done with them."""
import numpy as np
import torch

from tests.kv_reference import D, f64, mx4_values

FORMATS = ["bf16", "e4m3", "mx4"]
SCALES = (1.0 / 64, 0.0131)          # of E4M3 K and V; the second is no power of two


class Cache:
    """Random rows where the sequences have some; everywhere else rows of NaN.  token_major: a token's heads are neighbours in memory.
    missing: (sequence, page) pairs whose id is -1."""

    def __init__(self, ihip, fmt, lens, Hkv, page, seed, T=None, token_major=False, missing=()):
        g = torch.Generator().manual_seed(seed)
        B, T = len(lens), T or max(max(lens), 1)
        n, table = B, None
        if page:
            per = -(-T // page)
            n = B * per + 2
            table = torch.randperm(n, generator=g)[:B * per].to(torch.int32).view(B, per).contiguous()
        shape = (n, Hkv, page or T)
        def rows(width, dtype, fill):  # noqa: E306
            if token_major:
                return torch.full((shape[0], shape[2], shape[1], width), fill, dtype=dtype).permute(0, 2, 1, 3)
            return torch.full((*shape, width), fill, dtype=dtype)
        width, dtype, junk = {"bf16": (D, torch.bfloat16, float("nan")), "e4m3": (D, torch.uint8, 0x7f), "mx4": (D // 2, torch.uint8, 0)}[fmt]
        k, v = rows(width, dtype, junk), rows(width, dtype, junk)
        ks, vs = (rows(4, torch.uint8, 255), rows(4, torch.uint8, 255)) if fmt == "mx4" else (None, None)
        for b, t in enumerate(lens):
            for first in range(0, t, page or max(t, 1)):
                m = min(t - first, page or t)
                p = b if table is None else int(table[b, first // page])
                for x, s in ((k, ks), (v, vs)):
                    if fmt == "bf16":
                        x[p, :, :m] = torch.randn((Hkv, m, D), generator=g).bfloat16()
                    elif fmt == "e4m3":
                        x[p, :, :m] = (torch.randint(0, 115, (Hkv, m, D), generator=g) + 128 * torch.randint(0, 2, (Hkv, m, D), generator=g)).to(torch.uint8)
                    else:
                        x[p, :, :m] = torch.randint(0, 256, (Hkv, m, D // 2), generator=g, dtype=torch.uint8)
                        s[p, :, :m] = torch.randint(123, 127, (Hkv, m, 4), generator=g, dtype=torch.uint8)
        for b, i in missing:
            table[b, i] = -1
        def place(x):                  # (cuda() keeps the strides of a dense permuted tensor)  # noqa: E306
            return None if x is None else x.cuda()
        self.k, self.v, self.ks, self.vs = place(k), place(v), place(ks), place(vs)
        self.table = None if table is None else table.cuda()
        if fmt == "bf16":
            self.store = ihip.KVStore.bf16(self.k, self.v, self.table)
        elif fmt == "e4m3":
            self.store = ihip.KVStore.e4m3(self.k, self.v, SCALES, self.table)
        else:
            self.store = ihip.KVStore.mx4(self.k, self.v, self.ks, self.vs, self.table)
        self.fmt, self.lens, self.B, self.T, self.Hkv, self.page = fmt, lens, B, T, Hkv, page
        self.seq_lens = torch.tensor(lens, dtype=torch.int32).cuda()

    def there(self, b, r):
        """Which rows r of sequence b are on a page."""
        return np.ones(len(r), dtype=bool) if self.table is None else self.table.cpu().numpy()[b][r // self.page] >= 0

    def rows(self, b, g, r):
        """Rows r of sequence b and KV head g as float64 (K, V)."""
        p, j = (np.full(len(r), b), r) if self.table is None else (self.table.cpu().numpy()[b][r // self.page], r % self.page)
        p, j = torch.from_numpy(p.astype(np.int64)), torch.from_numpy(np.asarray(j))
        if self.fmt == "bf16":
            return tuple(f64(x.cpu()[p, g, j]) for x in (self.k, self.v))
        if self.fmt == "e4m3":
            return tuple(f64(x.cpu()[p, g, j].view(torch.float8_e4m3fn)) * np.float32(s) for x, s in zip((self.k, self.v), SCALES))
        return tuple(mx4_values(x.cpu()[p, g, j], s.cpu()[p, g, j]) for x, s in ((self.k, self.ks), (self.v, self.vs)))

    def raw(self):
        """All of its memory, as bytes."""
        return [x.contiguous().view(torch.uint8).cpu().numpy().copy() for x in (self.k, self.v, self.ks, self.vs) if x is not None]


def key_weights(q, k, lse, scale, G, window):
    """One sequence and KV head in float64: q [n, G, D], k [t, D], lse [n, G] -> (weights [t], how far fp32 may be off, relative, [t])."""
    n, t = q.shape[0], k.shape[0]
    w, worst = np.zeros(t), np.zeros(t)
    first = max(0, n - window)
    seen = np.arange(t)[None, :] <= (np.arange(first, n) + t - n)[:, None]
    for h in range(G):
        s = q[first:, h] @ k.T * scale
        # 128 products and sums of fp32, the logarithm's base, and the difference, each rounded; exp2 itself
        off = 2.0 ** -17 * scale * (np.abs(q[first:, h]) @ np.abs(k).T) + 2.0 ** -22 * (np.abs(s) + np.abs(lse[first:, h])[:, None]) + 2.0 ** -22
        p = np.where(seen, np.exp(np.where(seen, s - lse[first:, h][:, None], 0.0)), 0.0)
        w += p.sum(axis=0)
        worst += (p * np.where(seen, off, 0.0)).sum(axis=0)
    # (fp32 sums of at most 64 terms at each of four levels)
    return w, worst + w * 4 * 64 * 2.0 ** -24 + 2.0 ** -120


def evicted(weights, positions, n, keep, n_sink, recent_from):
    """One (sequence, KV head): the row that each of the `keep` rows was, -1 behind the sequence."""
    kept = np.full(keep, -1, dtype=np.int64)
    if n <= keep:
        kept[:n] = np.arange(n)
        return kept
    def order(r):                    # noqa: E306
        w, p = float(weights[r]), int(positions[r])
        fixed = p < n_sink or p >= recent_from
        return (0 if fixed else 2 if np.isnan(w) else 1, 0.0 if fixed or np.isnan(w) else -w, r)
    best = sorted(range(n), key=order)[:keep]
    stays, movers = {r for r in best if r < keep}, sorted(r for r in best if r >= keep)
    kept[:] = np.arange(keep)
    kept[[r for r in range(keep) if r not in stays]] = movers
    return kept
