"""Cache filling (ihip_kv_append) and reading back (ihip_kv_gather) against plain forms: the rotation in float32 with every
product and sum rounded, as the header says, so that what is stored is equal bit for bit; and in float64 within the roundings."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.kv_reference import D, f64, fp32_turned, mx4_rounded, mx4_values, turned  # noqa: E402
from workloads import gen  # noqa: E402

FORMATS = ["bf16", "e4m3", "mx4"]
SCALES = (1.0 / 64, 0.0131)          # of E4M3 K and V; the second is no power of two


@pytest.fixture(scope="module")
def ihip():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_08910_amd as pkg
    pkg.lib()
    return pkg


def normal(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).bfloat16()


class Cache:
    """A cache of the format full of junk (finite values), on the GPU."""

    def __init__(self, ihip, fmt, B, Hkv, T, page, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.fmt, self.page, self.T, self.Hkv = fmt, page, T, Hkv
        self.table, n = None, B
        if page:
            per = -(-T // page)
            n = B * per + 3
            self.table = torch.randperm(n, generator=g)[:B * per].to(torch.int32).view(B, per).contiguous().cuda()
        shape = (n, Hkv, page or T)
        if fmt == "bf16":
            self.k, self.v = (torch.randn((*shape, D), generator=g).bfloat16().cuda() for _ in range(2))
            self.store = ihip.KVStore.bf16(self.k, self.v, self.table)
        elif fmt == "e4m3":
            self.k, self.v = (torch.randint(0, 120, (*shape, D), generator=g, dtype=torch.uint8).cuda() for _ in range(2))
            self.store = ihip.KVStore.e4m3(self.k, self.v, SCALES, self.table)
        else:
            self.k, self.v = (torch.randint(0, 256, (*shape, D // 2), generator=g, dtype=torch.uint8).cuda() for _ in range(2))
            self.ks, self.vs = (torch.randint(100, 140, (*shape, 4), generator=g, dtype=torch.uint8).cuda() for _ in range(2))
            self.store = ihip.KVStore.mx4(self.k, self.v, self.ks, self.vs, self.table)

    def values(self):
        """K and V pools as float64."""
        if self.fmt == "bf16":
            return f64(self.k), f64(self.v)
        if self.fmt == "e4m3":
            return tuple(f64(t.view(torch.float8_e4m3fn)) * s for t, s in ((self.k, np.float32(SCALES[0])), (self.v, np.float32(SCALES[1]))))
        return mx4_values(self.k, self.ks), mx4_values(self.v, self.vs)

    def at(self, b, pos):
        return (b, pos) if self.table is None else (int(self.table[b, pos // self.page]), pos % self.page)


def stored(x, fmt, which):
    """float32-exact rows (float64 array) -> the values that the format keeps."""
    if fmt == "bf16":
        return f64(torch.from_numpy(x).float().bfloat16())
    if fmt == "e4m3":
        s = np.float32(SCALES[which])
        q = np.clip(x.astype(np.float32) / s, -448, 448)
        return f64(torch.from_numpy(q).to(torch.float8_e4m3fn)) * s
    return mx4_rounded(x)[0]


def offsets(new):
    return torch.tensor(np.concatenate(([0], np.cumsum(new))), dtype=torch.int32)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,Hq,Hkv,new,ctx,rope", [
    (0, 8, 2, [5, 0, 1, 33], [0, 7, 40, 3], True),
    (16, 8, 8, [1, 1, 1, 1, 1], [0, 15, 16, 31, 99], True),
    (64, 7, 1, [130, 1, 0, 66], [0, 63, 5, 62], True),
    (1, 5, 5, [3, 2], [0, 4], False),
    (16, 12, 4, [1], [0], False),
    (128, 40, 8, [300], [1], True),
])
def test_append(ihip, fmt, page, Hq, Hkv, new, ctx, rope):
    B, N = len(new), sum(new)
    total = [a + b for a, b in zip(new, ctx)]
    T = max(total)
    rows = N + 5                                     # rows behind the last sequence
    q, k, v = normal(1, rows, Hq, D), normal(2, rows, Hkv, D), normal(3, rows, Hkv, D)
    cos, sin = gen.rope_table(T, D)
    c = Cache(ihip, fmt, B, Hkv, T, page)
    before = c.values()
    q_out, k_out = (torch.full((rows, h, D), 5.0, dtype=torch.bfloat16).cuda() for h in (Hq, Hkv))
    ihip.kv_append(c.store, k.cuda(), v.cuda(), offsets(new).cuda(), torch.tensor(total, dtype=torch.int32).cuda(), T,
                   q=q.cuda(), rope=(cos.cuda(), sin.cuda()) if rope else None, q_out=q_out, k_out=k_out)
    want_k, want_v = (x.copy() for x in before)
    want_q, want_ko = (np.full((rows, h, D), 5.0) for h in (Hq, Hkv))
    cos, sin = f64(cos), f64(sin)
    t = 0
    for b in range(B):
        for i in range(new[b]):
            pos = ctx[b] + i
            kt, qt = f64(k[t]), f64(q[t])
            if rope:
                kt64, qt64 = turned(kt, cos[pos], sin[pos]), turned(qt, cos[pos], sin[pos])
                # bf16's half step, and three roundings of fp32 on values of at most |e| + |o| each
                tol = np.abs(qt64) * 2.0 ** -8 + 3 * 2.0 ** -24 * 2 * np.abs(qt).max()
                assert (np.abs(f64(q_out[t]) - qt64) <= tol).all()
                kt, qt = fp32_turned(kt, cos[pos], sin[pos]), fp32_turned(qt, cos[pos], sin[pos])
                assert np.abs(kt - kt64).max() <= 3 * 2.0 ** -24 * 2 * np.abs(f64(k[t])).max()
            want_q[t], want_ko[t] = stored(qt, "bf16", 0), stored(kt, "bf16", 0)
            p, j = c.at(b, pos)
            want_k[p, :, j], want_v[p, :, j] = stored(kt, fmt, 0), stored(f64(v[t]), fmt, 1)
            t += 1
    got_k, got_v = c.values()
    assert np.array_equal(f64(q_out), want_q) and np.array_equal(f64(k_out), want_ko)
    assert np.array_equal(got_k, want_k) and np.array_equal(got_v, want_v)


def test_append_in_place_of_a_fused_projection(ihip):
    """q, k and v are parts of one tensor's rows; q and k are rotated where they stand."""
    Hq, Hkv, N = 8, 2, 37
    x = normal(4, N, Hq + 2 * Hkv, D)
    y = x.cuda()
    q, k, v = y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:]
    cos, sin = gen.rope_table(64, D)
    c = Cache(ihip, "bf16", 1, Hkv, 64, 0)
    ihip.kv_append(c.store, k, v, offsets([N]).cuda(), torch.tensor([N + 10], dtype=torch.int32).cuda(), 64, q=q, rope=(cos.cuda(), sin.cuda()), q_out=q, k_out=k)
    pos = np.arange(10, 10 + N)
    want = f64(x)
    want[:, :Hq + Hkv] = stored(fp32_turned(want[:, :Hq + Hkv], f64(cos)[pos][:, None], f64(sin)[pos][:, None]), "bf16", 0)
    assert np.array_equal(f64(y), want)
    assert np.array_equal(f64(c.k[0, :, 10:10 + N]).transpose(1, 0, 2), want[:, Hq:Hq + Hkv])
    assert torch.equal(c.v[0, :, 10:10 + N].transpose(0, 1).cpu(), x[:, Hq + Hkv:])


@pytest.mark.parametrize("fmt", FORMATS)
def test_tokens_without_a_place_are_dropped(ihip, fmt):
    """Positions before 0 or at and behind max_seq_len, and pages with a negative id."""
    B, Hkv, page, T = 3, 2, 16, 48
    c = Cache(ihip, fmt, B, Hkv, T, page)
    c.table[1, 1] = -1                               # positions 16..31 of sequence 1
    new, lens = [4, 40, 6], [2, 40, 51]              # sequence 0: positions -2..1; 2: 45..50
    rows = sum(new)
    k, v = normal(5, rows, Hkv, D), normal(6, rows, Hkv, D)
    before = c.values()
    k_out = torch.full((rows, Hkv, D), 5.0, dtype=torch.bfloat16).cuda()
    cos, sin = gen.rope_table(T, D)
    ihip.kv_append(c.store, k.cuda(), v.cuda(), offsets(new).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), T,
                   rope=(cos.cuda(), sin.cuda()), k_out=k_out)
    want_k, want_v = (x.copy() for x in before)
    want_ko = np.full((rows, Hkv, D), 5.0)
    t = 0
    for b in range(B):
        for i in range(new[b]):
            pos = lens[b] - new[b] + i
            if 0 <= pos < T:
                kt = fp32_turned(f64(k[t]), f64(cos)[pos], f64(sin)[pos])
                want_ko[t] = stored(kt, "bf16", 0)
                p, j = c.at(b, pos)
                if p >= 0:
                    want_k[p, :, j], want_v[p, :, j] = stored(kt, fmt, 0), stored(f64(v[t]), fmt, 1)
            t += 1
    got_k, got_v = c.values()
    assert np.array_equal(got_k, want_k) and np.array_equal(got_v, want_v) and np.array_equal(f64(k_out), want_ko)


def test_values_at_the_ends_of_the_formats(ihip):
    """Zero, huge, tiny, infinite and NaN elements; the borders between 4-bit codes, where ties go to the even one."""
    x = torch.zeros((10, 1, D))
    x[1] = 7.0                                       # the largest magnitude that keeps its scale: rounds to 6
    x[2] = 7.03125                                   # one bf16 step more
    x[3, 0, :32] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0] * 4)
    x[3, 0, 32:64] = -x[3, 0, :32] * 8
    x[3, 0, 64:96] = torch.tensor([0.2490234375, 0.251953125, 0.74609375, 0.75390625, 4.96875, 5.03125, 3.515625, -6.0] * 4)
    x[4] = 3.0e38
    x[5] = 2.0 ** -101
    x[5, 0, 5] = 2.0 ** -98
    x[6, 0, 40] = float("inf")
    x[7, 0, 0] = float("nan")
    x[8] = 448.0 / 64
    x[9] = torch.linspace(-700, 700, D)
    xb = x.bfloat16()
    for fmt in ("mx4", "e4m3"):
        c = Cache(ihip, fmt, 1, 1, 16, 0)
        ihip.kv_append(c.store, xb.cuda(), xb.cuda(), offsets([10]).cuda(), torch.tensor([10], dtype=torch.int32).cuda(), 16)
        got = c.values()[0][0, 0]
        for t in range(10):
            w = f64(xb[t, 0])
            if fmt == "e4m3":
                want = stored(w, fmt, 0)             # (infinity: 448; NaN: NaN)
            else:
                want = np.full(D, np.nan)
                for g in range(4):
                    part = slice(32 * g, 32 * g + 32)
                    if np.isfinite(w[part]).all():
                        rows = np.zeros(D)
                        rows[part] = w[part]
                        want[part] = mx4_rounded(rows)[0][part]
            assert np.array_equal(got[t], want, equal_nan=True), (fmt, t)
        if fmt == "mx4":
            k_out, v_out = ihip.kv_gather(c.store, torch.tensor([10], dtype=torch.int32).cuda(), 16)
            assert np.array_equal(f64(k_out)[0, 0, :10], c.values()[0][0, 0, :10], equal_nan=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,Hkv,lens", [(0, 2, [77, 0, 1, 130]), (16, 8, [15, 16, 17, 200]), (1, 3, [5, 64]), (256, 1, [300])])
def test_gather(ihip, fmt, page, Hkv, lens):
    B, T = len(lens), max(lens) + 3
    c = Cache(ihip, fmt, B, Hkv, T, page, seed=7)
    if page:
        c.table[0, 0] = -1                           # rows left as they were
    k_out, v_out = (torch.full((B, Hkv, T, D + 8), 5.0, dtype=torch.bfloat16).cuda()[..., :D] for _ in range(2))
    ihip.kv_gather(c.store, torch.tensor(lens, dtype=torch.int32).cuda(), T, k_out=k_out, v_out=v_out)
    for which, (pool, out) in enumerate(zip(c.values(), (k_out, v_out))):
        want = np.full((B, Hkv, T, D), 5.0)
        for b in range(B):
            for t in range(lens[b]):
                p, j = c.at(b, t)
                if p >= 0:
                    want[b, :, t] = pool[p, :, j]
        want = f64(torch.from_numpy(want).float().bfloat16())        # E4M3: scale * value rounds once (the product is exact in fp32's 24 bits)
        if fmt == "e4m3" and which == 1:             # ... or, with a scale of 24 bits, twice: within a step of bf16
            assert (np.abs(f64(out) - want) <= np.abs(want) * 2.0 ** -7).all()
        else:
            assert np.array_equal(f64(out), want)


def test_gather_of_keys_alone_and_of_lengths_beyond_the_bound(ihip):
    from paper_2502_08910_amd.binding import NO_TENSOR, _tensor
    c = Cache(ihip, "mx4", 2, 2, 40, 0)
    lens = torch.tensor([1 << 30, 9], dtype=torch.int32).cuda()
    out = torch.full((2, 2, 24, D), 5.0, dtype=torch.bfloat16).cuda()
    L = ihip.lib()
    assert L.ihip_kv_gather(c.store.ref(), 2, 2, D, lens.data_ptr(), 20, _tensor(out, "k"), NO_TENSOR, torch.cuda.current_stream().cuda_stream) == 0
    want = np.full((2, 2, 24, D), 5.0)
    want[0, :, :20], want[1, :, :9] = c.values()[0][0, :, :20], c.values()[0][1, :, :9]
    assert np.array_equal(f64(out), want)


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_beyond_four_gigabytes(ihip, fmt):
    """Pages at the end of pools that 32-bit byte offsets do not reach."""
    width = {"bf16": 256, "e4m3": 128, "mx4": 64}[fmt]
    page, Hkv = 64, 8
    n = (5 << 30) // (page * Hkv * width) + 7
    dt = torch.bfloat16 if fmt == "bf16" else torch.uint8
    k, v = (torch.zeros((n, Hkv, page, width // (2 if fmt == "bf16" else 1)), dtype=dt, device="cuda") for _ in range(2))
    table = torch.tensor([[n - 1, 0, n - 3]], dtype=torch.int32).cuda()
    if fmt == "mx4":
        ks, vs = (torch.full((n, Hkv, page, 4), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
        store = ihip.KVStore.mx4(k, v, ks, vs, table)
    else:
        store = ihip.KVStore.bf16(k, v, table) if fmt == "bf16" else ihip.KVStore.e4m3(k, v, (1.0 / 64, 1.0 / 64), table)
    N = 150
    x, y = normal(8, N, Hkv, D), normal(9, N, Hkv, D)
    lens = torch.tensor([N], dtype=torch.int32).cuda()
    ihip.kv_append(store, x.cuda(), y.cuda(), offsets([N]).cuda(), lens, N)
    got = ihip.kv_gather(store, lens, N)
    for out, rows in zip(got, (x, y)):
        w = f64(rows)
        want = w if fmt == "bf16" else f64(torch.from_numpy(w * 64).float().to(torch.float8_e4m3fn)) / 64 if fmt == "e4m3" else mx4_rounded(w)[0]
        assert np.array_equal(f64(out)[0], want.transpose(1, 0, 2))
    assert int((k.view(torch.uint8).view(n, -1)[1:n - 3] != 0).sum()) == 0


def test_append_and_gather_on_another_stream_and_in_a_graph(ihip):
    """Replayed with new rows and lengths in the captured buffers, eager calls in between; every replay equals the eager call."""
    B, Hkv, T = 3, 2, 64
    c = Cache(ihip, "mx4", B, Hkv, T, 16)
    cu = offsets([1, 1, 1]).cuda()
    k, v = (torch.empty((B, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lens = torch.empty(B, dtype=torch.int32, device="cuda")
    q = torch.empty((B, 4, D), dtype=torch.bfloat16, device="cuda")
    cos, sin = (t.cuda() for t in gen.rope_table(T, D))
    q_out = torch.empty_like(q)
    k_out, v_out = (torch.zeros((B, Hkv, T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step():
        ihip.kv_append(c.store, k, v, cu, lens, T, q=q, rope=(cos, sin), q_out=q_out)
        ihip.kv_gather(c.store, lens, T, k_out=k_out, v_out=v_out)

    def fill(i):
        for j, t in enumerate((k, v, q)):
            t.copy_(normal(100 * i + j, *t.shape))
        lens.copy_(torch.tensor([1 + i, 20 + i, 47 + i], dtype=torch.int32))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(1, 5):
        fill(i)
        junk = c.k.clone()
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (q_out, k_out, v_out, c.k, c.ks)]
        c.k.copy_(junk)
        for t in (q_out, k_out, v_out):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for got, w in zip((q_out, c.k, c.ks), (want[0], want[3], want[4])):
            assert torch.equal(got, w), i
        for b, n in enumerate(lens.tolist()):
            assert torch.equal(k_out[b, :, :n], want[1][b, :, :n]) and torch.equal(v_out[b, :, :n], want[2][b, :, :n])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page", [0, 16])
def test_caches_whose_tokens_hold_all_heads(ihip, fmt, page):
    """[.., tokens, heads, d] in memory, more of it between the rows, a cache that begins inside a larger one: the same as head by head."""
    c = Cache(ihip, fmt, 2, 3, 64, page, seed=31)

    def spread(t):
        n, H, T, w = t.shape
        big = torch.full((n + 1, T, H + 2, w), 7, dtype=t.dtype, device="cuda")
        view = big[1:, :, 1:H + 1].transpose(1, 2)
        view.copy_(t)
        return big, view

    big_k, k = spread(c.k)
    big_v, v = spread(c.v)
    if fmt == "mx4":
        (big_ks, ks), (big_vs, vs) = spread(c.ks), spread(c.vs)
        other = ihip.KVStore.mx4(k, v, ks, vs, c.table)
    else:
        other = ihip.KVStore.bf16(k, v, c.table) if fmt == "bf16" else ihip.KVStore.e4m3(k, v, SCALES, c.table)
    new, lens = [9, 30], torch.tensor([40, 61], dtype=torch.int32).cuda()
    nk, nv = normal(32, 39, 3, D).cuda(), normal(33, 39, 3, D).cuda()
    angles = torch.rand((64, D // 2), generator=torch.Generator().manual_seed(34))
    rope = angles.cos().cuda(), angles.sin().cuda()
    got = []
    for store in (c.store, other):
        ihip.kv_append(store, nk, nv, offsets(new).cuda(), lens, 64, rope=rope)
        out = [torch.zeros((2, 3, 64, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        got.append(ihip.kv_gather(store, lens, 64, *out))
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    for a, b in ((c.k, k), (c.v, v)) + (((c.ks, ks), (c.vs, vs)) if fmt == "mx4" else ()):
        assert torch.equal(a.view(torch.int16) if fmt == "bf16" else a, b.contiguous().view(torch.int16) if fmt == "bf16" else b)
    for big in (big_k, big_v):                           # what lies between the rows
        assert bool((big[0] == 7).all()) and bool((big[:, :, 0] == 7).all()) and bool((big[:, :, 4:] == 7).all())
    if fmt == "mx4":
        q = normal(35, 2, 6, 1, D).cuda()
        a, b = (ihip.sparse_attn_decode_mx4(ihip.Layer(q, x, lens, 1, 0, 64, max_seq_len=64), q, x)[0] for x in (c.store, other))
        assert torch.equal(a, b)
