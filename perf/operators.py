"""Filling, reading back and attending over KV caches, as measurable cases: the library's operators and their plain forms.

  append    new tokens' keys and values written into a cache (contiguous or paged; bf16, E4M3 or 4-bit rows), the position
            rotation applied to keys and queries on the way
  prompt    dense causal attention of packed prompts, grouped heads, with or without tokens that are there already
  decode4   decode attention over a 4-bit cache: all keys, or sink, kept blocks and window
  gather    a cache's rows, widened to contiguous bf16

128 dims a head, as everywhere in the library.  4-bit rows are OCP MX FP4: E2M1 codes, element 2i in the low half of byte i, and a
scale 2^(s - 127) for every 32 of them, the smallest power of two with which the largest magnitude of the 32 is at most 7.
"""
import math

import torch

own = False

D = 128
FP8_SCALE = 1.0 / 64
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, op, **kw):
    c = dict(op=op, Hq=32, Hkv=8, fmt="bf16", page=0, new="", ctx="", rotate=True, gather=False, n_sink=0, n_stream=0, n_blocks=0, block=16)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def _text(xs):
    return ",".join(str(x) for x in xs)


def listed():
    return [
        # one decode step of a serving batch: a token of each sequence into 16-token E4M3 pages (what a step appends does not depend on
        # how long the contexts are; short ones let the whole pool be the output)
        _case("append-decode-fp8-b32", "append", fmt="fp8", page=16, new=_text([1] * 32), ctx=_text(37 + (i * 29) % 60 for i in range(32))),
        # prompts of a batch, one after the other, into 64-token bf16 pages
        _case("append-prompts-bf16", "append", page=64, new="1801,7,640,2048,1,903,0,1537"),
        # a long document into a 4-bit cache, and the cache's rows read back for the next chunk's prefill
        _case("append-gather-mx4-32k", "append", fmt="mx4", new="32768", gather=True),
        # a few chat turns, odd lengths, one place of the batch empty: a chain of latencies
        _case("prompt-short", "prompt", new="1,77,300,0,201"),
        # ordinary prompts of a batch
        _case("prompt-b8-2k", "prompt", new="1801,2048,640,1999,1203,903,1024,1537"),
        # one long document
        _case("prompt-32k", "prompt", new="32749"),
        # a turn on contexts that are there already, two heads a group
        _case("prompt-on-context", "prompt", Hq=16, new="1500,700", ctx="12000,20011"),
        # one short sequence, 16-token pages: a chain of latencies
        _case("decode4-4k", "decode4", fmt="mx4", page=16, ctx="4099"),
        # a serving batch that attends to all of its keys
        _case("decode4-b32-16k", "decode4", fmt="mx4", page=16, ctx=_text(16384 - (i * 577) % 9001 for i in range(32))),
        # long contexts, the keys that a pruning plan left: sink, 256 blocks of 16, window
        _case("decode4-blocks-b4-250k", "decode4", fmt="mx4", ctx="250007,250007,201111,187654", n_sink=128, n_stream=1024, n_blocks=256),
        # a long 4-bit context widened for a prefill chunk
        _case("gather-mx4-128k", "gather", fmt="mx4", page=64, ctx="131072"),
        # E4M3 pages of a batch, odd lengths
        _case("gather-fp8-b8", "gather", fmt="fp8", page=16, ctx="4001,2777,911,4096,1,1300,3500,77"),
    ]


def draw(rng):
    """One more case: an operator, then sizes spread over its range (logarithmically where it is wide)."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def ragged(B, longest):
        return [longest] + [max(1, int(longest * rng.uniform(0.3, 1.0))) for _ in range(B - 1)]

    op = rng.choice(["append", "append", "prompt", "prompt", "decode4", "decode4", "gather"])
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (64, 8), (16, 8), (8, 8), (16, 4), (16, 2)])
    page = rng.choice([0, 16, 64])
    base = dict(Hq=Hq, Hkv=Hkv, page=page)
    if op == "append":
        fmt = rng.choice(["bf16", "fp8", "mx4"])
        if rng.random() < 0.4:
            B = log(4, 64)
            return _case("", op, fmt=fmt, new=_text([1] * B), ctx=_text(rng.randrange(0, 120) for _ in range(B)), gather=fmt == "mx4", rotate=rng.random() < 0.8, **base)
        B = log(1, 8)
        return _case("", op, fmt=fmt, new=_text(ragged(B, log(64, 16384 // B))), gather=fmt == "mx4", rotate=rng.random() < 0.8, **base)
    if op == "prompt":
        base.pop("page")
        B = log(1, 8)
        new = ragged(B, log(32, 16384 // B))
        ctx = _text(rng.randrange(0, 8192) for _ in range(B)) if rng.random() < 0.3 else ""
        return _case("", op, new=_text(new), ctx=ctx, **base)
    if op == "decode4":
        if rng.random() < 0.4:
            B = log(1, 8)
            return _case("", op, fmt="mx4", ctx=_text(ragged(B, log(16384, 400000 // B) | 1)), n_sink=rng.choice([64, 128, 100]), n_stream=rng.choice([512, 1024, 1000]),
                         n_blocks=log(48, 400), block=rng.choice([8, 16, 32]), **base)
        B = log(1, 48)
        return _case("", op, fmt="mx4", ctx=_text(ragged(B, log(500, 400000 // B) | 1)), **base)
    B = log(1, 8)
    return _case("", op, fmt=rng.choice(["fp8", "mx4", "mx4"]), ctx=_text(ragged(B, log(500, 100000 // B) | 1)), **base)


# ---- inputs ------------------------------------------------------------------
def _lens(text):
    return [int(x) for x in text.split(",")] if text else []


def _totals(case):
    """(new tokens, context before them, keys after) of every sequence."""
    new, ctx = _lens(case["new"]), _lens(case["ctx"])
    new, ctx = new or [0] * len(ctx), ctx or [0] * len(new)
    return new, ctx, [a + b for a, b in zip(new, ctx)]


def _ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _offsets(xs):
    at = [0]
    for x in xs:
        at.append(at[-1] + x)
    return _ints(at)


def _rope_table(n_pos):
    j = torch.arange(D // 2, dtype=torch.float64, device="cuda")
    ang = torch.arange(n_pos, dtype=torch.float64, device="cuda").view(-1, 1) * 10000.0 ** (-2.0 * j / D).view(1, -1)
    return ang.cos().float().contiguous(), ang.sin().float().contiguous()


def _to_mx4(x):
    """Rows x [..., 128] -> codes uint8 [..., 64], scales uint8 [..., 4]."""
    g = x.unflatten(-1, (4, 32))
    m, e = torch.frexp(g.abs().amax(-1))
    e = torch.where(m <= 0.875, e - 3, e - 2).clamp(min=-100)
    e = torch.where(m == 0, torch.full_like(e, -100), e)
    a = torch.ldexp(g, -e.unsqueeze(-1))
    sign = (a < 0).to(torch.uint8) * 8
    a = a.abs()
    c = sign
    for border, tie_up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        c = c + ((a >= border) if tie_up else (a > border)).to(torch.uint8)
    c = c.flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _to_fp8(x):
    return (x / FP8_SCALE).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _rows(shape, fmt, gen):
    """Cache rows of N(0,1) values in the format: {"x": rows, "s": scales of 4-bit ones}."""
    x = torch.randn((*shape, D), dtype=torch.bfloat16, device="cuda", generator=gen)
    if fmt == "bf16":
        return {"x": x}
    if fmt == "fp8":
        return {"x": torch.cat([_to_fp8(p.float()) for p in x.split(max(1, shape[0] // 8))])}
    parts = [_to_mx4(p.float()) for p in x.flatten(0, -2).split(1 << 20)]
    return {"x": torch.cat([p[0] for p in parts]).view(*shape, D // 2), "s": torch.cat([p[1] for p in parts]).view(*shape, 4)}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 23)
    new, ctx, total = _totals(case)
    B, Hq, Hkv, N, T = len(new), case["Hq"], case["Hkv"], sum(new), max(total)
    s = {"case": case, "T": T, "seq_lens": _ints(total)}
    if case["op"] in ("append", "prompt"):
        K = sum(total) if case["op"] == "prompt" else N
        s["q"] = torch.randn((N, Hq, D), dtype=torch.bfloat16, device="cuda", generator=gen)
        s["k"] = torch.randn((K, Hkv, D), dtype=torch.bfloat16, device="cuda", generator=gen)
        s["v"] = torch.randn((K, Hkv, D), dtype=torch.bfloat16, device="cuda", generator=gen)
        s["cu_q"], s["cu_k"] = _offsets(new), _offsets(total)
        s["max_q"] = max(new)
        if case["op"] == "prompt":
            return s
        s["cos"], s["sin"] = _rope_table(T)
    page = case["page"]
    if page:
        n = -(-T // page)
        s["table"] = torch.randperm(B * n, device="cuda", generator=gen).to(torch.int32).view(B, n).contiguous()
        shape = (B * n, Hkv, page)
    else:
        s["table"], shape = None, (B, Hkv, T)
    s["kc"], s["vc"] = _rows(shape, case["fmt"], gen), _rows(shape, case["fmt"], gen)
    if case["op"] == "gather" or case["gather"]:
        s["k_out"] = torch.zeros((B, Hkv, T, D), dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.zeros((B, Hkv, T, D), dtype=torch.bfloat16, device="cuda")
    if case["op"] == "decode4":
        s["q"] = torch.randn((B, Hq, 1, D), dtype=torch.bfloat16, device="cuda", generator=gen)
        if case["n_blocks"]:                         # per (sequence, KV head) distinct blocks of its middle range, ascending
            n_blk = (s["seq_lens"].long() - case["n_stream"] - case["n_sink"]) // case["block"]
            pick = torch.rand((B, Hkv, int(n_blk.max())), device="cuda", generator=gen)
            pick.masked_fill_(torch.arange(pick.shape[2], device="cuda") >= n_blk.view(-1, 1, 1), 2.0)
            idx = pick.topk(case["n_blocks"], dim=2, largest=False).indices.sort(dim=2).values
            s["blocks"] = (case["n_sink"] + idx * case["block"]).to(torch.int32).view(B * Hkv, -1).contiguous()
    return s


# ---- the library's calls -------------------------------------------------------
def _store(s):
    import paper_2502_08910_amd as ih
    if "store" not in s:                             # the handle of a cache, made once as a program would
        f, k, v = s["case"]["fmt"], s["kc"], s["vc"]
        if f == "bf16":
            s["store"] = ih.KVStore.bf16(k["x"], v["x"], block_table=s["table"])
        elif f == "fp8":
            s["store"] = ih.KVStore.e4m3(k["x"], v["x"], (FP8_SCALE, FP8_SCALE), block_table=s["table"])
        else:
            s["store"] = ih.KVStore.mx4(k["x"], v["x"], k["s"], v["s"], block_table=s["table"])
    return s["store"]


def _run_own(s):
    import paper_2502_08910_amd as ih
    case = s["case"]
    if case["op"] == "prompt":
        out, lse = ih.prompt_attn(s["q"], s["k"], s["v"], s["cu_q"], s["max_q"], cu_k=s["cu_k"], want_lse=True)
        return {"out": out, "lse": lse}
    store = _store(s)
    if case["op"] == "append":
        rope = (s["cos"], s["sin"]) if case["rotate"] else None
        q, _ = ih.kv_append(store, s["k"], s["v"], s["cu_q"], s["seq_lens"], s["T"], q=s["q"] if rope else None, rope=rope)
        got = {"q": q} if rope else {}
        if case["gather"]:
            got["k"], got["v"] = ih.kv_gather(store, s["seq_lens"], s["T"], k_out=s["k_out"], v_out=s["v_out"])
            return got
        return {**got, **_pools(s)}
    if case["op"] == "gather":
        k, v = ih.kv_gather(store, s["seq_lens"], s["T"], k_out=s["k_out"], v_out=s["v_out"])
        return {"k": k, "v": v}
    if "layer" not in s:
        s["layer"] = ih.Layer(s["q"], store, s["seq_lens"], 1, case["n_sink"], case["n_stream"] or s["T"], max_seq_len=s["T"])
        s["ws"] = s["layer"].workspace(ih.OP_ATTN_DECODE_MX4, [case["block"]], [max(case["n_blocks"], 1)])
    out, lse = ih.sparse_attn_decode_mx4(s["layer"], s["q"], store, s.get("blocks"), case["block"], want_lse=True, ws=s["ws"])
    return {"out": out, "lse": lse}


# ---- the plain forms -------------------------------------------------------------
def _pools(s):
    """A bf16 or E4M3 cache as the values that it holds."""
    view = (lambda x: x.view(torch.float8_e4m3fn)) if s["case"]["fmt"] == "fp8" else (lambda x: x)
    return {"k": view(s["kc"]["x"]), "v": view(s["vc"]["x"])}


def _turned(x, pos, s):
    c, n = s["cos"][pos].unsqueeze(1), s["sin"][pos].unsqueeze(1)
    e, o = x[..., 0::2], x[..., 1::2]
    return torch.stack((e * c - o * n, e * n + o * c), dim=-1).flatten(-2)


def _row_index(s, b, pos):
    """Rows of (sequence b, all KV heads, position pos) in the flattened cache: [..., Hkv]."""
    case, h = s["case"], torch.arange(s["case"]["Hkv"], device="cuda")
    per = case["page"] or s["T"]
    first = b if s["table"] is None else s["table"].long()[b, pos // per]
    return (first.unsqueeze(-1) * case["Hkv"] + h) * per + (pos % per).unsqueeze(-1)


def _widened(c, fmt, rows):
    """Cache rows as fp32 values [..., 128]."""
    x = c["x"].flatten(0, -2)[rows]
    if fmt == "bf16":
        return x.float()
    if fmt == "fp8":
        return x.view(torch.float8_e4m3fn).float() * FP8_SCALE
    t = torch.tensor(E2M1 + tuple(-y for y in E2M1), device="cuda")
    codes = torch.stack((x & 15, x >> 4), dim=-1).flatten(-2)
    scale = torch.ldexp(torch.ones((), device="cuda"), c["s"].flatten(0, -2)[rows].int() - 127)
    return (t[codes.int()].unflatten(-1, (4, 32)) * scale.unsqueeze(-1)).flatten(-2)


def _token_places(s):
    """Sequence and position of every new token."""
    new = s["cu_q"].long().diff()
    b = torch.repeat_interleave(torch.arange(new.numel(), device="cuda"), new, output_size=s["k"].shape[0])
    i = torch.arange(s["k"].shape[0], device="cuda")
    return b, s["seq_lens"].long()[b] - new[b] + i - s["cu_q"].long()[b]


def _append(s):
    case = s["case"]
    b, pos = _token_places(s)
    rows = _row_index(s, b, pos)
    got = {}
    k, v = s["k"].float(), s["v"].float()
    if case["rotate"]:
        got["q"] = _turned(s["q"].float(), pos, s).bfloat16()
        k = _turned(k, pos, s)
    for x, c in ((k, s["kc"]), (v, s["vc"])):
        flat = c["x"].flatten(0, -2)
        if case["fmt"] == "bf16":
            flat[rows] = x.bfloat16()
        elif case["fmt"] == "fp8":
            flat[rows] = _to_fp8(x)
        else:
            flat[rows], c["s"].flatten(0, -2)[rows] = _to_mx4(x)
    return {**got, **(_gather(s) if case["gather"] else _pools(s))}


def _gather(s):
    B, T = s["seq_lens"].numel(), s["T"]
    pos = torch.arange(T, device="cuda").expand(B, T)
    rows = _row_index(s, torch.arange(B, device="cuda").view(-1, 1), pos).transpose(1, 2)        # [B, Hkv, T]
    there = (pos < s["seq_lens"].view(-1, 1)).view(B, 1, T, 1)
    for c, out in ((s["kc"], s["k_out"]), (s["vc"], s["v_out"])):
        out.copy_(torch.where(there, _widened(c, s["case"]["fmt"], rows).bfloat16(), out))
    return {"k": s["k_out"], "v": s["v_out"]}


def _softmax_rows(s, v):
    """Scores s with -inf where nothing is seen, values v -> weighted values (0 where a row sees nothing), log-sum-exp."""
    m = s.amax(-1, keepdim=True)
    p = (s - torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    l = p.sum(-1, keepdim=True)
    return (p @ v) / torch.where(l == 0, torch.ones_like(l), l), (m + l.log()).squeeze(-1)


PLAIN_ROWS = 4096             # queries of a sequence whose scores are held at once


def _prompt(s):
    case = s["case"]
    Hq, Hkv, G = case["Hq"], case["Hkv"], case["Hq"] // case["Hkv"]
    new, _, total = _totals(case)
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    q0 = k0 = 0
    for n, t in zip(new, total):
        k = s["k"][k0:k0 + t].float().permute(1, 2, 0).contiguous()       # [Hkv, D, t]
        v = s["v"][k0:k0 + t].float().transpose(0, 1).contiguous()
        for i in range(0, n, PLAIN_ROWS):
            j = min(n, i + PLAIN_ROWS)
            seen = t - n + j                         # keys that the last of these queries sees
            q = s["q"][q0 + i:q0 + j].float().view(j - i, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * (j - i), D)
            sc = (q @ k[:, :, :seen]).mul_(1 / math.sqrt(D)).view(Hkv, G, j - i, seen)
            sc.masked_fill_(torch.arange(seen, device="cuda") > (t - n + torch.arange(i, j, device="cuda")).view(-1, 1), -math.inf)
            o, r = _softmax_rows(sc.view(Hkv, G * (j - i), seen), v[:, :seen])
            out[q0 + i:q0 + j] = o.view(Hq, j - i, D).transpose(0, 1).bfloat16()
            lse[q0 + i:q0 + j] = r.view(Hq, j - i).t()
        q0, k0 = q0 + n, k0 + t
    return {"out": out, "lse": lse}


def _attended(s):
    """Positions [B, Hkv, S] that a decode step attends to, and which of them are there."""
    case, lens = s["case"], s["seq_lens"].long()
    B, Hkv = lens.numel(), case["Hkv"]
    if not case["n_blocks"]:
        pos = torch.arange(s["T"], device="cuda").expand(B, Hkv, -1)
        return pos, pos < lens.view(-1, 1, 1)
    sink = torch.arange(case["n_sink"], device="cuda").expand(B, Hkv, -1)
    mid = (s["blocks"].long().view(B, Hkv, -1, 1) + torch.arange(case["block"], device="cuda")).flatten(2)
    window = (lens.view(-1, 1, 1) - case["n_stream"] + torch.arange(case["n_stream"], device="cuda")).expand(-1, Hkv, -1)
    pos = torch.cat((sink, mid, window), dim=2)
    return pos, torch.ones_like(pos, dtype=torch.bool)


def _decode4(s):
    case = s["case"]
    B, Hq, Hkv = s["q"].shape[0], case["Hq"], case["Hkv"]
    pos, there = _attended(s)
    per = case["page"] or s["T"]
    b = torch.arange(B, device="cuda").view(-1, 1, 1)
    first = b.expand_as(pos) if s["table"] is None else s["table"].long()[b, pos // per]
    rows = (first * Hkv + torch.arange(Hkv, device="cuda").view(1, -1, 1)) * per + pos % per
    k = _widened(s["kc"], "mx4", rows).transpose(2, 3).contiguous()
    sc = (s["q"].float().view(B, Hkv, Hq // Hkv, D) @ k) / math.sqrt(D)
    del k
    sc = sc.masked_fill(~there.unsqueeze(2), -math.inf)
    o, r = _softmax_rows(sc, _widened(s["vc"], "mx4", rows))
    return {"out": o.view(B, Hq, 1, D).bfloat16(), "lse": r.view(B, Hq, 1)}


def run(s):
    if own:
        return _run_own(s)
    return {"append": _append, "gather": _gather, "prompt": _prompt, "decode4": _decode4}[s["case"]["op"]](s)


# ---- what a pass cannot do without -----------------------------------------------
ROW = {"bf16": 256, "fp8": 128, "mx4": 68}


def work(case):
    new, ctx, total = _totals(case)
    Hq, Hkv, N, row = case["Hq"], case["Hkv"], sum(new), ROW[case["fmt"]]
    if case["op"] == "prompt":
        pairs = sum(n * c + n * (n + 1) / 2 for n, c in zip(new, ctx))
        return {"bytes": 2.0 * D * (2 * N * Hq + 2 * sum(total) * Hkv) + 4.0 * N * Hq, "flops": 4.0 * D * Hq * pairs}
    if case["op"] == "decode4":
        keys = sum(total) if not case["n_blocks"] else len(total) * (case["n_sink"] + case["n_stream"] + case["n_blocks"] * case["block"])
        return {"bytes": 2.0 * row * Hkv * keys + len(total) * Hq * (4.0 * D + 4), "flops": 4.0 * D * Hq * keys}
    read_back = 2.0 * (row + 256) * Hkv * sum(total)
    if case["op"] == "gather":
        return {"bytes": read_back, "flops": 2.0 * D * Hkv * sum(total)}
    turned = N * Hq * 512.0 + 512.0 * min(N, max(total)) if case["rotate"] else 0.0
    return {"bytes": turned + 2.0 * (256 + row) * Hkv * N + (read_back if case["gather"] else 0.0), "flops": 3.0 * D * (Hq + Hkv) * N}


# ---- the same in 64 bits, from the definitions -----------------------------------
def _exact_values(c, fmt):
    """All rows of a cache as float64 values."""
    if fmt == "bf16":
        return c["x"].double()
    if fmt == "fp8":
        return c["x"].view(torch.float8_e4m3fn).double() * FP8_SCALE
    v = torch.empty((*c["x"].shape[:-1], D), dtype=torch.float64, device="cuda")
    for part, shift in ((0, 0), (1, 4)):
        code = (c["x"] >> shift) & 15
        mag, exp = (code & 1).double(), (code >> 1) & 3
        mag = torch.where(exp == 0, mag / 2, (2 + mag) / 2 * 2.0 ** (exp.double() - 1))
        v[..., part::2] = torch.where(code > 7, -mag, mag)
    return v * (2.0 ** (c["s"].double() - 127)).repeat_interleave(32, dim=-1)


def _nearest(x, borders, values):
    """x [...] >= 0 -> the nearest of `values`; borders are the middles, and a tie goes to the value with the even code."""
    i = torch.bucketize(x, borders)                  # borders below x
    at_border = torch.zeros_like(x, dtype=torch.bool)
    at_border[i < borders.numel()] = x[i < borders.numel()] == borders[i[i < borders.numel()]]
    i = torch.where(at_border & (i % 2 == 1), i + 1, i)
    return values[i]


def _exact_stored(x, fmt):
    """float64 rows as the values that a cache of the format keeps of them."""
    if fmt == "bf16":
        return x
    if fmt == "fp8":
        codes = torch.arange(127, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn).double()
        return torch.sign(x) * _nearest((x / FP8_SCALE).abs(), (codes[1:] + codes[:-1]) / 2, codes) * FP8_SCALE
    g = x.unflatten(-1, (4, 32))
    top = g.abs().amax(-1, keepdim=True).clamp(min=1e-300)
    e = torch.ceil(torch.log2(top / 7))
    e = torch.where(top > 7 * 2.0 ** e, e + 1, torch.where(top <= 7 * 2.0 ** (e - 1), e - 1, e)).clamp(min=-100)
    values = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    return (torch.sign(g) * _nearest(g.abs() / 2.0 ** e, (values[1:] + values[:-1]) / 2, values) * 2.0 ** e).flatten(-2)


def _exact_turned(x, pos, s):
    z = torch.view_as_complex(x.unflatten(-1, (D // 2, 2)).contiguous())
    return torch.view_as_real(z * torch.complex(s["cos"][pos].double(), s["sin"][pos].double()).unsqueeze(1)).flatten(-2)


def _exact_append(s, case):
    new, ctx, total = _totals(case)
    got, at = {}, 0
    pos = torch.cat([torch.arange(c, t, device="cuda") for c, t in zip(ctx, total)])
    k, v = s["k"].double(), s["v"].double()
    if case["rotate"]:
        got["q"] = _exact_turned(s["q"].double(), pos, s)
        k = _exact_turned(k, pos, s)
    kept = {"k": _exact_stored(k, case["fmt"]), "v": _exact_stored(v, case["fmt"])}
    per = case["page"] or s["T"]
    for name, c in (("k", s["kc"]), ("v", s["vc"])):
        pool, at = _exact_values(c, case["fmt"]), 0
        for b, (n, c0) in enumerate(zip(new, ctx)):
            p = torch.arange(c0, c0 + n, device="cuda")
            page = s["table"][b].long()[p // per] if s["table"] is not None else torch.full_like(p, b)
            pool[page, :, p % per] = kept[name][at:at + n]
            at += n
        got[name] = pool if not case["gather"] else _exact_contiguous(pool, s, case)
        if case["fmt"] == "fp8" and not case["gather"]:
            got[name] = got[name] / FP8_SCALE        # the pool's bytes, as values
    return got


def _exact_contiguous(pool, s, case):
    _, _, total = _totals(case)
    per = case["page"] or s["T"]
    out = torch.zeros((len(total), case["Hkv"], s["T"], D), dtype=torch.float64, device="cuda")
    for b, t in enumerate(total):
        p = torch.arange(t, device="cuda")
        page = s["table"][b].long()[p // per] if s["table"] is not None else torch.full_like(p, b)
        out[b, :, :t] = pool[page, :, p % per].transpose(0, 1)
    return out


def _exact_prompt(s, case):
    new, _, total = _totals(case)
    G = case["Hq"] // case["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    q0 = k0 = 0
    for n, t in zip(new, total):
        for h in range(case["Hq"]):
            q = s["q"][q0:q0 + n, h].double()
            k, v = (s[x][k0:k0 + t, h // G].double() for x in ("k", "v"))
            kt = k.t().contiguous()
            for i in range(0, n, 8192):
                j = min(n, i + 8192)
                last = t - n + torch.arange(i, j, device="cuda").view(-1, 1)
                sc = (q[i:j] @ kt / math.sqrt(D)).masked_fill_(torch.arange(t, device="cuda") > last, -math.inf)
                r = torch.logsumexp(sc, dim=1, keepdim=True)
                out[q0 + i:q0 + j, h] = torch.nan_to_num((sc - r).exp_()) @ v
                lse[q0 + i:q0 + j, h] = r.squeeze(1)
        q0, k0 = q0 + n, k0 + t
    return {"out": out, "lse": lse}


def _exact_decode4(s, case):
    _, _, total = _totals(case)
    G, per = case["Hq"] // case["Hkv"], case["page"] or s["T"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device="cuda")
    for b, t in enumerate(total):
        for g in range(case["Hkv"]):
            p = torch.arange(t, device="cuda")
            if case["n_blocks"]:
                keep = (p < case["n_sink"]) | (p >= t - case["n_stream"])
                st = s["blocks"][b * case["Hkv"] + g].long()
                keep[(st.view(-1, 1) + torch.arange(case["block"], device="cuda")).flatten()] = True
                p = p[keep]
            page = s["table"][b].long()[p // per] if s["table"] is not None else torch.full_like(p, b)
            k, v = (_exact_values({n: y[page, g, p % per] for n, y in c.items()}, "mx4") for c in (s["kc"], s["vc"]))
            sc = s["q"][b, g * G:(g + 1) * G, 0].double() @ k.t().contiguous() / math.sqrt(D)
            r = torch.logsumexp(sc, dim=1, keepdim=True)
            out[b, g * G:(g + 1) * G, 0] = (sc - r).exp() @ v
            lse[b, g * G:(g + 1) * G, 0] = r.squeeze(1)
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s, case)
    if case["op"] == "gather":
        return {n: _exact_contiguous(_exact_values(c, case["fmt"]), s, case) for n, c in (("k", s["kc"]), ("v", s["vc"]))}
    return _exact_prompt(s, case) if case["op"] == "prompt" else _exact_decode4(s, case)
