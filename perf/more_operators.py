"""Cases of the 4-bit paged KV cache: what its operators compute in plain torch, and the calls a user
makes for the same results.

  write   rows of the cache to 4 bits, and back into other pages of the cache
  read    rows held in 4 bits back into the cache
  decode  decode attention of one layer over a cache held in 4 bits
  rows    causal attention of several positions per sequence over the same cache

A row of d elements is held as d signed 4-bit floats (magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6) and one
scale per 16 of them, a positive float of 8 bits (5 of exponent, 3 of mantissa): the largest
magnitude of the 16 over 6, to the nearest.  ``prepare`` makes what a serving program holds: the
pools, the page tables, the lengths, the queries (and the session that wraps them, where the
framework's own calls are timed).  ``run`` is one pass.
"""
import math

import numpy as np
import torch

own = False

OPS = ("write", "read", "decode", "rows")


def _case(name, op, B, Hq, Hkv, d, page, ctx, ctx_lo=0, dtype="bf16", k=1, **more):
    return {"name": name, "op": op, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "ctx": ctx,
            "ctx_lo": ctx_lo or ctx, "dtype": dtype, "k": k, **more}


def listed():
    return [
        # a decode step's new tokens of the 6/3-head model, all 16 channels: the latency of an append
        _case("write tokens", "write", 16, 6, 3, 96, 16, 2048, 1027, k=16, span=1),
        # prompts of the 12-head model moved to 4 bits behind their prefill, ragged and odd
        _case("write prompts", "write", 8, 12, 12, 64, 16, 2047, 511, k=12, span=2047),
        # a small fp32 cache, its tail
        _case("write fp32", "write", 2, 4, 4, 64, 16, 128, 101, dtype="f32", k=2, span=77),
        # one turn of a chat brought back for a prefill behind it
        _case("read turn", "read", 1, 6, 3, 96, 16, 1031, k=2, span=509),
        # the 32-head model's whole contexts, two channels
        _case("read contexts", "read", 8, 32, 32, 128, 16, 8192, 4097, k=2, span=8192),
        # one chat of the 6/3-head model: the latency of a single token
        _case("decode one chat", "decode", 1, 6, 3, 96, 16, 2049, k=2),
        # a decode batch of the 32-layer workload's shape, ragged contexts
        _case("decode batch", "decode", 32, 32, 32, 128, 16, 8192, 4096),
        # 131072-slot contexts with four query heads per kv head
        _case("decode long", "decode", 8, 32, 8, 128, 64, 131072, 70001),
        # a small fp32 cache
        _case("decode fp32", "decode", 2, 4, 4, 64, 16, 128, 97, dtype="f32", k=2),
        # five drafted tokens per sequence checked at once, the 12-head workload's shape
        _case("rows draft", "rows", 16, 12, 12, 64, 16, 2048, 1543, rows=5),
        # four drafted tokens behind 32768-slot contexts, grouped query heads
        _case("rows draft long", "rows", 8, 32, 8, 128, 64, 32768, 30011, rows=4),
        # the next 509 tokens of a prompt behind those already held
        _case("rows chunk", "rows", 1, 32, 8, 128, 16, 8701, rows=509),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    caps = {op: max(_cost(work(c)) for c in listed() if c["op"] == op) for op in OPS}
    op = rng.choice(OPS)
    while True:
        Hkv = rng.choice([1, 2, 3, 4, 8, 12, 16, 32])
        G = rng.choice([1, 1, 2, 4, 8])
        d = rng.choice([64, 96, 128])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        page = rng.choice([4, 8, 16, 16, 32, 64, 128])
        c = dict(op=op, B=log(1, 64), Hq=Hkv * G, Hkv=Hkv, d=d, page=page, dtype=dtype, k=rng.choice([1, 1, 2]))
        if op in ("write", "read"):
            ctx, c["k"] = log(1, 16384), rng.choice([1, 2, 4, 8, 16])
            c.update(ctx=ctx, ctx_lo=rng.randint(max(1, ctx // 2), ctx), span=rng.choice([1, ctx, rng.randint(1, ctx)]))
        elif op == "decode":
            ctx = log(1, 131072)
            c.update(ctx=ctx, ctx_lo=rng.randint(max(1, ctx // 2), ctx))
        else:
            rows = log(2, 600) if dtype == "bf16" else log(2, 16)
            ctx = max(rows, log(32, 32768))
            c.update(ctx=ctx, ctx_lo=rng.randint(max(rows, ctx // 2), ctx), rows=rows)
        # plain forms hold every row in 32 or 64 bits, and all scores
        if op == "rows" and c["B"] * c["Hq"] * c["rows"] * c["ctx"] > 32 * 509 * 8701:
            continue
        if op in ("write", "read") and 2 * _pool_bytes(c) > 4.4e9:
            continue
        if _cost(work(c)) <= caps[op]:
            return c


def _cost(w):
    return max(w["bytes"], w["flops"] / 50)


def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def _lens(case):
    """Lengths spread evenly over [ctx_lo, ctx]; the seed only orders them."""
    B = case["B"]
    return [case["ctx"] - (case["ctx"] - case["ctx_lo"]) * i // max(1, B - 1) for i in range(B)]


def _max_pages(case):
    return case["ctx"] // case["page"] + 1


def _pages(case):
    return sum(n // case["page"] + 1 for n in _lens(case))


def _pool_bytes(case):
    """K (or V) pool of a cache that holds the batch once."""
    return case["k"] * _pages(case) * case["Hkv"] * case["page"] * case["d"] * _elem(case)


def work(case):
    B, Hq, Hkv, d, op, e = case["B"], case["Hq"], case["Hkv"], case["d"], case["op"], _elem(case)
    packed = 2 * Hkv * (d // 2 + d // 16)  # K and V of one slot in 4 bits
    if op in ("write", "read"):
        n = case["k"] * sum(min(x, case["span"]) for x in _lens(case))
        once = n * (packed + 2 * Hkv * d * e)
        return {"bytes": 2 * once if op == "write" else once, "flops": 0}
    rows = case.get("rows", 1)
    seen = sum(rows * n - rows * (rows - 1) // 2 for n in _lens(case))
    return {"bytes": sum(_lens(case)) * packed + 2 * B * rows * Hq * d * e, "flops": 4 * seen * Hq * d}


# ------------------------------------------------------------------ the 4-bit form
def _magnitudes(device, dtype=torch.float32):
    return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device=device, dtype=dtype)


def _quantise(x):
    """Codes (uint8, one each) and scale bytes of rows x [..., d], in 64 bits: what lies next to a
    border has to fall on its own side."""
    g = x.double().unflatten(-1, (-1, 16))
    top = g.abs().amax(-1, keepdim=True)
    step = torch.exp2((torch.frexp(top / 6).exponent.clamp(min=-13) - 4).double())
    scale = (torch.round(top / 6 / step) * step).clamp(max=10240)
    y = (g / scale).abs()
    code = (y > .25).byte() + (y >= .75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)
    code = code + 8 * torch.signbit(g)
    return (code * (scale > 0)).flatten(-2), (scale.half().view(torch.int16) >> 7).byte().squeeze(-1)


def _values(code, scale):
    """Rows in 32 bits from codes [..., d] and scale bytes [..., d / 16]."""
    signed = torch.cat([_magnitudes(code.device), -_magnitudes(code.device)])
    s = (scale.short() << 7).view(torch.float16).float()
    return (signed[code.int()].unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)


def _tile(case):
    """Slots of a tile, and its bytes: codes of K, codes of V, scales of K, scales of V."""
    n = min(case["page"], 16)
    return n, (2 * n * (case["d"] // 2 + case["d"] // 16) + 15) // 16 * 16


def _pack(case, out, kv):
    """Rows kv (K, V) [pages][Hkv][P][d] as tiles out [pages][Hkv][P / n][bytes]."""
    n, d = _tile(case)[0], case["d"]
    at = 0
    parts = [_quantise(x.unflatten(2, (-1, n))) for x in kv]
    for part in [c[..., 0::2] + 16 * c[..., 1::2] for c, _ in parts] + [s for _, s in parts]:
        size = n * part.shape[-1]
        out[..., at:at + size] = part.flatten(-2)
        at += size


def _unpack(case, tiles):
    """K and V rows [..., P, d] in 32 bits of tiles [..., P / n, bytes]."""
    n, d = _tile(case)[0], case["d"]
    a, b = n * d // 2, n * d // 16
    codes = (tiles[..., :a], tiles[..., a:2 * a])
    scales = (tiles[..., 2 * a:2 * a + b], tiles[..., 2 * a + b:2 * a + 2 * b])
    return tuple(_values(torch.stack([c & 15, c >> 4], -1).flatten(-2).unflatten(-1, (n, d)),
                         s.unflatten(-1, (n, d // 16))).flatten(-3, -2) for c, s in zip(codes, scales))


# ------------------------------------------------------------------ what a program has in hand
def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 17)
    host = np.random.default_rng(int(seed) + 5)
    op, B, Hq, Hkv, d, P, k = (case[x] for x in ("op", "B", "Hq", "Hkv", "d", "page", "k"))
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    lens = host.permutation(np.array(_lens(case), dtype=np.int32))
    maxp, pages = _max_pages(case), _pages(case)

    def table(first=0):  # physical pages in no order
        order, out, at = host.permutation(pages).astype(np.int32) + first, np.full((B, maxp), -1, dtype=np.int32), 0
        for b in range(B):
            n = int(lens[b]) // P + 1
            out[b, :n] = order[at:at + n]
            at += n
        return torch.from_numpy(out).to(dev)

    s = {"case": case, "table": table(), "seq_lens": torch.from_numpy(lens).to(dev)}
    n, size = _tile(case)
    s["packed"] = torch.zeros((k, pages, Hkv, P // n, size), dtype=torch.uint8, device=dev)
    if op in ("write", "read"):
        # one cache: the rows' pages (write), and behind them the pages that they are read back into
        half = pages if op == "write" else 0
        s["src"], s["dst"] = table(), table(half)
        s["first"] = s["seq_lens"] - case["span"]
        s["first"].clamp_(min=0)
        cached = half + pages
    else:
        cached = 1  # attention over the 4-bit cache needs no other
    shape = (k, cached, Hkv, P, d)
    count = math.prod(shape) * _elem(case)
    v_at = (count + 255) // 256 * 256  # K pool, then V pool, each from a 256-byte boundary
    buf = torch.zeros(2 * v_at, dtype=torch.uint8, device=dev)
    s["k_pool"], s["v_pool"] = (buf[o:o + count].view(dt).view(shape) for o in (0, v_at))

    def rows(shape):
        # some features larger than others, as normed and rotated keys have them
        x = torch.randn(shape, generator=g, device=dev)
        return x * torch.exp(0.5 * torch.randn(shape[-1], generator=g, device=dev))

    if op == "write":
        for c in range(k):
            for pool in (s["k_pool"], s["v_pool"]):
                pool[c, :pages] = rows((pages, Hkv, P, d))
    else:
        some = max(1, (1 << 26) // (Hkv * P * d))
        for c in range(k):
            for at in range(0, pages, some):
                to = s["packed"][c, at:at + some]
                _pack(case, to, [rows((to.shape[0], Hkv, P, d)) for _ in range(2)])
    if op in ("decode", "rows"):
        lead = (B, case["rows"]) if op == "rows" else (B,)
        s["q"] = torch.randn((*lead, Hq, d), generator=g, device=dev).to(dt)
        s["out"] = torch.empty_like(s["q"])
        if op == "rows":  # the last positions of each sequence: position i sees slots 0 .. i
            s["pos"] = s["seq_lens"][:, None] - case["rows"] + torch.arange(case["rows"], device=dev, dtype=torch.int32)
    if own:  # the handles a serving program makes once for its caches
        from paper_2608_18486_gb300 import _lib
        from paper_2608_18486_gb300.session import DecodeSession, Q4Cache
        cfg = _lib.make_config(k, k, 64, Hq, Hkv, d, 1, P, case["dtype"], list(range(k)))
        s["session"] = DecodeSession(cfg, B, cached, maxp, dev, cache_buf=buf)
        s["q4"] = Q4Cache(cfg, pages, dev, cache_buf=s["packed"].view(-1))
    return s


def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


# ------------------------------------------------------------------ the framework's calls
def _own_write(s):
    c = s["case"]
    s["session"].q4_write(s["q4"], s["src"], s["table"], s["first"], s["seq_lens"], span=c["span"])
    return _own_read(s)


def _own_read(s):
    s["session"].q4_read(s["q4"], s["table"], s["dst"], s["first"], s["seq_lens"], span=s["case"]["span"])
    return s["k_pool"], s["v_pool"]


def _own_decode(s):
    s["session"].q4_decode_attn(s["case"]["k"] - 1, s["q"], s["q4"], s["table"], s["seq_lens"], s["out"])
    return s["out"]


def _own_rows(s):
    s["session"].q4_rows_attn(s["case"]["k"] - 1, s["q"], s["pos"], s["q4"], s["table"], s["out"])
    return s["out"]


_own = {"write": _own_write, "read": _own_read, "decode": _own_decode, "rows": _own_rows}


# ------------------------------------------------------------------ plain forms
def _ranged(s):
    """(sequence, page of the sequence, slot in page) of every slot in the sequences' ranges."""
    P = s["case"]["page"]
    t = torch.arange(s["table"].shape[1] * P, device=s["table"].device)
    b, t = torch.nonzero((t >= s["first"][:, None]) & (t < s["seq_lens"][:, None]), as_tuple=True)
    return b, t // P, t % P


def _plain_write(s):
    b, p, o = _ranged(s)
    src, dst = s["src"][b, p], s["dst"][b, p]
    for pool in (s["k_pool"], s["v_pool"]):
        pool[:, dst, :, o] = _values(*_quantise(pool[:, src, :, o])).to(pool.dtype)
    return s["k_pool"], s["v_pool"]


def _plain_read(s):
    b, p, o = _ranged(s)
    src, dst, n = s["table"][b, p], s["dst"][b, p], _tile(s["case"])[0]
    case = {**s["case"], "page": 1}
    a, z = n * case["d"] // 2, n * case["d"] // 16
    tiles = s["packed"][:, src, :, o // n]  # one tile per slot: the slot's own parts of it
    row = o % n
    part = lambda at, size: tiles[..., at:at + n * size].unflatten(-1, (n, size))[torch.arange(len(o)), :, :, row]  # noqa: E731
    slots = torch.cat([part(0, a // n), part(a, a // n), part(2 * a, z // n), part(2 * a + z, z // n)], -1)
    for pool, x in zip((s["k_pool"], s["v_pool"]), _unpack(case, slots[..., None, :])):
        pool[:, dst, :, o] = x.squeeze(-2).to(pool.dtype)
    return s["k_pool"], s["v_pool"]


def _cached(s):
    """K and V of the batch's slots, [B][Hkv][T][d] in 32 bits."""
    tiles = s["packed"][s["case"]["k"] - 1][s["table"].long().clamp(min=0)]
    return tuple(x.transpose(1, 2).flatten(2, 3) for x in _unpack(s["case"], tiles))


def _attend(q, K, V, seen):
    """Rows q [B][Hkv][G][R][d] over K, V [B][Hkv][T][d] where seen [B][R][T]; none: zeros."""
    scores = (q.flatten(2, 3) / math.sqrt(q.shape[-1]) @ K.transpose(-1, -2)).unflatten(2, q.shape[2:4])
    scores = scores.masked_fill(~seen[:, None, None], -math.inf)
    e = torch.exp(scores - scores.amax(-1, keepdim=True).clamp(min=-3e38))
    p = e / e.sum(-1, keepdim=True).clamp(min=1e-30)
    return (p.flatten(2, 3) @ V).unflatten(2, q.shape[2:4])


def _plain_decode(s):
    c, (K, V) = s["case"], _cached(s)
    seen = torch.arange(K.shape[2], device=K.device) < s["seq_lens"][:, None, None]
    q = s["q"].float().view(c["B"], c["Hkv"], -1, 1, c["d"])
    return _attend(q, K, V, seen).reshape(s["q"].shape).to(s["q"].dtype)


def _plain_rows(s):
    c, (K, V) = s["case"], _cached(s)
    seen = torch.arange(K.shape[2], device=K.device) <= s["pos"][..., None]
    q = s["q"].float().view(c["B"], c["rows"], c["Hkv"], -1, c["d"]).permute(0, 2, 3, 1, 4)
    return _attend(q, K, V, seen).permute(0, 3, 1, 2, 4).reshape(s["q"].shape).to(s["q"].dtype)


_plain = {"write": _plain_write, "read": _plain_read, "decode": _plain_decode, "rows": _plain_rows}


# ------------------------------------------------------------------ the definitions in 64 bits
def _nearest(x, grid):
    """Index of the nearest grid value, ties to the even index; grid ascending, x finite and >= 0."""
    mid = (grid[1:] + grid[:-1]) / 2
    low, high = torch.bucketize(x, mid, out_int32=True), torch.bucketize(x, mid, right=True, out_int32=True)
    return torch.where(low % 2 == 0, low, high)


def _held(x):
    """Rows as the 4-bit form holds them."""
    x = x.double().unflatten(-1, (-1, 16))
    byte = torch.arange(227, device=x.device)
    scales = torch.where(byte < 8, byte / 8 * 2.0 ** -14, (1 + byte % 8 / 8) * torch.exp2((byte // 8 - 15).double()))
    s = scales[_nearest(x.abs().amax(-1), 6 * scales)][..., None]
    m = _magnitudes(x.device, torch.float64)[_nearest(x.abs() / s.clamp(min=2.0 ** -20), _magnitudes(x.device, torch.float64))]
    return (torch.sign(x) * m * s).flatten(-2)


def _slot_rows(case, tiles, t):
    """K and V rows of slots t in 64 bits; tiles [pages of the sequence][P / n][bytes], one head."""
    n, d, P = _tile(case)[0], case["d"], case["page"]
    tile, r = tiles[t // P, t % P // n], t % n
    got = []
    for x in range(2):
        at = (x * n + r)[:, None] * (d // 2) + torch.arange(d // 2, device=t.device)
        byte = tile.gather(1, at).int()
        code = torch.stack([byte % 16, byte // 16], -1).flatten(1)
        e, m = code % 8 // 2, code % 2
        mag = torch.where(e == 0, m * 0.5, (1 + m * 0.5) * torch.exp2((e - 1).double()))
        at = 2 * n * (d // 2) + (x * n + r)[:, None] * (d // 16) + torch.arange(d // 16, device=t.device)
        b = tile.gather(1, at).int()
        s = torch.where(b < 8, b / 8 * 2.0 ** -14, (1 + b % 8 / 8) * torch.exp2((b // 8 - 15).double()))
        got.append(torch.where(code >= 8, -mag, mag) * s.double().repeat_interleave(16, 1))
    return got


def exact(case, seed):
    """One sequence (attention: and kv head) at a time, in 64 bits; None where those are too many."""
    s = prepare(case, seed)
    B, Hkv, d, P, k = (case[x] for x in ("B", "Hkv", "d", "page", "k"))
    lens, table, G = s["seq_lens"].tolist(), s["table"].long(), case["Hq"] // Hkv
    if case["op"] in ("write", "read"):
        if case["op"] == "read" and k * B * Hkv > 4096:
            return None
        out = [s["k_pool"].double(), s["v_pool"].double()]
        for b, n in enumerate(lens):
            t = torch.arange(max(0, n - case["span"]), n, device="cuda")
            dst, o = s["dst"].long()[b, t // P], t % P
            for c in range(k):
                if case["op"] == "write":
                    src = s["src"].long()[b, t // P]
                    for x, pool in enumerate((s["k_pool"], s["v_pool"])):
                        out[x][c, dst, :, o] = _held(pool[c, src, :, o])
                else:
                    for h in range(Hkv):
                        for x, v in enumerate(_slot_rows(case, s["packed"][c, table[b].clamp(min=0), h], t)):
                            out[x][c, dst, h, o] = v
        return out
    if B * Hkv > 4096:
        return None
    q, out = s["q"].double(), torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        t = torch.arange(n, device="cuda")
        for h in range(Hkv):
            K, V = _slot_rows(case, s["packed"][k - 1, table[b].clamp(min=0), h], t)
            for g in range(h * G, h * G + G):
                z = q[b, ..., g, :] @ K.T / d ** 0.5
                if case["op"] == "rows":
                    z = torch.where(t > s["pos"][b].long()[:, None], -math.inf, z)
                out[b, ..., g, :] = torch.softmax(z, -1) @ V
    return out
