"""Cases of the long-context operators of the paged KV cache: what they compute in plain torch, and
the calls a user makes for the same results.

  window          decode attention over a sliding window and the first slots (sinks)
  window_prefill  the same mask for many query positions at once
  prefix          decode attention of a batch whose sequences share their first pages
  mass            decode attention that also adds each slot's attention weight to its sum
  evict           compaction of the cache to a budget by those sums

``prepare`` makes what a serving program holds: the cache pools, the page table, the lengths, the
queries (and the session that wraps them, where the framework's own calls are timed).  ``run`` is one
call.
"""
import math

import numpy as np
import torch

own = False

OPS = ("window", "window_prefill", "prefix", "mass", "evict")


def _case(name, op, B, Hq, Hkv, d, page, ctx, ctx_lo=0, dtype="bf16", k=1, **more):
    return {"name": name, "op": op, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "ctx": ctx,
            "ctx_lo": ctx_lo or ctx, "dtype": dtype, "k": k, **more}


def listed():
    return [
        # one chat of the 6/3-head model past its window: the latency of a single token
        _case("window one chat", "window", 1, 6, 3, 96, 16, 2049, k=2, sinks=4, window=509),
        # a decode batch of the 32-layer workload's shape, ragged contexts
        _case("window batch", "window", 32, 32, 32, 128, 16, 8192, 4096, sinks=4, window=1024),
        # 131072-slot contexts with four query heads per kv head
        _case("window long", "window", 8, 32, 8, 128, 64, 131072, 70001, sinks=16, window=4096),
        # short prompts of the 6/3-head model, an odd number of tokens
        _case("prefill short", "window_prefill", 2, 6, 3, 96, 16, 509, sinks=4, window=128, rows=509),
        # a long prompt in one call
        _case("prefill long", "window_prefill", 1, 32, 32, 128, 16, 8192, sinks=4, window=1024, rows=8192),
        # a few sequences behind a system prompt
        _case("prefix few", "prefix", 4, 6, 3, 96, 16, 589, 519, k=2, shared=32),
        # a batch of the 12-head workload's shape sampling from one prompt
        _case("prefix batch", "prefix", 16, 12, 12, 64, 16, 2177, 1921, shared=120),
        # many requests over one long document, grouped query heads
        _case("prefix long", "prefix", 64, 32, 8, 128, 64, 33792, 32833, shared=512),
        # a small fp32 cache
        _case("mass small", "mass", 2, 4, 4, 64, 16, 128, 97, dtype="f32", k=2),
        # 32768-slot contexts, the sums kept for a later eviction
        _case("mass long", "mass", 8, 32, 32, 128, 64, 32768, 30011),
        # one sequence of a small model cut to half
        _case("evict small", "evict", 1, 6, 3, 96, 16, 1031, k=4, budget=509, sinks=4, recent=64),
        # the same heads, every channel of a whole batch
        _case("evict batch", "evict", 16, 6, 3, 96, 16, 2048, 1543, k=16, budget=1024, sinks=4, recent=256),
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
        page = rng.choice([8, 16, 16, 32, 64, 128])
        B = log(1, 64)
        c = dict(op=op, B=B, Hq=Hkv * G, Hkv=Hkv, d=d, page=page, dtype=dtype, k=rng.choice([1, 1, 2]))
        if op == "window":
            ctx = log(64, 131072)
            c.update(ctx=ctx, ctx_lo=rng.randint(max(1, ctx // 2), ctx), sinks=rng.choice([0, 1, 4, 16, 64]),
                     window=log(32, 4096))
        elif op == "window_prefill":
            ctx, c["B"], c["dtype"] = log(32, 8192), log(1, 8), "bf16"
            c.update(ctx=ctx, ctx_lo=ctx, sinks=rng.choice([0, 1, 4, 16, 64]), window=log(32, 2048),
                     rows=rng.randint(max(1, ctx // 3), ctx))
        elif op == "prefix":
            c["B"], shared = log(2, 64), max(1, log(128, 32768) // page)
            ctx = shared * page + log(8, 1024)
            c.update(shared=shared, ctx=ctx, ctx_lo=rng.randint(shared * page + 1, ctx))
        elif op == "mass":
            ctx = log(64, 32768)
            c.update(ctx=ctx, ctx_lo=rng.randint(max(1, ctx // 2), ctx))
        else:
            ctx = log(128, 32768)
            budget = rng.randint(ctx // 4, ctx - 8)
            c.update(ctx=ctx, ctx_lo=rng.randint(ctx - (ctx - budget) // 2, ctx), budget=budget, k=rng.choice([1, 2, 4, 8]),
                     sinks=rng.choice([0, 1, 4, 16]), recent=rng.randint(0, budget // 4))
        # plain forms of a prefill hold all scores: as many as the largest listed case at most
        if op == "window_prefill" and c["B"] * c["Hq"] * c["rows"] * c["ctx"] > 32 * 8192 * 8192:
            continue
        if _cost(work(c)) <= caps[op] and 2 * _pool_bytes(c) <= 4.4e9:
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


def _pool_pages(case):
    shared = case.get("shared", 0)
    return shared + sum(n // case["page"] + 1 - shared for n in _lens(case))


def _pool_bytes(case):
    return case["k"] * _pool_pages(case) * case["Hkv"] * case["page"] * case["d"] * _elem(case)


def work(case):
    B, Hq, Hkv, d, op, e = case["B"], case["Hq"], case["Hkv"], case["d"], case["op"], _elem(case)
    row = 2 * Hkv * d * e  # K and V of one slot
    if op == "evict":
        # every sum read, every new sum and kept index written, every kept row behind the sinks moved
        units, T = case["k"] * Hkv, _max_pages(case) * case["page"]
        moved = sum(min(n, case["budget"]) - case["sinks"] for n in _lens(case) if n > case["budget"])
        return {"bytes": 4 * units * (sum(_lens(case)) + B * T + B * case["budget"]) + 2 * case["k"] * moved * row,
                "flops": 0}
    if op == "window_prefill":
        s, w, first = case["sinks"], case["window"], case["ctx"] - case["rows"]
        seen = sum(min(p + 1, s + w) for p in range(first, case["ctx"]))
        read = min(case["ctx"], s + w - 1 + case["rows"])
        return {"bytes": B * (read * row + 2 * case["rows"] * Hq * d * e), "flops": 4 * B * seen * Hq * d}
    if op == "window":
        seen = read = sum(min(n, case["sinks"] + case["window"]) for n in _lens(case))
    else:
        seen = read = sum(_lens(case))
    if op == "prefix":
        read -= (B - 1) * case["shared"] * case["page"]
    return {"bytes": read * row + 2 * B * Hq * d * e + (8 * read * Hkv if op == "mass" else 0), "flops": 4 * seen * Hq * d}


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 17)
    host = np.random.default_rng(int(seed) + 5)
    B, Hq, Hkv, d, P, k = (case[x] for x in ("B", "Hq", "Hkv", "d", "page", "k"))
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    lens = host.permutation(np.array(_lens(case), dtype=np.int32))
    maxp, pages, shared = _max_pages(case), _pool_pages(case), case.get("shared", 0)
    order = host.permutation(pages).astype(np.int32)  # physical pages in no order
    table = np.full((B, maxp), -1, dtype=np.int32)
    table[:, :shared] = order[:shared]
    at = shared
    for b in range(B):
        n = int(lens[b]) // P + 1
        table[b, shared:n] = order[at:at + n - shared]
        at += n - shared
    # one buffer, K pool then V pool, each from a 256-byte boundary
    half = (_pool_bytes(case) + 255) // 256 * 256
    buf = torch.empty(2 * half, dtype=torch.uint8, device=dev)
    shape = (k, pages, Hkv, P, d)
    kp, vp = (buf[o:o + _pool_bytes(case)].view(dt).view(shape) for o in (0, half))
    kp.normal_(generator=g)
    vp.normal_(generator=g)
    s = {"case": case, "k_pool": kp, "v_pool": vp, "page_table": torch.from_numpy(table).to(dev),
         "seq_lens": torch.from_numpy(lens).to(dev)}
    rows = (B, case["rows"], Hq, d) if case["op"] == "window_prefill" else (B, Hq, d)
    s["q"] = torch.randn(rows, generator=g, device=dev).to(dt)
    s["out"] = torch.empty_like(s["q"])
    if case["op"] == "window_prefill":
        pos = torch.arange(case["ctx"] - case["rows"], case["ctx"], dtype=torch.int32, device=dev)
        s["pos"] = pos.expand(B, -1).contiguous()
    if case["op"] in ("mass", "evict"):
        # sums of attention weights: most slots little, a few much, some nothing at all
        m = torch.exp(1.5 * torch.randn((k, B, Hkv, maxp * P), generator=g, device=dev)) / 64
        m *= torch.rand(m.shape, generator=g, device=dev) > 0.125
        m *= torch.arange(maxp * P, device=dev) < s["seq_lens"][None, :, None, None]
        s["mass"] = m
    if case["op"] == "evict":
        s["mass_out"] = torch.empty_like(m)
        s["kept"] = torch.empty((k, B, Hkv, case["budget"]), dtype=torch.int32, device=dev)
        s["new_lens"] = torch.empty(B, dtype=torch.int32, device=dev)
    if own:  # the handle a serving program makes once for its cache
        from paper_2608_18486_gb300 import _lib
        from paper_2608_18486_gb300.session import DecodeSession
        cfg = _lib.make_config(k, k, 64, Hq, Hkv, d, 1, P, case["dtype"], list(range(k)))
        s["session"] = DecodeSession(cfg, B, pages, maxp, dev, cache_buf=buf)
    return s


def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


# ------------------------------------------------------------------ the framework's calls
def _own_window(s):
    c = s["case"]
    s["session"].window_attn(c["k"] - 1, s["q"], s["page_table"], s["seq_lens"], s["out"], sinks=c["sinks"],
                             window=c["window"])
    return s["out"]


def _own_window_prefill(s):
    c = s["case"]
    s["session"].window_prefill_attn(c["k"] - 1, s["q"], s["pos"], s["page_table"], s["out"], sinks=c["sinks"],
                                     window=c["window"])
    return s["out"]


def _own_prefix(s):
    c = s["case"]
    s["session"].prefix_attn(c["k"] - 1, s["q"], s["page_table"], s["seq_lens"], s["out"], shared_pages=c["shared"])
    return s["out"]


def _own_mass(s):
    c = s["case"]
    s["session"].decode_attn_mass(c["k"] - 1, s["q"], s["page_table"], s["seq_lens"], s["mass"], s["out"])
    return s["out"], s["mass"]


def _own_evict(s):
    c = s["case"]
    s["session"].evict(s["mass"], s["page_table"], s["seq_lens"], s["mass_out"], s["kept"], s["new_lens"],
                       budget=c["budget"], sinks=c["sinks"], recent=c["recent"])
    return s["k_pool"], s["v_pool"], s["mass_out"], s["kept"], s["new_lens"]


_own = {"window": _own_window, "window_prefill": _own_window_prefill, "prefix": _own_prefix, "mass": _own_mass,
        "evict": _own_evict}


# ------------------------------------------------------------------ plain forms
def _weights(scores, seen):
    """Softmax over the last axis where ``seen``; rows that see nothing get zeros."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    e = torch.exp(scores - top)
    return e / e.sum(-1, keepdim=True).clamp(min=1e-30)


def _slots(pool, table, slot):
    """Rows [B][Hkv][n][d] of the slots ``slot`` [B][n] in 32 bits, through the page table."""
    P = pool.shape[2]
    page = table.long().gather(1, slot // P).clamp(min=0)
    return pool[page, :, slot % P].transpose(1, 2).float()


def _cached(pool, table):
    """Every row of the batch's cache, [B][Hkv][T][d] in 32 bits."""
    x = pool[table.long().clamp(min=0)].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1]).float()


def _grouped(s):
    c = s["case"]
    return s["q"].float().view(c["B"], c["Hkv"], -1, c["d"]) / math.sqrt(c["d"])


def _plain_window(s):
    c, n = s["case"], s["seq_lens"].long()[:, None]
    near = n - c["window"] + torch.arange(c["window"], device=n.device)
    first = torch.arange(c["sinks"], device=n.device).expand(c["B"], -1)
    slot = torch.cat([first, near], 1)
    seen = torch.cat([first < n, near >= c["sinks"]], 1)
    slot = slot.clamp(min=0).minimum(n - 1)
    K, V = (_slots(s[x][c["k"] - 1], s["page_table"], slot) for x in ("k_pool", "v_pool"))
    p = _weights(_grouped(s) @ K.transpose(-1, -2), seen[:, None, None])
    return (p @ V).reshape(s["q"].shape).to(s["q"].dtype)


def _plain_window_prefill(s):
    c = s["case"]
    K, V = (_cached(s[x][c["k"] - 1], s["page_table"]) for x in ("k_pool", "v_pool"))
    t, pos = torch.arange(K.shape[2], device=K.device), s["pos"].long()[..., None]
    seen = (t <= pos) & ((t < c["sinks"]) | (t > pos - c["window"]))
    q = s["q"].float().view(c["B"], c["rows"], c["Hkv"], -1, c["d"]).permute(0, 2, 3, 1, 4) / math.sqrt(c["d"])
    V = V * seen.any(1)[:, None, :, None]
    p = _weights(q @ K.transpose(-1, -2)[:, :, None], seen[:, None, None])
    return (p @ V[:, :, None]).permute(0, 3, 1, 2, 4).reshape(s["q"].shape).to(s["q"].dtype)


def _plain_prefix(s):
    c, n = s["case"], s["seq_lens"].long()[:, None]
    start, table = c["shared"] * c["page"], s["page_table"]
    slot = start + torch.arange(int(c["ctx"]) - start, device=n.device).expand(c["B"], -1)
    seen, slot = slot < n, slot.minimum(n - 1)
    q, kp, vp = _grouped(s), s["k_pool"][c["k"] - 1], s["v_pool"][c["k"] - 1]
    K0, V0 = (_cached(x, table[:1, :c["shared"]])[0] for x in (kp, vp))
    K1, V1 = (_slots(x, table, slot) for x in (kp, vp))
    scores = torch.cat([torch.einsum("bhgd,htd->bhgt", q, K0), q @ K1.transpose(-1, -2)], -1)
    p = _weights(scores, torch.cat([torch.ones_like(seen[:, :1]).expand(-1, start), seen], 1)[:, None, None])
    o = torch.einsum("bhgt,htd->bhgd", p[..., :start], V0) + p[..., start:] @ V1
    return o.reshape(s["q"].shape).to(s["q"].dtype)


def _plain_mass(s):
    c = s["case"]
    K, V = (_cached(s[x][c["k"] - 1], s["page_table"]) for x in ("k_pool", "v_pool"))
    seen = torch.arange(K.shape[2], device=K.device) < s["seq_lens"][:, None]
    p = _weights(_grouped(s) @ K.transpose(-1, -2), seen[:, None, None])
    s["mass"][c["k"] - 1] += p.sum(2)
    return (p @ V).reshape(s["q"].shape).to(s["q"].dtype), s["mass"]


def _plain_evict(s):
    c, n = s["case"], s["seq_lens"].long()[:, None, None]
    mass, budget = s["mass"], c["budget"]
    t = torch.arange(mass.shape[-1], device=mass.device)
    cut = n > budget
    value = torch.where((t < c["sinks"]) | (t >= n - c["recent"]) | ~cut, math.inf, mass)
    value = torch.where(t < n, value, -math.inf)
    kept = torch.sort(value, dim=-1, descending=True, stable=True).indices[..., :budget].sort(-1).values
    live = torch.arange(budget, device=mass.device) < n
    page = s["page_table"].long()[None, :, None].expand(*kept.shape[:3], -1)
    P = c["page"]
    channel = torch.arange(c["k"], device=mass.device)[:, None, None, None]
    head = torch.arange(c["Hkv"], device=mass.device)[None, None, :, None]
    new = torch.arange(budget, device=mass.device).expand(kept.shape)
    moves = (cut & live).expand(kept.shape)
    source = tuple(x.expand(kept.shape)[moves] for x in (channel, page.gather(-1, kept // P), head, kept % P))
    target = tuple(x.expand(kept.shape)[moves] for x in (channel, page.gather(-1, new // P), head, new % P))
    s["k_pool"][target] = s["k_pool"][source]
    s["v_pool"][target] = s["v_pool"][source]
    s["mass_out"].zero_()
    s["mass_out"][..., :budget] = torch.where(live, mass.gather(-1, kept), 0.0)
    s["kept"].copy_(torch.where(live, kept, -1))
    s["new_lens"].copy_(s["seq_lens"].clamp(max=budget))
    return s["k_pool"], s["v_pool"], s["mass_out"], s["kept"], s["new_lens"]


_plain = {"window": _plain_window, "window_prefill": _plain_window_prefill, "prefix": _plain_prefix,
          "mass": _plain_mass, "evict": _plain_evict}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    """One (sequence, kv head) at a time, in 64 bits; None where that are too many."""
    if case["k"] * case["B"] * case["Hq"] > 8192:
        return None
    s = prepare(case, seed)
    B, Hq, Hkv, d, P = (case[x] for x in ("B", "Hq", "Hkv", "d", "page"))
    G, table, lens = Hq // Hkv, s["page_table"].long(), s["seq_lens"].tolist()
    if case["op"] == "evict":
        return _exact_evict(s, case, lens)
    K, V = s["k_pool"][case["k"] - 1], s["v_pool"][case["k"] - 1]
    q, out = s["q"].double(), torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if case["op"] == "mass" else None
    for b in range(B):
        n = lens[b]
        t = torch.arange(n, device="cuda")
        if case["op"] == "window":
            t = t[(t < case["sinks"]) | (t >= n - case["window"])]
        page, off = table[b, t // P], t % P
        for h in range(Hkv):
            Kh, Vh = K[page, h, off].double(), V[page, h, off].double()
            for g in range(h * G, h * G + G):
                if case["op"] == "window_prefill":
                    z = q[b, :, g] @ Kh.T / d ** 0.5
                    i = s["pos"][b].long()[:, None]
                    z = torch.where((t > i) | ((t >= case["sinks"]) & (t + case["window"] <= i)), -math.inf, z)
                    out[b, :, g] = torch.softmax(z, 1) @ Vh
                else:
                    w = torch.softmax(Kh @ q[b, g] / d ** 0.5, 0)
                    out[b, g] = w @ Vh
                    if mass is not None:
                        mass[case["k"] - 1, b, h, :n] += w
    return out if mass is None else (out, mass)


def _exact_evict(s, case, lens):
    K, V, P, budget = s["k_pool"].clone(), s["v_pool"].clone(), case["page"], case["budget"]
    mass, out, table = s["mass"].cpu().numpy(), np.zeros(s["mass"].shape), s["page_table"].long()
    kept = np.full(s["kept"].shape, -1, dtype=np.int32)
    for c in range(case["k"]):
        for b, n in enumerate(lens):
            for h in range(case["Hkv"]):
                keep = list(range(n))
                if n > budget:
                    lo, hi = case["sinks"], n - case["recent"]
                    best = np.lexsort((np.arange(lo, hi), -mass[c, b, h, lo:hi]))[:budget - lo - case["recent"]] + lo
                    keep = sorted(list(range(lo)) + best.tolist() + list(range(hi, n)))
                    a, z = torch.tensor(keep, device="cuda"), torch.arange(budget, device="cuda")
                    K[c, table[b, z // P], h, z % P] = s["k_pool"][c, table[b, a // P], h, a % P]
                    V[c, table[b, z // P], h, z % P] = s["v_pool"][c, table[b, a // P], h, a % P]
                out[c, b, h, :len(keep)] = mass[c, b, h, keep]
                kept[c, b, h, :len(keep)] = keep
    return K.double(), V.double(), out, kept, np.minimum(np.array(lens, dtype=np.int32), budget)
