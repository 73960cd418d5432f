"""Long-context decoding on one paged cache: window layers, a shared prompt, eviction.

A small random decoder (Sec. 4.1-style blocks in plain torch) runs on the library's cache of two
channels.  Even layers read channel 0 through a sliding window with sinks, odd layers read all of
channel 1:

  1. one sequence decodes the prompt; its pages are what later sequences share;
  2. the prompt's states are evaluated again for all positions at once (window_prefill_attn and
     prefill_attn), which must give what the single steps gave;
  3. a batch continues from the shared prompt (window_attn, prefix_attn);
  4. each sequence gets pages of its own, sums its slots' attention weights while it decodes
     (decode_attn_mass), and is cut to a budget (evict); decoding goes on at the true positions
     (kv_mix with pos).

Run:  python examples/long_context.py     (needs the GPU and the built library)
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_18486_gb300 import _lib as W  # noqa: E402
from paper_2608_18486_gb300.session import DecodeSession  # noqa: E402

L, K, D, HQ, HKV, HD, PAGE = 4, 2, 256, 8, 4, 64, 16
SINKS, WINDOW, THETA = 4, 24, 1e4
PROMPT, BATCH = 111, 4              # the prompt and the dummy fill 7 pages
SHARED = (PROMPT + 1) // PAGE
MAX_PAGES = 16


class Model:
    def __init__(self, dev, seed=0):
        g = torch.Generator(device=dev).manual_seed(seed)

        def w(*shape):
            return (torch.randn(shape, generator=g, device=dev) * shape[-1] ** -0.5).to(torch.bfloat16)

        ones = torch.ones(D, dtype=torch.bfloat16, device=dev)
        self.Wq, self.Wo = w(L, HQ * HD, D), w(L, D, HQ * HD)
        self.Wu, self.Wd = w(L, 2 * D, D), w(L, D, 2 * D)
        self.tokens = torch.randn((4096, D), generator=g, device=dev).to(torch.bfloat16)
        lp = -(-L // 2)
        bias = torch.zeros((K, L), device=dev)
        bias[torch.arange(L) % K, torch.arange(L)] = 1.0  # layer l feeds channel l mod k
        pair = lambda make: (make(), make())  # noqa: E731  (K branch, V branch)
        self.pool = dict(pre_g=pair(lambda: ones), Wr=pair(lambda: 0.3 * w(K * L, lp * D)),
                         br=pair(lambda: bias.reshape(-1).to(torch.bfloat16)),
                         ch_g=pair(lambda: ones.repeat(K, 1).contiguous()),
                         Wkv=pair(lambda: w(K, HKV * HD, D)),
                         qk_g=torch.ones((K, HD), dtype=torch.bfloat16, device=dev))

    @staticmethod
    def norm(x):
        x = x.float()
        return x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)

    def query(self, l, h, pos):
        """Normed, rotated queries [..., HQ, HD] of states h [..., D] at positions pos [...]."""
        q = self.norm((self.norm(h).to(torch.bfloat16) @ self.Wq[l].T).unflatten(-1, (HQ, HD)))
        inv = THETA ** (-torch.arange(0, HD // 2, device=h.device, dtype=torch.float64) * 2 / HD)
        a = (pos.double()[..., None] * inv)[..., None, :].float()
        x, y = q[..., :HD // 2], q[..., HD // 2:]
        return torch.cat([x * a.cos() - y * a.sin(), y * a.cos() + x * a.sin()], -1).to(torch.bfloat16).contiguous()

    def stack(self, h, pos, attend):
        """One pass through the layers; attend(l, q, out) fills out.  States entering the layers
        [..., L, D] and the last state."""
        states = []
        for l in range(L):
            states.append(h)
            q = self.query(l, h, pos)
            out = torch.empty_like(q)
            attend(l, q, out)
            h = h + out.flatten(-2) @ self.Wo[l].T
            u = self.norm(h).to(torch.bfloat16) @ self.Wu[l].T
            h = h + torch.nn.functional.silu(u) @ self.Wd[l].T
        return torch.stack(states, -2).contiguous(), h


def main():
    dev = torch.device("cuda:0")
    model = Model(dev)
    cfg = W.make_config(L, K, D, HQ, HKV, HD, 2, PAGE, "bf16", [l % K for l in range(L)], rope_theta=THETA)
    pages = SHARED + BATCH * MAX_PAGES
    sess = DecodeSession(cfg, BATCH, pages, MAX_PAGES, dev)
    sess.set_weights(**model.pool)
    sess.k_pool.normal_()  # (slot 0 holds the dummy; everything else is written before it is read)
    sess.v_pool.normal_()
    ids = torch.randint(4096, (BATCH, 512), generator=torch.Generator().manual_seed(1)).to(dev)
    table = torch.full((BATCH, MAX_PAGES), -1, dtype=torch.int32)
    table[:, :SHARED] = torch.arange(SHARED)
    for b in range(BATCH):
        table[b, SHARED:] = SHARED + b * MAX_PAGES + torch.arange(MAX_PAGES - SHARED)
    table = table.to(dev)
    lens = torch.ones(BATCH, dtype=torch.int32, device=dev)  # the dummy

    def window(l, q, out, B=BATCH):
        sess.window_attn(l, q, table, lens, out, sinks=SINKS, window=WINDOW, B=B)

    # 1. the prompt, one token at a time, in the pages that will be shared
    prompt_states = []
    for i in range(PROMPT):
        def attend(l, q, out):
            if l % 2 == 0:
                window(l, q, out, B=1)
            else:
                sess.decode_attn(l, q, table, lens, out, B=1)
        pos = lens[:1] - 1
        H, _ = model.stack(model.tokens[ids[0, i]][None], pos, attend)
        sess.kv_mix(H, table, lens, B=1)
        prompt_states.append(H[0])
        lens[0] += 1

    # 2. every position of the prompt at once
    pos = torch.arange(PROMPT, dtype=torch.int32, device=dev)[None].contiguous()

    def attend(l, q, out):
        if l % 2 == 0:
            sess.window_prefill_attn(l, q, pos, table, out, sinks=SINKS, window=WINDOW)
        else:
            sess.prefill_attn(l, q, pos, table, out)
    H, _ = model.stack(model.tokens[ids[0, :PROMPT]][None], pos, attend)
    one = torch.stack(prompt_states).float()
    parallel = float((H[0].float() - one).norm() / one.norm())

    # 3. a batch continues from the shared prompt
    lens.fill_(PROMPT + 1)
    for i in range(40):
        def attend(l, q, out):
            if l % 2 == 0:
                window(l, q, out)
            else:
                sess.prefix_attn(l, q, table, lens, out, shared_pages=SHARED)
        H, _ = model.stack(model.tokens[ids[:, PROMPT + i]], lens - 1, attend)
        sess.kv_mix(H, table, lens)
        lens += 1
    q = model.query(1, model.tokens[ids[:, 0]], lens)
    a, z = torch.empty_like(q), torch.empty_like(q)
    sess.prefix_attn(1, q, table, lens, a, shared_pages=SHARED)
    sess.decode_attn(1, q, table, lens, z)
    shared = float((a.float() - z.float()).norm() / z.float().norm())

    # 4. pages of its own for each sequence, weights summed, then the cut
    own = SHARED + torch.arange(BATCH)[:, None] * MAX_PAGES + MAX_PAGES - SHARED + torch.arange(SHARED)
    for pool in (sess.k_pool, sess.v_pool):
        pool[:, own.to(dev)] = pool[:, :SHARED][:, None]
    table[:, :SHARED] = own.to(dev).int()
    mass = torch.zeros((K, BATCH, HKV, MAX_PAGES * PAGE), device=dev)
    position = lens - 1
    kept = torch.empty((K, BATCH, HKV, 96), dtype=torch.int32, device=dev)
    for i in range(48):
        def attend(l, q, out):
            if l % 2 == 0:
                window(l, q, out)
            else:
                sess.decode_attn_mass(l, q, table, lens, mass, out)
        H, h = model.stack(model.tokens[ids[:, PROMPT + 40 + i]], position, attend)
        sess.kv_mix(H, table, lens, pos=position)
        lens, position = lens + 1, position + 1
        if i == 31:
            total = mass[1].sum(-1)  # 32 steps, two layers, two query heads per kv head
            new = torch.empty_like(lens)
            sess.evict(mass, table, lens, mass, kept, new, budget=96, sinks=SINKS, recent=WINDOW + 8)
            before, lens = lens, new
    torch.cuda.synchronize()
    assert sess.read_status() == 0
    report = {"parallel_vs_steps": parallel, "prefix_vs_decode": shared,
              "weight_per_head": float((total / (32 * 2 * 2) - 1).abs().max()),
              "cut": (int(before[0]), 96), "slots_now": int(lens[0]), "position": int(position[0]),
              "finite": bool(torch.isfinite(h.float()).all())}
    print("the prompt's states, all positions at once against single steps: %.2g" % parallel)
    print("attention over the shared prompt against per-sequence attention: %.2g" % shared)
    print("weights summed over 32 steps, off 1 per query head by at most %.2g" % report["weight_per_head"])
    print("cut from %d to %d slots; now %d slots at position %d" % (*report["cut"], report["slots_now"],
                                                                   report["position"]))
    assert math.isfinite(parallel) and report["finite"]
    return report


if __name__ == "__main__":
    main()
