"""Calls that follow each other on one stream with nothing between them.

Launches are chained so that one may start while the one before it finishes; what a call writes
has to be there for every later one, the second after it included, which with inputs_ready reads
the cache before it waits."""
import numpy as np
import pytest
import torch

from tests._longctx import Cache

pytestmark = pytest.mark.gpu


class Cut:
    """Two channels of one long sequence and the arguments of a cut to half.  The cut's few
    clusters leave most SMs to the calls behind it and keep moving rows meanwhile."""

    def __init__(self, seed):
        self.c = c = Cache([9001], Hkv=2, G=2, d=64, page=16, k=2, seed=seed)
        self.s, (self.table, self.lens) = c.session(), c.dev()
        self.pools = self.s.k_pool.clone(), self.s.v_pool.clone()
        self.mass = torch.from_numpy(np.abs(c.rng.standard_normal((2, 1, 2, c.T))).astype(np.float32)).cuda()
        self.kept = torch.empty((2, 1, 2, 4500), dtype=torch.int32, device="cuda")
        self.new = torch.empty_like(self.lens)
        self.out_mass = torch.empty_like(self.mass)
        self.q = c.queries(2, 1).cuda()
        self.outs = torch.empty_like(self.q)

    def reset(self):
        self.s.k_pool.copy_(self.pools[0])
        self.s.v_pool.copy_(self.pools[1])
        self.new.copy_(self.lens)
        self.outs.fill_(7.0)
        torch.cuda.synchronize()

    def cut(self):
        self.s.evict(self.mass, self.table, self.lens, self.out_mass, self.kept, self.new, budget=4500, sinks=4,
                     recent=256)

    def attend(self, layer, ready, **flags):
        self.s.decode_attn(layer, self.q[layer], self.table, self.new, self.outs[layer], inputs_ready=ready, **flags)


SPLITS = [dict(unit_split=True), dict(dynamic_split=True), dict()]


@pytest.mark.parametrize("flags", SPLITS)
def test_the_second_attention_after_an_eviction_sees_all_of_it(flags):
    x = Cut(1)
    x.reset()
    x.cut()
    torch.cuda.synchronize()
    for layer in (0, 1):
        x.attend(layer, False, **flags)
        torch.cuda.synchronize()
    want = x.outs.clone()
    for _ in range(20):
        x.reset()
        x.cut()
        x.attend(0, False, **flags)  # (it wrote no cache, table or length: what follows may say so)
        x.attend(1, True, **flags)
        torch.cuda.synchronize()
        assert torch.equal(x.outs, want)
    assert x.s.read_status() == 0


def test_attention_after_an_eviction_and_a_prefill_pass_sees_all_of_it():
    x = Cut(2)
    rows, pos = x.c.queries(1, 3).cuda(), torch.tensor([[5, 900, 4000]], dtype=torch.int32, device="cuda")
    out = torch.empty_like(rows)

    def calls(wait):
        x.cut()
        wait()
        x.s.prefill_attn(0, rows, pos, x.table, out)
        wait()
        x.attend(1, True, unit_split=True)
        torch.cuda.synchronize()

    x.reset()
    calls(torch.cuda.synchronize)
    want, want_rows = x.outs.clone(), out.clone()
    for _ in range(20):
        x.reset()
        calls(lambda: None)
        assert torch.equal(x.outs[1], want[1]) and torch.equal(out, want_rows)
    assert x.s.read_status() == 0


def test_attention_after_an_eviction_and_each_long_context_call():
    x = Cut(3)
    c, s = x.c, x.s
    out = torch.empty_like(x.q[0])
    sums = torch.zeros_like(x.mass)
    rows, pos = c.queries(1, 130).cuda(), torch.arange(4200, 4330, dtype=torch.int32, device="cuda")[None].contiguous()
    rows_out = torch.empty_like(rows)
    between = {
        "window": lambda: s.window_attn(0, x.q[0], x.table, x.new, out, sinks=4, window=700),
        "rows": lambda: s.window_prefill_attn(0, rows, pos, x.table, rows_out, sinks=4, window=300),
        "prefix": lambda: s.prefix_attn(0, x.q[0], x.table, x.new, out, shared_pages=40),
        "mass": lambda: s.decode_attn_mass(0, x.q[0], x.table, x.new, sums, out)}
    for name, call in between.items():
        def calls(wait):
            x.cut()
            wait()
            call()
            wait()
            x.attend(1, True, unit_split=True)
            torch.cuda.synchronize()
        x.reset()
        calls(torch.cuda.synchronize)
        want, want_out, want_rows = x.outs.clone(), out.clone(), rows_out.clone()
        for _ in range(10):
            x.reset()
            calls(lambda: None)
            assert torch.equal(x.outs[1], want[1]) and torch.equal(out, want_out), name
            assert torch.equal(rows_out, want_rows), name
    assert s.read_status() == 0


def test_the_second_attention_after_a_pool_update_sees_all_of_it():
    from tests import _harness as H
    from wm_synth import configs
    w = configs.get("paper_k16").with_(B=2, ctx=300)
    prob, s, dp = H.setup(w)
    pools = s.k_pool.clone(), s.v_pool.clone()
    outs = torch.empty((2, w.B, w.Hq, w.d), dtype=s.dtype, device="cuda")
    lens = dp.slot + 1  # the new token's slot included

    def calls(wait):
        s.k_pool.copy_(pools[0])
        s.v_pool.copy_(pools[1])
        outs.fill_(7.0)
        torch.cuda.synchronize()
        s.kv_mix(dp.h, dp.page_table, dp.slot)
        wait()
        s.decode_attn(0, dp.q[0], dp.page_table, lens, outs[0])
        wait()
        s.decode_attn(1, dp.q[1], dp.page_table, lens, outs[1], inputs_ready=True)
        torch.cuda.synchronize()

    calls(torch.cuda.synchronize)
    want = outs.clone()
    for _ in range(20):
        calls(lambda: None)
        assert torch.equal(outs, want)
    assert s.read_status() == 0
