"""The 4-bit cache's calls together, as a server uses them: the pool appended to it, contexts moved
to it behind a prefill, decode steps over it (eager and replayed), rows read back for the calls over
other caches; streams, graphs, workspaces and places past 32 bits."""
import numpy as np
import pytest
import torch

from paper_2608_18486_gb300 import _lib as W
from paper_2608_18486_gb300.session import DecodeSession, Q4Cache
from tests import _harness as H
from tests import _q4 as Q
from tests._longctx import to_f64
from wm_synth import configs

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).cuda()


@pytest.mark.parametrize("name,B,page", [("tiny_f32", 2, 16), ("paper_k16", 3, 16), ("paper_k16", 70, 4),
                                         ("no_compression", 5, 64)])
@pytest.mark.parametrize("given", [False, True])
def test_pool_in_4_bits_is_the_pool_written_in_4_bits(name, B, page, given):
    w = configs.get(name).with_(B=B, ctx=100, page=page)
    prob, s, dp = H.setup(w)
    one, two = Q4Cache(s.cfg, s.num_pages), Q4Cache(s.cfg, s.num_pages)
    for q4 in (one, two):
        q4.cache_buf.fill_(0x5A)
    pos = i32(7 + 3 * np.arange(B)) if given else None
    s.q4_kv_mix(dp.h, one, dp.page_table, dp.slot, pos=pos)
    s.kv_mix(dp.h, dp.page_table, dp.slot, pos=pos)
    s.q4_write(two, dp.page_table, dp.page_table, dp.slot, dp.slot + 1, span=1)
    assert s.read_status() == 0
    assert torch.equal(one.cache_buf, two.cache_buf) and not bool((one.cache_buf == 0x5A).all())
    # tokens without a place are left out and reported
    slot = dp.slot.clone()
    slot[0] = 0
    slot[-1] = s.max_pages * page
    three = Q4Cache(s.cfg, s.num_pages)
    three.cache_buf.copy_(one.cache_buf)
    s.q4_kv_mix(dp.h, three, dp.page_table, slot, pos=pos)
    assert s.read_status() == W.WM_ERR_BOUNDS and torch.equal(one.cache_buf, three.cache_buf)


def decode_close(got, want, rel):
    assert np.abs(got - want).max() <= rel * np.abs(want).max()


@pytest.mark.parametrize("name", ["paper_k8", "tiny_f32", "no_compression"])
def test_decode_steps_over_a_prompt_moved_to_4_bits(name):
    """A prompt behind its prefill is moved; three steps of all layers and the pool, eager and
    from a graph; the same steps over what is read back."""
    w = configs.get(name).with_(B=3, ctx=90, ctx_lo=41)
    prob, s, dp = H.setup(w)
    table, n0 = dp.page_table, dp.seq_lens.clone()
    q4 = Q4Cache(s.cfg, s.num_pages)
    q4.cache_buf.fill_(0xFF)
    zero = torch.zeros_like(n0)
    s.q4_write(q4, table, table, zero, n0, span=int(n0.max()))
    start = q4.cache_buf.clone()
    outs = torch.zeros((3, w.L, w.B, w.Hq, w.d), dtype=s.dtype, device="cuda")
    lens, slot = n0.clone(), n0.clone()

    def steps():
        lens.copy_(n0)
        for i in range(3):
            for layer in range(w.L):
                s.q4_decode_attn(layer, dp.q[layer], q4, table, lens, outs[i, layer])
            slot.copy_(lens)
            s.q4_kv_mix(dp.h, q4, table, slot)
            lens.add_(1)

    steps()
    assert s.read_status() == 0
    eager, held = outs.clone(), q4.cache_buf.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        steps()  # (its scratch is there before the capture)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            steps()
        for _ in range(3):
            q4.cache_buf.copy_(start)
            outs.fill_(float("nan"))
            g.replay()
    torch.cuda.synchronize()
    assert s.read_status() == 0
    assert torch.equal(outs, eager) and torch.equal(q4.cache_buf, held)

    # the calls over other caches, on the rows read back
    s.k_pool.fill_(float("nan"))
    s.v_pool.fill_(float("nan"))
    s.q4_read(q4, table, table, zero, lens, span=int(lens.max()))
    rel = 2e-5 if w.dtype == "f32" else 2.0 ** -6  # (each call's own rounding of weights and results)
    for layer in (0, w.L - 1):
        out = torch.empty_like(outs[0, 0])
        s.q4_decode_attn(layer, dp.q[layer], q4, table, lens, out)
        want = torch.empty_like(out)
        s.decode_attn(layer, dp.q[layer], table, lens, want)
        decode_close(to_f64(out), to_f64(want), rel)
        # one row at the last position, and several
        pos = (lens[:, None] - 1 - torch.arange(3, device="cuda")).int().contiguous()
        q = dp.q[layer][:, None].expand(-1, 3, -1, -1).contiguous()
        rows = torch.empty_like(q)
        s.q4_rows_attn(layer, q, pos, q4, table, rows)
        decode_close(to_f64(rows[:, 0]), to_f64(out), rel)
        if w.dtype == "bf16":
            ref = torch.empty_like(q)
            s.prefill_attn(layer, q, pos, table, ref)
            decode_close(to_f64(rows), to_f64(ref), rel)
    assert s.read_status() == 0


def many_rows_case():
    x = Q.Q4([600, 520], Hkv=2, G=4, d=64, page=16, k=1, max_pages=4096)
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    pos = i32(np.stack([np.arange(n - 300, n) for n in x.lens]))
    return x, s, q4, table, pos, x.queries(2, 300).cuda()


def test_graphs_of_every_call_and_their_scratch():
    """Graphs captured on one stream share its scratch; larger calls afterwards leave it to them."""
    x, s, q4, table, pos, q = many_rows_case()
    lens = i32(x.lens)
    qd = x.queries(2).cuda()
    want, wantd = torch.empty_like(q), torch.empty_like(qd)
    s.q4_rows_attn(0, q, pos, q4, table, want)
    s.q4_decode_attn(0, qd, q4, table, lens, wantd)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    out, outd = torch.zeros_like(q), torch.zeros_like(qd)
    graphs = []
    with torch.cuda.stream(stream):
        s.q4_decode_attn(0, qd, q4, table, lens, outd)
        for call in (lambda: s.q4_decode_attn(0, qd, q4, table, lens, outd),
                     lambda: s.q4_rows_attn(0, q, pos, q4, table, out)):
            call()  # (the scratch of this size, before the capture)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                call()
            graphs.append(g)
        for _ in range(2):
            out.zero_()
            outd.zero_()
            for g in graphs:
                g.replay()
    torch.cuda.synchronize()
    assert s.read_status() == 0 and torch.equal(out, want) and torch.equal(outd, wantd)


def test_two_streams_at_once():
    x, s, q4, table, pos, q = many_rows_case()
    lens = i32(x.lens)
    qd = x.queries(2).cuda()
    want, wantd = torch.empty_like(q), torch.empty_like(qd)
    s.q4_rows_attn(0, q, pos, q4, table, want)
    s.q4_decode_attn(0, qd, q4, table, lens, wantd)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(t) for _ in range(6)] for t in (q, qd)]
    for i in range(6):
        s.q4_rows_attn(0, q, pos, q4, table, outs[0][i], stream=streams[0])
        s.q4_decode_attn(0, qd, q4, table, lens, outs[1][i], stream=streams[1])
    torch.cuda.synchronize()
    assert s.read_status() == 0
    assert all(torch.equal(o, want) for o in outs[0]) and all(torch.equal(o, wantd) for o in outs[1])


def test_what_a_write_leaves_is_there_for_the_next_call():
    """A long write, then attention over what it wrote, launch behind launch."""
    x = Q.Q4([3000] * 8, Hkv=4, G=2, d=128, page=16, k=1)
    s, q4 = x.session(), Q4Cache(x.session_cfg(), x.q4_pages)
    table, lens = x.q4_dev()
    src = torch.from_numpy(x.table).cuda()
    q = x.queries(8).cuda()
    zero = torch.zeros_like(lens)
    want = torch.empty_like(q)
    s.q4_decode_attn(0, q, x.q4(), table, lens, want)
    for _ in range(5):
        q4.cache_buf.fill_(0xFF)
        out = torch.empty_like(q)
        s.q4_write(q4, src, table, zero, lens, span=3000)
        s.q4_decode_attn(0, q, q4, table, lens, out)
        assert torch.equal(out, want)
    assert s.read_status() == 0


def test_places_past_32_bits():
    """Pages behind 2^32 bytes of codes and 2^32 elements of rows."""
    d, page, Hkv, pages = 64, 4096, 1, 17000
    cfg = W.make_config(1, 1, 64, 2, Hkv, d, 1, page, "bf16", [0])
    s, q4 = DecodeSession(cfg, 1, pages, 3), Q4Cache(cfg, pages)
    assert s.k_pool.numel() > 2 ** 32 and q4.cache_buf.numel() > 2 ** 32
    far, near = i32([[pages - 1, 3, pages - 2]]), i32([[pages - 3, pages - 1, 0]])
    n = 2 * page + 700
    g = torch.Generator(device="cuda").manual_seed(0)
    for pool in (s.k_pool, s.v_pool):
        for pg in far[0].tolist():
            pool[0, pg] = torch.randn((Hkv, page, d), generator=g, device="cuda")
    rows = [torch.cat([p[0, pg, 0] for pg in far[0].tolist()])[:n].double().cpu().numpy() for p in (s.k_pool, s.v_pool)]
    lens, zero = i32([n]), i32([0])
    s.q4_write(q4, far, near, zero, lens, span=n)
    q = torch.randn((1, 2, d), generator=g, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    s.q4_decode_attn(0, q, q4, near, lens, out)
    back = i32([[0, pages - 4, 5]])
    s.q4_read(q4, near, back, zero, lens, span=n)
    assert s.read_status() == 0
    held = [Q.values(*Q.quantise(x)) for x in rows]
    for pool, want in zip((s.k_pool, s.v_pool), held):
        got = torch.cat([pool[0, pg, 0] for pg in back[0].tolist()])[:n]
        assert np.array_equal(to_f64(got), want)
    for h in range(2):
        z = held[0] @ to_f64(q[0, h]) / np.sqrt(d)
        p = np.exp(z - z.max())
        want = p / p.sum() @ held[1]
        assert np.abs(to_f64(out[0, h]) - want).max() <= 2.0 ** -8 * np.abs(want).max() + 2.0 ** -10 * np.abs(held[1]).max()
    del s, q4
    torch.cuda.empty_cache()
