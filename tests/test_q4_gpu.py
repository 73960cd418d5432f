"""The cache held in 4 bits: rows to it and back, and attention over it, against numpy in
64 bits.  Rows are compared bit for bit; attention within bounds derived in tests/_q4.py."""
import numpy as np
import pytest
import torch

from paper_2608_18486_gb300 import _lib as W
from paper_2608_18486_gb300.session import DecodeSession, Q4Cache
from tests import _q4 as Q
from tests._longctx import to_f64

pytestmark = pytest.mark.gpu

KINDS = [("bf16", 64), ("bf16", 96), ("bf16", 128), ("f32", 64), ("f32", 96), ("f32", 128)]


def special_rows(rng, n, d, dtype):
    """Rows of many sizes, with ties, zeros of both signs, tiny, huge and missing values."""
    x = rng.standard_normal((n, d)) * np.exp(4 * rng.standard_normal((n, d // 16)).repeat(16, 1))
    g = x.reshape(n, d // 16, 16)
    for i in range(n):
        y = g[i, i % (d // 16)]
        kind = i % 12
        if kind == 0:    # every border of a code, scale 1
            y[:] = [6, .25, -.25, .75, -.75, 1.25, -1.25, 1.75, 2.5, -2.5, 3.5, -3.5, 5, -5, 0, -0.0]
        elif kind == 1:  # the same times another scale
            y[:] = 1.375 * 2.0 ** rng.integers(-12, 12) * np.array([6, .25, -.25, .75, -.75, 1.25, -1.25, 1.75, 2.5, -2.5,
                                                                    3.5, -3.5, 5, -5, 0, -0.0])
        elif kind == 2:  # a tie of the scale
            y *= 6 * (1 + (2 * rng.integers(0, 8) + 1) / 16) / np.abs(y).max()
            y[0] = 6 * (1 + (2 * rng.integers(0, 8) + 1) / 16)
            y[1:] = np.clip(y[1:], -6, 6)
        elif kind == 3:
            y[:] = 0
        elif kind == 4:  # around the smallest scales
            y *= 2.0 ** rng.integers(-22, -12)
        elif kind == 5:
            y *= 2.0 ** rng.integers(12, 40)
        elif kind == 6:
            y[rng.integers(16)] = np.nan
        elif kind == 7:
            y[rng.integers(16)] = -np.inf
        elif kind == 8:
            y *= 1e-42 if dtype == "f32" else 1e-39
        elif kind == 9:  # neighbours of the borders
            s = (1 + rng.integers(0, 8) / 8) * 2.0 ** rng.integers(-6, 6)
            y[:] = s * np.array([6, .25, .25, .75, .75, 1.25, 1.25, 1.75, 1.75, 2.5, 2.5, 3.5, 3.5, 5, 5, 6])
            t = torch.from_numpy(y).to(torch.float32 if dtype == "f32" else torch.bfloat16)
            up = torch.from_numpy(rng.integers(-1, 2, 16))
            up[0] = 0
            if dtype == "f32":
                t = (t.view(torch.int32) + up.int()).view(torch.float32)
            else:
                t = (t.view(torch.int16) + up.short()).view(torch.bfloat16)
            y[:] = t.double().numpy()
    return x


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("page", [1, 2, 8, 16, 64])
def test_write_holds_the_nearest_values(dtype, d, page):
    rng = np.random.default_rng(d + page)
    k, Hkv, B = 2, 3, 3
    lens = np.array([37, 1, 90])
    first = np.array([5, 0, 33])
    maxp = 90 // page + 2
    pages = B * maxp
    tdt = torch.float32 if dtype == "f32" else torch.bfloat16
    cfg = W.make_config(k, k, 64, Hkv, Hkv, d, 1, page, dtype, [0, 1])
    s, q4 = DecodeSession(cfg, B, pages, maxp), Q4Cache(cfg, pages + 1)
    table = rng.permutation(pages).reshape(B, maxp).astype(np.int32)
    qtable = rng.permutation(pages).reshape(B, maxp).astype(np.int32) + 1
    rows = special_rows(rng, 2 * k * pages * Hkv * page, d, dtype).reshape(2, k, pages, Hkv, page, d)
    for pool, x in zip((s.k_pool, s.v_pool), rows):
        pool.copy_(torch.from_numpy(x).to(tdt))
    held = [to_f64(s.k_pool), to_f64(s.v_pool)]
    q4.cache_buf.fill_(0xA5)
    want = q4.cache_buf.cpu().numpy().copy()
    view = Q.pool_view(want, k, pages + 1, Hkv, page, d)
    dev = [torch.from_numpy(x.astype(np.int32)).cuda() for x in (table, qtable, first, lens)]
    s.q4_write(q4, *dev, span=57)
    for x in range(2):
        code, byte = Q.quantise(held[x])
        for b in range(B):
            for t in range(first[b], lens[b]):
                at = table[b, t // page], slice(None), t % page
                for c in range(k):
                    for h in range(Hkv):
                        Q.put_row(view, c, qtable[b, t // page], h, t % page, x, code[c][at][h], byte[c][at][h])
    got = q4.cache_buf.cpu().numpy()
    assert s.read_status() == 0
    assert np.array_equal(got, want), int((got != want).sum())

    # and back: into other pages, exactly, nothing else touched
    back = rng.permutation(pages).reshape(B, maxp).astype(np.int32)
    s.k_pool.fill_(-3)
    s.v_pool.fill_(7)
    s.q4_read(q4, dev[1], torch.from_numpy(back).cuda(), dev[2], dev[3], span=90)
    for x, pool in enumerate((s.k_pool, s.v_pool)):
        ref = np.full(held[x].shape, -3.0 if x == 0 else 7.0)
        v = Q.values(*Q.quantise(held[x]))
        for b in range(B):
            for t in range(first[b], lens[b]):
                ref[:, back[b, t // page], :, t % page] = v[:, table[b, t // page], :, t % page]
        assert np.array_equal(to_f64(pool), ref, equal_nan=True)
    assert s.read_status() == 0
    # what is read back is held again as it is, from scales of 2^-15 (byte 4) on
    again = Q4Cache(cfg, pages + 1)
    again.cache_buf.fill_(0xA5)
    s.q4_write(again, torch.from_numpy(back).cuda(), *dev[1:], span=90)
    v1, byte = decode_pool(Q.pool_view(got, k, pages + 1, Hkv, page, d), d)
    v2, _ = decode_pool(Q.pool_view(again.cache_buf.cpu().numpy(), k, pages + 1, Hkv, page, d), d)
    small = ((byte > 0) & (byte < 4)).repeat(16, -1)
    assert np.array_equal(np.where(small, 0, v1), np.where(small, 0, v2), equal_nan=True)


def decode_pool(pool, d):
    n = Q.tile_shape_of(pool, d)
    codes = pool[..., :n * d]
    code = np.stack([codes & 15, codes >> 4], -1).reshape(*pool.shape[:-1], 2 * n, d)
    byte = pool[..., n * d:n * d + 2 * n * (d // 16)].reshape(*pool.shape[:-1], 2 * n, d // 16)
    return Q.values(code, byte), byte


def test_copies_leave_out_what_is_bad():
    cfg = W.make_config(1, 1, 64, 2, 2, 64, 1, 16, "bf16", [0])
    s, q4 = DecodeSession(cfg, 4, 8, 3), Q4Cache(cfg, 8)
    s.k_pool.fill_(1)
    s.v_pool.fill_(2)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = i32([[0, 1, -1], [2, 3, 9], [4, 5, -1], [6, 7, -1]])
    good = (i32([0, 0, 5, 0]), i32([20, 32, 5, 32]))

    def written():
        view = Q.pool_view(q4.cache_buf.cpu().numpy(), 1, 8, 2, 16, 64)
        n = (view[0, :, 0, 0, :16 * 32].reshape(8, 16, 32) != 0).any(-1).sum(-1)
        q4.cache_buf.zero_()
        return n.tolist()

    q4.cache_buf.zero_()
    s.q4_write(q4, table, table, *good, span=32)
    assert s.read_status() == 0 and written() == [16, 4, 16, 16, 0, 0, 16, 16]
    s.q4_write(q4, table, table, *good, span=20)  # longer ones are cut
    assert s.read_status() == W.WM_ERR_BOUNDS and written() == [16, 4, 16, 4, 0, 0, 16, 4]
    s.q4_write(q4, table, table, i32([-1, 3, 9, 0]), i32([20, 2, 49, 16]), span=48)  # bad ranges
    assert s.read_status() == W.WM_ERR_BOUNDS and written() == [0, 0, 0, 0, 0, 0, 16, 0]
    s.q4_write(q4, table, table, i32([30, 30, 0, 0]), i32([34, 34, 0, 0]), span=48)  # bad pages of either sign
    assert s.read_status() == W.WM_ERR_BOUNDS and written() == [0, 2, 0, 2, 0, 0, 0, 0]
    bad = table.clone()
    bad[3, 0] = -1
    s.q4_write(q4, table, bad, *good, span=32)
    assert s.read_status() == W.WM_ERR_BOUNDS and written() == [16, 4, 16, 16, 0, 0, 0, 16]
    s.q4_write(q4, table, table, *good, span=0)
    assert s.read_status() == 0 and written() == [0] * 8


def attend_all(x, s, q4, q, lens, got, layer, steps):
    worst = 0.0
    for b in range(x.B):
        for hq in range(x.Hq):
            want, tol = x.bound(layer, b, hq, to_f64(q[b, hq]), list(range(int(lens[b]))), steps)
            err = np.abs(got[b, hq] - want).max()
            assert np.isfinite(got[b, hq]).all() and err <= tol, (b, hq, err, tol)
            worst = max(worst, err / max(tol, 1e-30))
    return worst


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("page", [1, 4, 16, 64])
def test_decode_attention(dtype, d, G, page):
    lens = [0, 1, 15, 16, 17, 97, 200]
    x = Q.Q4(lens, Hkv=2, G=G, d=d, page=page, dtype=dtype, seed=d + G + page)
    s, q4 = x.session(), x.q4()
    table, n = x.q4_dev()
    q = x.queries(x.B)
    out = torch.full((x.B, x.Hq, d), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_decode_attn(1, q.cuda(), q4, table, n, out)
    got = to_f64(out)
    assert s.read_status() == 0
    assert (got[0] == 0).all()
    attend_all(x, s, q4, q, lens, got, 1, 4)


@pytest.mark.parametrize("dtype,G,lens,page", [("bf16", 4, [5003, 3000, 1], 16), ("bf16", 1, [9001], 8),
                                               ("f32", 2, [5003, 17], 64), ("f32", 1, [4100], 4),
                                               ("bf16", 8, [1600] * 12 + [3, 0], 32)])
def test_decode_attention_of_long_contexts(dtype, G, lens, page):
    x = Q.Q4(lens, Hkv=1, G=G, d=64, page=page, dtype=dtype, k=1, seed=G)
    s, q4 = x.session(), x.q4()
    table, n = x.q4_dev()
    q = x.queries(x.B, scale=3.0)
    out = torch.full((x.B, x.Hq, 64), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_decode_attn(0, q.cuda(), q4, table, n, out)
    assert s.read_status() == 0
    attend_all(x, s, q4, q, lens, to_f64(out), 0, max(lens) / 16)
    again = torch.empty_like(out)
    s.q4_decode_attn(0, q.cuda(), q4, table, n, again)
    assert torch.equal(out, again)


def spread(x, Tq=1):
    """Whether the steps of this call are spread over the CTAs: it needs records then."""
    ws = W.wm_q4_rows_attn_workspace(x.session_cfg(), x.B, Tq, x.max_pages)
    return 256 < ws < 1 << 24


@pytest.mark.parametrize("dtype,Hkv,G,d,page,lens", [
    ("bf16", 3, 1, 64, 16, [0, 1, 31, 32, 33, 700, 0, 2500]),
    ("bf16", 1, 8, 128, 32, [5003, 0, 17]),
    ("bf16", 2, 4, 96, 4, [999]),
    ("bf16", 1, 2, 64, 16, [(7 * i) % 90 for i in range(300)]),  # more sequences than threads
    ("bf16", 2, 1, 64, 16, [(11 * i) % 200 for i in range(350)]),  # more units than CTAs
    ("bf16", 2, 1, 64, 16, [0] * 5),
    ("bf16", 1, 1, 64, 64, [100001]),                            # one unit, all records its own
    ("f32", 2, 1, 64, 16, [0, 1, 31, 32, 33, 700, 0, 2500]),
    ("f32", 1, 4, 128, 2, [600, 3, 5])])
def test_decode_attention_spread_over_the_ctas(dtype, Hkv, G, d, page, lens):
    x = Q.Q4(lens, Hkv=Hkv, G=G, d=d, page=page, dtype=dtype, k=1, seed=d, max_pages=-(-max(150000, 12 * max(lens)) // page))
    assert spread(x)
    s, q4 = x.session(), x.q4()
    table, n = x.q4_dev()
    q = x.queries(x.B)
    out = torch.full((x.B, x.Hq, d), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_decode_attn(0, q.cuda(), q4, table, n, out)
    assert s.read_status() == 0
    attend_all(x, s, q4, q, lens, to_f64(out), 0, max(lens) / 16)
    again = torch.empty_like(out)
    s.q4_decode_attn(0, q.cuda(), q4, table, n, again)
    assert torch.equal(out, again)
    # bad lengths beside good ones
    n[0], n[-1] = -3, x.T + 1
    s.q4_decode_attn(0, q.cuda(), q4, table, n, again)
    assert s.read_status() == W.WM_ERR_BOUNDS
    assert bool((again[0] == 0).all()) and bool((again[-1] == 0).all())
    got = to_f64(again)
    for b in range(1, x.B - 1):
        want, tol = x.bound(0, b, 0, to_f64(q[b, 0]), list(range(lens[b])), max(lens) / 16)
        assert np.abs(got[b, 0] - want).max() <= tol


@pytest.mark.parametrize("dtype,G,B", [("bf16", 4, 76), ("bf16", 1, 100), ("bf16", 2, 200), ("f32", 1, 56), ("f32", 4, 40)])
def test_decode_attention_where_larger_clusters_do_not_all_fit(dtype, G, B):
    lens = [(37 * i) % 300 for i in range(B)]
    x = Q.Q4(lens, Hkv=1, G=G, d=64, page=16, dtype=dtype, k=1, seed=B, max_pages=128)
    assert not spread(x)
    s, q4 = x.session(), x.q4()
    table, n = x.q4_dev()
    q = x.queries(x.B)
    out = torch.full((x.B, x.Hq, 64), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_decode_attn(0, q.cuda(), q4, table, n, out)
    assert s.read_status() == 0
    attend_all(x, s, q4, q, lens, to_f64(out), 0, 8)
    again = torch.empty_like(out)
    s.q4_decode_attn(0, q.cuda(), q4, table, n, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("G,Tq,d,page,lens,slots", [
    (4, 4, 128, 16, [900, 40, 33], 400000), (1, 13, 64, 8, [600, 13], 900000), (8, 2, 96, 64, [70, 2, 500], 400000),
    (1, 40, 64, 16, [300, 41], 120000), (4, 9, 128, 32, [200, 90], 100000), (2, 10, 96, 4, [100, 33], 150000)])
def test_rows_of_16_columns(G, Tq, d, page, lens, slots):
    """Few columns are spread over the CTAs, more make several units per kv head."""
    x = Q.Q4(lens, Hkv=2, G=G, d=d, page=page, k=1, max_pages=slots // page)
    assert spread(x, Tq) == (Tq * G <= 16) and not (on_tiles(x, Tq) and Tq * G > 16)
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    pos = np.stack([np.arange(n - Tq, n)[::-1] for n in lens]).astype(np.int32)
    pos[0, 1] = 0
    q = x.queries(x.B, Tq)
    dev = torch.from_numpy(pos).cuda()
    out = torch.full((x.B, Tq, x.Hq, d), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_rows_attn(0, q.cuda(), dev, q4, table, out)
    assert s.read_status() == 0
    first = to_f64(out)
    dev[-1, 0] = -1  # (the cuts go by the lengths, so the others may change in their last bits)
    s.q4_rows_attn(0, q.cuda(), dev, q4, table, out)
    assert s.read_status() == W.WM_ERR_BOUNDS and bool((out[-1, 0] == 0).all())
    second = to_f64(out)
    for b in range(x.B):
        for r in range(Tq):
            for hq in range(x.Hq):
                want, tol = x.bound(0, b, hq, to_f64(q[b, r, hq]), list(range(int(pos[b, r]) + 1)), max(lens) / 16)
                assert np.abs(first[b, r, hq] - want).max() <= tol, (b, r, hq)
                if b < x.B - 1 or r > 0:
                    assert np.abs(second[b, r, hq] - want).max() <= tol, (b, r, hq)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("G,Tq,page", [(1, 3, 16), (4, 5, 16), (8, 1, 8), (2, 19, 32), (1, 33, 2)])
def test_rows_attention(dtype, d, G, Tq, page):
    lens = [Tq, 41 + Tq, 130 + Tq]
    x = Q.Q4(lens, Hkv=2, G=G, d=d, page=page, dtype=dtype, seed=d + G)
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    rng = np.random.default_rng(Tq)
    pos = np.stack([rng.permutation(n)[:Tq] for n in lens]).astype(np.int32)  # any order
    pos[1, 0] = lens[1] - 1
    q = x.queries(x.B, Tq)
    out = torch.full((x.B, Tq, x.Hq, d), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_rows_attn(0, q.cuda(), torch.from_numpy(pos).cuda(), q4, table, out)
    assert s.read_status() == 0
    got = to_f64(out)
    for b in range(x.B):
        for r in range(Tq):
            for hq in range(x.Hq):
                want, tol = x.bound(0, b, hq, to_f64(q[b, r, hq]), list(range(int(pos[b, r]) + 1)), 12)
                err = np.abs(got[b, r, hq] - want).max()
                assert err <= tol, (b, r, hq, err, tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_leaves_out_what_is_bad(dtype):
    lens = [70, 60, 80, 50]
    x = Q.Q4(lens, Hkv=2, G=2, d=64, page=16, dtype=dtype)
    s, q4 = x.session(), x.q4()
    table, n = x.q4_dev()
    q = x.queries(x.B)
    table[0, 1] = -1
    table[2, 4] = x.q4_pages
    n[1], n[3] = -1, x.T + 1
    out = torch.full((x.B, x.Hq, 64), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_decode_attn(0, q.cuda(), q4, table, n, out)
    assert s.read_status() == W.WM_ERR_BOUNDS
    got = to_f64(out)
    assert (got[1] == 0).all() and (got[3] == 0).all()
    for b, ts in ((0, [t for t in range(70) if t // 16 != 1]), (2, list(range(64)))):
        for hq in range(x.Hq):
            want, tol = x.bound(0, b, hq, to_f64(q[b, hq]), ts, 4)
            assert np.abs(got[b, hq] - want).max() <= tol
    pos = torch.tensor([[69, -1], [59, x.T], [79, 3], [49, 0]], dtype=torch.int32, device="cuda")
    q2 = x.queries(x.B, 2)
    out = torch.full((x.B, 2, x.Hq, 64), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_rows_attn(0, q2.cuda(), pos, q4, table, out)
    assert s.read_status() == W.WM_ERR_BOUNDS
    got = to_f64(out)
    assert (got[0, 1] == 0).all() and (got[1, 1] == 0).all()
    for b, r, ts in ((0, 0, [t for t in range(70) if t // 16 != 1]), (1, 0, list(range(60))), (2, 0, list(range(64))),
                     (2, 1, list(range(4))), (3, 0, list(range(50))), (3, 1, [0])):
        for hq in range(x.Hq):
            want, tol = x.bound(0, b, hq, to_f64(q2[b, r, hq]), ts, 4)
            assert np.abs(got[b, r, hq] - want).max() <= tol


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_any_size(dtype):
    """Peaked, flat and rising scores; queries from 2^-100 to 2^60."""
    x = Q.Q4([300] * 4, Hkv=1, G=1, d=64, page=16, dtype=dtype, k=1)
    s, q4 = x.session(), x.q4()
    table, n = x.q4_dev()
    q = x.queries(x.B)
    for scale in (2.0 ** -100, 2.0 ** -8, 32.0, 0.0):
        y = q * scale
        out = torch.empty((x.B, 1, 64), dtype=x.tdt, device="cuda")
        s.q4_decode_attn(0, y.cuda(), q4, table, n, out)
        attend_all(x, s, q4, y, [300] * 4, to_f64(out), 0, 8)
    # so peaked that one slot takes all
    y = q * 2.0 ** 60
    s.q4_decode_attn(0, y.cuda(), q4, table, n, out)
    for b in range(x.B):
        K, V = (x.rows(p, 0, b, 0, np.arange(300)) for p in (x.kd, x.vd))
        assert np.allclose(to_f64(out)[b, 0], V[np.argmax(K @ to_f64(y[b, 0]))], rtol=0, atol=1e-6)
    y = q.clone()
    y[1, 0, 5], y[2, 0, 9] = float("nan"), float("inf")
    s.q4_decode_attn(0, y.cuda(), q4, table, n, out)
    got = to_f64(out)
    assert np.isnan(got[1]).all() and np.isnan(got[2]).all() and np.isfinite(got[[0, 3]]).all()


def on_tiles(x, Tq):
    """Whether rows of this shape run on the tensor-core kernel: its workspace holds rows read back."""
    c = x.session_cfg()
    return W.wm_q4_rows_attn_workspace(c, x.B, Tq, x.max_pages) >= x.max_pages * x.P * x.Hkv * x.d * 4


def check_many(x, q, pos, got, layer=0):
    """All rows at once, against 64 bits.  Weights enter the product as bf16 (2^-8), sums of its 128-slot
    steps are cut as in tests/_q4.py, the result is rounded by 2^-8 of itself."""
    T = int(pos.max()) + 1
    for b in range(x.B):
        n = int(pos[b].max()) + 1
        for h in range(x.Hkv):
            ts = np.arange(n)
            K, V = (x.rows(p, layer, b, h, ts) for p in (x.kd, x.vd))
            for g in range(x.G):
                Q_ = to_f64(q[b, :, h * x.G + g])
                s = Q_ @ K.T / np.sqrt(x.d)
                s[np.arange(n)[None] > pos[b][:, None]] = -np.inf
                p = np.exp(s - s.max(1, keepdims=True))
                want = p / p.sum(1, keepdims=True) @ V
                ds = (110 + x.d) * 2.0 ** -24 * (np.abs(Q_) @ np.abs(K).T).max() / np.sqrt(x.d)
                tol = (2 * ds + 2.0 ** -8 + T / 16 * 17 * 2.0 ** -23) * np.abs(V).max() + 2.0 ** -8 * np.abs(want).max()
                err = np.abs(got[b, :, h * x.G + g] - want).max()
                assert err <= tol, (b, h, g, err, tol)


@pytest.mark.parametrize("G,Tq,lens,Hkv,d,page,maxp,order", [
    (4, 300, [4001], 2, 128, 16, 1024, "last"),         # KV tiles cut, 256 rows per item
    (8, 16, [700, 90], 8, 64, 32, 4096, "last"),        # at most 128 rows: their even and odd KV tiles
    (1, 257, [300, 1500, 257], 2, 64, 8, 16384, "any"),  # more than one group of sequences, any order
    (2, 200, [611, 200], 3, 96, 64, 1024, "last"),
    (8, 260, [300] * 8, 4, 64, 16, 400, "last"),        # items enough: no cuts
    (1, 513, [513, 600], 32, 64, 128, 100, "last")])
def test_many_rows(G, Tq, lens, Hkv, d, page, maxp, order):
    x = Q.Q4(lens, Hkv=Hkv, G=G, d=d, page=page, k=1, max_pages=maxp, seed=G)
    assert on_tiles(x, Tq)
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    rng = np.random.default_rng(1)
    pos = np.stack([rng.integers(0, n, Tq) if order == "any" else np.arange(n - Tq, n) for n in lens]).astype(np.int32)
    q = x.queries(x.B, Tq)
    out = torch.full((x.B, Tq, x.Hq, d), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_rows_attn(0, q.cuda(), torch.from_numpy(pos).cuda(), q4, table, out)
    assert s.read_status() == 0
    check_many(x, q, pos, to_f64(out))


@pytest.mark.parametrize("G,Tq,lens,Hkv,maxp", [
    (4, 300, [400, 300, 350, 333, 500], 8, 512),  # up to four sequences at once
    (8, 70, [71, 300, 70], 8, 2048)])             # one after the other
def test_many_rows_in_groups(G, Tq, lens, Hkv, maxp):
    x = Q.Q4(lens, Hkv=Hkv, G=G, d=128, page=64, k=1, max_pages=maxp, seed=G)
    one, ws = maxp * 64 * Hkv * 128 * 4, W.wm_q4_rows_attn_workspace(x.session_cfg(), x.B, Tq, maxp)
    assert on_tiles(x, Tq) and ws < one * x.B
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    pos = np.stack([np.arange(n - Tq, n) for n in lens]).astype(np.int32)
    q = x.queries(x.B, Tq)
    out = torch.full((x.B, Tq, x.Hq, 128), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_rows_attn(0, q.cuda(), torch.from_numpy(pos).cuda(), q4, table, out)
    assert s.read_status() == 0
    check_many(x, q, pos, to_f64(out))


@pytest.mark.parametrize("G,Tq,B,maxp", [(8, 260, 8, 400), (4, 300, 2, 4096)])
def test_many_rows_leave_out_what_is_bad(G, Tq, B, maxp):
    x = Q.Q4([Tq] * B, Hkv=4, G=G, d=64, page=16, k=1, max_pages=maxp)
    assert on_tiles(x, Tq)
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    table[1, 3], table[0, 5] = -1, x.q4_pages
    pos = np.tile(np.arange(Tq, dtype=np.int32), (B, 1))
    q = x.queries(B, Tq)
    dev = torch.from_numpy(pos).cuda()
    dev[0, 7], dev[1, 9] = -1, x.T
    out = torch.full((B, Tq, x.Hq, 64), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_rows_attn(0, q.cuda(), dev, q4, table, out)
    assert s.read_status() == W.WM_ERR_BOUNDS
    got = to_f64(out)
    assert (got[0, 7] == 0).all() and (got[1, 9] == 0).all()
    for b, page in ((0, 5), (1, 3)):
        for r in (0, 15, 47, 48, 100, Tq - 1):
            ts = [t for t in range(r + 1) if t // 16 != page]
            for hq in (0, x.Hq - 1):
                want, tol = x.bound(0, b, hq, to_f64(q[b, r, hq]), ts, Tq / 16)
                assert np.abs(got[b, r, hq] - want).max() <= tol + 2.0 ** -8 * np.abs(x.vd[np.isfinite(x.vd)]).max(), (b, r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 2])
def test_scores_past_24_bits(dtype, G):
    """Scores so large that the reference is rounded: the largest one takes all, at every size."""
    x = Q.Q4([100] * 3, Hkv=2, G=G, d=64, page=16, dtype=dtype, k=1)
    s, q4 = x.session(), x.q4()
    table, n = x.q4_dev()
    q = x.queries(x.B)
    best = np.empty((x.B, x.Hq, 64))
    for b in range(x.B):
        for hq in range(x.Hq):
            K, V = (x.rows(p, 0, b, hq // G, np.arange(100)) for p in (x.kd, x.vd))
            z = np.sort(K @ to_f64(q[b, hq]))
            assert z[-1] - z[-2] > 1e-3  # (2^17 of it are 128 and more: nothing is left of the others)
            best[b, hq] = V[np.argmax(K @ to_f64(q[b, hq]))]
    for e in range(20, 40):
        y = q * 2.0 ** e
        out = torch.empty((x.B, x.Hq, 64), dtype=x.tdt, device="cuda")
        s.q4_decode_attn(0, y.cuda(), q4, table, n, out)
        assert np.array_equal(to_f64(out), best), e
    assert s.read_status() == 0
