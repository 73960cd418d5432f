"""Long-context operators against plain 64-bit references: windowed attention
(one row and many), shared prefixes, summed attention weights, eviction."""
import numpy as np
import pytest
import torch

from paper_2608_18486_gb300 import _lib as W
from tests._longctx import Cache, check_rows, to_f64

pytestmark = pytest.mark.gpu
BIG = 2 ** 31 - 1


def window_slots(n, sinks, window):
    return [t for t in range(n) if t < sinks or t >= n - window]


def run_window(c, layer=1, sinks=2, window=5, scale=1.0, stream=None):
    s = c.session()
    table, lens = c.dev()
    q = c.queries(c.B, scale=scale)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    s.window_attn(layer, q.cuda(), table, lens, out, sinks=sinks, window=window, stream=stream)
    torch.cuda.synchronize()
    return s, q.double().numpy(), to_f64(out)


# ------------------------------------------------------------------ window, one row
@pytest.mark.parametrize("dtype,d,G,page", [
    ("bf16", 64, 1, 16), ("bf16", 96, 2, 16), ("bf16", 128, 8, 64), ("bf16", 128, 4, 1),
    ("f32", 64, 1, 16), ("f32", 96, 8, 4), ("f32", 128, 2, 64), ("bf16", 96, 8, 2), ("f32", 128, 8, 32)])
@pytest.mark.parametrize("sinks,window", [(0, 0), (4, 0), (0, 1), (1, 33), (4, 17), (70, 40), (0, 300), (5, BIG), (BIG, BIG)])
def test_window_matches_reference(dtype, d, G, page, sinks, window):
    lens = [0, 1, 2, 31, 64, 129, 200]
    vis = lambda b: window_slots(lens[b], sinks, window)
    c = Cache(lens, Hkv=2, G=G, d=d, page=page, dtype=dtype, visible=vis, seed=d + G + page)
    for b, n in enumerate(lens):  # pages without a visible slot may be gone
        seen = {t // page for t in vis(b)}
        for x in range(c.max_pages):
            if x not in seen:
                c.table[b, x] = [-1, BIG, c.num_pages][x % 3]
    s, q, got = run_window(c, 1, sinks, window)
    assert s.read_status() == 0
    for b, n in enumerate(lens):
        for hq in range(c.Hq):
            want, _, ds, vmax = c.attend(1, b, hq, q[b, hq], vis(b))
            check_rows(c, got[b, hq], want, ds, vmax)


@pytest.mark.parametrize("B,Hkv", [(1, 1), (1, 3), (3, 7), (20, 4), (90, 4)])
def test_window_every_cluster_size(B, Hkv):
    lens = [700 - 3 * b for b in range(B)]
    c = Cache(lens, Hkv=Hkv, G=2, d=64, page=16, k=1, visible=lambda b: window_slots(lens[b], 3, 300), seed=B)
    s, q, got = run_window(c, 0, 3, 300)
    assert s.read_status() == 0
    for b in range(0, B, max(1, B // 5)):
        for hq in range(c.Hq):
            want, _, ds, vmax = c.attend(0, b, hq, q[b, hq], window_slots(lens[b], 3, 300))
            check_rows(c, got[b, hq], want, ds, vmax)


def test_window_peaked_queries_and_equal_keys():
    c = Cache([150, 97], Hkv=2, G=2, d=128, page=16, seed=5)
    s, q, got = run_window(c, 0, 4, 90, scale=20.0)
    for b in range(2):
        for hq in range(c.Hq):
            want, _, ds, vmax = c.attend(0, b, hq, q[b, hq], window_slots(int(c.lens[b]), 4, 90))
            check_rows(c, got[b, hq], want, ds, vmax)


def test_window_of_everything_is_decode_attention():
    c = Cache([300, 1, 77], Hkv=3, G=2, d=96, page=16, seed=2)
    s = c.session()
    table, lens = c.dev()
    q = c.queries(3).cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    s.window_attn(1, q, table, lens, a, sinks=0, window=BIG)
    s.decode_attn(1, q, table, lens, b)
    torch.cuda.synchronize()
    assert (a.float() - b.float()).abs().max() <= 3 * 2.0 ** -9 * float(np.nanmax(np.abs(c.vd)))


def test_window_bad_lengths_and_pages_are_reported():
    c = Cache([40, 40, 40, 40], Hkv=2, G=1, d=64, page=16, seed=3)
    s = c.session()
    table, lens = c.dev()
    q = c.queries(4).cuda()
    out = torch.full_like(q, 7.0)
    bad = lens.clone()
    bad[1], bad[2] = -1, c.max_pages * 16 + 1
    s.window_attn(0, q, table, bad, out, sinks=1, window=20)
    assert s.read_status() == W.WM_ERR_BOUNDS
    assert (out[1] == 0).all() and (out[2] == 0).all() and torch.isfinite(out.float()).all()
    t2 = table.clone()
    t2[3, 2] = c.num_pages  # holds slots 32 .. 39 of the window 20 .. 39
    s.window_attn(0, q, t2, lens, out, sinks=1, window=20)
    assert s.read_status() == W.WM_ERR_BOUNDS
    qd, got = to_f64(q), to_f64(out)
    for hq in range(2):
        want, _, ds, vmax = c.attend(0, 3, hq, qd[3, hq], [0] + list(range(20, 32)))
        check_rows(c, got[3, hq], want, ds, vmax)


def test_window_on_another_stream_and_in_a_graph():
    c = Cache([513, 300], Hkv=2, G=2, d=64, page=16, seed=9)
    side = torch.cuda.Stream()
    s, q, got = run_window(c, 1, 4, 200, stream=side)
    qd = torch.from_numpy(q).to(torch.bfloat16).cuda()
    table, lens = c.dev()
    out = torch.empty_like(qd)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        s.window_attn(1, qd, table, lens, out, sinks=4, window=200)
    g.replay()
    torch.cuda.synchronize()
    assert np.array_equal(to_f64(out), got)
    lens.copy_(torch.tensor([100, 11], dtype=torch.int32))
    g.replay()
    torch.cuda.synchronize()
    for b, n in enumerate([100, 11]):
        want, _, ds, vmax = c.attend(1, b, 1, q[b, 1], window_slots(n, 4, 200))
        check_rows(c, to_f64(out)[b, 1], want, ds, vmax)


# ------------------------------------------------------------------ window, many rows
def prefill_slots(i, sinks, window):
    return [t for t in range(i + 1) if t < sinks or t > i - window]


def run_prefill(c, pos, sinks, window, layer=0):
    s = c.session()
    table, _ = c.dev()
    q = c.queries(*pos.shape)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    s.window_prefill_attn(layer, q.cuda(), torch.from_numpy(pos).cuda(), table, out, sinks=sinks, window=window)
    torch.cuda.synchronize()
    return s, q.double().numpy(), to_f64(out)


def check_prefill(c, pos, sinks, window, q, got, layer=0, rows=None):
    B, Tq = pos.shape
    for b in range(B):
        for r in (range(Tq) if rows is None else rows):
            for hq in range(c.Hq):
                want, _, ds, vmax = c.attend(layer, b, hq, q[b, r, hq], prefill_slots(int(pos[b, r]), sinks, window))
                check_rows(c, got[b, r, hq], want, ds, vmax)


@pytest.mark.parametrize("dtype,d,G,page", [("bf16", 64, 1, 16), ("bf16", 96, 2, 16), ("bf16", 128, 4, 64),
                                            ("bf16", 64, 8, 4), ("f32", 64, 2, 16), ("bf16", 128, 1, 256)])
@pytest.mark.parametrize("sinks,window,Tq,first", [(0, 0, 5, 0), (3, 0, 9, 2), (0, 1, 40, 0), (4, 50, 150, 0),
                                                  (130, 20, 140, 150), (2, 200, 65, 333), (1, 128, 257, 40),
                                                  (5, BIG, 129, 0)])
def test_window_prefill_matches_reference(dtype, d, G, page, sinks, window, Tq, first):
    n = first + Tq
    seen = sorted({t for i in range(first, n) for t in prefill_slots(i, sinks, window)})
    c = Cache([n, n], Hkv=1, G=G, d=d, page=page, dtype=dtype, k=1, visible=lambda b: seen, seed=Tq + d)
    pages = {t // page for t in seen}
    for x in range(c.max_pages):
        if x not in pages:
            c.table[:, x] = [-1, BIG, c.num_pages][x % 3]
    pos = np.stack([np.arange(first, n, dtype=np.int32)] * 2)
    s, q, got = run_prefill(c, pos, sinks, window)
    assert s.read_status() == 0
    rows = sorted(set(range(0, Tq, 7)) | {0, 1, Tq - 1, min(Tq - 1, 127), min(Tq - 1, 128)} - {Tq})
    check_prefill(c, pos, sinks, window, q, got, rows=[r for r in rows if r < Tq])


@pytest.mark.parametrize("order", ["shuffled", "strided", "reversed"])
def test_window_prefill_positions_in_any_order(order):
    n = 420
    c = Cache([n], Hkv=2, G=2, d=64, page=16, k=1, seed=4)
    pos = np.arange(0, n, 8 if order == "strided" else 1, dtype=np.int32)
    if order == "shuffled":
        pos = np.random.default_rng(0).permutation(pos)
    if order == "reversed":
        pos = pos[::-1].copy()
    s, q, got = run_prefill(c, pos[None], 3, 60)
    assert s.read_status() == 0
    check_prefill(c, pos[None], 3, 60, q, got, rows=range(0, len(pos), 5))


@pytest.mark.parametrize("G", [1, 2])
def test_window_prefill_of_scattered_positions_reads_only_visible_slots(G):
    pos = np.array([300, 5, 171, 172, 40, 600, 601, 333] * 20, dtype=np.int32)
    seen = sorted({t for i in set(pos.tolist()) for t in prefill_slots(i, 2, 6)})
    c = Cache([602], Hkv=1, G=G, d=64, page=8, k=1, visible=lambda b: seen, seed=4)
    for x in range(c.max_pages):
        if x not in {t // 8 for t in seen}:
            c.table[:, x] = [-1, BIG, c.num_pages][x % 3]
    s, q, got = run_prefill(c, pos[None], 2, 6)
    assert s.read_status() == 0
    check_prefill(c, pos[None], 2, 6, q, got, rows=list(range(8)) + [127, 128, 159])


@pytest.mark.parametrize("Hkv,G", [(32, 1), (16, 2), (8, 4)])
@pytest.mark.parametrize("sinks,window", [(0, 40), (4, 200), (300, 1)])
def test_window_prefill_more_tiles_than_sms(Hkv, G, sinks, window):
    """Several items per CTA, items of a single step among them."""
    n, B = 1000, 2
    c = Cache([n] * B, Hkv=Hkv, G=G, d=64, page=64, k=1, seed=Hkv)
    pos = np.stack([np.arange(n, dtype=np.int32)] * B)
    s, q, got = run_prefill(c, pos, sinks, window)
    assert s.read_status() == 0
    check_prefill(c, pos, sinks, window, q, got, rows=[0, 100, 128, 255, 256, 511, 700, 999])


def test_window_prefill_bad_positions_zero_their_rows():
    c = Cache([60], Hkv=1, G=2, d=64, page=16, k=1, seed=8)
    pos = np.arange(0, 60, dtype=np.int32)[None].copy()
    pos[0, 7], pos[0, 30] = -1, c.max_pages * 16
    s, q, got = run_prefill(c, pos, 2, 9)
    assert s.read_status() == W.WM_ERR_BOUNDS
    assert (got[0, [7, 30]] == 0).all()
    check_prefill(c, pos, 2, 9, q, got, rows=[0, 6, 8, 29, 31, 59])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_prefill_bad_pages_are_left_out(dtype):
    c = Cache([200], Hkv=1, G=2, d=64, page=16, k=1, dtype=dtype, seed=8)
    good = c.table.copy()
    c.table[0, [0, 5]] = [-1, c.num_pages]  # slots 0 .. 15 and 80 .. 95
    pos = np.arange(200, dtype=np.int32)[None]
    s, q, got = run_prefill(c, pos, 20, 60)
    assert s.read_status() == W.WM_ERR_BOUNDS
    c.table = good
    for r in (0, 15, 16, 90, 95, 96, 199):
        ts = [t for t in prefill_slots(r, 20, 60) if t // 16 not in (0, 5)]
        for hq in range(2):
            want, _, ds, vmax = c.attend(0, 0, hq, q[0, r, hq], ts)
            check_rows(c, got[0, r, hq], want, ds, vmax)


def test_window_prefill_rows_equal_decode_rows():
    n = 300
    c = Cache([n], Hkv=1, G=2, d=96, page=16, k=1, seed=6)
    pos = np.arange(n, dtype=np.int32)[None]
    s, q, got = run_prefill(c, pos, 4, 70)
    table, _ = c.dev()
    out = torch.empty((1, 2, 96), dtype=torch.bfloat16, device="cuda")
    for r in (0, 3, 73, 74, 75, 200, 299):
        s.window_attn(0, torch.from_numpy(q[:, r]).to(torch.bfloat16).cuda(), table,
                      torch.tensor([r + 1], dtype=torch.int32, device="cuda"), out, sinks=4, window=70)
        assert np.abs(to_f64(out)[0] - got[0, r]).max() <= 4 * 2.0 ** -9 * float(np.nanmax(np.abs(c.vd)))


# ------------------------------------------------------------------ shared prefix
def run_prefix(c, shared, layer=0, scale=1.0):
    s = c.session()
    table, lens = c.dev()
    q = c.queries(c.B, scale=scale)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    s.prefix_attn(layer, q.cuda(), table, lens, out, shared_pages=shared)
    torch.cuda.synchronize()
    return s, q.double().numpy(), to_f64(out)


@pytest.mark.parametrize("dtype,d,G,page,shared", [
    ("bf16", 64, 1, 16, 8), ("bf16", 96, 2, 16, 21), ("bf16", 128, 8, 64, 3), ("bf16", 128, 4, 8, 19),
    ("f32", 64, 1, 16, 5), ("f32", 96, 4, 16, 9), ("bf16", 64, 2, 2, 37), ("bf16", 64, 1, 256, 2), ("f32", 128, 8, 32, 3)])
@pytest.mark.parametrize("tail", [[1], [0, 3, 40], [1, 2, 70, 0, 33, 5, 1, 90, 16, 17, 64]])
def test_prefix_matches_reference(dtype, d, G, page, shared, tail):
    base = shared * page
    lens = [base + t for t in tail]
    c = Cache(lens, Hkv=2, G=G, d=d, page=page, dtype=dtype, shared=shared, seed=len(tail) + d)
    s, q, got = run_prefix(c, shared, layer=1)
    assert s.read_status() == 0
    for b, n in enumerate(lens):
        for hq in range(c.Hq):
            want, _, ds, vmax = c.attend(1, b, hq, q[b, hq], range(n))
            check_rows(c, got[b, hq], want, ds, vmax)


@pytest.mark.parametrize("lens", [[0, 1, 64, 63, 65, 200], [17, 3, 40, 5], [0, 0], [150]])
def test_prefix_sequences_that_end_inside_it(lens):
    shared, page = 4, 16
    c = Cache(lens, Hkv=2, G=2, d=64, page=page, shared=shared, k=1, seed=len(lens))
    s, q, got = run_prefix(c, shared)
    assert s.read_status() == 0
    for b, n in enumerate(lens):
        for hq in range(c.Hq):
            want, _, ds, vmax = c.attend(0, b, hq, q[b, hq], range(n))
            check_rows(c, got[b, hq], want, ds, vmax)


@pytest.mark.parametrize("B,G,Hkv,d", [(70, 1, 2, 64), (150, 2, 1, 96), (40, 8, 1, 128), (33, 4, 2, 128)])
def test_prefix_many_rows(B, G, Hkv, d):
    shared, page = 50, 16
    lens = [shared * page + (5 * b) % 23 for b in range(B)]
    c = Cache(lens, Hkv=Hkv, G=G, d=d, page=page, shared=shared, k=1, seed=B)
    s, q, got = run_prefix(c, shared)
    assert s.read_status() == 0
    for b in range(0, B, 7):
        for hq in range(c.Hq):
            want, _, ds, vmax = c.attend(0, b, hq, q[b, hq], range(lens[b]))
            check_rows(c, got[b, hq], want, ds, vmax)


@pytest.mark.parametrize("shared", [0, 6])
def test_prefix_of_nothing_and_of_everything(shared):
    c = Cache([96] * 3, Hkv=2, G=2, d=128, page=16, shared=shared, k=1, seed=1, max_pages=6)
    s, q, got = run_prefix(c, shared)
    assert s.read_status() == 0
    for b in range(3):
        for hq in range(c.Hq):
            want, _, ds, vmax = c.attend(0, b, hq, q[b, hq], range(96))
            check_rows(c, got[b, hq], want, ds, vmax)


# Prefixes large enough for the tensor-core kernel (over 40 MB of K/V times
# groups of 8 rows): more and fewer than 128 rows per kv head, several row
# blocks, sequences that end inside the prefix, a page that does not exist.
@pytest.mark.parametrize("B,G,Hkv,d,page,shared,drop", [
    (64, 8, 1, 64, 16, 210, None), (37, 4, 2, 96, 8, 401, 100), (100, 1, 4, 64, 64, 53, None),
    (75, 4, 1, 128, 256, 10, None), (4, 2, 4, 128, 64, 330, 7), (9, 8, 2, 96, 128, 50, None)])
def test_prefix_on_the_tensor_cores(B, G, Hkv, d, page, shared, drop):
    base = shared * page
    lens = [base + (7 * b) % 29 for b in range(B)]
    lens[1], lens[B // 2], lens[B - 1] = base // 2 + 3, 5, 0  # (sequence 0 holds the whole prefix)
    assert base * Hkv * d * 4 * -(-B * G // 8) > 40 << 20
    c = Cache(lens, Hkv=Hkv, G=G, d=d, page=page, shared=shared, k=1, seed=B)
    good = c.table.copy()
    if drop is not None:
        c.table[:, drop] = c.num_pages
    s, q, got = run_prefix(c, shared)
    assert s.read_status() == (0 if drop is None else W.WM_ERR_BOUNDS)
    c.table = good
    for b in sorted({0, 1, 2, B // 2, B - 1, B - 2, B // 3}):
        ts = [t for t in range(lens[b]) if drop is None or t // page != drop]
        for hq in {0, G - 1, c.Hq - 1}:
            want, _, ds, vmax = c.attend(0, b, hq, q[b, hq], ts)
            check_rows(c, got[b, hq], want, ds, vmax)


def test_prefix_peaked_queries():
    c = Cache([500, 433, 401], Hkv=2, G=2, d=128, page=16, shared=25, k=1, seed=12)
    s, q, got = run_prefix(c, 25, scale=20.0)
    for b in range(3):
        for hq in range(c.Hq):
            want, _, ds, vmax = c.attend(0, b, hq, q[b, hq], range(int(c.lens[b])))
            check_rows(c, got[b, hq], want, ds, vmax)


def test_prefix_bad_lengths_and_pages_are_reported():
    c = Cache([100, 110, 90], Hkv=1, G=2, d=64, page=16, shared=4, k=1, seed=3)
    s = c.session()
    table, lens = c.dev()
    q = c.queries(3).cuda()
    out = torch.full_like(q, 7.0)
    bad = lens.clone()
    bad[1] = -5
    s.prefix_attn(0, q, table, bad, out, shared_pages=4)
    assert s.read_status() == W.WM_ERR_BOUNDS
    assert (out[1] == 0).all() and (out[0] != 7).all()
    t2 = table.clone()
    t2[:, 1] = c.num_pages + 3  # slots 16 .. 31 of the prefix
    s.prefix_attn(0, q, t2, lens, out, shared_pages=4)
    assert s.read_status() == W.WM_ERR_BOUNDS
    qd, got = to_f64(q), to_f64(out)
    for b in range(3):
        for hq in range(2):
            want, _, ds, vmax = c.attend(0, b, hq, qd[b, hq], [t for t in range(int(lens[b])) if t // 16 != 1])
            check_rows(c, got[b, hq], want, ds, vmax)


# ------------------------------------------------------------------ summed weights
@pytest.mark.parametrize("dtype,d,G,page", [("bf16", 64, 1, 16), ("bf16", 96, 2, 16), ("bf16", 128, 8, 64),
                                            ("bf16", 128, 4, 2), ("f32", 64, 2, 16), ("f32", 128, 8, 32)])
def test_mass_matches_reference_and_adds_up(dtype, d, G, page):
    lens = [0, 1, 5, 100, 257]
    c = Cache(lens, Hkv=2, G=G, d=d, page=page, dtype=dtype, k=2, seed=d + G)
    s = c.session()
    table, dl = c.dev()
    start = np.abs(c.rng.standard_normal((2, 5, 2, c.T))).astype(np.float32)
    mass = torch.from_numpy(start).cuda()
    want = start.astype(np.float64)
    tol = np.zeros_like(want)
    for step in range(2):
        q = c.queries(5)
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        s.decode_attn_mass(1, q.cuda(), table, dl, mass, out)
        qd, got = q.double().numpy(), to_f64(out)
        for b, n in enumerate(lens):
            for hq in range(c.Hq):
                o, p, ds, vmax = c.attend(1, b, hq, qd[b, hq], range(n))
                check_rows(c, got[b, hq], o, ds, vmax)
                want[1, b, hq // G, :n] += p
                # each weight off by a factor e^(2 ds) and a few roundings; the
                # sum rounds once per call
                tol[1, b, hq // G, :n] += p * (2 * ds + 64 * 2.0 ** -24)
        tol[1] += 2.0 ** -23 * want[1]
    assert s.read_status() == 0
    assert (np.abs(to_f64(mass) - want) <= tol).all()
    assert np.array_equal(to_f64(mass)[0], start[0].astype(np.float64))  # other channel untouched


def test_mass_long_split_is_reproducible():
    c = Cache([5000, 4097], Hkv=1, G=2, d=64, page=64, k=1, seed=3)
    s = c.session()
    table, dl = c.dev()
    q = c.queries(2).cuda()
    res = []
    for _ in range(2):
        mass, out = torch.zeros((1, 2, 1, c.T), device="cuda"), torch.empty_like(q)
        s.decode_attn_mass(0, q, table, dl, mass, out)
        res.append((mass, out))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
    assert torch.allclose(res[0][0].sum(-1), torch.full((1, 2, 1), 2.0, device="cuda"), atol=1e-4)
    assert (res[0][0][0, 1, 0, 4097:] == 0).all()
    for b in range(2):
        for hq in range(2):
            want, _, ds, vmax = c.attend(0, b, hq, to_f64(q)[b, hq], range(int(c.lens[b])))
            check_rows(c, to_f64(res[0][1])[b, hq], want, ds, vmax)


def test_mass_bad_page_gets_no_weight():
    c = Cache([64], Hkv=1, G=2, d=64, page=16, k=1, seed=3)
    s = c.session()
    table, dl = c.dev()
    table[0, 2] = -1
    q = c.queries(1)
    mass, out = torch.zeros((1, 1, 1, c.T), device="cuda"), torch.empty((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    s.decode_attn_mass(0, q.cuda(), table, dl, mass, out)
    assert s.read_status() == W.WM_ERR_BOUNDS
    got = to_f64(mass)[0, 0, 0]
    assert (got[32:48] == 0).all() and abs(got.sum() - 2) < 1e-4


# ------------------------------------------------------------------ eviction
def evict_reference(c, mass, budget, sinks, recent):
    kd, vd = c.kp.clone(), c.vp.clone()
    out, kept = np.zeros_like(mass), np.full((c.k, c.B, c.Hkv, budget), -1, dtype=np.int32)
    for ch in range(c.k):
        for b in range(c.B):
            n = int(c.lens[b])
            for h in range(c.Hkv):
                m = mass[ch, b, h]
                keep = list(range(n))
                if n > budget:
                    mid = range(sinks, n - recent)
                    rank = sorted(mid, key=lambda t: (np.isnan(m[t]), -m[t] if not np.isnan(m[t]) else 0.0, t))
                    keep = sorted(list(range(sinks)) + rank[:budget - sinks - recent] + list(range(n - recent, n)))
                for j, t in enumerate(keep):
                    a, z = c.table[b, t // c.P], c.table[b, j // c.P]
                    kd[ch, z, h, j % c.P] = c.kp[ch, a, h, t % c.P]
                    vd[ch, z, h, j % c.P] = c.vp[ch, a, h, t % c.P]
                    out[ch, b, h, j], kept[ch, b, h, j] = m[t], t
    return kd, vd, out, kept, np.minimum(c.lens, budget)


def same_bits(a, b):
    it = {4: torch.int32, 2: torch.int16}[a.element_size()]
    return torch.equal(a.cpu().contiguous().view(it), b.cpu().contiguous().view(it))


@pytest.mark.parametrize("dtype,d,page", [("bf16", 64, 16), ("bf16", 96, 16), ("bf16", 128, 4), ("f32", 64, 1),
                                          ("f32", 96, 64), ("f32", 128, 16)])
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (40, 4, 8), (40, 0, 40), (40, 20, 20),
                                                 (100, 0, 0), (129, 4, 64), (255, 1, 100)])
@pytest.mark.parametrize("alias", [False, True])
def test_evict_matches_reference(dtype, d, page, budget, sinks, recent, alias):
    lens = [0, 1, 40, 41, 129, 130, 300, 700]
    c = Cache(lens, Hkv=2, G=1, d=d, page=page, dtype=dtype, k=2, seed=budget + d)
    mass = np.abs(c.rng.standard_normal((2, 8, 2, c.T))).astype(np.float32)
    mass = np.where(c.rng.random(mass.shape) < 0.3, np.float32(0.0), mass)   # ties at zero
    mass = np.where(c.rng.random(mass.shape) < 0.3, np.float32(0.75), mass)  # and elsewhere
    mass[1, :, :, 3::11] = np.nan
    mass[0, :, 1, 5::13] = -0.0
    mass[1, :, 1, 6::17] = np.inf
    s = c.session()
    table, dl = c.dev()
    m = torch.from_numpy(mass).cuda()
    mo = m if alias else torch.full_like(m, 9.0)
    kept = torch.full((2, 8, 2, budget), 77, dtype=torch.int32, device="cuda")
    nl = torch.full((8,), 77, dtype=torch.int32, device="cuda")
    s.evict(m, table, dl, mo, kept, nl, budget=budget, sinks=sinks, recent=recent)
    assert s.read_status() == 0
    kd, vd, out, want, wl = evict_reference(c, mass, budget, sinks, recent)
    assert np.array_equal(kept.cpu().numpy(), want)
    assert np.array_equal(nl.cpu().numpy(), wl)
    assert np.array_equal(mo.cpu().numpy(), out, equal_nan=True)
    assert same_bits(s.k_pool, kd) and same_bits(s.v_pool, vd)


def test_evict_long_sequence():
    c = Cache([9001], Hkv=1, G=1, d=64, page=64, k=1, seed=1)
    mass = np.abs(c.rng.standard_normal((1, 1, 1, c.T))).astype(np.float32)
    s = c.session()
    table, dl = c.dev()
    mo, kept = torch.empty((1, 1, 1, c.T), device="cuda"), torch.empty((1, 1, 1, 5003), dtype=torch.int32, device="cuda")
    nl = torch.empty(1, dtype=torch.int32, device="cuda")
    s.evict(torch.from_numpy(mass).cuda(), table, dl, mo, kept, nl, budget=5003, sinks=3, recent=777)
    kd, vd, out, want, wl = evict_reference(c, mass, 5003, 3, 777)
    assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(mo.cpu().numpy(), out)
    assert same_bits(s.k_pool, kd) and same_bits(s.v_pool, vd)


@pytest.mark.parametrize("B,k,Hkv,d", [(30, 3, 4, 64), (3, 2, 5, 96)])
def test_evict_many_units_and_clusters(B, k, Hkv, d):
    """More units than two per SM, and few enough for clusters, several waves each."""
    lens = [500 - 7 * b for b in range(B)]
    c = Cache(lens, Hkv=Hkv, G=1, d=d, page=16, k=k, seed=B)
    mass = np.abs(c.rng.standard_normal((k, B, Hkv, c.T))).astype(np.float32)
    s = c.session()
    table, dl = c.dev()
    m = torch.from_numpy(mass).cuda()
    kept, nl = torch.empty((k, B, Hkv, 260), dtype=torch.int32, device="cuda"), torch.empty_like(dl)
    s.evict(m, table, dl, m, kept, nl, budget=260, sinks=4, recent=30)
    kd, vd, out, want, wl = evict_reference(c, mass, 260, 4, 30)
    assert s.read_status() == 0
    assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(m.cpu().numpy(), out)
    assert same_bits(s.k_pool, kd) and same_bits(s.v_pool, vd)


def evict_masses(c, kind):
    shape = (c.k, c.B, c.Hkv, c.T)
    m = np.abs(c.rng.standard_normal(shape))
    if kind == "equal":
        m[:] = 0.3
    elif kind == "few":  # ties of many slots
        m = c.rng.integers(0, 3, shape) * 0.25
    elif kind == "wide":  # every exponent, both signs, what is no number
        m = np.exp2(c.rng.uniform(-140, 120, shape)) * c.rng.choice([-1.0, 1.0], shape)
        m[..., 5::19], m[..., 7::23], m[..., 9::29] = np.inf, -np.inf, np.nan
    elif kind == "close":  # neighbours of one value
        m = np.float32(0.5) * (1 + c.rng.integers(0, 40, shape) * 2.0 ** -23)
    return m.astype(np.float32)


# units of one to eight CTAs, whose CTAs hold up to 2048 sums each, up to 8192, or more than that
@pytest.mark.parametrize("B,Hkv,lens,page", [(1, 1, 2050, 16), (2, 3, 5011, 4), (1, 1, 16381, 64), (1, 2, 30001, 64),
                                             (1, 1, 65505, 64), (40, 1, 4099, 32), (40, 2, 9001, 16),
                                             (1, 1, 4001, 1), (3, 4, 1023, 8), (160, 1, 2048, 16), (160, 1, 2049, 16)])
@pytest.mark.parametrize("kind", ["random", "equal", "few", "wide", "close"])
@pytest.mark.parametrize("alias", [False, True])
def test_evict_selects_the_largest_sums_at_every_split(B, Hkv, lens, page, kind, alias):
    """kept and the sums against a stable sort, the rows against kept."""
    if lens * B * Hkv > 200000 and kind not in ("random", "few"):
        pytest.skip("the large ones at two kinds")
    c = Cache([lens - 3 * (b % 5) for b in range(B)], Hkv=Hkv, G=1, d=64, page=page, k=1, seed=lens)
    mass = evict_masses(c, kind)
    budget, sinks, recent = lens * 3 // 7, 5, lens // 9
    s = c.session()
    table, dl = c.dev()
    m = torch.from_numpy(mass).cuda()
    mo = m if alias else torch.full_like(m, 9.0)
    kept = torch.full((1, B, Hkv, budget), 77, dtype=torch.int32, device="cuda")
    nl = torch.empty_like(dl)
    s.evict(m, table, dl, mo, kept, nl, budget=budget, sinks=sinks, recent=recent)
    assert s.read_status() == 0 and (nl == budget).all()
    kept, mo = kept.cpu().numpy(), mo.cpu().numpy()
    kd, vd = s.k_pool.cpu(), s.v_pool.cpu()
    for b in range(B):
        n, tab = int(c.lens[b]), c.table[b]
        for h in range(Hkv):
            x = mass[0, b, h]
            mid = np.where(np.isnan(x[sinks:n - recent]), -np.inf, x[sinks:n - recent]).astype(np.float64)
            nan = np.isnan(x[sinks:n - recent])
            order = sinks + np.lexsort((np.arange(len(mid)), -mid, nan))
            want = np.sort(np.concatenate([np.arange(sinks), order[:budget - sinks - recent], np.arange(n - recent, n)]))
            assert np.array_equal(kept[0, b, h], want)
            assert np.array_equal(mo[0, b, h, :budget], x[want], equal_nan=True) and (mo[0, b, h, budget:] == 0).all()
            to = np.arange(budget)
            for got, was in ((kd, c.kp), (vd, c.vp)):
                assert same_bits(got[0, tab[to // page], h, to % page], was[0, tab[want // page], h, want % page])


def test_evict_bad_lengths_and_pages_are_reported():
    c = Cache([60, 60, 60], Hkv=1, G=1, d=64, page=16, k=1, seed=2)
    s = c.session()
    table, dl = c.dev()
    mass = torch.rand((1, 3, 1, c.T), device="cuda")
    mo, kept = torch.empty_like(mass), torch.empty((1, 3, 1, 20), dtype=torch.int32, device="cuda")
    nl = torch.empty(3, dtype=torch.int32, device="cuda")
    bad = dl.clone()
    bad[0], bad[1] = -3, c.T + 1
    s.evict(mass, table, bad, mo, kept, nl, budget=20, sinks=2, recent=2)
    assert s.read_status() == W.WM_ERR_BOUNDS
    assert nl.tolist() == [0, 0, 20] and (kept[:, :2] == -1).all() and (mo[:, :2] == 0).all()
    # the first two sequences' rows did not move
    for b in (0, 1):
        for pg in c.table[b, :4]:
            assert same_bits(s.k_pool[:, pg], c.kp[:, pg])


def test_attention_over_an_evicted_cache_equals_attention_over_the_kept_slots():
    c = Cache([200, 150], Hkv=2, G=2, d=64, page=16, k=1, seed=7)
    s = c.session()
    table, dl = c.dev()
    mass = torch.zeros((1, 2, 2, c.T), device="cuda")
    out = torch.empty((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    for _ in range(3):
        s.decode_attn_mass(0, c.queries(2).cuda(), table, dl, mass, out)
    kept, nl = torch.empty((1, 2, 2, 64), dtype=torch.int32, device="cuda"), torch.empty_like(dl)
    s.evict(mass, table, dl, mass, kept, nl, budget=64, sinks=4, recent=16)
    q = c.queries(2)
    s.decode_attn(0, q.cuda(), table, nl, out)
    got, ks = to_f64(out), kept.cpu().numpy()
    for b in range(2):
        for hq in range(4):
            want, _, ds, vmax = c.attend(0, b, hq, q.double().numpy()[b, hq], ks[0, b, hq // 2])
            check_rows(c, got[b, hq], want, ds, vmax)


# ------------------------------------------------------------------ offsets past 32 bits
def test_cache_rows_past_32_bits():
    """Pages whose elements lie past 2^32 of their pool (17 GB in all)."""
    Hkv, P, d, n = 32, 64, 128, 150
    pages = 2 ** 32 // (Hkv * P * d) + 8
    c = Cache([n, n], Hkv=Hkv, G=1, d=d, page=P, k=1, seed=0)
    small = c.num_pages
    cfg = W.make_config(1, 1, 64, Hkv, Hkv, d, 1, P, "bf16", [0])
    from paper_2608_18486_gb300.session import DecodeSession
    s = DecodeSession(cfg, 2, pages, c.max_pages)
    far = torch.arange(small) + pages - small
    far[::2] -= pages - small  # every other page stays at the start
    s.k_pool[0, far] = c.kp[0].cuda()
    s.v_pool[0, far] = c.vp[0].cuda()
    table = torch.from_numpy(np.where(c.table >= 0, far.numpy()[c.table], -1).astype(np.int32)).cuda()
    lens = torch.from_numpy(c.lens).cuda()
    q = c.queries(2)
    qd, dq, out = q.double().numpy(), q.cuda(), torch.empty_like(q, device="cuda")
    mass = torch.zeros((1, 2, Hkv, c.T), device="cuda")

    def check(slots):
        got = to_f64(out)
        for b in range(2):
            for hq in (0, 17, 31):
                want, _, ds, vmax = c.attend(0, b, hq, qd[b, hq], slots(b, hq))
                check_rows(c, got[b, hq], want, ds, vmax)

    s.window_attn(0, dq, table, lens, out, sinks=3, window=100)
    check(lambda b, hq: window_slots(n, 3, 100))
    s.prefix_attn(0, dq, table, lens, out, shared_pages=0)
    check(lambda b, hq: range(n))
    s.decode_attn_mass(0, dq, table, lens, mass, out)
    check(lambda b, hq: range(n))
    pos = torch.full((2, 1), n - 1, dtype=torch.int32, device="cuda")
    s.window_prefill_attn(0, dq[:, None].contiguous(), pos, table, out.view(2, 1, Hkv, d), sinks=3, window=100)
    check(lambda b, hq: window_slots(n, 3, 100))
    kept, nl = torch.empty((1, 2, Hkv, 50), dtype=torch.int32, device="cuda"), torch.empty_like(lens)
    s.evict(mass, table, lens, mass, kept, nl, budget=50, sinks=1, recent=9)
    s.decode_attn(0, dq, table, nl, out)
    ks = kept.cpu().numpy()
    check(lambda b, hq: ks[0, b, hq])
    assert s.read_status() == 0


# ------------------------------------------------------------------ the pool at given positions
@pytest.mark.parametrize("name,B", [("tiny_f32", 2), ("paper_k16", 3), ("paper_k16", 70)])
def test_pool_at_given_positions(name, B):
    """wm_kv_mix_at: the same keys as wm_kv_mix when pos = slot - 1; else the
    keys that wm_kv_mix writes at the slot of that position; V unchanged."""
    from tests import _harness as H
    from wm_synth import configs
    w = configs.get(name).with_(B=B, ctx=100)
    prob, s, dp = H.setup(w)
    at = lambda: H.gpu_written_kv(s, prob, 1, w.k - 1)
    s.kv_mix(dp.h, dp.page_table, dp.slot)
    k0, v0 = at()
    s.kv_mix(dp.h, dp.page_table, dp.slot, pos=dp.slot - 1)
    k1, v1 = at()
    assert np.array_equal(k0, k1) and np.array_equal(v0, v1)
    s.kv_mix(dp.h, dp.page_table, dp.slot, pos=torch.full_like(dp.slot, 36))
    k2, v2 = at()
    assert np.array_equal(v0, v2) and not np.array_equal(k0, k2)
    # at slot 37 the pool itself uses position 36
    s.kv_mix(dp.h, dp.page_table, torch.full_like(dp.slot, 37))
    pg = int(prob.page_table[1, 37 // w.page])
    assert np.array_equal(to_f64(s.k_pool[w.k - 1, pg, :, 37 % w.page]), k2)
    assert s.read_status() == 0


def test_views_with_gaps_are_refused():
    c = Cache([40, 20], Hkv=2, G=2, d=64, page=16, k=1, seed=1)
    s = c.session()
    table, lens = c.dev()
    wide = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    mass = torch.zeros((1, 2, 2, c.T), device="cuda")
    for call in (lambda: s.window_attn(0, wide[..., :64], table, lens, out, sinks=1, window=4),
                 lambda: s.window_attn(0, out, table, lens, wide[..., ::2], sinks=1, window=4),
                 lambda: s.prefix_attn(0, wide[..., :64], table, lens, out, shared_pages=0),
                 lambda: s.window_prefill_attn(0, wide[:, None, :, :64], lens[:, None], table, out, sinks=1, window=4),
                 lambda: s.decode_attn_mass(0, out, table, lens, mass[..., ::2], out),
                 lambda: s.evict(mass, table.t(), lens, mass, table, lens, budget=8, sinks=1, recent=1)):
        with pytest.raises(ValueError):
            call()


def test_scratch_outgrown_by_a_later_call_stays_with_its_graph():
    c = Cache([90] * 6, Hkv=2, G=2, d=64, page=16, shared=3, seed=8)
    s = c.session()
    table, lens = c.dev()
    q = c.queries(6).cuda()
    want, out = torch.empty_like(q), torch.empty_like(q)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def call(B, out, stream=None):
        s.prefix_attn(1, q, table, lens, out, shared_pages=3, B=B, stream=stream)

    call(1, want, stream)  # (allocates before the capture)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=stream):
        call(1, out)
    small = s._scratch[stream.cuda_stream].numel()
    call(6, want, stream)
    torch.cuda.synchronize()
    assert s._scratch[stream.cuda_stream].numel() > small
    with torch.cuda.stream(stream):  # what the allocator hands out next is not the graph's
        others = [torch.full((small,), 77, dtype=torch.uint8, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0])
    assert all(bool((x == 77).all()) for x in others)
