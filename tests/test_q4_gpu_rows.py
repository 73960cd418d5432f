"""Many rows over a 4-bit cache: the size of the workspace, and the forms in which they run on the
tensor cores (whole KV ranges per item, or cut ones with partial records)."""
import numpy as np
import pytest
import torch

from paper_2608_18486_gb300 import _lib as W
from tests import _q4 as Q
from tests._longctx import to_f64

pytestmark = pytest.mark.gpu

ROWS, RECORDS = 2 ** 29, 2 ** 28  # bytes of rows read back at once (or one sequence's), of partial records


def config(Hq, Hkv, d, page):
    return W.make_config(1, 1, 64, Hq, Hkv, d, 1, page, "bf16", [0])


def up(n):
    return (n + 255) // 256 * 256


def one_sequence(c, maxp):
    return 4 * maxp * c.page_size * c.Hkv * c.d


def form(c, B, Tq, maxp):
    """(sequences read back at once, bytes of partial records): 0 of them, not cut; None: streamed."""
    ws = W.wm_q4_rows_attn_workspace(c, B, Tq, maxp)
    one = one_sequence(c, maxp)
    if ws < one:
        return None
    for g in range(min(B, max(1, ROWS // one)), 0, -1):
        rest = ws - 2 * up(g * one // 2) - up(4 * g * maxp) - up(4 * g) - up(4 * g * Tq)
        # the rows are most of it, and their records a multiple of one part's
        if rest >= 0:
            part = 4 * c.Hkv * Tq * (c.Hq // c.Hkv) * (c.d + 8)
            if rest == 0 or any(up(part * n) == rest for n in range(1, max(1, rest // part) + 1)):
                return g, rest
    raise AssertionError("no such workspace")


# (B, positions, slots, query heads, kv heads, head size)
LARGE = [(1, 4096, 65536, 64, 8, 128), (1, 8034, 65536, 256, 32, 128), (22, 3280, 62112, 24, 3, 128),
         (32, 300, 8192, 32, 4, 128), (8, 4096, 65536, 16, 2, 128), (1, 509, 8701, 32, 8, 128), (64, 64, 2048, 32, 8, 128),
         (1, 128, 1 << 20, 32, 32, 128), (4096, 1000, 512, 8, 8, 64), (1, 1 << 20, 1 << 20, 8, 1, 64)]


def draw(rng):
    Hkv, d = int(rng.choice([1, 2, 3, 4, 8, 12, 32])), int(rng.choice([64, 96, 128]))
    log = lambda lo, hi: int(np.exp(rng.uniform(np.log(lo), np.log(hi))))  # noqa: E731
    return log(1, 600), log(2, 20000), log(16, 200000), Hkv * int(rng.choice([1, 2, 4, 8])), Hkv, d


def test_workspace_of_many_rows_stays_within_its_bound():
    rng = np.random.default_rng(0)
    tiles = 0
    for B, Tq, slots, Hq, Hkv, d in LARGE + [draw(rng) for _ in range(600)]:
        page = 16
        c, maxp = config(Hq, Hkv, d, page), -(-slots // page)
        ws, one = W.wm_q4_rows_attn_workspace(c, B, Tq, maxp), one_sequence(c, maxp)
        assert ws > 0 and ws % 256 == 0
        if ws < one:
            continue
        tiles += 1
        g = min(B, max(1, ROWS // one))
        assert ws <= max(ROWS, one) + RECORDS + 4 * g * (maxp + 1 + Tq) + 6 * 256, (B, Tq, slots, Hq, Hkv, d)
    assert tiles > 100


def run(x, pos):
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    q = x.queries(x.B, pos.shape[1])
    out = torch.full((x.B, pos.shape[1], x.Hq, x.d), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_rows_attn(0, q.cuda(), torch.from_numpy(pos).cuda(), q4, table, out)
    assert s.read_status() == 0
    return q, to_f64(out)


def test_cut_rows_of_more_sequences_than_their_records_fit():
    x = Q.Q4([300, 411, 300, 333, 300, 517, 300, 340] * 2, Hkv=4, G=8, d=64, page=16, k=1, max_pages=1600)
    g, records = form(x.session_cfg(), x.B, 300, x.max_pages)
    part = 4 * x.Hkv * 300 * x.G * (x.d + 8)
    assert g == x.B and 0 < records <= RECORDS and round(records / part) % x.B != 0
    pos = np.stack([np.arange(n - 300, n) for n in x.lens]).astype(np.int32)
    q, got = run(x, pos)
    check_rows(x, q, pos, got)


# (group size, positions, lengths, kv heads, head size, page, pages of a row of the table, whether cut)
FORMS = [(2, 128, [256] * 38, 8, 64, 16, 16, False), (1, 128, [256] * 38, 8, 64, 16, 16, False),
         (1, 257, [600] * 10, 8, 64, 8, 75, False), (4, 130, [200, 190, 130, 140] * 3, 6, 96, 32, 7, False),
         (8, 40, [60] * 40, 2, 128, 64, 3, False),
         (4, 300, [400], 2, 128, 16, 1024, True), (8, 16, [70, 90], 8, 64, 32, 4096, True), (2, 200, [211, 200], 3, 96, 64, 1024, True)]


def case(G, Tq, lens, Hkv, d, page, maxp, cut, seed=3):
    x = Q.Q4(lens, Hkv=Hkv, G=G, d=d, page=page, k=1, max_pages=maxp, seed=seed)
    at = form(x.session_cfg(), x.B, Tq, maxp)
    assert at is not None and (at[1] > 0) == cut
    return x


def check_rows(x, q, pos, got, visible=None):
    """Every element within what the arithmetic may move it: scores as in tests/_q4.py, weights rounded to 11
    bits (2^-11; below 2^-22 of the largest to a multiple of 2^-32 of it), sums of steps cut by 17 *
    2^-23, the result rounded by 2^-8 of itself."""
    T = int(pos.max()) + 1
    for b in range(x.B):
        n = max(int(pos[b].max()) + 1, 1)
        ts = np.arange(n)
        see = ts[None] <= pos[b][:, None]
        if visible is not None:
            see &= visible[b][:n]
        for h in range(x.Hkv):
            K, V = (np.where(see.any(0)[:, None], x.rows(p, 0, b, h, ts), 0) for p in (x.kd, x.vd))
            for g in range(x.G):
                y = to_f64(q[b, :, h * x.G + g])
                s = np.where(see, y @ K.T / np.sqrt(x.d), -np.inf)
                p = np.where(see, np.exp(s - np.maximum(s.max(1, keepdims=True), -1e300)), 0)
                p /= np.maximum(p.sum(1, keepdims=True), 1e-300)
                want = p @ V
                ds = (110 + x.d) * 2.0 ** -24 * (np.abs(y) @ np.abs(K).T).max(1, keepdims=True) / np.sqrt(x.d)
                rel = 2 * ds + 2.0 ** -11 + T / 16 * 17 * 2.0 ** -23 + 64 * 2.0 ** -24
                tol = rel * (p @ np.abs(V)) + n * 2.0 ** -32 * np.abs(V).max() + 2.0 ** -8 * np.abs(want)
                over = (np.abs(got[b, :, h * x.G + g] - want) - tol).max()
                assert over <= 0, (b, h, g, over)


@pytest.mark.parametrize("order", ["last", "any", "few"])
@pytest.mark.parametrize("f", FORMS)
def test_both_forms_element_by_element(f, order):
    """few: rows that see so few slots that a weight's own rounding shows."""
    x, Tq = case(*f), f[1]
    rng = np.random.default_rng(2)
    pos = np.stack([np.arange(n - Tq, n) if order == "last" else rng.integers(0, n if order == "any" else 6, Tq)
                    for n in x.lens]).astype(np.int32)
    q, got = run(x, pos)
    check_rows(x, q, pos, got)


@pytest.mark.parametrize("f", FORMS)
def test_both_forms_leave_out_what_is_bad(f):
    """Pages and positions out of range, positions in no order, sequences of which no row sees a slot."""
    x, Tq = case(*f), f[1]
    rng = np.random.default_rng(4)
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    pos = np.stack([rng.integers(0, n, Tq) for n in x.lens]).astype(np.int32)
    visible = np.ones((x.B, x.T), dtype=bool)
    for b in range(0, x.B, 2):
        page = int(rng.integers(0, -(-int(x.lens[b]) // x.P)))
        table[b, page] = (-1, x.q4_pages, -2 ** 31, 2 ** 31 - 1)[b // 2 % 4]
        visible[b, page * x.P:(page + 1) * x.P] = False
    for b in range(x.B):
        pos[b, rng.integers(0, Tq, 3)] = (-1, x.T, -2 ** 31)
    if x.B > 2:
        pos[2] = -5
    q = x.queries(x.B, Tq)
    out = torch.full((x.B, Tq, x.Hq, x.d), float("nan"), dtype=x.tdt, device="cuda")
    s.q4_rows_attn(0, q.cuda(), torch.from_numpy(pos).cuda(), q4, table, out)
    assert s.read_status() == W.WM_ERR_BOUNDS
    got = to_f64(out)
    bad = (pos < 0) | (pos >= x.T)
    assert (got[bad] == 0).all()
    check_rows(x, q, np.where(bad, -1, pos), got, visible)


def test_whole_ranges_in_several_groups():
    rng = np.random.default_rng(6)
    x = Q.Q4(rng.integers(128, 200, 70).tolist(), Hkv=8, G=2, d=64, page=16, k=1, max_pages=256, seed=5)
    g, records = form(x.session_cfg(), x.B, 128, x.max_pages)
    assert g < x.B and records == 0
    pos = np.stack([np.arange(n - 128, n) for n in x.lens]).astype(np.int32)
    q, got = run(x, pos)
    check_rows(x, q, pos, got)


@pytest.mark.parametrize("f", [FORMS[0], FORMS[5], FORMS[6]])
def test_scores_of_any_size_in_both_forms(f):
    """Scores so large that a reference is rounded: the largest one takes all, whichever step it comes in."""
    x, Tq = case(*f), f[1]
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    pos = np.stack([np.arange(n - Tq, n) for n in x.lens]).astype(np.int32)
    q = x.queries(x.B, Tq)
    best = np.full((x.B, Tq, x.Hq, x.d), np.nan)
    for b in range(x.B):
        for hq in range(x.Hq):
            K, V = (x.rows(p, 0, b, hq // x.G, np.arange(x.lens[b])) for p in (x.kd, x.vd))
            z = to_f64(q[b, :, hq]) @ K.T
            z[np.arange(len(K))[None] > pos[b][:, None]] = -np.inf
            top = np.sort(z, 1)
            clear = top[:, -1] - top[:, -2] > 0.05  # (2^18 of it are 1000 and more: nothing is left of the others)
            best[b, clear, hq] = V[z.argmax(1)][clear]
    clear = ~np.isnan(best)
    assert clear.mean() > 0.5
    for e in range(18, 42):
        out = torch.full(q.shape, float("nan"), dtype=x.tdt, device="cuda")
        s.q4_rows_attn(0, (q * 2.0 ** e).cuda(), torch.from_numpy(pos).cuda(), q4, table, out)
        got = to_f64(out)
        # (its weight in fp16 against the sum of the unrounded one, and the result in bf16)
        assert (np.abs(got - best)[clear] <= (2.0 ** -11 + 2.0 ** -8 + 2.0 ** -16) * np.abs(best)[clear]).all(), e
        assert np.isfinite(got).all(), e
    assert s.read_status() == 0


@pytest.mark.parametrize("f", [FORMS[0], FORMS[5], FORMS[6]])
def test_rows_of_nan_queries_are_nan_in_both_forms(f):
    x, Tq = case(*f), f[1]
    pos = np.stack([np.arange(n - Tq, n) for n in x.lens]).astype(np.int32)
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    q = x.queries(x.B, Tq)
    q[0, 3, 1, 5], q[-1, Tq - 1, 0, 7] = float("nan"), float("inf")
    out = torch.zeros(q.shape, dtype=x.tdt, device="cuda")
    s.q4_rows_attn(0, q.cuda(), torch.from_numpy(pos).cuda(), q4, table, out)
    assert s.read_status() == 0
    nan = np.isnan(to_f64(out))
    assert nan[0, 3, 1].all() and nan[-1, Tq - 1, 0].all() and nan.sum() == 2 * x.d


@pytest.mark.parametrize("B,Tq,slots,Hq,Hkv,d,want", [
    (1, 32, 8192, 32, 8, 128, "stream"), (1, 64, 8192, 32, 8, 128, "cut"), (1, 256, 8192, 32, 8, 128, "cut"),
    (8, 16, 32768, 32, 8, 128, "stream"), (8, 64, 32768, 32, 8, 128, "cut"), (32, 16, 1024, 32, 8, 128, "stream"),
    (32, 32, 1024, 32, 8, 128, "whole"), (16, 256, 4096, 32, 8, 128, "whole"), (32, 300, 8192, 32, 4, 128, "whole"),
    (1, 64, 131072, 32, 8, 128, "cut"), (4, 200, 8192, 6, 3, 96, "stream"), (32, 32, 131072, 32, 8, 128, "stream")])
def test_calls_take_the_form_that_measured_fastest(B, Tq, slots, Hq, Hkv, d, want):
    """By 10% and more (us: streamed, whole, cut): 28 118 33; 47 119 35; 157 122 50; 296 1407 531; 1059 1064 557;
    63 118 320; 116 97 381; 1141 293 515; 4841 1478 1717; 582 1779 225; 68 159 85; the last one's estimates are
    close, and 1024 slots in such a table take 116 and 1028."""
    at = form(config(Hq, Hkv, d, 16), B, Tq, slots // 16)
    assert ("stream" if at is None else "cut" if at[1] else "whole") == want


@pytest.mark.parametrize("f", [FORMS[1], FORMS[5], FORMS[6]])
def test_large_scores_of_few_slots_of_either_sign(f):
    """Rows that see one to three slots, so that the largest score is as often negative; ties at every size."""
    x, Tq = case(*f), f[1]
    s, q4 = x.session(), x.q4()
    table, _ = x.q4_dev()
    pos = np.random.default_rng(8).integers(0, 3, (x.B, Tq)).astype(np.int32)
    q = x.queries(x.B, Tq)
    best, clear = np.empty((x.B, Tq, x.Hq, x.d)), np.empty((x.B, Tq, x.Hq), dtype=bool)
    for b in range(x.B):
        for hq in range(x.Hq):
            K, V = (x.rows(p, 0, b, hq // x.G, np.arange(3)) for p in (x.kd, x.vd))
            z = np.where(np.arange(3)[None] <= pos[b][:, None], to_f64(q[b, :, hq]) @ K.T, -np.inf)
            top = np.sort(z, 1)
            clear[b, :, hq] = top[:, -1] - top[:, -2] > 0.05
            best[b, :, hq] = V[z.argmax(1)]
    assert clear.mean() > 0.5 and (pos == 0).any()
    for e in range(18, 100, 3):
        out = torch.full(q.shape, float("nan"), dtype=x.tdt, device="cuda")
        s.q4_rows_attn(0, (q * 2.0 ** e).cuda(), torch.from_numpy(pos).cuda(), q4, table, out)
        got = to_f64(out)
        assert (np.abs(got - best) <= (2.0 ** -11 + 2.0 ** -8 + 2.0 ** -16) * np.abs(best))[clear].all(), e
        assert np.isfinite(got).all(), e
    assert s.read_status() == 0
