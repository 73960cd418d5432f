"""Many rows over a 4-bit cache: the size of the workspace, and the forms in which they run on the
tensor cores (whole KV ranges per item, or cut ones with partial records)."""
import numpy as np
import pytest
import torch

from paper_2608_18486_gb300 import _lib as W
from tests import _q4 as Q
from tests._longctx import to_f64
from tests.test_q4_gpu import check_many

pytestmark = pytest.mark.gpu

ROWS, RECORDS = 2 ** 29, 2 ** 27  # bytes of rows read back at once (or one sequence's), of partial records


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
    x = Q.Q4([300, 411, 300, 333, 300, 517, 300, 340], Hkv=4, G=8, d=64, page=16, k=1, max_pages=1600)
    g, records = form(x.session_cfg(), x.B, 300, x.max_pages)
    part = 4 * x.Hkv * 300 * x.G * (x.d + 8)
    assert g == x.B and 0 < records <= RECORDS and round(records / part) % x.B != 0
    pos = np.stack([np.arange(n - 300, n) for n in x.lens]).astype(np.int32)
    q, got = run(x, pos)
    check_many(x, q, pos, got)
