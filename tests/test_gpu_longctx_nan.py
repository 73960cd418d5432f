"""Query rows that hold NaN: their results are NaN, as the definition's are, and no other row's."""
import numpy as np
import pytest
import torch

from tests._longctx import Cache, check_rows, to_f64

pytestmark = pytest.mark.gpu


# lens: some sequences end inside the prefix or with it, so that nothing of theirs lies behind;
# the last is large enough for the tensor-core kernel
@pytest.mark.parametrize("dtype,d,G,Hkv,page,shared,lens", [
    ("bf16", 64, 2, 2, 16, 6, [96, 40, 130, 96, 0]), ("f32", 64, 2, 2, 16, 6, [96, 40, 130, 96, 0]),
    ("f32", 96, 8, 1, 16, 5, [80, 33, 100]),
    ("bf16", 128, 4, 4, 64, 104, [6656, 6656, 3001, 6700, 6656, 200, 6657, 6656])])
def test_prefix_rows_of_nan_queries(dtype, d, G, Hkv, page, shared, lens):
    c = Cache(lens, Hkv=Hkv, G=G, d=d, page=page, dtype=dtype, shared=shared, k=1, seed=d)
    if d == 128:  # (the rule of the kernels' choice)
        assert shared * page * Hkv * d * 4 * -(-len(lens) * G // 8) > 40 << 20
    s, (table, dl) = c.session(), c.dev()
    q = c.queries(len(lens))
    bad = {(0, 1), (1, 0), (2, c.Hq - 1)}  # (sequence, query head)
    for b, hq in bad:
        q[b, hq, 3] = float("nan")
    out = torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    s.prefix_attn(0, q.cuda(), table, dl, out, shared_pages=shared)
    assert s.read_status() == 0
    got, qd = to_f64(out), q.double().numpy()
    for b, n in enumerate(lens):
        for hq in range(c.Hq):
            if (b, hq) in bad:
                assert np.isnan(got[b, hq]).all(), (b, hq)
            elif d < 128 or hq % 5 == 0:
                want, _, ds, vmax = c.attend(0, b, hq, qd[b, hq], range(n))
                check_rows(c, got[b, hq], want, ds, vmax)


@pytest.mark.parametrize("dtype,G", [("bf16", 2), ("f32", 2), ("f32", 8)])
@pytest.mark.parametrize("n", [1, 90, 3000])
def test_window_and_mass_rows_of_nan_queries(dtype, G, n):
    c = Cache([n, n], Hkv=1, G=G, d=64, page=16, dtype=dtype, k=1, seed=n)
    s, (table, dl) = c.session(), c.dev()
    q = c.queries(2)
    q[0, G - 1, 5] = float("nan")
    out, summed = (torch.zeros(q.shape, dtype=q.dtype, device="cuda") for _ in range(2))
    mass = torch.zeros((1, 2, 1, c.T), device="cuda")
    s.window_attn(0, q.cuda(), table, dl, out, sinks=2, window=500)
    s.decode_attn_mass(0, q.cuda(), table, dl, mass, summed)
    assert s.read_status() == 0
    qd = q.double().numpy()
    for got, seen in ((to_f64(out), [t for t in range(n) if t < 2 or t >= n - 500]), (to_f64(summed), range(n))):
        for b in range(2):
            for hq in range(G):
                if (b, hq) == (0, G - 1):
                    assert np.isnan(got[b, hq]).all()
                else:
                    want, _, ds, vmax = c.attend(0, b, hq, qd[b, hq], seen)
                    check_rows(c, got[b, hq], want, ds, vmax)
    sums = to_f64(mass)[0, :, 0]
    assert np.isnan(sums[0, :n]).all() and np.isfinite(sums[1]).all() and (sums[:, n:] == 0).all()


@pytest.mark.parametrize("dtype,G", [("bf16", 1), ("bf16", 2), ("f32", 2)])
def test_prefill_rows_of_nan_queries(dtype, G):
    c = Cache([300], Hkv=1, G=G, d=64, page=16, dtype=dtype, k=1, seed=5)
    s, (table, _) = c.session(), c.dev()
    q = c.queries(1, 300)
    for r in (0, 40, 299):
        q[0, r, G - 1, 7] = float("nan")
    pos = torch.arange(300, dtype=torch.int32, device="cuda")[None].contiguous()
    out = torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    s.window_prefill_attn(0, q.cuda(), pos, table, out, sinks=3, window=70)
    assert s.read_status() == 0
    got, qd = to_f64(out), q.double().numpy()
    for r in (0, 1, 39, 40, 41, 127, 128, 298, 299):
        for hq in range(G):
            if r in (0, 40, 299) and hq == G - 1:
                assert np.isnan(got[0, r, hq]).all()
            else:
                seen = [t for t in range(r + 1) if t < 3 or t > r - 70]
                want, _, ds, vmax = c.attend(0, 0, hq, qd[0, r, hq], seen)
                check_rows(c, got[0, r, hq], want, ds, vmax)
