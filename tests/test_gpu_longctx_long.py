"""Contexts past what the on-chip forms hold: summed weights through the workspace, evictions whose
sums no cluster holds at once."""
import numpy as np
import pytest
import torch

from paper_2608_18486_gb300 import _lib as W
from paper_2608_18486_gb300.session import DecodeSession
from tests._longctx import Cache, to_f64

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ summed weights
def check_mass(c, mass, calls=2, layer=1):
    """Outputs and every sum against 64 bits.  Each weight is off by a factor e^(2 ds) and by
    roundings: those of its exponential and scale, and of the row's sum, which a lane adds up in at
    most 64 terms and 64 records join (2^-24 each, relative); a sum rounds once per call."""
    s, (table, dl) = c.session(), c.dev()
    # the records and a score per query head and slot go through the workspace
    assert W.wm_decode_attn_mass_workspace(s.cfg, c.B, c.max_pages) > 4 * c.B * c.Hq * c.T
    start = to_f64(mass)
    want, tol = start.copy(), np.zeros_like(start)
    for _ in range(calls):
        q = c.queries(c.B)
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        s.decode_attn_mass(layer, q.cuda(), table, dl, mass, out)
        qd, got = q.double().numpy(), to_f64(out)
        for b, n in enumerate(c.lens):
            for hq in range(c.Hq):
                o, p, ds, vmax = c.attend(layer, b, hq, qd[b, hq], range(int(n)))
                t = 2 * ds + 160 * 2.0 ** -24
                assert np.abs(got[b, hq] - o).max() <= (t + (2.0 ** -8 if c.dtype == "bf16" else 0.0)) * vmax
                want[layer, b, hq // c.G, :n] += p
                tol[layer, b, hq // c.G, :n] += p * t
        tol[layer] += 2.0 ** -23 * want[layer]
    assert s.read_status() == 0
    assert (np.abs(to_f64(mass) - want) <= tol).all()
    still = np.ones(start.shape, bool)  # other channels, and slots behind a sequence's end
    for b, n in enumerate(c.lens):
        still[layer, b, :, :n] = False
    assert np.array_equal(to_f64(mass)[still], start[still])


def start_mass(c):
    return torch.from_numpy(np.abs(c.rng.standard_normal((c.k, c.B, c.Hkv, c.T))).astype(np.float32)).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_long_mass_matches_reference(dtype, G, d):
    c = Cache([6001, 0, 1, 4097, 7100], Hkv=2, G=G, d=d, page=64 if d == 64 else 16, dtype=dtype, k=2, seed=d + G,
              max_pages=20000 // (64 if d == 64 else 16))
    check_mass(c, start_mass(c))


@pytest.mark.parametrize("dtype,G", [("bf16", 2), ("f32", 4)])
def test_long_mass_of_slots_that_are_no_multiple_of_four(dtype, G):
    c = Cache([5000, 3, 17002], Hkv=1, G=G, d=64, page=1, dtype=dtype, k=2, seed=G, max_pages=17003)
    check_mass(c, start_mass(c))


def test_long_mass_that_starts_between_16_byte_boundaries():
    c = Cache([5000, 16999], Hkv=1, G=2, d=64, page=8, k=2, seed=1, max_pages=2200)
    wide = torch.empty(2 * 2 * c.T + 1, device="cuda")
    mass = wide[1:].view(2, 2, 1, c.T)
    mass.copy_(start_mass(c))
    check_mass(c, mass)


def test_long_mass_of_a_bad_page_and_a_bad_length():
    c = Cache([6000, 6000], Hkv=1, G=2, d=64, page=16, k=1, seed=3, max_pages=1250)
    s, (table, dl) = c.session(), c.dev()
    table[0, 100], dl[1] = -1, c.T + 1
    q = c.queries(2)
    mass, out = torch.zeros((1, 2, 1, c.T), device="cuda"), torch.full((2, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    s.decode_attn_mass(0, q.cuda(), table, dl, mass, out)
    assert s.read_status() == W.WM_ERR_BOUNDS
    got = to_f64(mass)[0, :, 0]
    assert (got[0, 1600:1616] == 0).all() and abs(got[0].sum() - 2) < 1e-4 and (got[1] == 0).all()
    assert (out[1] == 0).all()


# ------------------------------------------------------------------ eviction
def cluster_of(units, budget, row_bytes):
    """CTAs per unit of a launch (the rule that the library documents beside it)."""
    sms, c = torch.cuda.get_device_properties(0).multi_processor_count, 1
    while c < 8 and units * c * 2 <= 2 * sms and c * 512 * 2 < budget * row_bytes // 16:
        c *= 2
    return c


def sums(rng, kind, shape):
    m = np.abs(rng.standard_normal(shape, dtype=np.float32))
    if kind == "equal":
        m[:] = 0.3
    elif kind == "few":  # ties of many slots, on both sides of every tile's end
        m = rng.integers(0, 3, shape) * np.float32(0.25)
    elif kind == "close":  # neighbours of one value
        m = np.float32(0.5) * (1 + rng.integers(0, 40, shape) * 2.0 ** -23)
    elif kind == "wide":  # every exponent, both signs, what is no number
        m = np.exp2(rng.uniform(-140, 120, shape)) * rng.choice([-1.0, 1.0], shape)
        m[..., 5::19], m[..., 7::23], m[..., 9::29] = np.inf, -np.inf, np.nan
    elif kind == "step":  # what stays lies in the last tile, and a tie runs across the tile before
        m = np.broadcast_to(np.where(np.arange(shape[-1]) > 0.8 * shape[-1], 2.0, 1.0), shape)
    return np.ascontiguousarray(m, dtype=np.float32)


# CTAs that hold 8192 sums each: several tiles per CTA where every unit has one, and units past what
# eight of them hold; slots that are no multiple of four
@pytest.mark.parametrize("B,Hkv,n,page,extra", [(10, 16, 9001, 16, 0), (5, 32, 20003, 64, 3), (160, 1, 8193, 1, 2),
                                                (1, 1, 70001, 64, 0), (1, 2, 131072, 64, 1), (1, 1, 66001, 1, 2)])
@pytest.mark.parametrize("kind", ["random", "few", "equal", "close", "wide", "step"])
@pytest.mark.parametrize("alias", [False, True])
def test_evict_of_sums_that_no_cluster_holds(B, Hkv, n, page, extra, kind, alias):
    rng = np.random.default_rng(n)
    d, lens = 64, np.array([n - 5 * (b % 7) if n > 8200 else n for b in range(B)], dtype=np.int32)
    budget, sinks, recent = n * 3 // 7, 5, n // 9
    assert n > 8192 * cluster_of(B * Hkv, budget, 2 * d)
    per = -(-n // page)
    maxp, pages = per + extra, B * per + 2
    T = maxp * page
    assert T % 4 == 0 or page == 1
    order = rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)
    table = np.full((B, maxp), -1, dtype=np.int32)
    table[:, :per] = order
    cfg = W.make_config(1, 1, 64, Hkv, Hkv, d, 1, page, "bf16", [0])
    s = DecodeSession(cfg, B, pages, maxp)
    gen = torch.Generator(device="cuda").manual_seed(n)
    s.k_pool.normal_(generator=gen)
    s.v_pool.normal_(generator=gen)
    was = s.k_pool.clone(), s.v_pool.clone()
    mass = sums(rng, kind, (1, B, Hkv, T))
    m = torch.from_numpy(mass).cuda()
    mo = m if alias else torch.full_like(m, 9.0)
    kept = torch.full((1, B, Hkv, budget), 77, dtype=torch.int32, device="cuda")
    dl = torch.from_numpy(lens).cuda()
    nl = torch.empty_like(dl)
    s.evict(m, torch.from_numpy(table).cuda(), dl, mo, kept, nl, budget=budget, sinks=sinks, recent=recent)
    assert s.read_status() == 0 and (nl == budget).all()
    kept, mo = kept.cpu().numpy(), mo.cpu().numpy()
    for b in range(B):
        end = int(lens[b])
        for h in range(Hkv):
            x = mass[0, b, h]
            mid = x[sinks:end - recent]
            nan = np.isnan(mid)
            first = np.lexsort((np.arange(len(mid)), -np.where(nan, -np.inf, mid).astype(np.float64), nan))
            want = np.sort(np.concatenate([np.arange(sinks), sinks + first[:budget - sinks - recent],
                                           np.arange(end - recent, end)]))
            assert np.array_equal(kept[0, b, h], want), (b, h)
            assert np.array_equal(mo[0, b, h, :budget], x[want], equal_nan=True)
            assert (mo[0, b, h, budget:] == 0).all()
    # every row that stayed is where its place in the list says, every other one is as it was
    to = torch.arange(budget, device="cuda")
    at, h = torch.from_numpy(table).cuda().long(), torch.arange(Hkv, device="cuda")[:, None]
    k = torch.from_numpy(kept[0]).cuda().long()
    for got, old in zip((s.k_pool, s.v_pool), was):
        want = old.clone()
        for b in range(B):
            want[0, at[b, to // page][None], h, (to % page)[None]] = old[0, at[b][k[b] // page], h, k[b] % page]
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
