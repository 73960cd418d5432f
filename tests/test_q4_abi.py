"""Host-side refusals of the 4-bit cache's entry points (nothing launched), and its numpy model."""
import numpy as np
import pytest

from paper_2608_18486_gb300 import _lib as W
from tests import _q4 as Q
from tests.test_abi import cfg, host_refusals_only

FAKE = 1 << 41
INV, UNS, OK = W.WM_ERR_INVALID_ARG, W.WM_ERR_UNSUPPORTED, W.WM_OK


def parts(**kw):
    c = cfg(**kw)
    return (c, W.wm_cache_alloc(c, 1 << 40, W.wm_cache_bytes(c, 4), 4),
            W.wm_q4_cache_alloc(c, 1 << 42, W.wm_q4_cache_bytes(c, 4), 4))


def write(c, cache, q4, table=FAKE, q4_table=FAKE, first=FAKE, last=FAKE, span=3, B=2, maxp=4):
    return W.wm_q4_write(c, cache, table, q4, q4_table, first, last, span, B, maxp, None, None)


def read(c, cache, q4, table=FAKE, q4_table=FAKE, first=FAKE, last=FAKE, span=3, B=2, maxp=4):
    return W.wm_q4_read(c, q4, q4_table, cache, table, first, last, span, B, maxp, None, None)


def decode(c, cache, q4, layer=0, q=FAKE, table=FAKE, lens=FAKE, B=2, maxp=4, out=FAKE, ws=FAKE, n=None):
    n = W.wm_q4_decode_attn_workspace(c, 2, 4) if n is None else n
    return W.wm_q4_decode_attn(c, q4, layer, q, table, lens, B, maxp, out, ws, n, None, None)


def rows(c, cache, q4, layer=0, q=FAKE, pos=FAKE, table=FAKE, B=2, Tq=3, maxp=4, out=FAKE, ws=FAKE, n=None):
    n = W.wm_q4_rows_attn_workspace(c, 2, 3, 4) if n is None else n
    return W.wm_q4_rows_attn(c, q4, layer, q, pos, table, B, Tq, maxp, out, ws, n, None, None)


def mix(c, cache, q4, h=FAKE, table=FAKE, slot=FAKE, pos=None, B=2, maxp=4, ws=FAKE, n=None, w=FAKE, g=FAKE):
    n = W.wm_q4_kv_mix_workspace(c, 2) if n is None else n
    weights = W.mix_weights((g, g), (w, w), (FAKE, FAKE), (FAKE, FAKE), (FAKE, FAKE), FAKE)
    return W.wm_q4_kv_mix(c, q4, weights, h, table, slot, pos, B, maxp, ws, n, None, None)


CALLS = {"write": write, "read": read, "decode": decode, "rows": rows, "mix": mix}


@host_refusals_only
@pytest.mark.parametrize("name,bad", [
    *((n, b) for n in ("write", "read") for b in (dict(table=None), dict(q4_table=None), dict(first=None), dict(last=None),
                                                   dict(span=-1), dict(B=-1), dict(maxp=0), dict(maxp=1 << 27))),
    ("decode", dict(layer=-1)), ("decode", dict(layer=32)), ("decode", dict(q=None)), ("decode", dict(q=FAKE + 8)),
    ("decode", dict(out=None)), ("decode", dict(out=FAKE + 2)), ("decode", dict(table=None)), ("decode", dict(lens=None)),
    ("decode", dict(ws=None)), ("decode", dict(ws=FAKE + 16)), ("decode", dict(n=0)), ("decode", dict(B=-1)),
    ("decode", dict(maxp=0)), ("rows", dict(Tq=-1)), ("rows", dict(pos=None)), ("rows", dict(layer=32)),
    ("mix", dict(h=None)), ("mix", dict(h=FAKE + 8)), ("mix", dict(table=None)), ("mix", dict(slot=None)),
    ("mix", dict(ws=None)), ("mix", dict(ws=FAKE + 128)), ("mix", dict(n=256)), ("mix", dict(w=None)), ("mix", dict(g=FAKE + 4)),
    ("mix", dict(B=-1)), ("mix", dict(maxp=0)),
    ("rows", dict(q=FAKE + 4)), ("rows", dict(out=None)), ("rows", dict(ws=None)), ("rows", dict(n=0))])
def test_bad_arguments_are_refused(name, bad):
    assert CALLS[name](*parts(), **bad) == INV


@host_refusals_only
@pytest.mark.parametrize("name", list(CALLS))
def test_configs_and_caches_are_checked(name):
    c, cache, q4 = parts()
    assert CALLS[name](cfg(k=8), cache, q4) == INV  # caches of another config
    assert CALLS[name](cfg(d=80), cache, q4) == UNS
    assert CALLS[name](c, cache, q4, B=0) == OK
    for field, value in (("pool", None), ("pool", (1 << 42) + 8), ("num_pages", 0), ("page_size", 8), ("Hkv", 1), ("d", 64)):
        other = W.wm_q4_cache_alloc(c, 1 << 42, W.wm_q4_cache_bytes(c, 4), 4)
        if getattr(other, field) == value:
            continue
        setattr(other, field, value)
        assert CALLS[name](c, cache, other) == INV, field
    q4.num_pages = 1 << 30
    assert CALLS[name](c, cache, q4) == UNS


@host_refusals_only
def test_nothing_to_do_and_too_much():
    p = parts()
    assert write(*p, span=0) == OK and read(*p, span=0) == OK and rows(*p, Tq=0) == OK
    assert decode(*p, B=4097) == UNS and rows(*p, B=4097) == UNS and rows(*p, B=4096, Tq=1 << 20) == UNS
    assert write(*p, B=4096, span=1 << 24, maxp=1 << 20) == UNS
    assert mix(*p, B=65536, n=1 << 50) == UNS and W.wm_q4_kv_mix_workspace(p[0], -1) == 0
    assert W.wm_q4_kv_mix_workspace(p[0], 2) > W.wm_kv_mix_workspace(p[0], 2)


def test_sizes():
    for d in (64, 96, 128):
        for page in (1, 2, 4, 8, 16, 32, 4096):
            c = cfg(d=d, page_size=page)
            n, tile = Q.tile_shape(page, d)
            assert tile % 16 == 0
            need = c.k * 5 * c.Hkv * (page // n) * tile
            assert W.wm_q4_cache_bytes(c, 5) == (need + 255) // 256 * 256
    assert W.wm_q4_cache_bytes(c, 0) == 0 and W.wm_q4_cache_bytes(cfg(d=80), 4) == 0
    assert W.wm_q4_decode_attn_workspace(c, 2, 0) == 0 and W.wm_q4_decode_attn_workspace(c, -1, 4) == 0
    assert W.wm_q4_rows_attn_workspace(c, 2, -1, 4) == 0
    for b in (1, 3, 64):
        assert 0 < W.wm_q4_decode_attn_workspace(c, b, 8192) % 256 == 0 or W.wm_q4_decode_attn_workspace(c, b, 8192) > 0
    for bad in (dict(dev_buf=None), dict(dev_buf=(1 << 40) + 16), dict(nbytes=100), dict(num_pages=0)):
        args = dict(dev_buf=1 << 40, nbytes=1 << 50, num_pages=4, **{}) | bad
        with pytest.raises(W.WMError):
            W.wm_q4_cache_alloc(c, args["dev_buf"], args["nbytes"], args["num_pages"])


def test_model_rounds_as_defined():
    """Codes and scales of the numpy model against the nearest of all, one by one."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((64, 16)) * np.exp(3 * rng.standard_normal((64, 1)))
    code, byte = Q.quantise(x)
    s = Q.SCALES[byte[:, 0]]
    want = np.abs(6 * Q.SCALES[None] - np.abs(x).max(1)[:, None]).argmin(1)
    assert np.array_equal(byte[:, 0], want)
    assert np.array_equal(code & 7, np.abs(np.abs(x)[..., None] - Q.MAGS * s[:, None, None]).argmin(-1))
    assert np.array_equal(Q.quantise(Q.values(code, byte))[0] & 7, code & 7)
    err = Q.values(code, byte) - x
    assert np.sqrt((err ** 2).mean(1) / (x ** 2).mean(1)).max() < 0.25
    y = np.zeros((1, 16))
    y[0, :8] = [6, -.25, .75, 1.25, -1.75, 2.5, 3.5, -5]  # ties
    assert (Q.quantise(y)[0][0, :8] == [7, 8, 2, 2, 12, 4, 6, 14]).all() and Q.quantise(y)[1][0, 0] == 15 * 8
    y[0, 3] = np.nan
    assert Q.quantise(y)[1][0, 0] == 255 and (Q.quantise(y)[0] == 0).all()
