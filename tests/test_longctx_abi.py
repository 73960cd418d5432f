"""Host-side refusals of the long-context entry points (nothing launched)."""
import pytest

from paper_2608_18486_gb300 import _lib as W
from tests.test_abi import cfg, host_refusals_only

FAKE = 1 << 41
INV, UNS, OK = W.WM_ERR_INVALID_ARG, W.WM_ERR_UNSUPPORTED, W.WM_OK


def parts(**kw):
    c = cfg(**kw)
    return c, W.wm_cache_alloc(c, 1 << 40, W.wm_cache_bytes(c, 4), 4)


def window(c, cache, layer=0, q=FAKE, table=FAKE, lens=FAKE, sinks=1, window=8, B=2, maxp=4, out=FAKE):
    return W.wm_window_attn(c, cache, layer, q, table, lens, sinks, window, B, maxp, out, None, None)


def prefill(c, cache, layer=0, q=FAKE, pos=FAKE, table=FAKE, sinks=1, window=8, B=2, Tq=3, maxp=4, out=FAKE):
    return W.wm_window_prefill_attn(c, cache, layer, q, pos, table, sinks, window, B, Tq, maxp, out, None, None)


def prefix(c, cache, layer=0, q=FAKE, table=FAKE, lens=FAKE, shared=1, B=2, maxp=4, out=FAKE, ws=FAKE, n=None):
    n = W.wm_prefix_attn_workspace(c, 2, 4, 1) if n is None else n
    return W.wm_prefix_attn(c, cache, layer, q, table, lens, shared, B, maxp, out, ws, n, None, None)


def mass(c, cache, layer=0, q=FAKE, table=FAKE, lens=FAKE, mass=FAKE, B=2, maxp=4, out=FAKE, ws=FAKE, n=None):
    n = W.wm_decode_attn_mass_workspace(c, 2, 4) if n is None else n
    return W.wm_decode_attn_mass(c, cache, layer, q, table, lens, mass, B, maxp, out, ws, n, None, None)


def evict(c, cache, mass=FAKE, out=FAKE, table=FAKE, lens=FAKE, budget=8, sinks=1, recent=2, B=2, maxp=4, kept=FAKE,
          new=FAKE + 64):
    return W.wm_cache_evict(c, cache, mass, out, table, lens, budget, sinks, recent, B, maxp, kept, new, None, None)


CALLS = {"window": window, "prefill": prefill, "prefix": prefix, "mass": mass, "evict": evict}


@host_refusals_only
@pytest.mark.parametrize("name,bad", [
    ("window", dict(layer=-1)), ("window", dict(layer=32)), ("window", dict(sinks=-1)), ("window", dict(window=-1)),
    ("window", dict(q=None)), ("window", dict(table=None)), ("window", dict(lens=None)), ("window", dict(out=None)),
    ("window", dict(q=FAKE + 8)), ("window", dict(out=FAKE + 2)), ("window", dict(B=-1)), ("window", dict(maxp=0)),
    ("window", dict(maxp=1 << 27)),
    ("prefill", dict(Tq=-1)), ("prefill", dict(pos=None)), ("prefill", dict(sinks=-2)), ("prefill", dict(window=-2)),
    ("prefill", dict(layer=32)), ("prefill", dict(q=FAKE + 4)), ("prefill", dict(out=None)),
    ("prefix", dict(shared=-1)), ("prefix", dict(shared=5)), ("prefix", dict(ws=None)), ("prefix", dict(ws=FAKE + 128)),
    ("prefix", dict(n=0)), ("prefix", dict(lens=None)), ("prefix", dict(out=FAKE + 2)), ("prefix", dict(layer=40)),
    ("mass", dict(mass=None)), ("mass", dict(mass=FAKE + 2)), ("mass", dict(n=64)), ("mass", dict(ws=None)),
    ("mass", dict(q=None)), ("mass", dict(B=-3)),
    ("evict", dict(budget=0)), ("evict", dict(sinks=-1)), ("evict", dict(recent=-1)), ("evict", dict(sinks=7)),
    ("evict", dict(budget=65)), ("evict", dict(mass=None)), ("evict", dict(out=None)), ("evict", dict(kept=None)),
    ("evict", dict(new=None)), ("evict", dict(new=FAKE)), ("evict", dict(table=None)), ("evict", dict(lens=None)),
    ("evict", dict(mass=FAKE + 1)), ("evict", dict(B=-1))])
def test_bad_arguments_are_refused(name, bad):
    c, cache = parts()
    assert CALLS[name](c, cache, **bad) == INV


@host_refusals_only
@pytest.mark.parametrize("name", list(CALLS))
def test_configs_and_caches_are_checked(name):
    c, cache = parts()
    other = cfg(k=8)
    assert CALLS[name](other, cache) == INV  # a cache of another config
    bad = cfg(d=80)
    assert CALLS[name](bad, cache) == UNS
    assert CALLS[name](c, cache, B=0) == OK  # nothing to do


@host_refusals_only
def test_batches_past_the_grid_are_refused():
    c, cache = parts()
    assert window(c, cache, B=4097) == UNS
    assert prefix(c, cache, B=4097) == UNS
    assert mass(c, cache, B=4097) == UNS
    assert prefill(c, cache, B=1 << 14, Tq=1 << 14) == UNS
    assert prefill(c, cache, Tq=0) == OK


@host_refusals_only
def test_pool_positions_are_required():
    c, cache = parts()
    w = W.mix_weights((FAKE, FAKE), (FAKE, FAKE), (FAKE, FAKE), (FAKE, FAKE), (FAKE, FAKE), FAKE)
    ws = W.wm_kv_mix_workspace(c, 2)
    assert W.wm_kv_mix_at(c, cache, w, FAKE, FAKE, FAKE, None, 2, 4, FAKE, ws, None, None) == INV
    assert W.wm_kv_mix_at(c, cache, w, None, None, None, None, 0, 4, None, 0, None, None) == OK


def test_workspace_queries():
    c = cfg()
    assert W.wm_prefix_attn_workspace(c, 2, 4, 5) == 0 and W.wm_prefix_attn_workspace(c, 2, 4, -1) == 0
    assert W.wm_decode_attn_mass_workspace(c, 2, 0) == 0 and W.wm_decode_attn_mass_workspace(c, -1, 4) == 0
    for b in (1, 3, 64):
        assert W.wm_prefix_attn_workspace(c, b, 40, 7) % 256 == 0
        # short contexts keep their scores on chip
        assert W.wm_decode_attn_mass_workspace(c, b, 40) % 256 == 0 < W.wm_decode_attn_mass_workspace(c, b, 40)
        # long ones: a score per query head and slot, and at least one record per unit
        assert W.wm_decode_attn_mass_workspace(c, b, 8192) >= 4 * b * (c.Hq * 8192 * c.page_size + c.Hkv * (c.d + 2))
