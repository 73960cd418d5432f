"""What DecodeSession checks before a call on a 4-bit cache (no GPU, nothing launched)."""
import pytest
import torch

from paper_2608_18486_gb300 import _lib as W
from paper_2608_18486_gb300.session import Q4Cache
from tests.test_session_cpu import Far, config, host_session

B, MAXP, TQ = 3, 4, 2


def host_q4(cfg, pages):
    n = W.wm_q4_cache_bytes(cfg, pages)
    buf = torch.zeros(n + 256, dtype=torch.uint8)
    at = -buf.data_ptr() % 256
    return Q4Cache(cfg, pages, "cpu", cache_buf=buf[at:at + n])


class Calls:
    """A session, a 4-bit cache and right tensors; what reaches the library is recorded."""

    def __init__(self, monkeypatch, dtype="bf16"):
        cfg = config(k=2, dtype=dtype)
        self.s = s = host_session(cfg, B, 16, MAXP)
        self.q4 = host_q4(cfg, 16)
        monkeypatch.setattr(s, "_raw_stream", lambda stream: 0)
        monkeypatch.setattr(s, "_scratch_for", lambda n, raw, stream: 0)
        self.reached = []
        calls = self

        class Lib:
            def __getattr__(self, name):
                return lambda *a: calls.reached.append((name, a)) or W.WM_OK

        s._lib = Lib()
        s._weights = W.wm_mix_weights()
        td = s.dtype
        i = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
        f = lambda *shape: torch.zeros(shape, dtype=td)  # noqa: E731
        row = (cfg.Hq, cfg.d)
        copy = dict(src=i(B, MAXP), dst=i(B, MAXP), first=i(B), last=i(B))
        self.t = {"write": copy, "read": dict(copy),
                  "mix": dict(h=f(B, cfg.L, cfg.D), table=i(B, MAXP), slot=i(B), pos=i(B)),
                  "decode": dict(q=f(B, *row), table=i(B, MAXP), lens=i(B), out=f(B, *row)),
                  "rows": dict(q=f(B, TQ, *row), pos=i(B, TQ), table=i(B, MAXP), out=f(B, TQ, *row))}

    def run(self, name, span=5, **other):
        t = self.t[name] | other
        s = self.s
        if name == "write":
            s.q4_write(self.q4, t["src"], t["dst"], t["first"], t["last"], span=span)
        elif name == "read":
            s.q4_read(self.q4, t["src"], t["dst"], t["first"], t["last"], span=span)
        elif name == "mix":
            s.q4_kv_mix(t["h"], self.q4, t["table"], t["slot"], pos=t["pos"])
        elif name == "decode":
            s.q4_decode_attn(0, t["q"], self.q4, t["table"], t["lens"], t["out"])
        else:
            s.q4_rows_attn(0, t["q"], t["pos"], self.q4, t["table"], t["out"])


NAMES = {"write": ("src", "dst", "first", "last"), "read": ("src", "dst", "first", "last"),
         "mix": ("h", "table", "slot", "pos"), "decode": ("q", "table", "lens", "out"), "rows": ("q", "pos", "table", "out")}
EACH = [(n, w) for n, ws in NAMES.items() for w in ws]
ENTRY = {"write": "wm_q4_write", "read": "wm_q4_read", "mix": "wm_q4_kv_mix", "decode": "wm_q4_decode_attn",
         "rows": "wm_q4_rows_attn"}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(NAMES))
def test_right_tensors_reach_the_library(monkeypatch, name, dtype):
    c = Calls(monkeypatch, dtype)
    c.run(name)
    assert [x[0] for x in c.reached] == [ENTRY[name]]
    for w, t in c.t[name].items():
        assert t.data_ptr() in c.reached[0][1], w
    if name in ("write", "read"):  # which table is the cache's
        order = ("src", "dst") if name == "write" else ("src", "dst")
        at = [c.reached[0][1].index(c.t[name][w].data_ptr()) for w in order]
        assert at == [2, 4]


@pytest.mark.parametrize("name,what", EACH)
def test_another_type_is_refused(monkeypatch, name, what):
    c = Calls(monkeypatch)
    t = c.t[name][what]
    other = {torch.int32: torch.int64, torch.bfloat16: torch.float16}[t.dtype]
    with pytest.raises(ValueError):
        c.run(name, **{what: t.to(other)})
    assert not c.reached


@pytest.mark.parametrize("name,what", EACH)
def test_too_few_elements_and_gaps_are_refused(monkeypatch, name, what):
    c = Calls(monkeypatch)
    t = c.t[name][what]
    if what not in ("q", "pos") or name != "rows":  # (a call's rows are its query's)
        with pytest.raises(ValueError):
            c.run(name, **{what: t[:-1].contiguous()})
    wide = torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype)[..., ::2]
    with pytest.raises(ValueError):
        c.run(name, **{what: wide})
    assert not c.reached


@pytest.mark.parametrize("name,what", EACH)
def test_another_device_is_refused(monkeypatch, name, what):
    c = Calls(monkeypatch)
    with pytest.raises(ValueError):
        c.run(name, **{what: c.t[name][what].as_subclass(Far)})
    assert not c.reached


@pytest.mark.parametrize("name", list(NAMES))
def test_a_4_bit_cache_on_another_device_is_refused(monkeypatch, name):
    c = Calls(monkeypatch)
    c.q4._index = 1
    with pytest.raises(ValueError):
        c.run(name)
    assert not c.reached


@pytest.mark.parametrize("name,what", [(n, w) for n, w in EACH if w in ("src", "dst", "table")])
def test_tables_of_another_width_are_refused(monkeypatch, name, what):
    c = Calls(monkeypatch)
    with pytest.raises(ValueError):
        c.run(name, **{what: torch.zeros((B, MAXP + 1), dtype=torch.int32)})
    assert not c.reached


@pytest.mark.parametrize("span,seen", [(0, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 40 + 3, 2 ** 31 - 1),
                                       (-1, -1), (-2 ** 32 + 5, -1)])
def test_spans_past_32_bits_keep_their_meaning(monkeypatch, span, seen):
    c = Calls(monkeypatch)
    c.run("write", span=span)
    assert c.reached[0][1][7] == seen


def test_buffers_of_a_4_bit_cache_are_checked():
    cfg = config()
    n = W.wm_q4_cache_bytes(cfg, 8)
    for bad in (torch.zeros(n, dtype=torch.int8), torch.zeros(2 * n, dtype=torch.uint8)[::2],
                torch.zeros(n, dtype=torch.uint8, device="meta")):
        with pytest.raises(ValueError):
            Q4Cache(cfg, 8, "cpu", cache_buf=bad)
    with pytest.raises(W.WMError):
        host_q4(cfg, 8).__class__(cfg, 9, "cpu", cache_buf=host_q4(cfg, 8).cache_buf)
    with pytest.raises(W.WMError):
        Q4Cache(cfg, 0, "cpu")
    bad = config()
    bad.d = 80
    with pytest.raises(W.WMError):
        Q4Cache(bad, 8, "cpu")
