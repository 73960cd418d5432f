"""Page counts and layers past 32 bits keep their meaning in the 4-bit cache's calls (no GPU)."""
import pytest

from paper_2608_18486_gb300 import _lib as W
from paper_2608_18486_gb300.session import Q4Cache
from tests.test_q4_session_cpu import Calls, config, host_q4


@pytest.mark.parametrize("pages", [2 ** 31, 2 ** 32 + 4, -2 ** 32 + 4, 2 ** 64 + 1])
def test_page_counts_past_32_bits_are_refused(pages):
    buf = host_q4(config(), 8).cache_buf  # (aligned, and large enough for the low 32 bits' pages)
    with pytest.raises(W.WMError):
        Q4Cache(config(), pages, "cpu", cache_buf=buf)


@pytest.mark.parametrize("layer,seen", [(0, 0), (3, 3), (-1, -1), (2 ** 31, -1), (2 ** 32, -1), (2 ** 32 + 1, -1), (-2 ** 32, -1)])
def test_layers_past_32_bits_are_no_others(monkeypatch, layer, seen):
    c = Calls(monkeypatch)
    t = c.t["decode"]
    c.s.q4_decode_attn(layer, t["q"], c.q4, t["table"], t["lens"], t["out"])
    t = c.t["rows"]
    c.s.q4_rows_attn(layer, t["q"], t["pos"], c.q4, t["table"], t["out"])
    assert [a[2] for _, a in c.reached] == [seen, seen]
