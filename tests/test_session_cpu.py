"""DecodeSession's host side: devices, streams, scratch and checks (no GPU, nothing launched)."""
import contextlib

import pytest
import torch

from paper_2608_18486_gb300 import _lib as W
from paper_2608_18486_gb300.session import DecodeSession


def config(k=1, Hkv=2, G=2, d=64, page=16, dtype="bf16"):
    return W.make_config(k, k, 64, Hkv * G, Hkv, d, 1, page, dtype, list(range(k)))


def host_session(cfg, B, pages, max_pages):
    """A session in host memory, its cache on a 256-byte boundary as device memory is."""
    n = W.wm_cache_bytes(cfg, pages)
    buf = torch.zeros(n + 256, dtype=torch.uint8)
    at = -buf.data_ptr() % 256
    return DecodeSession(cfg, B, pages, max_pages, "cpu", cache_buf=buf[at:at + n])


class Devices:
    current = 1


@pytest.fixture
def two_devices(monkeypatch):
    """A process whose current device is 1 at first; what it allocates lies in host memory."""
    devices = Devices()
    zeros = torch.zeros

    def on_host(n, dtype, device):  # on a 256-byte boundary, as device memory is
        x = zeros(n + 256, dtype=dtype)
        at = -x.data_ptr() % 256 // x.element_size()
        return x[at:at + n]
    monkeypatch.setattr(torch, "empty", on_host)
    monkeypatch.setattr(torch, "zeros", on_host)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: devices.current)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: devices.current, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index, raising=False)

    class Stream:
        def __init__(self, index):
            self.cuda_stream = 1000 + index

    def current_stream(device=None):
        index = None if device is None else torch.device(device).index
        return Stream(devices.current if index is None else index)
    monkeypatch.setattr(torch.cuda, "current_stream", current_stream)
    return devices


@pytest.mark.parametrize("device,index", [("cuda", 1), ("cuda:0", 0), ("cuda:1", 1)])
def test_every_call_takes_the_stream_of_the_sessions_device(two_devices, device, index):
    s = DecodeSession(config(), 2, 4, 2, device)
    assert s.device == torch.device("cuda", index)
    two_devices.current = index
    assert s._raw_stream(None) == 1000 + index
    assert s._stream(None).value == 1000 + index


@pytest.mark.parametrize("device,current", [("cuda", 0), ("cuda:0", 1), ("cuda:1", 0)])
def test_calls_while_another_device_is_current_are_refused(two_devices, device, current):
    """They would launch there, on this device's addresses."""
    s = DecodeSession(config(), 2, 4, 2, device)
    two_devices.current = current
    for stream in (None, torch.cuda.current_stream(s.device)):
        with pytest.raises(ValueError):
            s._raw_stream(stream)
        with pytest.raises(ValueError):
            s._stream(stream)


def test_a_cache_on_another_device_is_refused(two_devices):
    class Elsewhere:
        dtype, device = torch.uint8, torch.device("cuda:0")

        def is_contiguous(self):
            return True

        def numel(self):
            return 1 << 40

    with pytest.raises(ValueError):
        DecodeSession(config(), 2, 4, 2, "cuda", cache_buf=Elsewhere())


def test_scratch_kept_for_graphs_stays_below_what_is_in_use(monkeypatch):
    """A batch that grows one sequence at a time, the mass call's workspace on two streams."""
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: None)
    cfg = config(Hkv=2, G=2, page=64)
    s = host_session(cfg, 64, 4, 65)
    needs = [W.wm_decode_attn_mass_workspace(cfg, b, 65) for b in range(1, 65)]
    assert needs[-1] > 16 * needs[0]  # (the sizes do grow)
    for stream in (7, 8):
        for n in needs:
            assert s._scratch_for(n, stream, None) == s._scratch[stream].data_ptr()
            assert s._scratch[stream].numel() >= n
    live = sum(x.numel() for x in s._scratch.values())
    assert live < 2 * 2 * max(needs)
    assert sum(x.numel() for x in s._outgrown) < live
    again = [x.data_ptr() for x in s._scratch.values()]
    for n in reversed(needs):  # (smaller requests share what is there)
        s._scratch_for(n, 7, None)
    assert [x.data_ptr() for x in s._scratch.values()] == again


class Calls:
    """The long-context calls of a session of B sequences on right tensors, any of
    them replaced; what reaches the library is recorded, and not called."""

    def __init__(self, monkeypatch, B=3, dtype="bf16"):
        cfg = config(k=2, dtype=dtype)
        self.s = s = host_session(cfg, B, 16, 4)
        monkeypatch.setattr(s, "_raw_stream", lambda stream: 0)
        monkeypatch.setattr(s, "_scratch_for", lambda n, raw, stream: 0)
        self.reached = []

        class Library:
            def __getattr__(_, name):
                return lambda *a: self.reached.append((name, a)) or W.WM_OK
        s._lib = Library()
        i32 = torch.int32
        self.B, self.t = B, dict(
            q=torch.zeros(B, 4, 64, dtype=s.dtype), out=torch.zeros(B, 4, 64, dtype=s.dtype),
            table=torch.zeros(B, 4, dtype=i32), lens=torch.zeros(B, dtype=i32),
            rows=torch.zeros(B, 5, 4, 64, dtype=s.dtype), rows_out=torch.zeros(B, 5, 4, 64, dtype=s.dtype),
            pos=torch.zeros(B, 5, dtype=i32), mass=torch.zeros(2, B, 2, 64), mass_out=torch.zeros(2, B, 2, 64),
            kept=torch.zeros(2, B, 2, 24, dtype=i32), new_lens=torch.zeros(B, dtype=i32))

    def __call__(self, name, B=None, sinks=1, window=8, budget=24, recent=2, **other):
        t, s = {**self.t, **other}, self.s
        if name == "window":
            s.window_attn(0, t["q"], t["table"], t["lens"], t["out"], sinks=sinks, window=window, B=B)
        if name == "rows":
            s.window_prefill_attn(0, t["rows"], t["pos"], t["table"], t["rows_out"], sinks=sinks, window=window)
        if name == "prefix":
            s.prefix_attn(0, t["q"], t["table"], t["lens"], t["out"], shared_pages=1, B=B)
        if name == "mass":
            s.decode_attn_mass(0, t["q"], t["table"], t["lens"], t["mass"], t["out"], B=B)
        if name == "evict":
            s.evict(t["mass"], t["table"], t["lens"], t["mass_out"], t["kept"], t["new_lens"], budget=budget,
                    sinks=sinks, recent=recent, B=B)


READ = {"window": ["q", "table", "lens", "out"], "rows": ["rows", "pos", "table", "rows_out"],
        "prefix": ["q", "table", "lens", "out"], "mass": ["q", "table", "lens", "mass", "out"],
        "evict": ["mass", "table", "lens", "mass_out", "kept", "new_lens"]}
EACH = [(name, what) for name in READ for what in READ[name]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(READ))
def test_right_tensors_reach_the_library(monkeypatch, name, dtype):
    c = Calls(monkeypatch, dtype=dtype)
    c(name)
    assert len(c.reached) == 1
    if name not in ("rows", "mass", "evict"):  # part of a batch, in tensors made for all of it
        c(name, B=2)
        assert len(c.reached) == 2
    if name in ("mass", "evict"):
        small = {"mass": torch.zeros(2, 2, 2, 64), "mass_out": torch.zeros(2, 2, 2, 64),
                 "kept": torch.zeros(2, 2, 2, 24, dtype=torch.int32)}
        c(name, B=2, **small)
        assert len(c.reached) == 2
    flat = c.t["table"].reshape(-1)  # (the table's rows one behind the other)
    c(name, table=flat)


@pytest.mark.parametrize("name,what", EACH)
def test_another_type_is_refused(monkeypatch, name, what):
    c = Calls(monkeypatch)
    t = c.t[what]
    for dtype in (torch.int64, torch.float64, torch.float16, torch.uint8):
        with pytest.raises(ValueError):
            c(name, **{what: torch.zeros(4 * t.numel(), dtype=dtype).view(4, *t.shape)})
    assert not c.reached


@pytest.mark.parametrize("name,what", EACH)
def test_too_few_elements_and_gaps_are_refused(monkeypatch, name, what):
    c = Calls(monkeypatch)
    t = c.t[what]
    wide = torch.zeros(*t.shape, 2, dtype=t.dtype)[..., 0]
    fewer = t[1:] if what != "rows" else t[..., :63].contiguous()  # (the rows themselves give that call's sizes)
    for bad in (wide, fewer):
        with pytest.raises(ValueError):
            c(name, **{what: bad})
    assert not c.reached


class Far(torch.Tensor):
    """A tensor that says it is on device 1."""

    def get_device(self):
        return 1


@pytest.mark.parametrize("name,what", EACH)
def test_another_device_is_refused(monkeypatch, name, what):
    c = Calls(monkeypatch)
    with pytest.raises(ValueError):
        c(name, **{what: c.t[what].as_subclass(Far)})
    assert not c.reached


@pytest.mark.parametrize("name", list(READ))
def test_tables_of_another_width_are_refused(monkeypatch, name):
    c = Calls(monkeypatch)
    with pytest.raises(ValueError):
        c(name, table=torch.zeros(3, 6, dtype=torch.int32))
    assert not c.reached


@pytest.mark.parametrize("name,what", [("mass", "mass"), ("evict", "mass"), ("evict", "mass_out"), ("evict", "kept")])
def test_sums_made_for_another_batch_are_refused(monkeypatch, name, what):
    """Their channels lie where the call's own batch puts them."""
    c = Calls(monkeypatch)
    small = {"mass": torch.zeros(2, 2, 2, 64), "mass_out": torch.zeros(2, 2, 2, 64),
             "kept": torch.zeros(2, 2, 2, 24, dtype=torch.int32)}
    del small[what]
    with pytest.raises(ValueError):
        c(name, B=2, **small)
    assert not c.reached


def test_pool_positions_are_checked(monkeypatch):
    s = host_session(config(), 3, 16, 4)
    s._weights = W.wm_mix_weights()
    ran = []
    monkeypatch.setattr(W, "wm_kv_mix_at", lambda *a: ran.append(a) or W.WM_OK)
    monkeypatch.setattr(s, "_stream", lambda stream: None)
    s.kv_mix(None, None, None, pos=torch.zeros(3, dtype=torch.int32))
    assert len(ran) == 1
    for bad in (torch.zeros(3, dtype=torch.int64), torch.zeros(2, dtype=torch.int32),
                torch.zeros(3, 2, dtype=torch.int32)[:, 0], torch.zeros(3, dtype=torch.int32).as_subclass(Far)):
        with pytest.raises(ValueError):
            s.kv_mix(None, None, None, pos=bad)
    assert len(ran) == 1


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 40 + 1, 10 ** 30, -1, -2 ** 32, -2 ** 32 + 5])
@pytest.mark.parametrize("name,at", [("window", (6, 7)), ("rows", (6, 7))])
def test_counts_of_slots_past_32_bits_are_every_slot(monkeypatch, name, at, n):
    """Windows and sinks may be of any size; a negative one reaches the library as one, which refuses it."""
    c = Calls(monkeypatch)
    c(name, sinks=n, window=3)
    c(name, sinks=3, window=n)
    want = 2 ** 31 - 1 if n > 0 else -1
    assert [a[at[0]] for _, a in c.reached] == [want, 3] and [a[at[1]] for _, a in c.reached] == [3, want]


@pytest.mark.parametrize("what,at", [("sinks", 7), ("recent", 8)])
@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 32, -2 ** 32 + 1])
def test_evictions_of_counts_past_32_bits_are_refused_by_the_library(monkeypatch, what, at, n):
    c = Calls(monkeypatch)
    c("evict", **{what: n})
    (name, args), = c.reached
    assert name == "wm_cache_evict" and args[at] == (2 ** 31 - 1 if n > 0 else -1)  # over the budget, or below 0
