"""DecodeSession's host side: devices and streams (no GPU, nothing launched)."""
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


@pytest.fixture
def two_devices(monkeypatch):
    """A process whose current device is 1; what it allocates lies in host memory."""
    zeros = torch.zeros

    def on_host(n, dtype, device):  # on a 256-byte boundary, as device memory is
        x = zeros(n + 256, dtype=dtype)
        at = -x.data_ptr() % 256 // x.element_size()
        return x[at:at + n]
    monkeypatch.setattr(torch, "empty", on_host)
    monkeypatch.setattr(torch, "zeros", on_host)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index)

    class Stream:
        def __init__(self, index):
            self.cuda_stream = 1000 + index

    def current_stream(device=None):
        index = None if device is None else torch.device(device).index
        return Stream(1 if index is None else index)
    monkeypatch.setattr(torch.cuda, "current_stream", current_stream)


@pytest.mark.parametrize("device,index", [("cuda", 1), ("cuda:0", 0), ("cuda:1", 1)])
def test_every_call_takes_the_stream_of_the_sessions_device(two_devices, device, index):
    s = DecodeSession(config(), 2, 4, 2, device)
    assert s.device == torch.device("cuda", index)
    assert s._raw_stream(None) == 1000 + index
    assert s._stream(None).value == 1000 + index


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
