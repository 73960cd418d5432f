"""What a session keeps of large scratch, while calls grow (no GPU, nothing launched)."""
import contextlib

import pytest
import torch

from tests.test_session_cpu import config, host_session

MB = 1 << 20


@pytest.fixture
def capturing(monkeypatch):
    """Streams that record work into graphs: names in the set."""
    now, current = set(), [None]

    @contextlib.contextmanager
    def on(stream):
        before, current[0] = current[0], stream
        yield
        current[0] = before

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[0])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: current[0] in now)
    return now


def large(s):
    return getattr(s, "_large_scratch", s._scratch).values()


def held(s):
    return sum(x.numel() for x in {id(x): x for x in (*s._scratch.values(), *large(s), *s._outgrown)}.values())


def test_large_scratch_grows_to_what_is_asked_for(capturing):
    s = host_session(config(), 2, 4, 2)
    for n in (40 * MB, 41 * MB, 50 * MB, 50 * MB + 256, 64 * MB):
        p = s._scratch_for(n, 7, "seven")
        assert held(s) == n and p == s._scratch_for(n - 256, 7, "seven") == s._scratch_for(33 * MB, 7, "seven")
    assert s._scratch_for(65 * MB, 8, "eight") != s._scratch_for(64 * MB, 7, "seven")
    assert held(s) == 129 * MB


def test_large_scratch_that_a_graph_uses_stays(capturing):
    s = host_session(config(), 2, 4, 2)
    s._scratch_for(40 * MB, 7, "seven")  # (before the capture)
    capturing.add("seven")
    used = s._scratch_for(36 * MB, 7, "seven")
    capturing.clear()
    assert s._scratch_for(41 * MB, 7, "seven") != used
    assert [x.data_ptr() for x in s._outgrown] == [used] and held(s) <= 3 * 41 * MB
    s._scratch_for(100 * MB, 7, "seven")  # (no graph uses the one between)
    assert [x.data_ptr() for x in s._outgrown] == [used] and held(s) == 140 * MB


def test_captures_on_another_stream_keep_nothing_of_this_one(capturing):
    s = host_session(config(), 2, 4, 2)
    capturing.add("eight")
    s._scratch_for(40 * MB, 7, "seven")
    s._scratch_for(50 * MB, 7, "seven")
    assert not s._outgrown and held(s) == 50 * MB


def test_small_scratch_is_kept_beside_large(capturing):
    s = host_session(config(), 2, 4, 2)
    small = s._scratch_for(1000, 7, "seven")
    s._scratch_for(40 * MB, 7, "seven")
    assert s._scratch_for(1000, 7, "seven") == small and not s._outgrown


def test_growing_in_a_capture_stays_below_twice_what_is_in_use(capturing):
    s = host_session(config(), 2, 4, 2)
    capturing.add("seven")
    for n in range(33, 200, 5):
        s._scratch_for(n * MB, 7, "seven")
    live = sum(x.numel() for x in large(s))
    assert sum(x.numel() for x in s._outgrown) < live < 2 * 200 * MB
