"""The binding's scratch (kv8.Kv8Cache._scratch), on CPU tensors: which call gets which memory."""
import gc
import weakref

import pytest

from paper_2310_07240_amd import kv8

STREAM = 77                                    # a handle


@pytest.fixture
def cache():
    torch = pytest.importorskip("torch")
    c = kv8.Kv8Cache(4, 2, 64, device="cpu")
    c.capturing = False
    c._capturing = lambda *_: c.capturing
    c.zeros = lambda t: int(t[:4096].count_nonzero()) == 0
    c.torch = torch
    return c


def test_eager_calls_share_and_grow(cache):
    a = cache._scratch(None, STREAM, 5000)
    assert a[1] >= 5000 and cache.zeros(a[2]) and a[0] == a[2].data_ptr()
    assert cache._scratch(None, STREAM, 4096)[0] == a[0]
    b = cache._scratch(None, STREAM, 50000)
    assert b[1] >= 50000 and cache.zeros(b[2])
    assert cache._scratch(None, STREAM, 5000)[0] == b[0]
    assert cache._scratch(None, STREAM + 1, 5000)[0] != b[0]


def test_a_captured_call_takes_none_of_the_eager_calls_scratch(cache):
    """Whatever the stream has from a warm-up: a larger eager call would free it under the graph,
    and an eager call on it may run beside a replay."""
    eager = cache._scratch(None, STREAM, 5000)
    cache.capturing = True
    first = cache._scratch(None, STREAM, 5000)
    assert first[0] != eager[0] and first[1] >= 5000 and cache.zeros(first[2])
    second = cache._scratch(None, STREAM, 9000)
    assert second[0] not in (eager[0], first[0])
    cache.capturing = False
    assert cache._scratch(None, STREAM, 5000)[0] == eager[0]
    assert cache._scratch(None, STREAM, 60000)[0] not in (first[0], second[0])


def test_captures_leave_nothing_behind(cache):
    """The graph's pool keeps a captured call's scratch, the cache does not."""
    cache.capturing = True
    t = weakref.ref(cache._scratch(None, STREAM, 5000)[2])
    gc.collect()
    assert t() is None and not cache._ws


def test_a_need_that_grows_by_steps_is_not_met_step_by_step(cache):
    """A sequence of tokens needs a little more with every page."""
    need, seen = 100000, set()
    for _ in range(200):
        ws = cache._scratch(None, STREAM, need)
        assert ws[1] >= need
        seen.add(ws[1])
        need += 4096
    assert len(seen) <= 12                     # 9 times as much at the end: quarters, ten of them


def test_which_streams_are_captured(monkeypatch):
    """The runtime is asked about the call's own stream, whichever is current; what it cannot tell
    counts as captured, the null stream never does."""
    import ctypes
    pytest.importorskip("torch")
    states, asked = {5: (0, 0), 6: (0, 1), 7: (0, 2), 8: (900, 0)}, []

    class Lib:
        def hipStreamIsCapturing(self, handle, status):
            asked.append(handle)
            ctypes.c_int.from_address(status).value = states[handle][1]
            return states[handle][0]

    monkeypatch.setattr(kv8, "_lib", Lib)
    c = kv8.Kv8Cache(4, 2, 64, device="cpu")
    assert [c._capturing(h) for h in (0, 5, 6, 7, 8, 5)] == [False, False, True, True, True, False]
    assert asked == [5, 6, 7, 8, 5]
