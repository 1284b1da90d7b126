"""Which device a call of the serving cache's binding goes to (the library replaced by one that
notes its calls, CPU tensors): none for a cache of host memory, none on another GPU's stream, and
the cache's GPU is the current one while the library launches."""
import contextlib

import pytest

from paper_2310_07240_amd import kv8


class Noted:
    def __init__(self):
        self.calls = []
        self.current = 0

    def __getattr__(self, name):
        if name.endswith("_workspace_bytes"):
            return lambda *args: 8192
        if name.startswith("cg_kv8_"):
            return lambda *args: self.calls.append((name, self.current, args[-1])) or 0
        raise AttributeError(name)


class Stream:
    cuda_stream = 99

    def __init__(self, device):
        self.device = device


@pytest.fixture
def setup(monkeypatch):
    torch = pytest.importorskip("torch")
    w = Noted()
    monkeypatch.setattr(kv8, "_lib", lambda: w)
    c = kv8.Kv8Cache(6, 2, 64, device="cpu")
    t = torch.zeros((1, 2), dtype=torch.int32)
    n = torch.full((1,), 100, dtype=torch.int32)
    q = torch.zeros((1, 1, 4, 64), dtype=torch.float16)
    k = torch.zeros((1, 1, 2, 64), dtype=torch.float16)
    mass = torch.zeros((6, 2, 64))
    calls = [lambda **kw: c.store(k, k, t, n, **kw), lambda **kw: c.load(t, n, 3, k=None, v=None, **kw),
             lambda **kw: c.attend(q, t, n, out=q.clone(), **kw),
             lambda **kw: c.select(q, t, n, 1, out=n.view(1, 1, 1, 1).repeat(1, 1, 2, 1), **kw),
             lambda **kw: c.evict(t, n, mass, 64, 1, t, **kw)]
    return torch, w, c, calls


def test_host_memory_never_reaches_the_library(setup):
    torch, w, c, calls = setup
    for f in calls:
        with pytest.raises(ValueError):
            f()
    assert not w.calls


def test_streams_of_another_gpu_are_refused(setup, monkeypatch):
    torch, w, c, calls = setup
    c._empty = lambda shape, dtype, stream: torch.empty(shape, dtype=dtype)
    for f in calls:
        with pytest.raises(ValueError):
            f(stream=Stream(torch.device("cuda", 1)))
    assert not w.calls


def test_the_caches_gpu_is_current_for_the_launch(setup, monkeypatch):
    """A cache of GPU 1 while GPU 0 is current."""
    torch, w, c, calls = setup

    @contextlib.contextmanager
    def device(index):
        was, w.current = w.current, index
        yield
        w.current = was

    monkeypatch.setattr(torch.cuda, "device", device)
    c._capturing = lambda *_: False
    c._handle = lambda stream: 55
    c._index = 1
    c._current = lambda: w.current
    for f in calls:
        f()
    assert [x[1:] for x in w.calls] == [(1, 55)] * 5 and w.current == 0
