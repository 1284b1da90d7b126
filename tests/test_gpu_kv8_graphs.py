"""GPU: captured calls of the 8-bit cache whose stream has scratch already, and eager calls beside
and after the capture that need more of it."""
import numpy as np
import pytest

from gpu_helpers import say, torch_cuda
from test_gpu_kv8 import ints, make, tables

pytestmark = pytest.mark.gpu


class Small:
    """A call with weights and splits, a selection and attention over its pages."""

    def __init__(self, torch, seed):
        rng = np.random.default_rng(seed)
        _, self.table, n = tables(torch, rng, 2, 20)
        self.cache = make(torch, n, 2, 128)
        self.q = torch.randn(2, 1, 8, 128).half().cuda()
        self.L = ints(torch, [1100, 700])
        self.out, self.sparse = torch.zeros_like(self.q), torch.zeros_like(self.q)
        self.mass = torch.zeros((n, 2, 64), device="cuda")
        self.picks = torch.zeros((2, 1, 2, 3), dtype=torch.int32, device="cuda")

    def step(self):
        c = self.cache
        c.attend(self.q, self.table, self.L, out=self.out, mass=None, mass_out=self.mass)
        c.select(self.q, self.table, self.L, 3, out=self.picks)
        c.attend(self.q, self.table, self.L, out=self.sparse, picks=self.picks)

    def results(self):
        return [x.clone() for x in (self.out, self.mass, self.picks, self.sparse)]


def test_warm_up_capture_and_larger_calls_on_one_stream():
    torch = torch_cuda()
    s = Small(torch, 21)
    # a call of the same cache that needs far more scratch: a prompt of many splits
    big_q = torch.randn(2, 100, 8, 128).half().cuda()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        s.step()                               # the warm-up
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.step()
    kept = []
    for i in range(4):
        say(f"replay {i} behind a larger call")
        with torch.cuda.stream(stream):
            s.cache.attend(big_q, s.table, s.L)
            # what the larger call may have given back to the allocator is taken by others
            kept += [torch.full((m,), 0xff, dtype=torch.uint8, device="cuda")
                     for m in (4096, 1 << 16, 1 << 18, 1 << 20, 1 << 22)]
        s.q.copy_(torch.randn(s.q.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = s.results()
        assert all(bool((k == 0xff).all()) for k in kept)
        s.step()
        torch.cuda.synchronize()
        for a, b in zip(got, s.results()):
            assert torch.equal(a, b), i


def test_replays_beside_eager_calls_on_the_capture_stream():
    """The graph runs on one stream while the stream it was captured on goes on with eager calls."""
    torch = torch_cuda()
    s, e = Small(torch, 22), Small(torch, 23)
    e.cache = s.cache                          # one cache, other sequences and outputs
    e.table, e.mass = s.table.flip(0).contiguous(), torch.zeros_like(s.mass)
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        s.step()
        e.step()
    torch.cuda.synchronize()
    want, want_e = s.results(), e.results()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.step()
    for _ in range(3):
        for x in (s.out, s.mass, s.picks, s.sparse, e.out, e.mass, e.picks, e.sparse):
            x.zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            with torch.cuda.stream(other):
                graph.replay()
            with torch.cuda.stream(stream):
                e.step()
        torch.cuda.synchronize()
        for a, b in zip(s.results() + e.results(), want + want_e):
            assert torch.equal(a, b)
