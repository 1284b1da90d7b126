"""GPU: a whole step of requests over a shared context (pages, store, attention, drafts verified, pages
back) captured and replayed, on streams other than the current one, and from two threads: each run
against an eager twin on buffers of its own, bit for bit."""
import threading

import numpy as np
import pytest

from gpu_helpers import say, torch_cuda
from test_gpu_kv8 import ints

pytestmark = pytest.mark.gpu
H, D, HQ, R, K, VOCAB, T = 2, 64, 8, 6, 3, 6000, 250


class Requests:
    """Requests of two contexts with room for their answers, and the inputs of a step in place. `seed`
    makes them alike."""

    def __init__(self, torch, seed, stream=None, big=False):
        from paper_2310_07240_amd.kv8 import Kv8Cache
        self.torch, self.stream = torch, stream
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        P = 20000 if big else 120              # a pool that takes the launches of a large one
        self.cache = Kv8Cache(P, H, D)
        self.mass = torch.rand((P, H, 64), generator=g, device="cuda")
        self.refs = torch.zeros(P, dtype=torch.int32, device="cuda")
        self.table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
        zero, held = ints(torch, [0, 0]), ints(torch, [T, T])
        self.cache.reserve(self.table, zero, held, self.refs)
        k, v = (torch.randn((2, T, H, D), generator=g, device="cuda").half() for _ in "kv")
        self.cache.store(k, v, self.table, zero)
        self.shared, tails = self.table[:, :3].contiguous(), self.table[:, 3:]
        wide = torch.full((2, 3), -1, dtype=torch.int32, device="cuda")
        wide[:, :1] = tails
        self.rows, self.lengths = self.cache.fork(wide, ints(torch, [T % 64] * 2),
                                                  ints(torch, [0] * R + [1] * R), self.refs)
        self.shared_len, self.firsts = ints(torch, [192, 192]), ints(torch, [0, R, 2 * R])
        n, q = 2 * R, K + 1
        new = lambda *s: torch.zeros(s, device="cuda")
        self.k, self.v, self.q = new(n, q, H, D).half(), new(n, q, H, D).half(), new(n, q, HQ, D).half()
        self.target, self.draft = new(n, q, VOCAB), new(n, K, VOCAB)
        self.drafts, self.u = ints(torch, [[0] * K] * n), new(n, q)
        self.counts = ints(torch, [q] * n)
        self.out, self.lse = torch.zeros_like(self.q), new(n, q, HQ)
        self.tokens, self.accepted = ints(torch, [[0] * q] * n), ints(torch, [0] * n)
        self.missing = ints(torch, [0])

    def fill(self, seed):
        """The next step's inputs, in place."""
        g = self.torch.Generator(device="cuda").manual_seed(seed)
        for x in (self.k, self.v, self.q):
            x.copy_(self.torch.randn(x.shape, generator=g, device="cuda"))
        for x in (self.target, self.draft):
            x.copy_(self.torch.softmax(3 * self.torch.randn(x.shape, generator=g, device="cuda"), -1))
        self.drafts.copy_(self.torch.randint(0, VOCAB, self.drafts.shape, generator=g, device="cuda"))
        self.u.copy_(self.torch.rand(self.u.shape, generator=g, device="cuda"))
        # two drafts in three are accepted
        self.target[:, :K].scatter_(2, self.drafts.long()[..., None], 0.4)
        self.draft.scatter_(2, self.drafts.long()[..., None], 0.6)

    def step(self):
        c, s = self.cache, self.stream
        c.reserve(self.rows, self.lengths, self.counts, self.refs, mass=self.mass,
                  missing=self.missing, stream=s)
        c.store(self.k, self.v, self.rows, self.lengths, mass=self.mass, stream=s)
        with self.torch.cuda.stream(s or self.torch.cuda.current_stream()):
            self.lengths.add_(self.counts)
        c.attend_shared(self.q, self.shared, self.shared_len, self.firsts, table=self.rows,
                        lengths=self.lengths, out=self.out, lse=self.lse, stream=s)
        c.verify(self.target, self.drafts, self.u, draft=self.draft, lengths=self.lengths,
                 tokens=self.tokens, accepted=self.accepted, new_lengths=self.lengths, stream=s)
        c.release(self.rows, self.refs, keep=self.lengths, stream=s)
        # a look at what would be left in front (the pages moved are copies: the old ones stay)
        self.moved = c.compact(self.table, self.refs, mass=self.mass, stream=s)

    def results(self):
        c = self.cache
        return {k: x.clone() for k, x in {
            "rows": self.rows, "refs": self.refs, "lengths": self.lengths, "out": self.out,
            "lse": self.lse, "tokens": self.tokens, "accepted": self.accepted, "missing": self.missing,
            "mass": self.mass, "k": c.k_codes, "v": c.v_codes, "ks": c.k_scale, "vs": c.v_scale,
            "bounds": c.k_bounds, "table": self.moved[0], "new refs": self.moved[1],
            "moved": self.moved[2], "live": self.moved[3]}.items()}


def same(torch, a, b, what):
    x, y = a.results(), b.results()
    torch.cuda.synchronize()
    for k in x:
        assert torch.equal(x[k], y[k]), (what, k)


@pytest.mark.parametrize("big", [False, True])
def test_captured_steps(big):
    """Every replay against the eager twin; between replays eager calls of the same cache that need
    more scratch, and tensors that take what they give back."""
    torch = torch_cuda()
    a, b = Requests(torch, 5, big=big), Requests(torch, 5, big=big)
    other = Requests(torch, 6)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):                # the warm-up is a step of both
        a.fill(0)
        a.step()
    b.fill(0)
    b.step()
    torch.cuda.synchronize()
    same(torch, a, b, "warm-up")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.step()
    total, kept = 0, []
    for i in range(1, 7):
        say(f"replay {i}")
        a.fill(i)
        b.fill(i)
        other.fill(i)
        other.step()
        many = torch.randn(400, 1, HQ, D, device="cuda").half()
        a.cache.attend_shared(many, a.shared, a.shared_len, ints(torch, [0, 200, 400]))
        kept += [torch.full((m,), 0xff, dtype=torch.uint8, device="cuda") for m in (4096, 1 << 18)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b.step()
        same(torch, a, b, i)
        total += int(b.accepted.sum())
        assert int(b.missing) == 0 and all(bool((x == 0xff).all()) for x in kept)
    assert 0 < total < 6 * 2 * R * K
    assert int(b.lengths.max()) > 64               # pages were reserved on the way


def test_a_given_stream():
    torch = torch_cuda()
    s = torch.cuda.Stream()
    a, b = Requests(torch, 7, stream=s), Requests(torch, 7)
    for i in range(4):
        a.fill(i)
        b.fill(i)
        torch.cuda.synchronize()
        a.step()
        b.step()
        torch.cuda.synchronize()
        same(torch, a, b, i)


def test_two_threads_on_one_stream():
    """Threads that share a cache's scratch: their launches do not mix."""
    torch = torch_cuda()
    a, b, twin = Requests(torch, 8), Requests(torch, 9), Requests(torch, 8)
    b.cache._ws = a.cache._ws                      # one cache's scratch for both, as of one cache
    b.cache._lock = a.cache._lock
    for x in (a, b, twin):
        x.fill(1)
    torch.cuda.synchronize()
    errors = []

    def many(x, n):
        try:
            for _ in range(n):
                x.step()
        except Exception as e:                     # pragma: no cover
            errors.append(e)
    threads = [threading.Thread(target=many, args=(a, 6)), threading.Thread(target=many, args=(b, 6))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    many(twin, 6)
    torch.cuda.synchronize()
    same(torch, a, twin, "threads")
