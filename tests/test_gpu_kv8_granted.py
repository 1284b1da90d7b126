"""GPU: reservations that find too few pages, or rows without room: what they grant, and that a store
with it writes to no page that others hold (the pool is compared bit for bit)."""
import numpy as np
import pytest

import sharing_reference as S
from paper_2310_07240_amd import workloads as W
from gpu_helpers import say, torch_cuda
from test_gpu_kv8 import ints, make

pytestmark = pytest.mark.gpu
PAGE = 64


def pool(cache):
    return [x.clone() for x in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale,
                                cache.k_bounds)]


def same(torch, a, b, but=()):
    keep = torch.ones(len(a[0]), dtype=torch.bool, device="cuda")
    keep[list(but)] = False
    return all(torch.equal(x[keep].view(torch.uint8), y[keep].view(torch.uint8)) for x, y in zip(a, b))


def grants(lengths, counts, width, missing):
    """From the header's words, in whole numbers."""
    out = []
    for n, c in zip(lengths, counts):
        a = S.clip(n, width)
        out.append(0 if missing else S.clip(a + max(0, int(c)), width) - a)
    return out


# (pools of both kinds: planned by one workgroup, and by many)
@pytest.mark.parametrize("P", [40, 66000])
def test_a_store_after_too_few_pages(P):
    """Four requests fork a context that ends inside a page; three pages are free."""
    torch = torch_cuda()
    H, D, T = 1, 64, 100
    cache = make(torch, P, H, D)
    refs = torch.ones(P, dtype=torch.int32, device="cuda")
    free = [3, 20, P - 2]
    refs[free] = 0
    table = ints(torch, [[7, 11, -1]])
    rows, lengths = cache.fork(table, ints(torch, [T]), ints(torch, [0] * 4), refs)
    counts, granted = ints(torch, [5, 20, 0, 70]), ints(torch, [9] * 4)
    k, v = (torch.randn(4, 70, H, D, device="cuda").half() for _ in "kv")
    before, held, was = pool(cache), refs.clone(), rows.clone()
    # the third request wants nothing, the fourth two pages: four in all
    missing = cache.reserve(rows, lengths, counts, refs, granted=granted)
    cache.store(k, v, rows, lengths, counts=granted)
    assert int(missing) == 1 and granted.tolist() == [0] * 4
    assert torch.equal(refs, held) and torch.equal(rows, was) and same(torch, before, pool(cache))
    refs[P - 5] = 0
    missing = cache.reserve(rows, lengths, counts, refs, granted=granted)
    cache.store(k, v, rows, lengths, counts=granted)
    assert int(missing) == 0 and granted.tolist() == [5, 20, 0, 70]
    assert same(torch, before, pool(cache), free + [P - 5])
    assert rows.tolist() == [[7, 3, -1], [7, 20, -1], [7, 11, -1], [7, P - 5, P - 2]]
    # what was stored lies behind the copied tokens, which only a larger scale may have coded again
    got, _ = cache.load(rows, lengths, 70, counts=granted)
    for b, n in enumerate(granted.tolist()):
        # half a step of a code of the page's largest value
        assert float((got[b, :n].float() - k[b, :n].float()).abs().max() if n else 0) <= (
            float(cache.k_scale.max()) * 0.5 + 2.0 ** -11 * float(k.float().abs().max()))


@pytest.mark.parametrize("P,n", [(300, 60), (66000, 60), (3000, 2100), (300, 200)])
@pytest.mark.parametrize("free", [0, 4, None])
@pytest.mark.parametrize("alias", [False, True])
def test_what_is_granted(P, n, free, alias):
    """Counts below zero and past the row, lengths past it, for calls that want pages and that want
    none; written over the counts too."""
    torch = torch_cuda()
    rng = np.random.default_rng(P + n)
    width = 3
    cache = make(torch, P, 1, 64)
    refs = np.ones(P, np.int32)
    if free != 0:
        refs[rng.permutation(P)[:P // 2 if free is None else free]] = 0
    held = np.flatnonzero(refs)
    rows = rng.choice(held, (n, width)).astype(np.int32)
    if free != 0:                                      # else every page is its row's alone
        rows[rng.random((n, width)) < 0.1] = -1
    lengths = rng.integers(-3, width * PAGE + 20, n)
    counts = rng.integers(-3, 100, n)
    counts[rng.random(n) < 0.1] = 2 ** 31 - 1
    want = S.reserve(rows.tolist(), lengths, counts, refs.tolist(), P)
    table, r = torch.from_numpy(rows).cuda(), torch.from_numpy(refs).cuda()
    c = ints(torch, counts.tolist())
    granted = c if alias else ints(torch, [77] * n)
    missing = cache.reserve(table, ints(torch, lengths.tolist()), c, r, granted=granted)
    assert int(missing) == want[2] and table.tolist() == want[0] and r.tolist() == want[1]
    assert granted.tolist() == grants(lengths, counts, width, want[2])
    assert (want[2] > 0) == (sum(granted.tolist()) == 0)
    if n >= 200:                                       # (60 sequences do not want four pages)
        assert (want[2] > 0) == (free == 4)


def test_captured_steps_that_run_out():
    """Reserve, store and longer sequences in one graph: against an eager twin, while pages are there,
    when they are not, and when they are again."""
    torch = torch_cuda()
    H, D, n, P, q = 2, 64, 5, 14, 20

    class Twin:
        def __init__(self):
            torch.manual_seed(3)
            self.cache = make(torch, P, H, D)
            self.refs = torch.zeros(P, dtype=torch.int32, device="cuda")
            self.refs[0] = 1
            table = ints(torch, [[0, -1, -1, -1]])
            self.rows, self.lengths = self.cache.fork(table, ints(torch, [50]), ints(torch, [0] * n),
                                                      self.refs)
            self.counts, self.granted = ints(torch, [q] * n), ints(torch, [0] * n)
            self.missing = ints(torch, [0])
            self.k, self.v = (torch.zeros(n, q, H, D, device="cuda").half() for _ in "kv")

        def fill(self, seed):
            g = torch.Generator(device="cuda").manual_seed(seed)
            for x in (self.k, self.v):
                x.copy_(torch.randn(x.shape, generator=g, device="cuda"))

        def step(self):
            self.cache.reserve(self.rows, self.lengths, self.counts, self.refs, missing=self.missing,
                               granted=self.granted)
            self.cache.store(self.k, self.v, self.rows, self.lengths, counts=self.granted)
            self.lengths.add_(self.granted)

        def state(self):
            return [self.rows.clone(), self.refs.clone(), self.lengths.clone(), self.granted.clone(),
                    self.missing.clone()] + pool(self.cache)

    a, b = Twin(), Twin()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    a.fill(0)
    b.fill(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        a.step()
    b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.step()
    shorts = []
    for i in range(1, 10):
        say(f"replay {i}")
        if i == 7:                                     # two requests end
            for x in (a, b):
                x.cache.release(x.rows, x.refs, keep=ints(torch, [9999, 0, 9999, 0, 9999]))
                x.lengths[[1, 3]] = 0
        a.fill(i)
        b.fill(i)
        context = b.cache.k_codes[0].clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b.step()
        x, y = a.state(), b.state()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(x, y)), i
        assert torch.equal(a.cache.k_codes[0], context)        # the context's page: nobody's to write
        shorts.append(int(a.missing) > 0)
        assert (int(a.granted.sum()) == 0) == shorts[-1]
    assert not shorts[0] and shorts[5] and not shorts[6]


def test_answers_that_run_out_of_pages():
    torch_cuda()
    from paper_2310_07240_amd import serving
    w = W.small(name="answers", n_ctx=2, n_layers=3, n_tokens=300, n_channels=256, chunk_len=128)
    # a page for each of 30 requests at first, which holds some steps; then some want a second one
    r = serving.answer(w, kv_heads=4, q_heads=8, requests=5, drafts=3, steps=14, vocab=500, spare=32)
    say(r)
    assert r["missing"] > 0 and r["accepted"] > 0
    assert r["pages"]["after"] == r["pages"]["contexts"] == 6 * 5
    assert r["rel_error_8bit"] < 0.05 and r["rel_error_after"] < 0.05
    # none from the first step on: nobody writes to a context
    r = serving.answer(w, kv_heads=4, q_heads=8, requests=5, drafts=3, steps=3, vocab=500, spare=29)
    assert r["missing"] == 1 and r["accepted"] == 0 and r["pages"]["used"] == 30
    assert r["rel_error_after"] < 0.05
