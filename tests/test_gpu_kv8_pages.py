"""GPU: pages of the 8-bit cache that sequences share, get, give back, copy and move, against the
definitions in Python (tests/sharing_reference.py). Everything is whole numbers and copies: every
buffer is compared bit for bit, what no call may touch included."""
import numpy as np
import pytest

import sharing_reference as S
from gpu_helpers import say, torch_cuda
from test_gpu_kv8 import ints, make

pytestmark = pytest.mark.gpu
PAGE = 64
BUFFERS = ("k_codes", "v_codes", "k_scale", "v_scale", "k_bounds")


class Pool:
    """A cache with random pages, sequences in some of them, and host copies of it all."""

    def __init__(self, torch, rng, P, H, D, bounds=True, mass=True):
        self.cache = make(torch, P, H, D, bounds)
        self.mass = torch.rand((P, H, PAGE), device="cuda") if mass else None
        self.P = P
        self.host = {k: getattr(self.cache, k).cpu() for k in BUFFERS
                     if getattr(self.cache, k) is not None}
        if mass:
            self.host["mass"] = self.mass.cpu()

    def copied(self, copies):
        """The host's pages after copies (from, to) that were all read first."""
        for x in self.host.values():
            x[[b for _, b in copies]] = x[[a for a, _ in copies]].clone()

    def same(self):
        for k, x in self.host.items():
            got = (self.mass if k == "mass" else getattr(self.cache, k)).cpu()
            bad = (got != x).flatten(1).any(1).nonzero().flatten().tolist()
            assert not bad, (k, bad[:10])


def rows_of(rng, P, lengths, width, used=None):
    """A table with pages in no order for lengths, and the pages' counts."""
    order = list(rng.permutation(P))
    table = [[-1] * width for _ in lengths]
    refs = [0] * P
    for row, n in zip(table, lengths):
        for j in range(S.pages_of(n)):
            row[j] = int(order.pop())
            refs[row[j]] = 1
    return table, refs


def tensors(torch, *lists):
    return [torch.tensor(x, dtype=torch.int32, device="cuda") for x in lists]


def equal(name, got, want):
    got = got.cpu().numpy()
    assert np.array_equal(got, np.asarray(want, np.int32)), (name, got.tolist(), want)


@pytest.mark.parametrize("P,H,D,lengths,width,children,ends", [
    (64, 2, 64, [100, 640, 1, 0], 12, [0, 0, 1, 3, 2, 1, 9, -1], None),
    (300, 1, 128, [64, 1000, 128], 16, [1] * 40 + [0, 2], None),
    (300, 1, 128, [64, 1000, 5000], 16, [2, 1, 1, 0, 1, 1], [900, 65, 64, 63, 0, -5]),
    (40, 3, 256, [700], 300, [0] * 3, [4000, 700, 1]),
])
def test_fork(P, H, D, lengths, width, children, ends):
    torch = torch_cuda()
    rng = np.random.default_rng(P + H)
    pool = Pool(torch, rng, P, H, D)
    table, refs = rows_of(rng, P, [min(n, width * PAGE) for n in lengths], width)
    table[0][0] = P + 3                             # lost pages are nobody's
    if len(lengths) > 1:
        table[1][0] = -7
    t, r = tensors(torch, table, refs)
    new_width = width + 3
    to = torch.full((len(children) + 2, new_width), 77, dtype=torch.int32, device="cuda")
    got, got_n = pool.cache.fork(t, ints(torch, lengths), ints(torch, children), r,
                                 ends=None if ends is None else ints(torch, ends),
                                 new_table=to[1:-1])
    want, want_n, want_refs = S.fork(table, lengths, children, refs, P, new_width, ends)
    equal("table", got, want)
    equal("lengths", got_n, want_n)
    equal("refs", r, want_refs)
    equal("parents", t, table)
    assert bool((to[[0, -1]] == 77).all())
    pool.same()


@pytest.mark.parametrize("keep", [None, [0, 64, 65, 100000], [1, -3, 639, 64]])
def test_release(keep):
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    P = 70
    table, refs = rows_of(rng, P, [640, 640, 640, 70], 10)
    table[1][1:5] = table[0][1:5]                    # shared, and one that a row names twice
    table[3][2] = table[3][0]
    for p in table[0][1:5] + [table[3][0]]:
        refs[p] += 1
    refs[table[2][9]] = 0                            # a count that is 0 stays 0
    table[2][3], table[0][7] = P, -9
    t, r = tensors(torch, table, refs)
    cache = make(torch, P, 1, 64)
    cache.release(t, r, keep=None if keep is None else ints(torch, keep))
    want, want_refs = S.release(table, refs, P, keep)
    equal("table", t, want)
    equal("refs", r, want_refs)


RESERVE = [
    # P, H, D, parents' lengths, children of each, width, counts, mass, bounds
    (200, 2, 128, [100, 640, 1], 3, 14, [1, 64, 200, 0, 27, 28, 65, -4, 3], True, True),
    (64, 1, 64, [63, 64, 65, 0], 1, 4, [1, 1, 1, 1], False, True),
    (500, 3, 256, [1000], 20, 20, [1] * 20, True, False),
    (4096, 1, 64, [8000, 1], 2, 130, [130, 8000, 300, 1], True, True),
    (9000, 1, 64, [70, 700], 5, 120, [5000] * 10, False, True),
    (13000, 1, 64, [12000, 77], 4, 200, [1, 1, 2000, 5, 1, 1, 1, 1], True, True),
    # more sequences than one workgroup plans for, and more pages
    (6000, 1, 64, [70], 2100, 3, [1, 60] * 1050, False, True),
    (6000, 1, 64, [70, 5], 1000, 5, [1, 60] * 1000, False, True),
    (65536, 1, 64, [3000, 64], 5, 60, [700] * 10, False, False),
    (65537, 1, 64, [3000, 64], 5, 60, [700] * 10, True, False),
]


@pytest.mark.parametrize("P,H,D,lengths,children,width,counts,mass,bounds", RESERVE)
def test_reserve(P, H, D, lengths, children, width, counts, mass, bounds):
    """Children of shared contexts get copies and pages; then more, behind what they have got."""
    torch = torch_cuda()
    rng = np.random.default_rng(P + width)
    pool = Pool(torch, rng, P, H, D, bounds, mass)
    table, refs = rows_of(rng, P, lengths, width)
    parents = [i for i in range(len(lengths)) for _ in range(children)]
    rows, n, refs = S.fork(table, lengths, parents, refs, P, width)
    rows[0][-1] = P + 5                              # behind everything: replaced if it is reached
    t, r = tensors(torch, rows, refs)
    for step in range(3):
        say(f"step {step}")
        rows, refs, missing, copies = S.reserve(rows, n, counts, refs, P)
        got = pool.cache.reserve(t, ints(torch, n), ints(torch, counts), r, mass=pool.mass)
        pool.copied(copies)
        equal("missing", got, [missing])
        equal("table", t, rows)
        equal("refs", r, refs)
        pool.same()
        if not missing:
            n = [S.clip(a + max(0, c), width) for a, c in zip(n, counts)]


def test_reserve_more_than_there_is():
    """Nothing changes where pages are missing, also where only one is; then the last one goes."""
    torch = torch_cuda()
    rng = np.random.default_rng(3)
    for P, need in ((40, 40), (40, 41), (40, 400), (16385, 16385), (16385, 16500), (16500, 16499)):
        pool = Pool(torch, rng, P, 1, 64)
        width = need + 1
        table, refs = [[-1] * width, [-1] * width], [0] * P
        t, r = tensors(torch, table, refs)
        counts = [64 * (need - 3), 64 * 3 - 10]
        rows, after, missing, _ = S.reserve(table, [0, 0], counts, refs, P)
        got = pool.cache.reserve(t, ints(torch, [0, 0]), ints(torch, counts), r)
        equal("missing", got, [missing])
        assert missing == max(0, need - P)
        equal("table", t, rows)
        equal("refs", r, after)
        pool.same()


def test_reserve_counts_that_do_not_match():
    """Rows that name pages which nobody or somebody else holds, pages named twice, negative
    counts: the definition's answer, and nobody's page is handed out twice."""
    torch = torch_cuda()
    rng = np.random.default_rng(11)
    for case in range(20):
        P, B, width = 60, 6, 8
        pool = Pool(torch, rng, P, 1, 64)
        table = rng.integers(-3, P + 3, (B, width)).tolist()
        # (a count below the rows' that drop the page would depend on who asks first for what is
        # free: pages that rows name behind their tokens are counted at least as often)
        refs = rng.integers(-1, 3, P).tolist()
        n = rng.integers(-5, width * PAGE + 50, B).tolist()
        counts = rng.integers(-5, 200, B).tolist()
        t, r = tensors(torch, table, refs)
        rows, after, missing, copies = S.reserve(table, n, counts, refs, P)
        got = pool.cache.reserve(t, ints(torch, n), ints(torch, counts), r, mass=pool.mass)
        pool.copied(copies)
        equal("missing", got, [missing])
        equal("table", t, rows)
        equal("refs", r, after)
        pool.same()


@pytest.mark.parametrize("P,H,D,mass,bounds", [(64, 1, 64, True, True), (50, 5, 64, False, True),
                                               (40, 3, 128, True, False), (30, 2, 256, True, True)])
def test_copy(P, H, D, mass, bounds):
    torch = torch_cuda()
    rng = np.random.default_rng(P)
    pool = Pool(torch, rng, P, H, D, bounds, mass)
    order = rng.permutation(P).tolist()
    src, dst = order[:P // 3], order[P // 3:2 * (P // 3)]
    src[0], dst[1], src[2] = -1, P, P + 9            # pairs outside the pool
    dst[3] = src[3]                                  # a page onto itself
    src[5] = src[4]                                  # one to two
    pool.cache.copy(ints(torch, src), ints(torch, dst), mass=pool.mass)
    pool.copied([(a, b) for a, b in zip(src, dst) if 0 <= a < P and 0 <= b < P])
    pool.same()
    pool.cache.copy(ints(torch, []), ints(torch, []))


@pytest.mark.parametrize("P,H,D", [(1, 1, 64), (63, 2, 128), (4096, 1, 64), (4097, 1, 64),
                                   (16384, 1, 64), (16385, 1, 64), (21000, 1, 64)])
@pytest.mark.parametrize("live", [0.0, 0.1, 0.5, 0.97, 1.0])
def test_compact(P, H, D, live):
    torch = torch_cuda()
    rng = np.random.default_rng(P + int(100 * live))
    pool = Pool(torch, rng, P, H, D, mass=P < 5000)
    refs = np.where(rng.random(P) < live, rng.integers(1, 4, P), rng.integers(-1, 1, P)).tolist()
    table = rng.integers(-2, P + 2, (5, 70)).tolist()
    t, r = tensors(torch, table, refs)
    rows, after, moved, n, copies = S.compact(table, refs, P)
    got = pool.cache.compact(t, r, mass=pool.mass)
    pool.copied(copies)
    for name, a, b in zip(("table", "refs", "moved", "live"), got, (rows, after, moved, [n])):
        equal(name, a, b)
    equal("old table", t, table)
    equal("old refs", r, refs)
    pool.same()
    # once more: nothing is left to do
    again = pool.cache.compact(got[0], got[1], mass=pool.mass)
    equal("table again", again[0], rows)
    equal("refs again", again[1], after)
    pool.same()
