"""GPU: contexts read by unequal numbers of requests, with a bound that leaves room for all of them at
each (the default of max_users), against the definition in 64 bits; bounds as in
tests/test_gpu_kv8_shared.py."""
import numpy as np
import pytest

from gpu_helpers import torch_cuda
from test_gpu_kv8 import ints, make
from test_gpu_kv8_shared import check

pytestmark = pytest.mark.gpu


def uneven(rng, C, most, heavy=0):
    """Requests of each context, one of them with many, some with none."""
    users = rng.integers(0, most + 1, C)
    users[rng.integers(C)] = 0
    if heavy:
        users[rng.integers(C)] = heavy
    return [int(x) for x in users]


def ends(users, before=0):
    return [before] + [before + int(x) for x in np.cumsum(users)]


@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("H,group,D,Q", [(2, 4, 128, 1), (3, 1, 64, 3), (1, 8, 256, 2), (2, 5, 64, 1)])
def test_few_contexts(H, group, D, Q, own):
    users = [1, 30, 0, 2, 1, 1, 50, 0, 3, 1, 1, 7]
    tokens = [70, 300, 64, 1, 0, 129, 500, 64, 65, 200, 30, 128]
    firsts = ends(users, before=2)                         # (two without a context, and three behind)
    n = firsts[-1] + 3
    lengths = [Q + (7 * i) % 150 for i in range(n)] if own else None
    check(H, group, D, "float16" if D == 128 else "bfloat16", tokens, firsts, n, lengths,
          [1 + i % Q for i in range(n)], Q, seed=D)


@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("H,group,D", [(2, 24, 64), (1, 2, 128), (2, 12, 256)])
def test_more_contexts_than_a_wave_looks_at(H, group, D, own):
    """Of few rows each and of some, in one tile of a workgroup and in several."""
    rng = np.random.default_rng(D)
    users = uneven(rng, 150, 3, heavy=40)
    n = sum(users)
    tokens = [int(x) for x in rng.integers(0, 130, 150)]
    check(H, group, D, "float16", tokens, ends(users), n,
          [1 + i % 70 for i in range(n)] if own else None, seed=D + 1)


def test_thousands_of_contexts():
    rng = np.random.default_rng(9)
    users = uneven(rng, 5000, 1, heavy=9)
    n = sum(users)
    check(1, 1, 64, "float16", [int(x) for x in rng.integers(0, 66, 5000)], ends(users), n,
          [1 + i % 3 for i in range(n)], seed=10)


@pytest.mark.parametrize("own", [True, False])
def test_splits_of_uneven_contexts(own):
    """Long contexts in splits: few rows (joined by the last to come, in the contexts' own launch) and
    many, in tiles of half and of all of a workgroup's waves."""
    for seed, (H, group, D, users, tokens) in enumerate((
            (1, 2, 128, [1, 0, 9], [3000, 50, 2000]),
            (8, 4, 64, [30, 1, 0, 1, 40], [2500, 2000, 3000, 2100, 1300]),
            (4, 4, 256, [60, 1, 2], [1500, 1000, 1100]),
            (32, 8, 64, [170, 1, 1, 40], [256, 256, 70, 200]))):
        n = sum(users)
        check(H, group, D, "bfloat16", tokens, ends(users), n, [2 + i % 60 for i in range(n)]
              if own else None, seed=30 + seed)


@pytest.mark.parametrize("own", [True, False])
def test_bounds_below_some_contexts_requests(own):
    """More room than there are requests, and still less than some contexts have: those behind see none."""
    users = [12, 0, 1, 8, 5, 1, 1, 2, 0, 9]
    n = sum(users) + 1
    for most in (5, 8):
        check(2, 4, 64, "float16", [150 + i for i in range(10)], ends(users), n,
              [3 + i for i in range(n)] if own else None, max_users=most, seed=most)


def test_long_own_tokens_behind_uneven_contexts():
    users = [3, 1, 0, 20]
    n = sum(users)
    own = [1100] + [9] * (n - 1)
    check(1, 2, 128, "float16", [300, 64, 70, 100], ends(users), n, own, seed=40)
    check(1, 1, 64, "float16", [300, 64, 70, 100], ends(users), n, [900] + [90] * (n - 1), None, 80,
          seed=41)


@pytest.mark.parametrize("H,group", [(1, 2), (8, 64)])
@pytest.mark.parametrize("own", [True, False])
def test_firsts_in_no_order(H, group, own):
    """Only rows that exist are read and written, by either kernel."""
    torch = torch_cuda()
    rng = np.random.default_rng(3)
    n, C = 20, 30
    cache = make(torch, C + n, H, 64)
    q = torch.randn(n, 1, H * group, 64, device="cuda").half()
    around = torch.full((n + 2, 1, H * group, 64), 7.0, device="cuda").half()
    lse = torch.full((n + 2, 1, H * group), 7.0, device="cuda")
    more = {"table": ints(torch, [[C + i] for i in range(n)]), "lengths": ints(torch, [3] * n)} if own else {}
    for _ in range(20):
        firsts = rng.integers(-5, n + 6, C + 1).tolist()
        cache.attend_shared(q, ints(torch, [[i] for i in range(C)]), ints(torch, [60] * C),
                            ints(torch, firsts), out=around[1:-1], lse=lse[1:-1], **more)
        torch.cuda.synchronize()
        assert bool((around[[0, -1]] == 7).all()) and bool((lse[[0, -1]] == 7).all())


@pytest.mark.parametrize("C,Q,H,group,tokens", [(64, 448, 16, 1, 64), (420, 6, 8, 4, 200), (48, 1, 8, 4, 900)])
def test_contexts_of_a_request_each(C, Q, H, group, tokens):
    """Cross attention of a batch: without the bound, what it gives with the exact one. (The splits may be
    others. Both round weights to fp16, 2^-11 of them, and the output by half a step, 2^-11 of it: of
    the largest |V|, 4 2^-11 between them.)"""
    torch = torch_cuda()
    pages = -(-tokens // 64)
    cache = make(torch, C * pages, H, 64)
    q = torch.randn(C, Q, H * group, 64, device="cuda").half()
    args = (q, torch.arange(C * pages, dtype=torch.int32, device="cuda").view(C, pages),
            ints(torch, [tokens - i % 50 for i in range(C)]), ints(torch, list(range(C + 1))))
    a, b = cache.attend_shared(*args), cache.attend_shared(*args, max_users=1)
    off = (a.float() - b.float()).abs().max()
    assert float(off) <= 4 * 2.0 ** -11 * 127 * float(cache.v_scale.max())
    assert bool((a != 0).any())


@pytest.mark.parametrize("H,group,D,tokens,users,Q", [
    (1, 2, 64, 64, [1], 1), (3, 2, 128, 1200, [2, 1], 2), (8, 16, 64, 1000, [60], 1),
    (32, 8, 64, 256, [30, 200], 1), (2, 8, 256, 700, [70], 1),
])
def test_many_requests_without_a_context(H, group, D, tokens, users, Q):
    """In front of the first context's, behind the bound of each, and behind the last: zeros and -inf, and
    the others are what they are without them."""
    torch = torch_cuda()
    pages = -(-tokens // 64)
    cache = make(torch, len(users) * pages, H, D)
    firsts = [40] + [40 + 50 * (i + 1) + sum(users[:i + 1]) for i in range(len(users))]
    n, most = firsts[-1] + 333, max(users)
    q = torch.randn(n, Q, H * group, D, device="cuda").half()
    out, lse = torch.full_like(q, 7.0), torch.full((n, Q, H * group), 7.0, device="cuda")
    shared = torch.arange(len(users) * pages, dtype=torch.int32, device="cuda").view(len(users), pages)
    args = shared, ints(torch, [tokens] * len(users))
    cache.attend_shared(q, *args, ints(torch, firsts), out=out, lse=lse, max_users=most)
    has = torch.zeros(n, dtype=torch.bool, device="cuda")
    for a, b in zip(firsts, firsts[1:]):
        has[a:min(b, a + most)] = True
    assert bool((out[~has] == 0).all()) and bool((lse[~has] == -float("inf")).all())
    inner = [0]
    for a, b in zip(firsts, firsts[1:]):
        inner.append(inner[-1] + min(b - a, most))
    same = torch.empty_like(q[has])
    other = torch.empty_like(lse[has])
    cache.attend_shared(q[has].contiguous(), *args, ints(torch, inner), out=same, lse=other,
                        max_users=most)
    # (both off by 2^-11 of a weight and half a step of the output, as above)
    off = (out[has].float() - same.float()).abs().max()
    assert float(off) <= 4 * 2.0 ** -11 * 127 * float(cache.v_scale.max())
    assert bool(lse[has].isfinite().all())
