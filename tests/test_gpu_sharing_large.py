"""GPU: requests that share a context where offsets pass 32 bits: pools of more than 4 GiB of codes,
and rows that lie further apart than 2^31 elements. Each is compared with the same call where all is
small, bit for bit."""
import numpy as np
import pytest

import sharing_reference as S
from gpu_helpers import torch_cuda
from test_gpu_kv8 import ints, make

pytestmark = pytest.mark.gpu
PAGE = 64
P, H, D = 70000, 8, 128                       # 4.6 GB of K codes, and of V's


def large_pool(torch, pages):
    """A small cache, and a large one that holds its pages at the numbers `pages`."""
    from paper_2310_07240_amd.kv8 import Kv8Cache
    small = make(torch, len(pages), H, D)
    at = torch.tensor(pages, device="cuda")
    buffers = {}
    for k in ("k_codes", "v_codes", "k_scale", "v_scale", "k_bounds"):
        x = getattr(small, k)
        buffers[k] = torch.empty((P,) + tuple(x.shape[1:]), dtype=x.dtype, device="cuda")
        buffers[k][at] = x
    return small, Kv8Cache(P, H, D, buffers=buffers)


def same_pages(small, large, pairs):
    """Pages (of the small cache, of the large one) hold the same."""
    for k in ("k_codes", "v_codes", "k_scale", "v_scale", "k_bounds"):
        for i, j in pairs:
            assert bool((getattr(small, k)[i] == getattr(large, k)[j]).all()), (k, i, j)


def test_pages_behind_4_gib():
    torch = torch_cuda()
    pages = [69999, 3, 66001, 40000, 69000, 65990]
    small, large = large_pool(torch, pages)
    # copies up and down
    large.copy(ints(torch, [69999, 3]), ints(torch, [5, 69998]))
    same_pages(small, large, [(0, 5), (1, 69998)])
    # a copy on write to the lowest free page, and one high up
    refs = torch.ones(P, dtype=torch.int32, device="cuda")
    refs[66001] = 3
    refs[[7, 69500]] = 0
    table = ints(torch, [[66001, -1], [66001, -1], [66001, 69000]])
    missing = large.reserve(table, ints(torch, [10, 20, 70]), ints(torch, [1, 2, 3]), refs)
    assert missing.tolist() == [0]
    assert table.tolist() == [[7, -1], [69500, -1], [66001, 69000]]
    assert refs[[7, 69500, 66001, 69000]].tolist() == [1, 1, 1, 1]
    same_pages(small, large, [(2, 7), (2, 69500), (2, 66001)])
    missing = large.reserve(table, ints(torch, [64, 0, 70]), ints(torch, [1, 2, 3]), refs)
    assert missing.tolist() == [1]
    # the used ones to the front
    refs.zero_()
    refs[ints(torch, pages).long()] = 1
    table = ints(torch, [pages])
    new_table, new_refs, moved, live = large.compact(table, refs)
    rows, after, to, _, _ = S.compact([pages], refs.tolist(), P)
    assert new_table.tolist() == rows and live.tolist() == [6]
    assert new_refs.tolist() == after and moved.tolist() == to
    same_pages(small, large, list(enumerate(new_table[0].tolist())))


@pytest.mark.parametrize("users", [3, 40])
def test_attention_behind_4_gib(users):
    torch = torch_cuda()
    pages = [69999, 3, 66001, 40000] + list(range(69000, 69000 + users))
    small, large = large_pool(torch, pages)
    q = torch.randn(users, 2, 2 * H, D, device="cuda").half()
    first = ints(torch, [0, users])
    outs = []
    for cache, name in ((small, list(range(len(pages)))), (large, pages)):
        outs.append(cache.attend_shared(
            q, ints(torch, [name[:4]]), ints(torch, [230]), first,
            table=ints(torch, [[x] for x in name[4:]]), lengths=ints(torch, [5] * users)))
        outs.append(cache.attend_shared(q, ints(torch, [name[:4]]), ints(torch, [230]), first))
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
    assert not torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("users", [3, 40])
def test_queries_far_apart(users):
    """Sequences' rows 2^31 elements apart and more, queries and results."""
    torch = torch_cuda()
    cache = make(torch, 6 + users, 1, 64)
    gap = (1 << 31) // (users - 2)             # the last sequence lies behind 2^31 elements
    room = torch.zeros(gap * users, dtype=torch.float16, device="cuda")
    far = room.as_strided((users, 2, 2, 64), (gap, 128, 64, 1))
    q = torch.randn(users, 2, 2, 64, device="cuda").half()
    far.copy_(q)
    out = room.as_strided((users, 2, 2, 64), (gap, 128, 64, 1), 4096)
    args = ints(torch, [[0, 1, 2, 3, 4]]), ints(torch, [300]), ints(torch, [0, users])
    for more in ({}, {"table": ints(torch, [[5 + i] for i in range(users)]),
                      "lengths": ints(torch, [9] * users)}):
        want = cache.attend_shared(q, *args, **more)
        out.zero_()
        cache.attend_shared(far, *args, out=out, **more)
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_probabilities_far_apart(dtype):
    torch = torch_cuda()
    n, k, vocab = 4, 2, 5000
    gap = (1 << 30) + 12345
    room = torch.empty(gap * n, dtype=getattr(torch, dtype), device="cuda")
    target = torch.softmax(2 * torch.randn(n, k + 1, vocab, device="cuda"), -1).to(room.dtype)
    draft = torch.softmax(2 * torch.randn(n, k, vocab, device="cuda"), -1).to(room.dtype)
    far_t = room.as_strided((n, k + 1, vocab), (gap, vocab + 1, 1))
    far_d = room.as_strided((n, k, vocab), (gap, vocab + 3, 1), 100000)
    far_t.copy_(target)
    far_d.copy_(draft)
    rng = np.random.default_rng(3)
    drafts = ints(torch, rng.integers(0, vocab, (n, k)).tolist())
    u = torch.rand((n, k + 1), device="cuda")
    cache = make(torch, 1, 1, 64)
    near, far = cache.verify(target, drafts, u, draft=draft), cache.verify(far_t, drafts, u, draft=far_d)
    assert torch.equal(near[0], far[0]) and torch.equal(near[1], far[1])
