"""GPU: pages that go from one sequence to another, and the weights that stand in them."""
import numpy as np
import pytest

from gpu_helpers import assert_same, say, torch_cuda
from test_gpu_kv8 import PAGE, ints, make, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,H,T,starts,counts", [
    (64, 3, 1, [0, 1, 63, 64, 127, 5], [1, 1, 1, 1, 1, 0]),
    (128, 2, 150, [0, 70, 64], [150, 150, 3]),
    (256, 1, 65, [1, 62], None),
    (64, 32, 2200, [37, 64], None),            # new and kept pages in launches of their own
])
def test_store_clears_weights(D, H, T, starts, counts):
    """From a page's first new row on, and nothing else."""
    torch = torch_cuda()
    rng = np.random.default_rng(T)
    B = len(starts)
    t, table, n = tables(torch, rng, B, (max(starts) + T) // PAGE + 1)
    cache = make(torch, n, H, D)
    k = torch.randn(B, T, H, D).half().cuda()
    mass = torch.full((n, H, PAGE), float("nan"), device="cuda")
    mass[torch.rand(mass.shape, device="cuda") < 0.5] = 3.0
    want = mass.cpu().numpy().copy()
    cnt = [T] * B if counts is None else counts
    for b in range(B):
        if cnt[b] > 0:
            for j in range(starts[b] // PAGE, (starts[b] + cnt[b] - 1) // PAGE + 1):
                want[t[b, j], :, max(0, starts[b] - j * PAGE):] = 0
    say(f"store {D} {H} {T} with weights")
    args = (k, k, table, ints(torch, starts), None if counts is None else ints(torch, counts))
    cache.store(*args, mass=mass)
    assert_same("weights", mass.cpu().numpy().view(np.int32), want.view(np.int32))
    codes = [x.clone() for x in (cache.k_codes, cache.v_codes, cache.k_scale)]
    cache.store(*args)
    assert all(torch.equal(a, b) for a, b in zip(codes, (cache.k_codes, cache.v_codes,
                                                         cache.k_scale)))


def test_a_reused_page_evicts_as_a_fresh_one():
    """A sequence in pages that another one left its weights in keeps the tokens that it would keep
    in new pages."""
    torch = torch_cuda()
    H, D, T, keep = 2, 64, 300, 100
    width, new = -(-(T + 4) // PAGE), -(-keep // PAGE)
    n = width + new
    table = torch.arange(width, dtype=torch.int32, device="cuda")[None]
    to = torch.arange(width, n, dtype=torch.int32, device="cuda")[None]
    k, v = (torch.randn(1, T, H, D).half().cuda() for _ in range(2))
    rows = [tuple(torch.randn(1, 1, h, D).half().cuda() for h in (H, H, 4 * H)) for _ in range(4)]

    def serve(mass):
        cache = make(torch, n, H, D)
        cache.store(k, v, table, ints(torch, [0]), mass=mass)
        for i, (kn, vn, q) in enumerate(rows):
            cache.store(kn, vn, table, ints(torch, [T + i]), mass=mass)
            cache.attend(q, table, ints(torch, [T + i + 1]), mass=mass, decay=0.9)
        kept, _ = cache.evict(table, ints(torch, [T + 4]), mass, keep, 4, to)
        return kept.clone(), mass[to[0].long()].clone()

    fresh = serve(torch.zeros((n, H, PAGE), device="cuda"))
    left = torch.rand((n, H, PAGE), device="cuda") * 50
    left[0, 0, 3] = float("inf")
    left[1, 1, 7] = float("nan")
    again = serve(left)
    assert torch.equal(fresh[0], again[0]) and torch.equal(fresh[1], again[1])
