"""GPU: two threads whose calls go through one cache's scratch on one stream; what each of them does is
compared with an eager twin's, bit for bit."""
import threading

import pytest

from gpu_helpers import torch_cuda
from test_gpu_sharing_graphs import Requests, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("big", [False, True])
def test_both_threads(big):
    torch = torch_cuda()
    pairs = [(Requests(torch, seed, big=big), Requests(torch, seed, big=big)) for seed in (8, 9)]
    a, b = pairs[0][0], pairs[1][0]
    b.cache._ws, b.cache._lock = a.cache._ws, a.cache._lock    # as of one cache
    for i, pair in enumerate(pairs):
        for x in pair:
            x.fill(20 + i)
    torch.cuda.synchronize()
    errors = []

    def many(x, n):
        try:
            for _ in range(n):
                x.step()
        except Exception as e:                     # pragma: no cover
            errors.append(e)
    threads = [threading.Thread(target=many, args=(x, 6)) for x in (a, b)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for (x, twin), name in zip(pairs, "ab"):
        many(twin, 6)
        torch.cuda.synchronize()
        same(torch, x, twin, name)
    assert not errors
