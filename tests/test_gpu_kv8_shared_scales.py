"""GPU: attention over shared contexts where V scales are so large that a sum of values which are not
yet divided by the sum of weights would pass 32 bits, although every result is a finite number. The
bounds are those of tests/test_gpu_kv8_shared.py, which follow the size of the values."""
import pytest

from gpu_helpers import torch_cuda
from test_gpu_kv8_shared import check

pytestmark = pytest.mark.gpu


def large(scale, own_scale):
    def spoil(cache, shared, table):
        cache.v_scale[sorted(set(shared.ravel().tolist()) - {-1})] = scale
        if table is not None:
            cache.v_scale[sorted(set(table.ravel().tolist()) - {-1})] = own_scale
        cache.k_scale.mul_(0.01)                   # (weights alike: all tokens add up)
    return spoil


# few rows; those of half of a workgroup's waves, in one split and in several; those of all waves
@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("H,group,D,tokens,users", [
    (1, 2, 128, 256, 3), (1, 2, 128, 256, 40),
    (8, 8, 128, 250, 136), (8, 4, 128, 8192, 12), (8, 1, 64, 5000, 200), (32, 8, 64, 256, 300),
    (2, 8, 256, 1024, 130), (1, 8, 256, 4096, 40),
])
def test_v_scales_near_the_largest_numbers(H, group, D, tokens, users, own):
    torch_cuda()
    # (127 times 1e33 is 1.3e35; 8192 of those, the most that attend_kernel's and the own tokens' sums
    # of weights up to 1 take, pass 3.4e38, so long contexts have smaller ones)
    scale = 1e33 if tokens <= 1024 else 1e32
    out, _ = check(H, group, D, "bfloat16", [tokens], [0, users], users, [3] * users if own else None,
                   seed=D + users, spoil=large(scale, scale if users % 8 else 1e-3))
    assert bool(out.isfinite().all())


@pytest.mark.parametrize("H,D,context,own,Q", [(1, 64, 100, 1500, 80), (2, 128, 300, 2500, 1),
                                               (1, 128, 300, 6400, 300)])
def test_own_tokens_of_large_scales(H, D, context, own, Q):
    """Own tokens in splits, of few rows and of many, large beside a context that is not, and the other
    way round."""
    torch_cuda()
    for scales in ((1e32, 1e32), (1e-3, 1e32), (1e32, 1e-3)):
        out, _ = check(H, 1, D, "bfloat16", [context], [0, 2], 2, [own, 70 + Q], None, Q, seed=D + Q,
                       spoil=large(*scales))
        assert bool(out.isfinite().all())
