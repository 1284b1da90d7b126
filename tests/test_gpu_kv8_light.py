"""GPU: attention of many rows where the heaviest token has nothing in half of the channels, so that
light weights are all there is in them, and where V is small.

Bound: a weight goes to fp16 at 2^11 times the heaviest so far or more, so it is off by 2^-11 of
itself or, below fp16's normal numbers, by half a step, 2^-25 / 2^11 of the heaviest; sums in 32 bits
and the rounding of the exponential fit in as much again as the 2^-11. The result is rounded to its
type, whose subnormals are 2^-133 apart for bf16 and 2^-24 for fp16."""
import numpy as np
import pytest

import kv8_reference as R
from gpu_helpers import say, torch_cuda
from test_gpu_kv8 import UNIT, ints, make, much_room, tables

pytestmark = pytest.mark.gpu


def light_cache(torch, t, n, D, vs, steps=(19, 10, 1)):
    """One token a page above the others, by as many logits as `steps` says, without V in half of
    the channels."""
    cache = make(torch, n, 1, D)
    cache.k_codes.zero_()
    for j, s in enumerate(steps):
        cache.k_codes[int(t[0, j]), 0, 7, :] = s
        cache.v_codes[int(t[0, j]), 0, ::2, 7] = 0
    cache.k_scale.fill_(1.0)
    cache.v_scale.fill_(vs)
    return cache


def close(cache, out, q, t, length, kind):
    """One head of the first sequence against the definition (all have the same queries)."""
    want, _, _, size, _ = R.attend(R.Ref(cache), q[:1, :, :1].float().cpu().numpy(), t[:1], [length],
                                   [q.shape[1]], 1.0)
    got = out[:1, :, :1].float().cpu().numpy()
    v = R.Ref(cache).rows(t[:1], 0, 0, length)[1]
    small = 2.0 ** -134 if kind == "bfloat16" else 2.0 ** -25
    lim = UNIT[kind] * np.abs(want) + 2.0 ** -10 * size + 2.0 ** -36 * np.abs(v).sum(0) + small
    err = np.abs(got - want)
    say("worst", float((err / lim).max()))
    assert (err <= lim).all()
    assert bool((out == out[:1, :, :1]).all())


@pytest.mark.parametrize("vs,kind", [(1e-20, "bfloat16"), (1.0, "bfloat16"), (200.0, "float16")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_light_weights_of_split_prompts(D, vs, kind):
    """A page a split."""
    torch = torch_cuda()
    rng = np.random.default_rng(D)
    t, _, n = tables(torch, rng, 1, 3)
    cache = light_cache(torch, t, n, D, vs)
    t, table = much_room(torch, t)
    q = torch.full((1, 60, 3, D), 1 / D, dtype=getattr(torch, kind), device="cuda")
    out = cache.attend(q, table, ints(torch, [192]), scale=1.0)
    close(cache, out, q, t, 192, kind)


@pytest.mark.parametrize("vs,kind", [(1e-20, "bfloat16"), (200.0, "float16")])
@pytest.mark.parametrize("D,steps", [(64, (19, 10, 1)), (128, (19, 10, 1)), (128, (1, 10, 19)),
                                     (256, (5, 19, 10))])
def test_light_weights_of_whole_prompts(D, steps, vs, kind):
    """So many workgroups that no prompt is split: one reference goes through all of its pages,
    whichever holds the heaviest token."""
    torch = torch_cuda()
    rng = np.random.default_rng(D)
    t, _, n = tables(torch, rng, 1, 3)
    cache = light_cache(torch, t, n, D, vs, steps)
    t = np.repeat(t, 40, 0)
    q = torch.full((40, 100, 16, D), 1 / D, dtype=getattr(torch, kind), device="cuda")
    out = cache.attend(q, torch.from_numpy(t).cuda(), ints(torch, [192] * 40), scale=1.0)
    close(cache, out, q, t, 192, kind)


@pytest.mark.parametrize("vs", [1e-30, 1e-33, 1e-36])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("split", [True, False])
def test_tiny_values_of_prompts(D, vs, split):
    """V scales that bf16 results hold and that are far below 1."""
    torch = torch_cuda()
    rng = np.random.default_rng(D)
    t, _, n = tables(torch, rng, 1, 3)
    cache = light_cache(torch, t, n, D, vs, (6, 10, 1))
    B = 1 if split else 40
    if split:
        t, table = much_room(torch, t)
    else:
        t = np.repeat(t, B, 0)
        table = torch.from_numpy(t).cuda()
    q = torch.full((B, 100, 16, D), 1 / D, device="cuda").bfloat16()
    lse = torch.empty((B, 100, 16), device="cuda")
    out = cache.attend(q, table, ints(torch, [192] * B), scale=1.0, lse=lse)
    close(cache, out, q, t, 192, "bfloat16")
    want = R.attend(R.Ref(cache), q[:1, :, :1].float().cpu().numpy(), t[:1], [192], [100], 1.0)[1]
    assert np.abs(lse[:1, :, :1].cpu().numpy() - want).max() <= 1e-4


def test_tiny_values_beside_ordinary_ones():
    """Pages of V scales from 1e-36 to 1 in one prompt, in both orders."""
    torch = torch_cuda()
    for scales in ((1e-36, 1e-20, 1.0), (1.0, 1e-10, 1e-36), (0.0, 1e-36, 0.0), (1e-36, 0.0, 1e-14)):
        rng = np.random.default_rng(3)
        t, _, n = tables(torch, rng, 1, 3)
        cache = light_cache(torch, t, n, 64, 1.0, (3, 5, 4))
        for j, x in enumerate(scales):
            cache.v_scale[int(t[0, j])] = x
        t = np.repeat(t, 40, 0)
        q = torch.full((40, 100, 16, 64), 1 / 64, device="cuda").bfloat16()
        out = cache.attend(q, torch.from_numpy(t).cuda(), ints(torch, [192] * 40), scale=1.0)
        close(cache, out, q, t, 192, "bfloat16")
