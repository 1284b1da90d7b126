"""GPU: calls of the 8-bit cache that tests/test_gpu_kv8.py does not make: eviction with pages lost
and lengths past the host's bound, selection with strided and unaligned queries, weights of wide
groups in bf16, captured evictions and stores."""
import numpy as np
import pytest

import kv8_reference as R
from gpu_helpers import assert_same, say, torch_cuda
from test_gpu_kv8 import PAGE, check_attend, ints, make, much_room, same_cache, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,keep,recent", [(64, 100, 20), (128, 65, 0), (256, 300, 300)])
def test_evict_lost_pages(D, keep, recent):
    """Tokens of pages that do not exist weigh least, earlier ones first; one that stays all the same
    becomes a row of zeros without weight. A new page that does not exist gets nothing."""
    torch = torch_cuda()
    H, n, width, new = 2, 400, 7, 5
    rng = np.random.default_rng(D)
    order = rng.permutation(width + new).astype(np.int32)
    t, to = order[:width].copy(), order[width:].copy()
    cache = make(torch, width + new, H, D)
    mass = torch.rand((width + new, H, PAGE), device="cuda") - 0.5
    old, k_old, v_old = mass.cpu().numpy(), *cache.load(
        torch.from_numpy(t[None]).cuda(), ints(torch, [0]), n)
    t[1], t[4] = -1, 99
    to[1] = -7
    say(f"evict {D}, pages 1 and 4 of 7 and new page 1 lost")
    kept, length = cache.evict(torch.from_numpy(t[None]).cuda(), ints(torch, [n]), mass, keep,
                               recent, torch.from_numpy(to[None]).cuda())
    torch.cuda.synchronize()
    assert length.tolist() == [min(n, keep)]
    lost = np.isin(np.arange(n) // PAGE, (1, 4))
    k_new, v_new = cache.load(torch.from_numpy(to[None]).cuda(), ints(torch, [0]), min(n, keep))
    for h in range(H):
        w = np.array([np.nan if lost[j] else old[t[j // PAGE], h, j % PAGE] for j in range(n)])
        want = R.kept_tokens(list(w), n, keep, recent)
        assert_same("kept", kept[0, h].cpu().numpy(), np.asarray(want, np.int32))
        for i, j in enumerate(want):
            if i // PAGE == 1:
                assert not k_new[0, i, h].any() and not v_new[0, i, h].any()
                continue
            got = float(mass[int(to[i // PAGE]), h, i % PAGE])
            if lost[j]:
                assert got == 0 and not k_new[0, i, h].any() and not v_new[0, i, h].any()
            else:
                assert got == float(old[t[j // PAGE], h, j % PAGE])
                # coded again: half a step of the new page's scale, and fp16's rounding twice
                for a, b, s in ((k_new, k_old, cache.k_scale), (v_new, v_old, cache.v_scale)):
                    step = float(s[int(to[i // PAGE]), h])
                    err = (a[0, i, h].float() - b[0, j, h].float()).abs().max()
                    assert err <= 0.51 * step + 2.0 ** -10 * 127 * step


@pytest.mark.parametrize("max_len", [0, 1, 64, 130, 250])
def test_evict_lengths_past_the_bound(max_len):
    """Sequences longer than the host's bound are cut to it."""
    torch = torch_cuda()
    H, D, keep = 2, 64, 100
    lengths = [300, 130, 10, 10 ** 6]
    rng = np.random.default_rng(max_len)
    t, table, n = tables(torch, rng, 4, 7)
    t, to = t[:, :5].copy(), t[:, 5:].copy()
    cache = make(torch, n, H, D)
    mass = torch.rand((n, H, PAGE), device="cuda")
    ref, rm = R.Ref(cache), mass.cpu().numpy().copy()
    kept, new = cache.evict(torch.from_numpy(t).cuda(), ints(torch, lengths), mass, keep, 10,
                            torch.from_numpy(to).cuda(), max_len=max_len)
    torch.cuda.synchronize()
    wk, wn = R.evict(ref, t, [min(x, max_len) for x in lengths], rm, keep, 10, to)
    assert_same("kept", kept.cpu().numpy(), wk)
    assert_same("lengths", new.cpu().numpy(), wn)
    same_cache(cache, ref)
    assert_same("mass", mass.cpu().numpy().view(np.int32), rm.view(np.int32))


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D,HQ,H", [(64, 6, 2), (128, 4, 1), (256, 2, 2)])
def test_select_strided_queries(D, HQ, H, dtype, off):
    """Queries inside a [token][q, k, v][head] projection; off = 1: off 16-byte boundaries."""
    torch = torch_cuda()
    rng = np.random.default_rng(D)
    B, Q, lengths = 2, 3, [900, 700]
    t, table, n = tables(torch, rng, B, 15)
    cache = make(torch, n, H, D)
    flat = torch.randn(B * Q * 3 * HQ * D + 8).to(getattr(torch, dtype)).cuda()
    q = flat[off:off + B * Q * 3 * HQ * D].view(B, Q, 3, HQ, D)[:, :, 1]
    assert q.stride(1) == 3 * HQ * D
    picks = cache.select(q, table, ints(torch, lengths), 4, recent=2)
    want = R.select(R.Ref(cache), q.float().cpu().numpy(), t, lengths, [Q] * B, 4, 2)
    assert_same("picks", picks.cpu().numpy(), want)
    check_attend(torch, cache, q, table, t, lengths, picks=want)


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("D,HQ,H,Q,lengths", [(64, 64, 1, 3, [200]), (64, 40, 1, 5, [130, 64]),
                                              (128, 16, 2, 37, [100, 300]), (256, 5, 1, 30, [90]),
                                              (128, 24, 1, 9, [150])])
def test_weights_of_wide_groups_in_bf16(D, HQ, H, Q, lengths, off):
    torch = torch_cuda()
    rng = np.random.default_rng(HQ)
    t, table, n = tables(torch, rng, len(lengths), max(lengths) // PAGE + 1)
    cache = make(torch, n, H, D)
    shape = (len(lengths), Q, HQ, D)
    size = int(np.prod(shape))
    q = torch.randn(size + 8).bfloat16().cuda()[off:off + size].view(shape)
    check_attend(torch, cache, q, table, t, lengths, mass=True)
    t, table = much_room(torch, t)
    check_attend(torch, cache, q, table, t, lengths, mass=True)


def test_decode_step_replayed():
    """Store with weights, attention and an eviction captured together, replayed between eager work
    with other rows."""
    torch = torch_cuda()
    H, D, B = 2, 64, 3
    rng = np.random.default_rng(5)
    t, table, n = tables(torch, rng, B, 9)
    t, to = table[:, :7].contiguous(), table[:, 7:].contiguous()
    cache = make(torch, n, H, D)
    k, v = (torch.randn(B, 2, H, D).half().cuda() for _ in range(2))
    q = torch.randn(B, 2, 4 * H, D).half().cuda()
    starts, L = ints(torch, [190, 300, 63]), ints(torch, [192, 302, 65])
    buffers = (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale, cache.k_bounds)
    was = [x.clone() for x in buffers]
    first = torch.rand((n, H, PAGE), device="cuda")
    mass, out = first.clone(), torch.empty_like(q)
    kept = []

    def step():
        cache.store(k, v, t, starts, mass=mass)
        cache.attend(q, t, L, out=out, mass=mass, decay=0.75)
        kept[:] = cache.evict(t, L, mass, 100, 2, to)

    def reset():
        mass.copy_(first)
        for x, y in zip(buffers, was):
            x.copy_(y)

    def results():
        return [x.clone() for x in (out, mass, *kept, *buffers)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    captured = list(kept)
    for i in range(4):
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape))
        reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        kept[:] = captured
        got = results()
        reset()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, results()):
            assert torch.equal(a, b), i
