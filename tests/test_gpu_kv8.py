"""GPU: the 8-bit serving cache (store, load, attend, select, evict) against the definition in
numpy (tests/kv8_reference.py).

Codes, scales, bounds, picks, kept tokens and moved weights are compared bit for bit. Attention is
compared in 64 bits under bounds that follow from its arithmetic: products are exact, sums of D
products in fp32 are off by at most D 2^-24 of the sum of magnitudes (`spread`, in units of the
logits), a weight by that much relatively (twice, for the logit and for the sum of weights) plus
the exponential's and the references' roundings (2^-18 in all at these sizes), and rounding P to
fp16 by 2^-11; the output adds half a unit of its type."""
import numpy as np
import pytest

import kv8_reference as R
from gpu_helpers import assert_same, say, torch_cuda

pytestmark = pytest.mark.gpu

PAGE = 64
UNIT = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


def make(torch, n_pages, H, D, bounds=True):
    from paper_2310_07240_amd.kv8 import Kv8Cache
    dev = "cuda"
    buf = {"k_codes": torch.randint(-127, 128, (n_pages, H, PAGE, D), device=dev).to(torch.int8),
           "v_codes": torch.randint(-127, 128, (n_pages, H, D, PAGE), device=dev).to(torch.int8),
           "k_scale": torch.rand((n_pages, H), device=dev) * 0.02 + 0.001,
           "v_scale": torch.rand((n_pages, H), device=dev) * 0.02 + 0.001,
           "k_bounds": None}
    if bounds:
        buf["k_bounds"] = torch.stack([buf["k_codes"].amin(2), buf["k_codes"].amax(2)],
                                      2).contiguous()
    return Kv8Cache(n_pages, H, D, buffers=buf)


def tables(torch, rng, B, width, extra=2):
    """A table of distinct pages in no order, and how many pages the pool has."""
    n = B * width + extra
    t = rng.permutation(n)[:B * width].reshape(B, width).astype(np.int32)
    return t, torch.from_numpy(t).cuda(), n


def ints(torch, x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same_cache(cache, ref, pages=None):
    at = slice(None) if pages is None else pages
    assert_same("k codes", cache.k_codes.cpu().numpy()[at], ref.k[at])
    assert_same("v codes", cache.v_codes.cpu().numpy().transpose(0, 1, 3, 2)[at], ref.v[at])
    assert_same("k scale", cache.k_scale.cpu().numpy()[at], ref.ks[at])
    assert_same("v scale", cache.v_scale.cpu().numpy()[at], ref.vs[at])
    if ref.bounds is not None:
        assert_same("bounds", cache.k_bounds.cpu().numpy()[at], ref.bounds[at])


# ---- store and load ---------------------------------------------------------------------------
@pytest.mark.parametrize("D,H,dtype,T,starts,counts", [
    (128, 2, "float16", 200, [0, 5, 64], [200, 130, 64]),
    (64, 3, "bfloat16", 1, [0, 63, 64, 127], [1, 1, 1, 1]),
    (256, 1, "float16", 65, [1, 62, 100], [65, 3, 0]),
    (128, 5, "bfloat16", 129, [127, 0], None),
])
def test_store_and_load(D, H, dtype, T, starts, counts):
    torch = torch_cuda()
    rng = np.random.default_rng(D + T)
    B = len(starts)
    t, table, n = tables(torch, rng, B, (max(starts) + T) // PAGE + 1)
    cache = make(torch, n, H, D)
    ref = R.Ref(cache)
    dt = getattr(torch, dtype)
    k = (torch.randn(B, T, H, D) * torch.exp(torch.randn(H, D))).to(dt).cuda()
    v = torch.randn(B, T, H, D).to(dt).cuda()
    k[0, 0, 0] = 0                             # a row of zeros, and one far above the rest
    v[-1, 0, 0, 3] = 77.0
    cnt = [T] * B if counts is None else counts
    say(f"store {D} {H} {dtype} {T}")
    cache.store(k, v, table, ints(torch, starts), None if counts is None else ints(torch, counts))
    torch.cuda.synchronize()
    ref.store(k.float().cpu().numpy(), v.float().cpu().numpy(), t, starts, cnt)
    same_cache(cache, ref)
    # once more: what is stored already stays as it is
    cache.store(k, v, table, ints(torch, starts), ints(torch, cnt))
    ref.store(k.float().cpu().numpy(), v.float().cpu().numpy(), t, starts, cnt)
    same_cache(cache, ref)
    for out_type in ("float16", "bfloat16"):
        ot = getattr(torch, out_type)
        back = cache.load(table, ints(torch, starts), T, ints(torch, cnt), dtype=ot)
        torch.cuda.synchronize()
        for codes, scale, got in ((ref.k, ref.ks, back[0]), (ref.v, ref.vs, back[1])):
            want = np.zeros((B, T, H, D), np.float32)
            for b in range(B):
                for i in range(cnt[b]):
                    p = t[b, (starts[b] + i) // PAGE]
                    want[b, i] = codes[p, :, (starts[b] + i) % PAGE].astype(np.float32) \
                        * scale[p][:, None]
            assert_same(out_type, got.view(torch.int16).cpu().numpy(),
                        torch.from_numpy(want).to(ot).view(torch.int16).numpy())


def test_load_rounds_the_fp32_product():
    """Scales whose products with some codes lie so near the middle of two fp16 values that
    rounding once and rounding through fp32 differ: the definition goes through fp32."""
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    q = np.arange(1, 128, dtype=np.float64)
    s = (rng.random(400000) * 0.05 + 0.01).astype(np.float32)
    once = (q[None] * s[:, None].astype(np.float64)).astype(np.float16)
    twice = (q[None].astype(np.float32) * s[:, None]).astype(np.float16)
    found = s[(once != twice).any(1)][:40]
    assert len(found) >= 20
    n = len(found)
    cache = make(torch, n, 1, 128)
    codes = torch.arange(-63, 65, device="cuda").to(torch.int8)
    cache.k_codes.copy_(codes.view(1, 1, 1, 128).expand(n, 1, 64, 128))
    cache.k_codes[:, :, ::2] += 63                             # 0 .. 127 in every other row
    cache.v_codes.copy_(cache.k_codes.transpose(2, 3))
    for x in (cache.k_scale, cache.v_scale):
        x.copy_(torch.from_numpy(found).view(n, 1))
    table = torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1)
    k, v = cache.load(table, ints(torch, [0] * n), 64)
    ref = R.Ref(cache)
    want = (ref.k[:, 0].astype(np.float32) * ref.ks[:, :, None]).astype(np.float16)
    for got in (k, v):
        assert_same("rows", got[:, :, 0].view(torch.int16).cpu().numpy().view(np.uint16),
                    want.view(np.uint16))


@pytest.mark.parametrize("off", [0, 1])
def test_store_strides(off):
    """Rows inside a [ctx][layer][K/V][token][channel] cache; off = 1: not 16-byte aligned."""
    torch = torch_cuda()
    rng = np.random.default_rng(3)
    B, L, T, H, D = 2, 3, 70, 2, 64
    flat = torch.randn(B * L * 2 * T * H * D + 8).half().cuda()
    kv = flat[off:off + B * L * 2 * T * H * D].view(B * L, 2, T, H, D)
    t, table, n = tables(torch, rng, B * L, 2)
    cache = make(torch, n, H, D, bounds=False)
    ref = R.Ref(cache)
    zero = [0] * (B * L)
    cache.store(kv[:, 0], kv[:, 1], table, ints(torch, zero))
    x = kv.float().cpu().numpy()
    ref.store(x[:, 0], x[:, 1], t, zero, [T] * (B * L))
    same_cache(cache, ref)
    out = torch.zeros_like(flat)[off:off + kv.numel()].view(kv.shape)
    cache.load(table, ints(torch, zero), T, k=out[:, 0], v=out[:, 1])
    again = cache.load(table, ints(torch, zero), T)
    assert torch.equal(out[:, 0], again[0]) and torch.equal(out[:, 1], again[1])


def test_store_pages_and_values_out_of_place():
    """Page numbers off the pool are skipped, NaN and Inf set no scale and are reported."""
    torch = torch_cuda()
    from paper_2310_07240_amd.cachegen import cg_get_status
    t = np.array([[1, -1, 3], [99, 0, 5]], np.int32)
    table = torch.from_numpy(t).cuda()
    cache = make(torch, 6, 1, 64)
    ref = R.Ref(cache)
    k, v = torch.randn(2, 150, 1, 64).half(), torch.randn(2, 150, 1, 64).half()
    status = ints(torch, [7])
    args = (table, ints(torch, [0, 10]))
    cache.store(k.cuda(), v.cuda(), *args, status=status)
    assert cg_get_status(status) == 0
    ref.store(k.float().numpy(), v.float().numpy(), t, [0, 10], [150, 150])
    same_cache(cache, ref)
    k[0, 3, 0, 5], k[1, 140, 0, 1], v[0, 0, 0, 0] = float("nan"), float("-inf"), float("inf")
    v[1, 100:, 0] = float("nan")
    cache.store(k.cuda(), v.cuda(), *args, status=status)
    assert cg_get_status(status) == -4
    ref.store(k.float().numpy(), v.float().numpy(), t, [0, 10], [150, 150])
    same_cache(cache, ref)
    kb, vb = cache.load(table, ints(torch, [0, 10]), 150)
    assert (kb[0, 64:128] == 0).all() and (vb[1, :54] == 0).all()


@pytest.mark.parametrize("size", [1e-38, 1e-41, 3e38])
def test_store_extreme_sizes(size):
    """bf16 rows whose scale is subnormal, or near the largest."""
    torch = torch_cuda()
    cache = make(torch, 3, 1, 64)
    ref = R.Ref(cache)
    t = np.array([[2]], np.int32)
    k = (torch.rand(1, 64, 1, 64) * size).bfloat16()
    v = -k
    cache.store(k.cuda(), v.cuda(), torch.from_numpy(t).cuda(), ints(torch, [0]))
    ref.store(k.float().numpy(), v.float().numpy(), t, [0], [64])
    same_cache(cache, ref)


@pytest.mark.parametrize("D,H,dtype,T,starts", [(64, 2, "float16", 1, [0, 1, 37, 63, 64, 127]),
                                                (128, 3, "bfloat16", 30, [0, 1, 37, 63, 64, 127]),
                                                (256, 1, "float16", 130, [5, 64, 66]),
                                                (64, 32, "bfloat16", 2200, [37, 64])])
@pytest.mark.parametrize("size", [0.1, 30.0, 0.0, 1e-38, 1e38])
def test_store_behind_tokens(D, H, dtype, T, starts, size):
    """Rows behind tokens that a page keeps: far smaller (the scale stays), far larger (it grows and
    the codes are made anew), zero, subnormal or near the largest of their type."""
    torch = torch_cuda()
    rng = np.random.default_rng(T)
    B = len(starts)
    t, table, n = tables(torch, rng, B, (max(starts) + T) // PAGE + 1)
    cache = make(torch, n, H, D)
    ref = R.Ref(cache)
    dt = getattr(torch, dtype)
    rows = lambda m, f: ((torch.rand(B, m, H, D) * 2 - 1) * f).to(dt)
    top = min(size, 6e4) if dtype == "float16" else size
    for m, at, count, f in ((max(starts), [0] * B, starts, 1.0), (T, starts, [T] * B, top)):
        k, v = rows(m, f), rows(m, f)
        say(f"store {D} {H} {dtype} {m} rows of size {f}")
        cache.store(k.cuda(), v.cuda(), table, ints(torch, at), ints(torch, count))
        torch.cuda.synchronize()
        ref.store(k.float().numpy(), v.float().numpy(), t, at, count)
        same_cache(cache, ref)


@pytest.mark.parametrize("was", [0.0, 1e-39, 2.0 ** 121, float("inf")])
def test_store_behind_odd_scales(was):
    """A page whose scale is zero under codes that are not, subnormal, huge or infinite."""
    torch = torch_cuda()
    cache = make(torch, 3, 2, 64)
    t = np.array([[1]], np.int32)
    table = torch.from_numpy(t).cuda()
    k = torch.randn(1, 20, 2, 64).half()
    cache.store(k.cuda(), -k.cuda(), table, ints(torch, [0]))
    cache.k_scale[1], cache.v_scale[1, 1] = was, was
    for new in (torch.zeros_like(k), k):
        ref = R.Ref(cache)
        cache.store(new.cuda(), new.cuda(), table, ints(torch, [20]))
        torch.cuda.synchronize()
        ref.store(new.float().numpy(), new.float().numpy(), t, [20], [20])
        same_cache(cache, ref)


# ---- attention --------------------------------------------------------------------------------
def check_attend(torch, cache, q, table, t, lengths, q_lens=None, picks=None, mass=False,
                 scale=None, max_len=None, decay=0.5):
    B, Q, HQ, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    name = str(q.dtype).split(".")[1]
    lse = torch.full((B, Q, HQ), 7.0, device="cuda")
    out = torch.full_like(q, 7.0)
    more = {}
    if mass:
        old = torch.rand((cache.n_pages, cache.n_heads, PAGE), device="cuda")
        got_mass = torch.full_like(old, -1.0)
        more = {"mass": old, "mass_out": got_mass, "decay": decay}
    dev_picks = None if picks is None else torch.from_numpy(picks).cuda()
    say(f"attend {tuple(q.shape)} {name} lengths {list(lengths)[:4]} picks {picks is not None}")
    for _ in range(2):                        # the same bits each time
        first = out.clone()
        cache.attend(q, table, ints(torch, lengths), scale=scale, max_len=max_len, out=out,
                     q_lens=None if q_lens is None else ints(torch, q_lens), lse=lse,
                     picks=dev_picks, **more)
    torch.cuda.synchronize()
    assert torch.equal(first, out) or torch.isnan(out).any()
    ql = [Q] * B if q_lens is None else q_lens
    cut = [min(x, table.shape[1] * PAGE if max_len is None else max_len) for x in lengths]
    want, wl, wm, size, spread = R.attend(R.Ref(cache), q.float().cpu().numpy(), t, cut, ql, scale,
                                          picks)
    off = 4 * D * 2.0 ** -24 * spread + 2.0 ** -18
    bound = UNIT[name] * np.abs(want) + (2.0 ** -11 + off)[..., None] * size * 1.01 + 1e-7
    err = np.abs(out.float().cpu().numpy().astype(np.float64) - want)
    assert (err <= bound).all(), (err / bound).max()
    g = lse.cpu().numpy().astype(np.float64)
    assert (np.isinf(g) == np.isinf(wl)).all()
    fin = np.isfinite(wl)
    lerr = np.abs(np.where(fin, g - np.where(fin, wl, 0), 0))
    lim = off + 2.0 ** -20 * np.abs(np.where(fin, wl, 0))
    assert (lerr <= lim).all(), (lerr / lim).max()
    if mass:
        seen = np.zeros(wm.shape, bool)
        for b in range(B):
            for j in range(min(cut[b], table.shape[1] * PAGE)):
                p = t[b, j // PAGE]
                if 0 <= p < cache.n_pages:
                    seen[p, :, j % PAGE] = True
        gm = got_mass.cpu().numpy().astype(np.float64)
        wm = wm + decay * old.cpu().numpy().astype(np.float64)
        assert (gm[~seen] == -1.0).all()
        lim = (off.max(initial=0) * 2 + 2.0 ** -22 * Q * HQ + 2.0 ** -20) * wm + 1e-12
        assert (np.abs(gm - wm)[seen] <= lim[seen]).all()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D,HQ,H,lengths", [
    (128, 4, 1, [1, 2, 63, 64, 65, 0, 700]),
    (64, 8, 2, [300, 17]),
    (256, 3, 3, [129, 128]),
    (128, 17, 1, [200]),                      # a group past one 16-row tile
    (64, 40, 1, [333]),
])
def test_attend_one_token(dtype, D, HQ, H, lengths):
    torch = torch_cuda()
    rng = np.random.default_rng(D + HQ)
    t, table, n = tables(torch, rng, len(lengths), max(lengths) // PAGE + 2)
    cache = make(torch, n, H, D)
    q = (torch.randn(len(lengths), 1, HQ, D) * 2).to(getattr(torch, dtype)).cuda()
    check_attend(torch, cache, q, table, t, lengths, mass=True)
    check_attend(torch, cache, q, table, t, lengths, max_len=max(lengths))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D,HQ,H,Q,lengths,q_lens", [
    (128, 4, 2, 5, [5, 70, 3, 64], [5, 3, 3, 0]),
    (64, 2, 1, 33, [33, 200], None),
    (128, 8, 1, 40, [100, 40, 0], [40, 39, 0]),
    (256, 2, 2, 17, [130], None),
    (128, 3, 1, 90, [250, 90], None),
    (64, 6, 2, 130, [450], None),
    (128, 8, 2, 70, [513, 64, 300], [70, 1, 64]),
])
def test_attend_many_tokens(dtype, D, HQ, H, Q, lengths, q_lens):
    torch = torch_cuda()
    rng = np.random.default_rng(Q)
    t, table, n = tables(torch, rng, len(lengths), max(lengths) // PAGE + 1)
    cache = make(torch, n, H, D)
    q = (torch.randn(len(lengths), Q, HQ, D) * 2).to(getattr(torch, dtype)).cuda()
    check_attend(torch, cache, q, table, t, lengths, q_lens=q_lens, mass=True)


def test_attend_more_queries_than_tokens():
    """A call whose first queries stand before the sequence's first token: empty rows."""
    torch = torch_cuda()
    rng = np.random.default_rng(9)
    t, table, n = tables(torch, rng, 2, 2)
    cache = make(torch, n, 2, 64)
    q = torch.randn(2, 30, 4, 64).half().cuda()
    check_attend(torch, cache, q, table, t, [7, 29], mass=True)


def test_attend_strides_and_garbage_outside():
    """Strided queries and outputs, page numbers off the pool, lengths past the table, NaN scales
    in pages that no sequence reads, codes of all kinds behind the length."""
    torch = torch_cuda()
    t = np.array([[0, 3, 77, 2], [4, -5, 1, 6]], np.int32)
    table = torch.from_numpy(t).cuda()
    cache = make(torch, 9, 2, 128)
    cache.k_scale[5] = float("nan")
    cache.v_scale[7] = float("inf")
    big = torch.randn(2, 4, 3, 3, 128).half().cuda()
    q = big[:, :, 1, :2]
    check_attend(torch, cache, q, table, t, [1000, 200], mass=True)
    o = torch.full((2, 2, 4, 130), 5.0, dtype=torch.float16, device="cuda")
    view = o.permute(0, 2, 1, 3)[..., 1:129]
    a = cache.attend(q, table, ints(torch, [200, 90]))
    cache.attend(q, table, ints(torch, [200, 90]), out=view)
    assert torch.equal(a, view)
    assert (o[..., 0] == 5).all() and (o[..., 129] == 5).all()


def test_attend_nan_query_stays_in_its_row():
    torch = torch_cuda()
    for dtype in (torch.float16, torch.bfloat16):
        rng = np.random.default_rng(2)
        t, table, n = tables(torch, rng, 1, 3)
        cache = make(torch, n, 1, 128)
        q = torch.randn(1, 3, 4, 128).to(dtype).cuda()
        good = cache.attend(q, table, ints(torch, [150]))
        q[0, 1, 2, 7] = float("nan")
        q[0, 2, 3, 9] = float("inf")
        got = cache.attend(q, table, ints(torch, [150]))
        bad = torch.zeros((1, 3, 4), dtype=torch.bool, device="cuda")
        bad[0, 1, 2] = bad[0, 2, 3] = True
        assert torch.equal(got[~bad], good[~bad])
        assert torch.isnan(got[0, 1, 2]).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
@pytest.mark.parametrize("Q,HQ,D", [(8, 2, 128), (80, 3, 64), (70, 2, 256), (300, 1, 128)])
def test_attend_bad_scale_stays_with_who_sees_it(bad, which, Q, HQ, D):
    """NaN or Inf as the scale of the sequence's last page: the queries before it are as without
    it, bit for bit. Those that see it are not finite, except under an infinite K scale, whose
    logits of minus infinity are weights of 0."""
    torch = torch_cuda()
    rng = np.random.default_rng(13)
    t, table, n = tables(torch, rng, 1, 6)
    cache = make(torch, n, 1, D)
    q = torch.randn(1, Q, HQ, D).half().cuda()
    length = 5 * 64 + 3                        # the last three queries see the last page
    good = cache.attend(q, table, ints(torch, [length]))
    getattr(cache, which)[int(t[0, 5])] = bad
    mass = torch.zeros((n, 1, PAGE), device="cuda")
    got = cache.attend(q, table, ints(torch, [length]), mass=mass)
    assert torch.equal(got[:, :Q - 3], good[:, :Q - 3]) and not torch.isnan(good).any()
    if which == "v_scale" or bad != bad:
        assert not torch.isfinite(got[:, Q - 3:]).any()
    if which == "k_scale" and bad != bad:
        assert torch.isnan(mass[int(t[0, 5]), 0, 0])


@pytest.mark.parametrize("scale", [-0.3, 0.0, 3.0])
def test_attend_scales_and_extremes(scale):
    """Logits far apart (a few hundred), equal, and in reverse; one heavy token before a long
    light tail whose sum still counts."""
    torch = torch_cuda()
    rng = np.random.default_rng(4)
    t, table, n = tables(torch, rng, 1, 20)
    cache = make(torch, n, 1, 64)
    q = torch.randn(1, 2, 5, 64).half().cuda()
    check_attend(torch, cache, q, table, t, [1234], scale=scale, mass=True)
    cache.k_codes.zero_()
    cache.k_codes[int(t[0, 0]), 0, 5, :] = 100
    cache.k_scale.fill_(0.01)
    cache.v_scale[int(t[0, 3])] = 1e-4
    cache.v_scale[int(t[0, 4])] = 0.0
    q.fill_(0.25)
    check_attend(torch, cache, q, table, t, [1234], scale=1.0)


@pytest.mark.parametrize("D,dtype", [(128, "float16"), (64, "bfloat16"), (256, "float16")])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 2.0])
def test_attend_many_tokens_scales_and_extremes(D, dtype, scale):
    """The same for a prompt: pages of zeros, of V scales far apart and of none, lost pages, one
    heavy token before a light tail."""
    torch = torch_cuda()
    rng = np.random.default_rng(11)
    t, table, n = tables(torch, rng, 2, 12)
    cache = make(torch, n, 1, D)
    for j, f in enumerate((1.0, 30.0, 1e-3, 0.0, 1.0, 1e-25, 3.0, 1.0)):
        cache.v_scale[int(t[0, j])] *= f
    cache.k_scale[int(t[0, 2])] = 0.0
    cache.k_codes[int(t[1, 1])] = 0
    t[1, 3] = -1
    table[1, 3] = -1
    q = torch.randn(2, 70, 3, D).to(getattr(torch, dtype)).cuda()
    check_attend(torch, cache, q, table, t, [700, 333], scale=scale, mass=True)
    cache.k_codes.zero_()
    cache.k_codes[int(t[0, 0]), 0, 5, :] = 100
    cache.k_scale.fill_(0.01)
    q.fill_(0.25)
    check_attend(torch, cache, q, table, t, [700, 70], scale=scale * 8)


def much_room(torch, t):
    """The table with columns of no page behind it: the host lays such a call out as a large one,
    which shares the pages among the rows of a workgroup, in many splits."""
    t = np.concatenate([t, np.full((len(t), 2800 - t.shape[1]), -1, np.int32)], 1)
    return t, torch.from_numpy(t).cuda()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D,HQ,H,Q,lengths,q_lens", [
    (64, 2, 1, 33, [33, 200], None),
    (128, 8, 1, 40, [100, 40, 0], [40, 39, 0]),
    (256, 2, 2, 49, [130], None),
    (64, 6, 2, 130, [450], None),
    (128, 8, 2, 70, [513, 64, 300], [70, 1, 64]),
    (64, 4, 1, 30, [7, 29], None),             # queries before the first token
])
def test_attend_large_calls(dtype, D, HQ, H, Q, lengths, q_lens):
    torch = torch_cuda()
    rng = np.random.default_rng(Q)
    t, _, n = tables(torch, rng, len(lengths), max(lengths) // PAGE + 1)
    t, table = much_room(torch, t)
    cache = make(torch, n, H, D)
    q = (torch.randn(len(lengths), Q, HQ, D) * 2).to(getattr(torch, dtype)).cuda()
    check_attend(torch, cache, q, table, t, lengths, q_lens=q_lens, mass=True)


@pytest.mark.parametrize("D,H,Q,most", [(128, 8, 12, 150), (64, 12, 13, 100), (256, 4, 12, 200)])
def test_attend_many_sequences(D, H, Q, most):
    """More row tiles than the card holds workgroups: no splits."""
    torch = torch_cuda()
    rng = np.random.default_rng(Q)
    B = 22
    lengths = [int(x) for x in rng.integers(0, most, B)]
    t, table, n = tables(torch, rng, B, most // PAGE + 1)
    cache = make(torch, n, H, D)
    q = torch.randn(B, Q, 4 * H, D).half().cuda()
    check_attend(torch, cache, q, table, t, lengths, mass=True)


@pytest.mark.parametrize("D,dtype", [(128, "float16"), (64, "bfloat16"), (256, "float16")])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 2.0])
def test_attend_large_calls_scales_and_extremes(D, dtype, scale):
    torch = torch_cuda()
    rng = np.random.default_rng(11)
    t, _, n = tables(torch, rng, 2, 12)
    cache = make(torch, n, 1, D)
    for j, f in enumerate((1.0, 30.0, 1e-3, 0.0, 1.0, 1e-25, 3.0, 1.0)):
        cache.v_scale[int(t[0, j])] *= f
    cache.k_scale[int(t[0, 2])] = 0.0
    cache.k_codes[int(t[1, 1])] = 0
    t[1, 3] = -1
    t, table = much_room(torch, t)
    q = torch.randn(2, 70, 3, D).to(getattr(torch, dtype)).cuda()
    check_attend(torch, cache, q, table, t, [700, 333], scale=scale, mass=True)
    cache.k_codes.zero_()
    cache.k_codes[int(t[0, 0]), 0, 5, :] = 100
    cache.k_scale.fill_(0.01)
    q.fill_(0.25)
    check_attend(torch, cache, q, table, t, [700, 70], scale=scale * 8)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
@pytest.mark.parametrize("Q,HQ,D", [(80, 3, 64), (70, 2, 256), (300, 1, 128)])
def test_attend_large_calls_bad_scale(bad, which, Q, HQ, D):
    torch = torch_cuda()
    rng = np.random.default_rng(13)
    t, _, n = tables(torch, rng, 1, 6)
    t, table = much_room(torch, t)
    cache = make(torch, n, 1, D)
    q = torch.randn(1, Q, HQ, D).half().cuda()
    length = 5 * 64 + 3                        # the last three queries see the last page
    good = cache.attend(q, table, ints(torch, [length]))
    getattr(cache, which)[int(t[0, 5])] = bad
    mass = torch.zeros((n, 1, PAGE), device="cuda")
    got = cache.attend(q, table, ints(torch, [length]), mass=mass)
    assert torch.equal(got[:, :Q - 3], good[:, :Q - 3]) and not torch.isnan(good).any()
    if which == "v_scale" or bad != bad:
        assert not torch.isfinite(got[:, Q - 3:]).any()
    if which == "k_scale" and bad != bad:
        assert torch.isnan(mass[int(t[0, 5]), 0, 0])


def test_attend_large_call_split():
    """Splits of several pages each, of sequences of uneven length."""
    torch = torch_cuda()
    rng = np.random.default_rng(12)
    t, table, n = tables(torch, rng, 4, 60)
    cache = make(torch, n, 8, 64)
    q = torch.randn(4, 60, 8, 64).half().cuda()
    check_attend(torch, cache, q, table, t, [3800, 900, 200, 130], mass=True)


@pytest.mark.parametrize("vs", [1e-20, 1e-30, 1e-36])
@pytest.mark.parametrize("Q", [1, 30])
def test_attend_light_weights(vs, Q):
    """A heavy token with nothing in half of the channels: there the light ones are all there is,
    down to weights of 2^-28, and V is small."""
    torch = torch_cuda()
    rng = np.random.default_rng(14)
    t, table, n = tables(torch, rng, 1, 3)
    cache = make(torch, n, 1, 128)
    cache.k_codes.zero_()
    for j, steps in enumerate((19, 10, 1)):    # logits of one token a page above the others'
        cache.k_codes[int(t[0, j]), 0, 7, :] = steps
        cache.v_codes[int(t[0, j]), 0, ::2, 7] = 0
    cache.k_scale.fill_(1.0)
    cache.v_scale.fill_(vs)
    q = torch.full((1, Q, 3, 128), 1 / 128).bfloat16().cuda()
    lse = torch.empty((1, Q, 3), device="cuda")
    out = cache.attend(q, table, ints(torch, [192 - 30 + Q]), scale=1.0, lse=lse).float().cpu()
    want, wl, _, size, _ = R.attend(R.Ref(cache), q.float().cpu().numpy(), t, [192 - 30 + Q], [Q],
                                    1.0)
    # a weight's fp16 rounding, and the rounding to bf16, whose subnormals are 2^-133 apart
    lim = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * size + 2.0 ** -134
    assert (np.abs(out.numpy() - want) <= lim).all()
    assert np.abs(lse.cpu().numpy() - wl).max() <= 1e-4


def test_attend_long_prompt_split():
    torch = torch_cuda()
    rng = np.random.default_rng(12)
    t, table, n = tables(torch, rng, 1, 60)
    cache = make(torch, n, 1, 64)
    q = torch.randn(1, 100, 1, 64).half().cuda()
    check_attend(torch, cache, q, table, t, [3800], mass=True)


def test_attend_long_and_split():
    """Long enough for many splits; lengths far below the bound, so that splits stay empty."""
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    t, table, n = tables(torch, rng, 2, 160)
    cache = make(torch, n, 1, 64)
    q = torch.randn(2, 1, 2, 64).half().cuda()
    check_attend(torch, cache, q, table, t, [10171, 65], mass=True)


def test_attend_on_another_stream():
    torch = torch_cuda()
    rng = np.random.default_rng(6)
    t, table, n = tables(torch, rng, 2, 40)
    cache = make(torch, n, 2, 128)
    q = torch.randn(2, 1, 8, 128).half().cuda()
    L = ints(torch, [2500, 900])
    want = cache.attend(q, table, L)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    got = cache.attend(q, table, L, stream=other)
    other.synchronize()
    assert torch.equal(want, got)


def test_attend_graph_replay():
    """Captured once, replayed between eager work with new contents: the same as eager."""
    torch = torch_cuda()
    rng = np.random.default_rng(7)
    t, table, n = tables(torch, rng, 3, 30)
    cache = make(torch, n, 2, 128)
    q = torch.randn(3, 1, 8, 128).half().cuda()
    k, v = torch.randn(3, 1, 2, 128).half().cuda(), torch.randn(3, 1, 2, 128).half().cuda()
    starts, L = ints(torch, [100, 700, 1500]), ints(torch, [101, 701, 1501])
    out = torch.empty_like(q)
    mass = torch.zeros((n, 2, PAGE), device="cuda")
    got_mass = torch.zeros_like(mass)
    picks = torch.zeros((3, 1, 2, 4), dtype=torch.int32, device="cuda")
    sparse = torch.empty_like(q)

    def step():
        cache.store(k, v, table, starts)
        cache.attend(q, table, L, out=out, mass=mass, mass_out=got_mass)
        cache.select(q, table, L, 4, out=picks)
        cache.attend(q, table, L, out=sparse, picks=picks)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        q.copy_(torch.randn(q.shape))
        k.copy_(torch.randn(k.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, got_mass, picks, sparse)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, got_mass, picks, sparse)):
            assert torch.equal(a, b), i


# ---- select and sparse attention --------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D,HQ,H,Q,lengths,n_picks,recent", [
    (128, 8, 2, 1, [1, 64, 65, 1000, 0], 3, 1),
    (64, 3, 1, 2, [640, 641], 5, 2),
    (256, 2, 1, 1, [2000], 4, 0),
    (128, 16, 1, 3, [900], 2, 5),
    (64, 2, 2, 1, [20000], 70, 1),
    (64, 200, 1, 1, [700], 4, 1),
])
def test_select_and_sparse(dtype, D, HQ, H, Q, lengths, n_picks, recent):
    torch = torch_cuda()
    rng = np.random.default_rng(D + n_picks)
    B = len(lengths)
    t, table, n = tables(torch, rng, B, max(lengths) // PAGE + 1)
    cache = make(torch, n, H, D)
    # ranges that differ, some alike: scores that differ, and ties
    part = torch.randint(1, 9, (n, H, 1, 1), device="cuda") / 8.0
    cache.k_codes.copy_((cache.k_codes.float() * part).round())
    cache.k_codes[: n // 2] = cache.k_codes[0]
    cache.k_scale[: n // 2] = 0.01
    cache.k_bounds.copy_(torch.stack([cache.k_codes.amin(2), cache.k_codes.amax(2)], 2))
    q = torch.randn(B, Q, HQ, D).to(getattr(torch, dtype)).cuda()
    q[0, 0, 0, 0] = 0.0
    say(f"select {D} {HQ} {H} {lengths}")
    q_lens = [min(Q, x) for x in lengths]
    picks = cache.select(q, table, ints(torch, lengths), n_picks, recent=recent,
                         q_lens=ints(torch, q_lens))
    want = R.select(R.Ref(cache), q.float().cpu().numpy(), t, lengths, q_lens, n_picks, recent)
    assert_same("picks", picks.cpu().numpy(), want)
    check_attend(torch, cache, q, table, t, lengths, q_lens=q_lens, picks=want)


def test_sparse_with_odd_picks():
    """Entries outside the sequence are skipped; no entry at all gives an empty row."""
    torch = torch_cuda()
    rng = np.random.default_rng(8)
    t, table, n = tables(torch, rng, 2, 6)
    cache = make(torch, n, 1, 128)
    q = torch.randn(2, 1, 4, 128).half().cuda()
    picks = np.array([[[[5, -1, 0, 99, -7]]], [[[-1, 4, 77, -1, -1]]]], np.int32)
    check_attend(torch, cache, q, table, t, [330, 200], picks=picks)


def test_select_zero_queries_and_lost_pages():
    torch = torch_cuda()
    t = np.array([[0, 1, 50, 3, 4, -2, 6]], np.int32)
    table = torch.from_numpy(t).cuda()
    cache = make(torch, 8, 1, 64)
    q = torch.zeros(1, 1, 2, 64).half().cuda()
    for lengths in ([400], [7 * 64]):
        picks = cache.select(q, table, ints(torch, lengths), 3)
        want = R.select(R.Ref(cache), np.zeros((1, 1, 2, 64), np.float32), t, lengths, [1], 3, 1)
        assert_same("picks", picks.cpu().numpy(), want)


# ---- eviction ---------------------------------------------------------------------------------
@pytest.mark.parametrize("D,H,lengths,keep,recent", [
    (128, 2, [500, 64, 130, 0, 129], 130, 30),
    (64, 3, [300], 1, 0),
    (64, 1, [300, 299], 65, 65),
    (256, 1, [200], 100, 150),
    (128, 1, [5000, 4000], 1000, 100),
    (64, 1, [70000], 3000, 100),              # more keys than the lanes keep in registers
])
def test_evict(D, H, lengths, keep, recent):
    torch = torch_cuda()
    rng = np.random.default_rng(D + keep)
    B = len(lengths)
    width, new_width = max(lengths) // PAGE + 1, (keep + PAGE - 1) // PAGE
    n = B * (width + new_width) + 2
    order = rng.permutation(n).astype(np.int32)
    t = order[:B * width].reshape(B, width).copy()
    to = order[B * width:B * (width + new_width)].reshape(B, new_width).copy()
    cache = make(torch, n, H, D)
    mass = torch.rand((n, H, PAGE), device="cuda")
    mass[torch.rand(mass.shape, device="cuda") < 0.3] = 0.25          # ties
    mass[torch.rand(mass.shape, device="cuda") < 0.1] = 0.0
    mass[torch.rand(mass.shape, device="cuda") < 0.05] = -0.0
    mass[torch.rand(mass.shape, device="cuda") < 0.02] = float("nan")
    mass[torch.rand(mass.shape, device="cuda") < 0.02] = float("inf")
    ref, rm = R.Ref(cache), mass.cpu().numpy().copy()
    say(f"evict {D} {H} {lengths} {keep} {recent}")
    kept, new = cache.evict(torch.from_numpy(t).cuda(), ints(torch, lengths), mass, keep, recent,
                            torch.from_numpy(to).cuda())
    torch.cuda.synchronize()
    wk, wn = R.evict(ref, t, lengths, rm, keep, recent, to)
    assert_same("kept", kept.cpu().numpy(), wk)
    assert_same("lengths", new.cpu().numpy(), wn)
    same_cache(cache, ref)
    assert_same("mass", mass.cpu().numpy().view(np.int32), rm.view(np.int32))


@pytest.mark.parametrize("keep", [1, 2, 60, 128, 900, 999])
def test_evict_distributions(keep):
    """Which tokens stay, by heads whose weights are spread in ways that a search over them has to
    get right: mostly or all zero, all equal, one far above, neighbours in the last bit, over all
    magnitudes, negative, infinite, not a number."""
    torch = torch_cuda()
    n, D = 1000, 64
    rng = np.random.default_rng(keep)
    f = np.float32
    few = np.where(rng.random(n) < 0.05, rng.random(n), 0)
    bits = lambda a: np.asarray(a, np.uint32).view(f)
    rows = [few, np.zeros(n), np.full(n, 0.5), np.eye(1, n, 400)[0], -rng.random(n),
            bits(0x3f800000 + rng.integers(0, 3000, n)), bits(rng.integers(0, 0x7f800000, n)),
            bits(rng.integers(0, 1 << 32, n, dtype=np.uint64)),
            np.where(rng.random(n) < 0.5, np.inf, np.nan), np.full(n, np.nan),
            np.where(rng.random(n) < 0.5, -0.0, 0.0), np.where(np.arange(n) < 500, -1.0, 1.0),
            bits(rng.integers(0, 3, n)), np.where(rng.random(n) < 0.5, -np.inf, 3e38),
            np.exp(2 * rng.standard_normal(n)), np.arange(n), -np.arange(n)[::-1]]
    H, pages, new = len(rows), (n + PAGE - 1) // PAGE, (keep + PAGE - 1) // PAGE
    cache = make(torch, pages + new, H, D)
    w = np.zeros((H, pages * PAGE), f)
    for h, r in enumerate(rows):
        w[h, :n] = r
    mass = torch.zeros((pages + new, H, PAGE), device="cuda")
    mass[:pages] = torch.from_numpy(w.reshape(H, pages, PAGE).transpose(1, 0, 2).copy()).cuda()
    t = torch.arange(pages + new, dtype=torch.int32, device="cuda")
    for recent in (0, 1, keep // 2):
        say(f"evict {keep} of {n} by {H} distributions, the last {recent} kept")
        kept, _ = cache.evict(t[None, :pages].contiguous(), ints(torch, [n]), mass, keep, recent,
                              t[None, pages:].contiguous())
        torch.cuda.synchronize()
        for h in range(H):
            assert_same(f"distribution {h}", kept[0, h].cpu().numpy(),
                        np.asarray(R.kept_tokens(list(w[h, :n]), n, keep, recent), np.int32))


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("D,HQ,H,Q,lengths", [
    (64, 64, 1, 3, [200]),                     # a token is two tiles of 32 rows
    (64, 40, 1, 5, [130, 64]),                 # tiles begin inside a token
    (128, 16, 2, 37, [100, 300]),
    (256, 5, 1, 30, [90]),
])
def test_attend_weights_of_wide_groups(D, HQ, H, Q, lengths, off):
    """Weights of many rows, by groups that fill whole tiles and groups that do not; off = 1: rows
    off 16-byte boundaries."""
    torch = torch_cuda()
    rng = np.random.default_rng(HQ)
    t, table, n = tables(torch, rng, len(lengths), max(lengths) // PAGE + 1)
    cache = make(torch, n, H, D)
    shape = (len(lengths), Q, HQ, D)
    q = torch.randn(int(np.prod(shape)) + 8).half().cuda()[off:off + int(np.prod(shape))].view(shape)
    check_attend(torch, cache, q, table, t, lengths, mass=True)
