"""GPU: attention of sequences that share contexts (and cross attention, where they have nothing of
their own), against the definition in 64 bits (tests/sharing_reference.py). The bounds are those of
tests/test_gpu_kv8.py, which follow from the same arithmetic: products are exact, sums of D products
in 32 bits are off by at most D 2^-24 of the sum of magnitudes, weights by twice that and their
rounding to fp16, 2^-11; the output adds half a unit of its type. The join of a context's and a
sequence's own states is in 32 bits: of at most 256 states, within the 2^-18 for all of them."""
import numpy as np
import pytest

import kv8_reference as R
import sharing_reference as S
from gpu_helpers import say, torch_cuda
from test_gpu_kv8 import UNIT, ints, make

pytestmark = pytest.mark.gpu
PAGE = 64


def table_of(rng, order, lengths, width=None):
    width = width or max(1, max(S.pages_of(n) for n in lengths))
    t = np.full((len(lengths), width), -1, np.int32)
    for i, n in enumerate(lengths):
        for j in range(min(width, S.pages_of(n))):
            t[i, j] = order.pop()
    return t


def check(H, group, D, dtype, tokens, firsts, n, own, q_lens=None, Q=1, max_users=None, seed=0,
          scale=None, strided=False, lost=False, spoil=None, max_shared=None):
    """own: the sequences' own lengths, or None. Returns (out, lse) for further looks."""
    torch = torch_cuda()
    rng = np.random.default_rng(seed)
    total = sum(map(S.pages_of, tokens)) + sum(map(S.pages_of, own or [])) + 2
    order = rng.permutation(total).tolist()
    shared = table_of(rng, order, tokens)
    table = None if own is None else table_of(rng, order, own)
    if lost:
        shared[0, 0] = -1
        shared[-1, -1] = total + 5
    cache = make(torch, total, H, D)
    if spoil:
        spoil(cache, shared, table)
    ref = R.Ref(cache)
    HQ = H * group
    scale = D ** -0.5 if scale is None else scale
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = (torch.randn((n, Q, HQ, D), generator=g, device="cuda")).to(getattr(torch, dtype))
    out = torch.full_like(q, 7.0)
    if strided:                                # rows in other orders and apart, off 16 bytes
        wide = torch.full((Q, n, HQ, D + 3), 3.0, dtype=q.dtype, device="cuda")
        wide[..., 1:D + 1] = q.transpose(0, 1)
        q = wide.transpose(0, 1)[..., 1:D + 1]
        out = torch.full((HQ, n, Q, D + 5), 7.0, dtype=q.dtype, device="cuda"
                         ).permute(1, 2, 0, 3)[..., 2:D + 2]
    lse = torch.full((n, Q, HQ), 5.0, device="cuda")
    more = {} if own is None else {"table": torch.from_numpy(table).cuda(),
                                   "lengths": ints(torch, own)}
    args = (q, torch.from_numpy(shared).cuda(), ints(torch, tokens), ints(torch, firsts))
    more.update(scale=scale, q_lens=None if q_lens is None else ints(torch, q_lens), out=out,
                lse=lse, max_users=max_users, max_shared=max_shared)
    cache.attend_shared(*args, **more)
    first = out.clone()
    out.fill_(9.0)
    cache.attend_shared(*args, **more)
    assert torch.equal(first, out)             # whoever ends first
    users = n if max_users is None else max_users
    if max_shared is not None:
        tokens = [min(x, max_shared) for x in tokens]
    want, wl, size, spread = S.attend(ref, q.float().cpu().numpy(), shared, tokens, firsts, users,
                                      table, own, [Q] * n if q_lens is None else q_lens, scale)
    off = 4 * D * 2.0 ** -24 * spread + 2.0 ** -18
    bound = UNIT[dtype] * np.abs(want) + (2.0 ** -11 + off)[..., None] * size * 1.01 + 1e-7
    err = np.abs(out.float().cpu().numpy().astype(np.float64) - want)
    assert (err <= bound).all(), (np.argwhere(err > bound)[:5], (err / bound).max())
    got = lse.cpu().numpy().astype(np.float64)
    assert (np.isinf(got) == np.isinf(wl)).all()
    fin = np.isfinite(wl)
    lerr = np.abs(np.where(fin, got - np.where(fin, wl, 0), 0))
    assert (lerr <= off + 2.0 ** -20 * np.abs(np.where(fin, wl, 0))).all()
    say("err / bound", float((err / bound).max()))
    return out, lse


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("H,group,D", [(2, 4, 128), (1, 1, 64), (3, 3, 64), (1, 8, 256)])
@pytest.mark.parametrize("tokens,firsts,n,own", [
    ([100], [0, 3], 3, [1, 70, 64]),                       # one context, few rows
    ([130, 1, 64], [0, 4, 4, 9], 9, [1, 2, 3, 0, 65, 200, 1, 128, 5]),   # one nobody reads
    ([700], [0, 20], 20, [5 + i for i in range(20)]),       # many rows a head
    ([65, 300], [2, 3, 14], 16, None),                      # no own tokens, some without context
])
def test_one_token(H, group, D, dtype, tokens, firsts, n, own):
    check(H, group, D, dtype, tokens, firsts, n, own, seed=D + n)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("H,group,D,tokens,firsts,own,q_lens,Q", [
    (2, 4, 128, [300], [0, 4], [20, 7, 6, 64], [6, 1, 0, 3], 6),
    (1, 3, 64, [64, 200], [0, 1, 3], [50, 50, 50], None, 40),
    (2, 2, 128, [500, 30], [0, 1, 2], None, [100, 33], 100),
    (1, 2, 256, [200], [0, 2], [150, 140], [130, 140], 140),
    (1, 1, 64, [1500], [0, 1], None, None, 300),
    (2, 8, 128, [190], [0, 5], [3, 3, 9, 3, 70], [3, 3, 2, 3, 3], 3),
])
def test_query_tokens(H, group, D, dtype, tokens, firsts, own, q_lens, Q):
    check(H, group, D, dtype, tokens, firsts, firsts[-1], own, q_lens, Q, seed=Q)


def test_the_same_as_one_sequence():
    """A context and a sequence's own tokens are that sequence's attention over both: where the
    context fills its pages, ``attend`` over one row of them all."""
    torch = torch_cuda()
    rng = np.random.default_rng(1)
    H, D, HQ, T, own = 2, 128, 8, 640, 100
    order = rng.permutation(40)
    shared, tails = order[:10], order[10:16].reshape(3, 2)
    cache = make(torch, 40, H, D)
    q = torch.randn(3, 4, HQ, D, device="cuda").half()
    whole = np.concatenate([np.tile(shared, (3, 1)), tails], 1).astype(np.int32)
    a = cache.attend(q, torch.from_numpy(whole).cuda(), ints(torch, [T + own] * 3))
    b = cache.attend_shared(q, ints(torch, [shared.tolist()]), ints(torch, [T]), ints(torch, [0, 3]),
                            table=torch.from_numpy(tails.astype(np.int32)).cuda(),
                            lengths=ints(torch, [own] * 3))
    # both are within half a step and the weights' rounding of the same value
    assert float((a.float() - b.float()).abs().max()) <= 4 * 2.0 ** -11 * float(a.float().abs().max())


@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("group,Q", [(2, 1), (4, 20)])
def test_bounds_and_strides(own, group, Q):
    """More sequences than max_users: those behind see no context; rows with strides of their own."""
    lengths = [Q + 3 * i for i in range(7)] if own else None
    check(2, group, 64, "float16", [200, 90], [0, 5, 7], 7, lengths, None, Q, max_users=3,
          strided=True, seed=3)


@pytest.mark.parametrize("firsts", [[0, 0, 0], [4, 4, 4], [5, 2, 1], [-3, 2, 100], [1, 3, 2]])
@pytest.mark.parametrize("own", [True, False])
def test_firsts_are_not_trusted(firsts, own):
    """Whatever they say, only rows that exist are read and written; ascending ones that reach past
    the sequences are cut."""
    torch = torch_cuda()
    if firsts == sorted(firsts):
        check(1, 2, 64, "float16", [100, 70], firsts, 4, [3, 4, 5, 6] if own else None, seed=2)
        return
    cache = make(torch, 12, 1, 64)
    q = torch.randn(4, 1, 2, 64, device="cuda").half()
    around = torch.full((6, 1, 2, 64), 7.0, device="cuda").half()
    table = {"table": ints(torch, [[4], [5], [6], [7]]), "lengths": ints(torch, [3] * 4)} if own else {}
    cache.attend_shared(q, ints(torch, [[0, 1], [2, 3]]), ints(torch, [100, 70]), ints(torch, firsts),
                        out=around[1:5], **table)
    torch.cuda.synchronize()
    assert bool((around[[0, 5]] == 7).all())


@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("users,Q", [(2, 1), (30, 2)])
def test_lost_pages_and_what_is_not_seen(own, users, Q):
    """Pages that are no pages count as without tokens; behind lengths, NaN and Inf scales of pages
    that nobody sees reach nobody."""
    n = users + 1
    lengths = [Q + i for i in range(n)] if own else None

    def spoil(cache, shared, table):
        free = sorted(set(range(cache.n_pages)) - set(shared.ravel().tolist())
                      - set(() if table is None else table.ravel().tolist()))
        cache.k_scale[free], cache.v_scale[free] = float("nan"), float("inf")
    check(1, 4, 128, "bfloat16", [300, 100], [0, users, n], n, lengths, None, Q, lost=True,
          spoil=spoil, seed=8)


def test_empty_contexts_and_no_rows():
    """Contexts of no tokens; sequences whose own tokens are none and that have no context."""
    out, lse = check(1, 2, 64, "float16", [0, 5], [0, 2, 2], 4, [0, 3, 0, 2], seed=4)
    assert bool((out[0] == 0).all()) and bool((out[2] == 0).all())
    assert bool((lse[0] == -float("inf")).all())
    out, _ = check(1, 2, 64, "float16", [0], [0, 40], 41, None, None, 2, seed=4)
    assert bool((out == 0).all())


@pytest.mark.parametrize("own", [True, False])
def test_contexts_that_the_host_takes_for_empty(own):
    """max_shared 0 with more rows than fit the card at once, and a bound inside a page."""
    n = 300
    lengths = [1 + i % 60 for i in range(n)] if own else None
    for most in (0, 70):
        check(8, 8, 64, "float16", [100, 128], [0, 200, n], n, lengths, seed=17, max_shared=most)


@pytest.mark.parametrize("users", [3, 40])
@pytest.mark.parametrize("own", [True, False])
def test_v_scales_of_all_sizes(users, own):
    """V scales that are subnormal, zero, or far apart within a context: what a token adds is relative
    to what the others add, however small they are all."""
    for seed, scales in enumerate(([1e-41, 3e-42], [0.0, 0.0], [1e-30, 1e-2], [2.0 ** -120, 2.0 ** -127])):
        def spoil(cache, shared, table):
            at = shared.ravel().tolist()
            cache.v_scale[at[0::2]] = scales[0]
            cache.v_scale[at[1::2]] = scales[1]
            if table is not None:
                cache.v_scale[sorted(set(table.ravel().tolist()) - {-1})] = scales[0]
        out, _ = check(1, 2, 128, "bfloat16", [330], [0, users], users,
                       [3] * users if own else None, seed=seed, spoil=spoil)
        assert not bool(out.isnan().any())


def test_long_context_in_many_splits():
    check(1, 2, 128, "float16", [9000], [0, 2], 2, [300, 1], seed=6)
    check(1, 4, 64, "bfloat16", [7000, 64], [0, 30, 31], 31, [40] * 31, None, 3, seed=7)


def test_long_own_tokens():
    """Own tokens in splits of their own, of few rows and of many, behind contexts of both kinds."""
    check(1, 2, 128, "float16", [300], [0, 2], 2, [2500, 70], seed=10)
    check(1, 2, 64, "bfloat16", [300, 7], [0, 40, 41], 41, [1300] + [60] * 40, seed=11)
    check(1, 1, 64, "float16", [100], [0, 1], 1, [1500], [70], 80, seed=12)


def test_own_tokens_of_many_requests():
    """A wave for a request's own tokens and its join: pages by the dozen, none, a part of one; and own
    pages on both sides of where the waves of a workgroup take them."""
    own = [(37 * i) % 300 for i in range(110)]
    check(8, 2, 64, "float16", [150, 70], [0, 100, 109], 110, own, seed=20)
    check(8, 1, 128, "bfloat16", [90], [0, 97], 97, [1 + (91 * i) % 260 for i in range(97)],
          [(i % 4) for i in range(97)], 3, seed=21)
    check(7, 1, 256, "float16", [66], [0, 110], 110, [(53 * i) % 200 for i in range(110)], seed=22)
    for pages in (8, 9, 16, 17):
        check(2, 4, 128, "float16", [200], [0, 3], 3, [64 * pages, 64 * pages - 63, 5], seed=pages)


def test_many_rows_in_tiles():
    """More rows than a workgroup's: tiles of half and of all waves, with splits and without."""
    check(1, 4, 64, "float16", [500], [0, 40], 40, None, seed=13)
    check(2, 4, 128, "bfloat16", [700, 130], [0, 33, 70], 71, [9] * 71, None, 2, seed=14)
    check(8, 1, 64, "float16", [130] * 17, list(range(18)), 17, None, None, 270, seed=15)
    check(1, 2, 256, "float16", [900], [0, 80], 80, [3] * 80, seed=16)
    # few rows, of which two waves of a half have some, of contexts that fill the card
    check(8, 4, 128, "float16", [500] * 15 + [449], list(range(0, 161, 10)), 160, [3] * 160, seed=23)


def test_logits_far_apart():
    """A context whose logits lie far above or below the own tokens' (the join's references)."""
    for scale in (8.0, -8.0):
        def spoil(cache, shared, table):
            cache.k_scale[shared.ravel().tolist()] *= 20 if scale > 0 else 0.01
        check(1, 2, 64, "float16", [150], [0, 3], 3, [70, 1, 64], seed=9, scale=scale, spoil=spoil)


def test_room_for_more_requests_than_there_are():
    """max_users far above what a context has, with few requests and many: queries and results of
    requests that do not exist are neither read nor written (they would lie behind the tensors)."""
    for n, firsts, most in ((3, [0, 1, 3], 3), (400, [0, 390, 400], 400), (60, [0, 2, 60], 60)):
        check(1, 4, 64, "float16", [130, 64], firsts, n, None, seed=18, max_users=most)
        check(1, 4, 64, "float16", [130, 64], firsts, n, [2] * n, None, 2, seed=19, max_users=most)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("users,Q", [(3, 1), (40, 1), (9, 30)])
@pytest.mark.parametrize("own", [True, False])
def test_queries_that_are_no_numbers(own, users, Q, dtype):
    """NaN or Inf in one request's queries reach no other request (rows of one tile among them)."""
    torch = torch_cuda()
    H, D = 2, 128
    cache = make(torch, 10 + users, H, D)
    q = torch.randn(users, Q, 2 * H, D, device="cuda").to(getattr(torch, dtype))
    args = ints(torch, [list(range(9))]), ints(torch, [570]), ints(torch, [0, users])
    more = {"table": ints(torch, [[10 + i] for i in range(users)]),
            "lengths": ints(torch, [Q + 3] * users)} if own else {}
    want = cache.attend_shared(q, *args, **more).float()
    for value in (float("nan"), float("inf")):
        bad = q.clone()
        bad[1, Q - 1, 1, 5] = value
        got = cache.attend_shared(bad, *args, **more).float()
        assert bool(got[1, Q - 1, 1].isnan().any())
        got[1, Q - 1, 1] = want[1, Q - 1, 1]
        # both are within half a step and the weights' rounding of the same value
        most = (4 * 2.0 ** -11 + 2 * UNIT[dtype]) * float(want.abs().max())
        assert float((got - want).abs().max()) <= most
