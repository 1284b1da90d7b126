"""Contexts read by unequal numbers of requests, C ABI: scratch and refusals follow the requests that
there are, whatever the bound of a context's requests leaves room for. Host only."""
import pytest

from paper_2310_07240_amd import kv8
from test_kv8_abi import A, FAKE, L, attn, cache, seqs
from test_sharing_abi import BIG, contexts, kv8_code


def need(C, n, users, n_q=1, group=4, H=8, max_shared=1 << 14, max_len=64, own=True, D=128):
    x = contexts(seqs=seqs(C, 256), max_len=max_shared, max_users=users)
    s = seqs(n, 4) if own else seqs(n, 0, None)
    a = attn(n_q=n_q, n_q_heads=H * group, max_len=max_len)
    return L().cg_kv8_attend_shared_workspace_bytes(cache(n_heads=H, head_dim=D), x, s, a)


@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("C,each", [(64, 16), (32, 9), (200, 1), (3, 300)])
def test_scratch_follows_the_requests(C, each, own):
    """A state is D + 2 numbers of 32 bits; the rows of all requests and one tile of 16 of every context
    are the most that there can be, in 256 splits at most, and in no more than with the exact bound."""
    n = C * each
    exact, loose = need(C, n, each, own=own), need(C, n, n, own=own)
    assert loose >= exact > 0 or exact == loose == 0
    # (a context's last tile may be begun: as many tiles more as contexts)
    assert loose <= 2 * exact + 4096
    if own:
        tiles = n * 4 // 16 + C
        assert loose <= kv8.ZEROED + tiles * 8 * 256 * 16 * (128 + 2) * 4 + 4096


@pytest.mark.parametrize("kw", [
    dict(C=420, n=420, users=420, n_q=6),                  # contexts of a request each
    dict(C=64, n=64, users=64, n_q=448, H=16, group=1),    # (with own tokens, so that there is scratch)
    dict(C=1024, n=4096, users=4096),
])
def test_bounds_that_the_requests_do_not_reach(kw):
    x = contexts(seqs=seqs(kw["C"], 256), max_len=1 << 14, max_users=kw["users"])
    s = seqs(kw["n"], 4) if kw.get("own", True) else seqs(kw["n"], 0, None)
    H = kw.get("H", 8)
    a = attn(n_q=kw.get("n_q", 1), n_q_heads=H * kw.get("group", 4))
    # (nothing is refused but a workspace that is too small)
    assert need(**kw) > kv8.ZEROED
    assert L().cg_kv8_attend_shared(cache(n_heads=H), x, s, a, FAKE, kv8.ZEROED,
                                    None) == kv8_code("CAPACITY")


@pytest.mark.parametrize("n,C,n_q,bad", [(1 << 19, 1 << 19, 8, False), (1 << 19, 1 << 19, 9, True),
                                         (1, 1 << 20, 8, False), (2, 1 << 20, 8, True)])
def test_too_many_rows(n, C, n_q, bad):
    """The smaller of what the contexts have room for and n_seq + contexts, times the query tokens:
    2^23 at most."""
    kw = dict(n_q=n_q, group=1, H=1, max_shared=64, max_len=8)
    assert (need(C, n, n, **kw) == 0) == bad
    if bad:
        x = contexts(seqs=seqs(C, 1), max_len=64, max_users=n)
        a = attn(n_q=n_q, n_q_heads=1, max_len=8)
        assert L().cg_kv8_attend_shared(cache(n_heads=1), x, seqs(n, 4), a, FAKE, BIG, None) == -2
