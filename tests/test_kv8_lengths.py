"""A bound of the lengths above the table's row (INT32_MAX: the caller knows none) lays work and
scratch out for the row, and neither wraps where tokens are rounded up to pages."""
import pytest

from test_kv8_abi import A, FAKE, L, attn, cache, seqs

TOP = 2 ** 31 - 1


@pytest.mark.parametrize("width", [1, 4, 300])
@pytest.mark.parametrize("kw", [dict(), dict(mass_out=A), dict(n_q=40, n_q_heads=16), dict(n_picks=3)])
def test_scratch_is_for_the_tables_row(width, kw):
    s, c = seqs(width=width), cache()
    for query in (L().cg_kv8_attend_workspace_bytes, L().cg_kv8_select_workspace_bytes):
        want = query(c, s, attn(max_len=64 * width, **kw))
        assert query(c, s, attn(max_len=TOP, **kw)) == want
        assert query(c, s, attn(max_len=64 * width + 1, **kw)) == want
        assert query(c, s, attn(max_len=64 * width - 1, **kw)) == want


def test_rows_past_32_bits():
    """A row of 2^25 pages or more names 2^31 tokens: the bound stays below, in whole pages."""
    s, c = seqs(n=1, width=2 ** 26), cache()
    a = attn(max_len=TOP, n_picks=3)
    need = L().cg_kv8_select_workspace_bytes(c, s, a)
    assert need == L().cg_kv8_select_workspace_bytes(c, s, attn(max_len=TOP - 63, n_picks=3))


def test_eviction_asks_for_no_more_pages_than_the_row_has():
    # 100000 tokens are to be kept, but the row holds 256: four new pages will do (the refusal that
    # is left is the missing list of kept tokens)
    assert L().cg_kv8_evict(cache(), seqs(width=4), FAKE, TOP, FAKE, 100000, 10, seqs(width=3), FAKE,
                            FAKE, None) == -3
    assert L().cg_kv8_evict(cache(), seqs(width=4), FAKE, TOP, FAKE, 100000, 10, seqs(width=4), None,
                            FAKE, None) == -1


def test_binding_bounds_the_tables_row(monkeypatch):
    """A table of 2^25 columns names more tokens than the C ABI's bound holds."""
    torch = pytest.importorskip("torch")
    from paper_2310_07240_amd import kv8
    got = []

    class Lib:
        def cg_kv8_attend(self, cache, s, a, *_):
            got.append(kv8._ATTN.unpack(a)[5])
            return 0

        def cg_kv8_evict(self, cache, s, lengths, max_len, *_):
            got.append(max_len)
            return 0

        def cg_kv8_attend_workspace_bytes(self, *_):
            return 0

    monkeypatch.setattr(kv8, "_lib", Lib)
    c = kv8.Kv8Cache(4, 2, 64, device="cpu")
    c._handle = lambda stream: 0
    n = torch.zeros(1, dtype=torch.int32)
    q = torch.zeros((1, 1, 4, 64), dtype=torch.float16)
    mass = torch.zeros((4, 2, 64))
    for width in (3, 2 ** 25):
        t = torch.zeros((1, width), dtype=torch.int32)
        c.attend(q, t, n)
        c.evict(t, n, mass, 10, 1, t[:, :1].contiguous())
    assert got == [192, 192, TOP, TOP]
