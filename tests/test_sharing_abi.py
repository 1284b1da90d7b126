"""Requests that share a context, C ABI and binding: every refusal is decided on the host, before any
pointer is followed, and the binding refuses tensors of the wrong type, shape or device."""
import ctypes

import pytest

from paper_2310_07240_amd import kv8
from test_kv8_abi import A, BAD_CACHE, FAKE, L, attn, cache, seqs

BIG = 1 << 40


def contexts(n=2, width=4, **kw):
    d = dict(seqs=seqs(n, width), lengths=A, max_len=200, firsts=A, max_users=2)
    d.update(kw)
    return kv8._Contexts(**d)


def verify(**kw):
    d = dict(n_seq=2, n_drafts=3, vocab=100, dtype=2, target=A, t_seq_stride=400, t_row_stride=100,
             draft=A, d_seq_stride=300, d_row_stride=100, drafts=A, counts=A, u=A, tokens=A,
             accepted=A, lengths=A, new_lengths=A)
    d.update(kw)
    return kv8._Verify(**d)


def calls(c=None, s=None):
    """Every call with everything right but the workspace, which is missing where one is needed."""
    c, s = c or cache(), s or seqs()
    l = L()
    return {"fork": l.cg_kv8_fork(c, s, FAKE, FAKE, FAKE, seqs(3, 2), FAKE, FAKE, None),
            "reserve": l.cg_kv8_reserve(c, s, FAKE, FAKE, FAKE, FAKE, None, BIG, None),
            "release": l.cg_kv8_release(c, s, ctypes.c_void_p(A + 2), FAKE, None),
            "compact": l.cg_kv8_compact(c, s, FAKE, FAKE, ctypes.c_void_p(2 * A), FAKE, FAKE, None, BIG,
                                        None),
            "attend_shared": l.cg_kv8_attend_shared(c, contexts(), s, attn(), None, BIG, None)}


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_bad_caches(kw, code):
    c = cache(**kw)
    assert set(calls(c).values()) == {code}
    assert L().cg_kv8_copy(c, FAKE, FAKE, 3, None) == code
    assert L().cg_kv8_reserve_workspace_bytes(c, seqs()) == 0
    assert L().cg_kv8_compact_workspace_bytes(c) == 0
    assert L().cg_kv8_attend_shared_workspace_bytes(c, contexts(), seqs(), attn()) == 0


@pytest.mark.parametrize("kw,code", [(dict(n=0), -2), (dict(width=0), -2), (dict(n=1 << 21), -2),
                                     (dict(table=A + 2), -1)])
def test_bad_sequences(kw, code):
    assert set(calls(None, seqs(**kw)).values()) == {code}
    assert L().cg_kv8_fork(cache(), seqs(), FAKE, FAKE, FAKE, seqs(**kw), FAKE, FAKE, None) == code
    assert L().cg_kv8_reserve_workspace_bytes(cache(), seqs(**kw)) == 0
    assert L().cg_kv8_attend_shared(cache(), contexts(seqs=seqs(**kw)), seqs(), attn(), FAKE, BIG,
                                    None) == code


def test_null_structs():
    l, c = L(), cache()
    assert l.cg_kv8_fork(None, seqs(), FAKE, FAKE, None, seqs(), FAKE, FAKE, None) == -1
    assert l.cg_kv8_fork(c, None, FAKE, FAKE, None, seqs(), FAKE, FAKE, None) == -1
    assert l.cg_kv8_fork(c, seqs(), FAKE, FAKE, None, None, FAKE, FAKE, None) == -1
    assert l.cg_kv8_attend_shared(c, None, seqs(), attn(), FAKE, BIG, None) == -1
    assert l.cg_kv8_attend_shared(c, contexts(), None, attn(), FAKE, BIG, None) == -1
    assert l.cg_kv8_attend_shared(c, contexts(), seqs(), None, FAKE, BIG, None) == -1
    assert l.cg_verify_drafts(None, FAKE, BIG, None) == -1
    assert l.cg_verify_workspace_bytes(None) == 0


ODD = ctypes.c_void_p(A + 2)


@pytest.mark.parametrize("bad", [None, ODD])
def test_pointers_of_the_page_calls(bad):
    l, c, s = L(), cache(), seqs()
    for i in (0, 1):
        args = [FAKE, FAKE]
        args[i] = bad
        assert l.cg_kv8_fork(c, s, *args, None, seqs(), FAKE, FAKE, None) == -1
        assert l.cg_kv8_fork(c, s, FAKE, FAKE, None, seqs(), *args, None) == -1
        assert l.cg_kv8_copy(c, *args, 3, None) == -1
    for i in range(4):
        args = [FAKE] * 4
        args[i] = bad
        assert l.cg_kv8_reserve(c, s, *args, FAKE, BIG, None) == -1
    for i in range(5):
        args = [FAKE, FAKE, ctypes.c_void_p(2 * A), FAKE, FAKE]
        args[i] = bad
        assert l.cg_kv8_compact(c, s, *args, FAKE, BIG, None) == -1
    assert l.cg_kv8_release(c, s, None, bad, None) == -1
    assert l.cg_kv8_compact(c, s, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, BIG, None) == -1   # in place
    assert l.cg_kv8_fork(c, s, FAKE, FAKE, ODD, seqs(), FAKE, FAKE, None) == -1


def test_sizes_and_workspaces_of_the_page_calls():
    l, c, s = L(), cache(), seqs()
    assert l.cg_kv8_fork(c, s, FAKE, FAKE, None, seqs(3, 3), FAKE, FAKE, None) == kv8_code("CAPACITY")
    assert l.cg_kv8_copy(c, FAKE, FAKE, 0, None) == -2
    assert l.cg_kv8_copy(cache(n_heads=(1 << 21) + 1), FAKE, FAKE, 1, None) == -2
    need = l.cg_kv8_reserve_workspace_bytes(c, s)
    assert need > kv8.ZEROED
    assert l.cg_kv8_reserve(c, s, *[FAKE] * 4, None, BIG, None) == -1
    assert l.cg_kv8_reserve(c, s, *[FAKE] * 4, ctypes.c_void_p(A + 64), BIG, None) == -1
    assert l.cg_kv8_reserve(c, s, *[FAKE] * 4, FAKE, need - 1, None) == kv8_code("CAPACITY")
    need = l.cg_kv8_compact_workspace_bytes(c)
    out = [FAKE, FAKE, ctypes.c_void_p(2 * A), FAKE, FAKE]
    assert l.cg_kv8_compact(c, s, *out, None, BIG, None) == -1
    assert l.cg_kv8_compact(c, s, *out, FAKE, need - 1, None) == kv8_code("CAPACITY")
    # a large pool and many sequences: sizes are 64-bit
    many = cache(n_pages=(1 << 31) - 1, n_heads=1)
    assert l.cg_kv8_compact_workspace_bytes(many) > 8 * ((1 << 31) - 1)
    assert l.cg_kv8_reserve_workspace_bytes(many, seqs(1 << 20, 1 << 14)) > 4 * ((1 << 31) - 1)


def kv8_code(name):
    from paper_2310_07240_amd.cachegen import ERRORS
    return next(code for code, text in ERRORS.items() if text == "CG_ERR_" + name)


@pytest.mark.parametrize("x,a,code", [
    (dict(lengths=None), {}, -1), (dict(firsts=None), {}, -1), (dict(firsts=A + 1), {}, -1),
    (dict(max_users=0), {}, -2), (dict(max_len=-1), {}, -2),
    ({}, dict(picks=A, n_picks=2), -1), ({}, dict(mass_out=A), -1), ({}, dict(lengths=None), -1),
    ({}, dict(n_q_heads=7), -2), ({}, dict(dtype=2), -1), ({}, dict(n_q=0), -2),
    ({}, dict(max_len=-1), -2), ({}, dict(lse=A + 2), -1), ({}, dict(q_lens=A + 2), -1),
    # rows of all users of a context past 2^30
    (dict(max_users=2, seqs=seqs(1 << 19, 4)), dict(n_q=128), -2),
])
def test_bad_attention(x, a, code):
    assert L().cg_kv8_attend_shared(cache(), contexts(**x), seqs(), attn(**a), FAKE, BIG, None) == code
    assert L().cg_kv8_attend_shared_workspace_bytes(cache(), contexts(**x), seqs(), attn(**a)) == 0


def test_attention_without_own_pages():
    """table NULL: the columns and the lengths are not looked at, everything else is."""
    l, none = L(), seqs(2, 0, None)
    assert l.cg_kv8_attend_shared(cache(), contexts(), none, attn(lengths=None, q_lens=A + 2), FAKE,
                                  BIG, None) == -1
    assert l.cg_kv8_attend_shared(cache(), contexts(lengths=None), none, attn(), FAKE, BIG, None) == -1
    assert l.cg_kv8_attend_shared(cache(), contexts(), seqs(0, 0, None), attn(), FAKE, BIG, None) == -2
    # short own tokens are joined where they are read; long ones have states, and scratch, of their own
    x = contexts(seqs=seqs(2, 100), max_len=6400)
    own = l.cg_kv8_attend_shared_workspace_bytes(cache(), x, seqs(), attn())
    alone = l.cg_kv8_attend_shared_workspace_bytes(cache(), x, none, attn(lengths=None))
    long = l.cg_kv8_attend_shared_workspace_bytes(cache(), x, seqs(2, 100), attn(max_len=6400))
    assert long > own >= alone > kv8.ZEROED
    assert l.cg_kv8_attend_shared(cache(), x, none, attn(), FAKE, alone - 1, None) == kv8_code("CAPACITY")
    assert l.cg_kv8_attend_shared(cache(), x, none, attn(), None, BIG, None) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(n_seq=0), -2), (dict(n_seq=(1 << 21) + 1), -2), (dict(n_drafts=-1), -2),
    (dict(n_drafts=1025), -2), (dict(vocab=0), -2), (dict(vocab=(1 << 20) + 1), -2),
    (dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(target=None), -1), (dict(target=A + 2), -1),
    (dict(dtype=0, target=A + 1), -1), (dict(draft=A + 2), -1), (dict(drafts=None), -1),
    (dict(drafts=A + 2), -1), (dict(counts=A + 1), -1), (dict(u=None), -1), (dict(u=A + 2), -1),
    (dict(tokens=None), -1), (dict(accepted=None), -1), (dict(lengths=None), -1),
    (dict(lengths=A + 2), -1), (dict(new_lengths=A + 2), -1),
])
def test_bad_drafts(kw, code):
    assert L().cg_verify_drafts(verify(**kw), FAKE, BIG, None) == code


def test_workspace_of_the_drafts():
    l = L()
    need = l.cg_verify_workspace_bytes(verify())
    assert need == kv8.ZEROED + 2 * 8
    assert l.cg_verify_workspace_bytes(verify(n_seq=1 << 21, vocab=1 << 20)) == (
        kv8.ZEROED + 1024 * 256 * 8)
    assert l.cg_verify_drafts(verify(), None, BIG, None) == -1
    assert l.cg_verify_drafts(verify(), FAKE, need - 1, None) == kv8_code("CAPACITY")
    assert l.cg_verify_drafts(verify(), ctypes.c_void_p(A + 16), BIG, None) == -1


# ---- the binding --------------------------------------------------------------------------------
class Noted:
    """The library replaced by one that notes its calls."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_workspace_bytes"):
            return lambda *args: 8192
        return lambda *args: self.calls.append(name) or 0


@pytest.fixture
def bound(monkeypatch):
    torch = pytest.importorskip("torch")
    w = Noted()
    monkeypatch.setattr(kv8, "_lib", lambda: w)
    c = kv8.Kv8Cache(6, 2, 64, device="cpu")
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    f = lambda *s: torch.zeros(s)
    good = {
        "fork": dict(table=i(2, 3), lengths=i(2), parents=i(4), refs=i(6), ends=i(4),
                     new_table=i(4, 3)),
        "reserve": dict(table=i(2, 3), lengths=i(2), counts=i(2), refs=i(6), mass=f(6, 2, 64),
                        missing=i(1)),
        "release": dict(table=i(2, 3), refs=i(6), keep=i(2)),
        "copy": dict(src=i(3), dst=i(3), mass=f(6, 2, 64)),
        "compact": dict(table=i(2, 3), refs=i(6), mass=f(6, 2, 64)),
        "attend_shared": dict(q=f(2, 1, 4, 64).half(), shared=i(1, 3), shared_lengths=i(1),
                              firsts=i(2), table=i(2, 3), lengths=i(2), q_lens=i(2),
                              out=f(2, 1, 4, 64).half(), lse=f(2, 1, 4)),
        "verify": dict(target=f(2, 3, 50), drafts=i(2, 2), u=f(2, 3), draft=f(2, 2, 50), counts=i(2),
                       lengths=i(2), tokens=i(2, 3), accepted=i(2), new_lengths=i(2)),
    }
    return torch, w, c, good


def test_host_memory_never_reaches_the_library(bound):
    torch, w, c, good = bound
    for name, kw in good.items():
        with pytest.raises(ValueError, match="GPU"):
            getattr(c, name)(**kw)
    assert not w.calls


def test_tensors_of_the_wrong_kind(bound, monkeypatch):
    torch, w, c, good = bound
    monkeypatch.setattr(c, "_handle", lambda stream: 0)
    monkeypatch.setattr(c, "_scratch", lambda *a: (0, 8192, None))
    for name, kw in good.items():
        getattr(c, name)(**kw)                          # all of it is right
        n = len(w.calls)
        for key, t in kw.items():
            for bad in (t.double() if t.is_floating_point() else t.long(),
                        torch.cat([t, t]) if t.dim() == 1 else t[..., None], t[:0],
                        t.to("meta")):
                if name == "compact" and key == "table" and len(bad) == 0:
                    continue                            # (no sequences: the library refuses it)
                with pytest.raises(ValueError):
                    getattr(c, name)(**{**kw, key: bad})
        assert len(w.calls) == n, name
    with pytest.raises(ValueError):
        c.attend_shared(**{**good["attend_shared"], "lengths": None})
    with pytest.raises(ValueError):
        c.verify(**{**good["verify"], "lengths": None})
    with pytest.raises(ValueError):
        c.verify(**{**good["verify"], "draft": good["verify"]["draft"].transpose(1, 2)})
    with pytest.raises(ValueError):
        c.reserve(**{**good["reserve"], "refs": good["reserve"]["refs"].repeat_interleave(2)[::2]})


def test_optional_arguments(bound, monkeypatch):
    torch, w, c, good = bound
    monkeypatch.setattr(c, "_handle", lambda stream: 0)
    monkeypatch.setattr(c, "_scratch", lambda *a: (0, 8192, None))
    drop = {"fork": ("ends", "new_table"), "reserve": ("mass", "missing"), "release": ("keep",),
            "copy": ("mass",), "compact": ("mass",), "attend_shared": ("q_lens", "out", "lse"),
            "verify": ("draft", "counts", "tokens", "accepted")}
    for name, keys in drop.items():
        getattr(c, name)(**{k: v for k, v in good[name].items() if k not in keys})
    kw = {k: v for k, v in good["verify"].items() if k not in ("lengths", "new_lengths")}
    assert len(c.verify(**kw)) == 2 and len(c.verify(**good["verify"])) == 3
    kw = {k: v for k, v in good["attend_shared"].items() if k not in ("table", "lengths")}
    assert c.attend_shared(**kw) is kw["out"]
    assert len(w.calls) == len(drop) + 3
    c.copy(torch.zeros(0, dtype=torch.int32), torch.zeros(0, dtype=torch.int32))   # nothing to do
    assert len(w.calls) == len(drop) + 3
