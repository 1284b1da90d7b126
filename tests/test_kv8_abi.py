"""The 8-bit serving cache's C ABI: every refusal is decided on the host, before any pointer is
followed, and the binding refuses tensors of the wrong type, shape or layout."""
import ctypes
import math

import pytest

from paper_2310_07240_amd import kv8

A = 1 << 20
FAKE = ctypes.c_void_p(A)


def cache(**kw):
    d = dict(n_pages=10, n_heads=2, head_dim=128, k_codes=A, v_codes=A, k_scale=A, v_scale=A,
             k_bounds=A)
    d.update(kw)
    return kv8._Cache(**d)


def seqs(n=2, width=4, table=A):
    return kv8._Seqs(n, width, table)


def rows(data=A):
    return kv8._Rows(data, 1000, 100, 128)


def attn(**kw):
    a = kv8._Attn()
    d = dict(n_q=1, n_q_heads=8, dtype=0, scale=0.1, lengths=A, max_len=200, q=rows(), out=rows())
    d.update(kw)
    for k, v in d.items():
        setattr(a, k, v)
    return a


class Checked:
    """The library with the structures passed by address."""

    def __getattr__(self, name):
        fn = getattr(kv8._lib(), name)

        def call(*args):
            return fn(*(ctypes.addressof(a) if isinstance(a, ctypes.Structure) else a
                        for a in args))
        return call


def L():
    return Checked()


BAD_CACHE = [(dict(n_pages=0), -2), (dict(n_heads=-1), -2), (dict(head_dim=96), -2),
             (dict(k_codes=None), -1), (dict(v_codes=A + 8), -1), (dict(k_scale=A + 2), -1),
             (dict(v_scale=None), -1), (dict(k_bounds=A + 4), -1)]


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_bad_caches(kw, code):
    c = cache(**kw)
    r = rows()
    assert L().cg_kv8_store(c, seqs(), FAKE, None, 5, 0, r, r, None, None) == code
    assert L().cg_kv8_load(c, seqs(), FAKE, None, 5, 0, r, r, None) == code
    assert L().cg_kv8_attend(c, seqs(), attn(), FAKE, 1 << 40, None) == code
    assert L().cg_kv8_attend_workspace_bytes(c, seqs(), attn()) == 0
    assert L().cg_kv8_select(c, seqs(), attn(n_picks=2), 1, FAKE, FAKE, 1 << 40, None) == code
    assert L().cg_kv8_select_workspace_bytes(c, seqs(), attn(n_picks=2)) == 0
    assert L().cg_kv8_evict(c, seqs(), FAKE, 200, FAKE, 100, 10, seqs(), FAKE, FAKE, None) == code


@pytest.mark.parametrize("s,code", [(seqs(n=0), -2), (seqs(width=0), -2), (seqs(table=None), -1),
                                    (seqs(table=A + 2), -1), (seqs(n=1 << 21), -2)])
def test_bad_sequences(s, code):
    r = rows()
    assert L().cg_kv8_store(cache(), s, FAKE, None, 5, 0, r, r, None, None) == code
    assert L().cg_kv8_load(cache(), s, FAKE, None, 5, 0, r, r, None) == code
    assert L().cg_kv8_attend(cache(), s, attn(), FAKE, 1 << 40, None) == code
    assert L().cg_kv8_evict(cache(), s, FAKE, 200, FAKE, 100, 10, seqs(), FAKE, FAKE, None) == code
    assert L().cg_kv8_evict(cache(), seqs(), FAKE, 200, FAKE, 100, 10, s, FAKE, FAKE, None) == code


def test_store_and_load_refusals():
    c, s, r = cache(), seqs(), rows()
    for fn in (lambda *a: L().cg_kv8_store(c, s, *a, None, None),
               lambda *a: L().cg_kv8_load(c, s, *a, None)):
        assert fn(None, None, 5, 0, r, r) == -1
        assert fn(FAKE, None, 0, 0, r, r) == -2
        assert fn(FAKE, None, 5, 2, r, r) == -1
        assert fn(FAKE, None, 5, 0, rows(None), r) == -1
        assert fn(FAKE, None, 5, 0, r, rows(A + 1)) == -1
        assert fn(FAKE, ctypes.c_void_p(A + 1), 5, 0, r, r) == -1
        assert fn(FAKE, None, 5, 0, None, r) == -1
    assert L().cg_kv8_store(c, s, FAKE, None, 5, 0, r, r, ctypes.c_void_p(A + 2), None) == -1
    assert L().cg_kv8_store(None, s, FAKE, None, 5, 0, r, r, None, None) == -1
    assert L().cg_kv8_store(c, None, FAKE, None, 5, 0, r, r, None, None) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(n_q=0), -2), (dict(n_q_heads=7), -2), (dict(n_q_heads=0), -2), (dict(max_len=-1), -2),
    (dict(n_q=1 << 30), -2), (dict(dtype=3), -1), (dict(q=rows(None)), -1),
    (dict(lengths=None), -1), (dict(lengths=A + 1), -1), (dict(q_lens=A + 2), -1),
    (dict(out=rows(A + 1)), -1), (dict(lse=A + 2), -1), (dict(scale=math.nan), -6),
    (dict(decay=math.inf), -6), (dict(picks=A, n_picks=0), -2), (dict(picks=A + 1, n_picks=1), -1),
    (dict(mass_in=A), -1), (dict(mass_out=A + 1), -1),
    (dict(mass_out=A, picks=A, n_picks=3), -1)])
def test_attend_refusals(kw, code):
    a = attn(**kw)
    assert L().cg_kv8_attend(cache(), seqs(), a, FAKE, 1 << 40, None) == code
    assert L().cg_kv8_attend_workspace_bytes(cache(), seqs(), a) == 0
    assert L().cg_kv8_attend(cache(), seqs(), None, FAKE, 1 << 40, None) == -1


def test_attend_workspace():
    a = attn(max_len=100000, mass_out=A)
    s = seqs(width=2000)
    need = L().cg_kv8_attend_workspace_bytes(cache(), s, a)
    assert need > 0
    assert L().cg_kv8_attend(cache(), s, a, FAKE, need - 1, None) == -3
    assert L().cg_kv8_attend(cache(), s, a, None, need, None) == -1
    assert L().cg_kv8_attend(cache(), s, a, ctypes.c_void_p(A + 64), need, None) == -1


def test_select_refusals():
    s = seqs()
    a = attn(n_picks=2)
    need = L().cg_kv8_select_workspace_bytes(cache(), s, a)

    def sel(c=None, a=a, recent=1, out=FAKE, ws=FAKE, size=need):
        return L().cg_kv8_select(c or cache(), s, a, recent, out, ws, size, None)

    assert need > 0 and sel(size=need - 1) == -3
    assert sel(c=cache(k_bounds=None)) == -1
    assert sel(a=attn(n_picks=0)) == -2
    assert sel(recent=-1) == -2
    assert sel(out=None) == -1 and sel(out=ctypes.c_void_p(A + 2)) == -1
    assert sel(ws=ctypes.c_void_p(A + 8)) == -1


def test_evict_refusals():
    def ev(lengths=FAKE, max_len=200, mass=FAKE, keep=100, recent=10, to=None, kept=FAKE, new=FAKE):
        return L().cg_kv8_evict(cache(), seqs(), lengths, max_len, mass, keep, recent,
                                to or seqs(), kept, new, None)

    assert ev(keep=0) == -2 and ev(recent=-1) == -2 and ev(max_len=-5) == -2
    assert ev(to=seqs(n=3)) == -2
    assert ev(to=seqs(width=1)) == -3                     # 100 tokens need two pages
    assert ev(lengths=None) == -1 and ev(mass=ctypes.c_void_p(A + 2)) == -1
    assert ev(kept=None) == -1 and ev(new=ctypes.c_void_p(A + 1)) == -1


def test_binding_refuses_tensors():
    """Shapes, types and layouts, on CPU tensors: nothing reaches the library."""
    import torch
    with pytest.raises(RuntimeError):
        kv8.Kv8Cache(4, 2, 96, device="cpu")
    c = kv8.Kv8Cache(4, 2, 64, device="cpu")
    t = torch.zeros((3, 2), dtype=torch.int32)
    n = torch.zeros(3, dtype=torch.int32)
    q = torch.zeros((3, 1, 4, 64), dtype=torch.float16)
    k = torch.zeros((3, 5, 2, 64), dtype=torch.float16)
    bad = [lambda: c.attend(q.float(), t, n), lambda: c.attend(q[..., ::2], t, n),
           lambda: c.attend(q, t.long(), n), lambda: c.attend(q, t, n[:2]),
           lambda: c.attend(q, t.t(), n), lambda: c.attend(q, t, None),
           lambda: c.attend(q[:2], t, n), lambda: c.attend(q[0], t, n),
           lambda: c.store(k.float(), k, t, n), lambda: c.store(k, k.bfloat16(), t, n),
           lambda: c.store(k[:, :, :1], k, t, n), lambda: c.store(k, k[:, :4], t, n),
           lambda: c.store(k, k, t, n.long()), lambda: c.store(k, k, t, None),
           lambda: c.store(k, k, t, n, counts=n[:1]),
           lambda: c.store(k, k, t[0], n)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(ValueError):
        kv8.Kv8Cache(4, 2, 64, buffers={"k_codes": torch.zeros((4, 2, 64, 64), dtype=torch.int8)})
