"""What a reservation grants, C ABI and binding: refusals, decided on the host."""
import ctypes

import pytest

from paper_2310_07240_amd import kv8
from test_kv8_abi import A, BAD_CACHE, FAKE, L, cache, seqs
from test_sharing_abi import BIG, bound, kv8_code  # noqa: F401  (a fixture)

ODD = ctypes.c_void_p(A + 2)


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_bad_caches(kw, code):
    assert L().cg_kv8_reserve_granted(cache(**kw), seqs(), *[FAKE] * 5, FAKE, BIG, None) == code


@pytest.mark.parametrize("kw,code", [(dict(n=0), -2), (dict(width=0), -2), (dict(n=1 << 21), -2),
                                     (dict(table=A + 2), -1)])
def test_bad_sequences(kw, code):
    assert L().cg_kv8_reserve_granted(cache(), seqs(**kw), *[FAKE] * 5, FAKE, BIG, None) == code


def test_pointers_and_workspace():
    l, c, s = L(), cache(), seqs()
    for bad in (None, ODD):
        for i in range(5):
            args = [FAKE] * 5
            args[i] = bad
            # (without a workspace: no call gets past the checks)
            assert l.cg_kv8_reserve_granted(c, s, *args, None, BIG, None) == -1
    need = l.cg_kv8_reserve_workspace_bytes(c, s)
    for granted in (FAKE, None):
        assert l.cg_kv8_reserve_granted(c, s, *[FAKE] * 4, granted, FAKE, need - 1,
                                        None) == kv8_code("CAPACITY")
    assert l.cg_kv8_reserve_granted(c, s, *[FAKE] * 4, ODD, FAKE, need - 1, None) == -1


def test_the_binding(bound, monkeypatch):  # noqa: F811
    torch, w, c, good = bound
    monkeypatch.setattr(c, "_handle", lambda stream: 0)
    monkeypatch.setattr(c, "_scratch", lambda *a: (0, 8192, None))
    kw = good["reserve"]
    c.reserve(**kw, granted=torch.zeros(2, dtype=torch.int32))
    c.reserve(**kw)
    assert w.calls == ["cg_kv8_reserve_granted"] * 2
    for bad in (torch.zeros(2), torch.zeros(3, dtype=torch.int32),
                torch.zeros(2, dtype=torch.int32, device="meta")):
        with pytest.raises(ValueError):
            c.reserve(**kw, granted=bad)
    assert len(w.calls) == 2
