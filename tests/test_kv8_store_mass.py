"""store's weights argument: refusals, on the host."""
import ctypes

import pytest

from paper_2310_07240_amd import kv8
from test_kv8_abi import A, FAKE, L, cache, rows, seqs


def test_misaligned_weights_are_refused():
    r = rows()
    for mass in (A + 1, A + 2):
        assert L().cg_kv8_store(cache(mass=mass), seqs(), FAKE, None, 5, 0, r, r, None, None) == -1


def test_binding_refuses_weights():
    torch = pytest.importorskip("torch")
    c = kv8.Kv8Cache(4, 2, 64, device="cpu")
    c._handle = lambda stream: pytest.fail("reached the launch")
    t = torch.zeros((3, 2), dtype=torch.int32)
    n = torch.zeros(3, dtype=torch.int32)
    k = torch.zeros((3, 5, 2, 64), dtype=torch.float16)
    good = torch.zeros((4, 2, 64))
    for bad in (good[:3], good.half(), good[:, :, :32], good.transpose(0, 1)):
        with pytest.raises(ValueError):
            c.store(k, k, t, n, mass=bad)


def test_store_hands_the_weights_on(monkeypatch):
    torch = pytest.importorskip("torch")
    c = kv8.Kv8Cache(4, 2, 64, device="cpu")
    got = []

    class Lib:
        def cg_kv8_store(self, cache, *args):
            p = cache if isinstance(cache, int) else ctypes.addressof(cache._obj)
            got.append(kv8._Cache.from_address(p).mass)
            return 0

    monkeypatch.setattr(kv8, "_lib", Lib)
    c._handle = lambda stream: 0
    t = torch.zeros((3, 2), dtype=torch.int32)
    n = torch.zeros(3, dtype=torch.int32)
    k = torch.zeros((3, 5, 2, 64), dtype=torch.float16)
    mass = torch.zeros((4, 2, 64))
    c.store(k, k, t, n, mass=mass)
    c.store(k, k, t, n)
    assert got == [mass.data_ptr(), None]
