"""Threads that share a cache and a stream: a call's launches go through one scratch, so no other
call may come between them. The library is replaced by one that watches (CPU tensors)."""
import threading
import time

import pytest

from paper_2310_07240_amd import kv8


class Watcher:
    """Stands for the library: how many calls are inside it at once, and the scratch they got."""

    def __init__(self):
        self.inside = self.most = 0
        self.seen = []

    def need(self, cache, seqs, attn):
        return 4096 + 4096 * (threading.get_ident() % 7)

    cg_kv8_attend_workspace_bytes = cg_kv8_select_workspace_bytes = need

    def run(self, *args):
        self.inside += 1
        self.most = max(self.most, self.inside)
        self.seen.append(args[-3:])
        time.sleep(0.002)                      # the GIL is free, as in a call through ctypes
        self.inside -= 1
        return 0

    cg_kv8_attend = cg_kv8_select = run


def test_launches_of_one_call_stay_together(monkeypatch):
    torch = pytest.importorskip("torch")
    w = Watcher()
    monkeypatch.setattr(kv8, "_lib", lambda: w)
    c = kv8.Kv8Cache(4, 2, 64, device="cpu")
    c._handle = lambda stream: 77
    c._capturing = lambda *_: False
    table = torch.zeros((1, 2), dtype=torch.int32)
    n = torch.full((1,), 100, dtype=torch.int32)
    q = torch.zeros((1, 1, 4, 64), dtype=torch.float16)

    def work():
        for _ in range(10):
            c.attend(q, table, n)
            c.select(q, table, n, 1)

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(w.seen) == 80 and w.most == 1
    for address, size, handle in w.seen:
        assert address and size >= 4096 and handle == 77


def test_a_refused_call_lets_others_in(monkeypatch):
    torch = pytest.importorskip("torch")
    w = Watcher()
    w.cg_kv8_attend = lambda *args: -1
    monkeypatch.setattr(kv8, "_lib", lambda: w)
    c = kv8.Kv8Cache(4, 2, 64, device="cpu")
    c._handle = lambda stream: 77
    c._capturing = lambda *_: False
    table = torch.zeros((1, 2), dtype=torch.int32)
    n = torch.full((1,), 100, dtype=torch.int32)
    q = torch.zeros((1, 1, 4, 64), dtype=torch.float16)
    for _ in range(2):
        with pytest.raises(RuntimeError):
            c.attend(q, table, n)
    c.select(q, table, n, 1)
    assert len(w.seen) == 1
