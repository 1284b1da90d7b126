"""Python binding of the 8-bit serving cache (include/cachegen.h, cg_kv8_*): a pool of 64-token
pages that holds decoded contexts as int8 codes under a scale per page and head, and the operators
on it — rows in and out (``store``, ``load``), attention of one or many query tokens
(``attend``), eviction by accumulated weight (``evict``) and the choice of the pages a query reads
(``select``).

Argument marshalling only, as in ``cachegen``: every step runs in the HIP kernels of
``libcachegen.so``, torch supplies buffers and the stream handle, and there is no CPU fallback.
Tensors are checked for type, shape and device before their addresses are passed on.
"""
from __future__ import annotations

import ctypes
import math

from .cachegen import CodecError, _check, lib

PAGE = 64
_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_I32 = ctypes.c_int32


class _Cache(ctypes.Structure):
    _fields_ = [("n_pages", _I32), ("n_heads", _I32), ("head_dim", _I32), ("k_codes", _P),
                ("v_codes", _P), ("k_scale", _P), ("v_scale", _P), ("k_bounds", _P)]


class _Seqs(ctypes.Structure):
    _fields_ = [("n_seq", _I32), ("max_pages", _I32), ("table", _P)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", _P), ("seq_stride", _I64), ("token_stride", _I64),
                ("head_stride", _I64)]


class _Attn(ctypes.Structure):
    _fields_ = [("n_q", _I32), ("n_q_heads", _I32), ("dtype", _I32), ("scale", ctypes.c_float),
                ("lengths", _P), ("max_len", _I32), ("q_lens", _P), ("q", _Rows), ("out", _Rows),
                ("lse", _P), ("picks", _P), ("n_picks", _I32), ("mass_in", _P), ("mass_out", _P),
                ("decay", ctypes.c_float)]


_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        L = lib()
        C, S, R, A = (ctypes.POINTER(t) for t in (_Cache, _Seqs, _Rows, _Attn))
        L.cg_kv8_store.argtypes = [C, S, _P, _P, _I32, _I32, R, R, _P, _P]
        L.cg_kv8_load.argtypes = [C, S, _P, _P, _I32, _I32, R, R, _P]
        L.cg_kv8_attend_workspace_bytes.argtypes = [C, S, A]
        L.cg_kv8_attend_workspace_bytes.restype = ctypes.c_uint64
        L.cg_kv8_attend.argtypes = [C, S, A, _P, ctypes.c_uint64, _P]
        L.cg_kv8_select_workspace_bytes.argtypes = [C, S, A]
        L.cg_kv8_select_workspace_bytes.restype = ctypes.c_uint64
        L.cg_kv8_select.argtypes = [C, S, A, _I32, _P, _P, ctypes.c_uint64, _P]
        L.cg_kv8_evict.argtypes = [C, S, _P, _I32, _P, _I32, _I32, S, _P, _P, _P]
        for n in ("store", "load", "attend", "select", "evict"):
            getattr(L, "cg_kv8_" + n).restype = ctypes.c_int
        _LIB = L
    return _LIB


def _need(ok, what):
    if not ok:
        raise ValueError(what)


class Kv8Cache:
    """A pool of pages on one GPU and the operators on it.

    Sequences are given by ``table`` [n_seq, columns] (int32 page numbers) and the number of
    tokens they hold. Lengths, starts and counts are int32 [n_seq]; everything is a contiguous
    tensor on the cache's device except rows of K, V, queries and outputs, which may have any
    strides as long as the head dimension is contiguous. Calls are asynchronous on ``stream``
    (default: the current one). Scratch is kept per stream and grows as needed.

    ``buffers``: tensors ``k_codes``, ``v_codes``, ``k_scale``, ``v_scale`` and (or None)
    ``k_bounds`` to use as the pool; without it they are allocated, zeroed.
    """

    def __init__(self, n_pages, n_heads, head_dim, device="cuda", buffers=None):
        import torch
        self.torch = torch
        P, H, D = int(n_pages), int(n_heads), int(head_dim)
        self.n_pages, self.n_heads, self.head_dim = P, H, D
        if P <= 0 or H <= 0 or D not in (64, 128, 256):
            raise CodecError(-2, "Kv8Cache")
        want = {"k_codes": ((P, H, PAGE, D), torch.int8), "v_codes": ((P, H, D, PAGE), torch.int8),
                "k_scale": ((P, H), torch.float32), "v_scale": ((P, H), torch.float32),
                "k_bounds": ((P, H, 2, D), torch.int8)}
        if buffers is None:
            buffers = {n: torch.zeros(s, dtype=t, device=device) for n, (s, t) in want.items()}
        self.device = buffers["k_codes"].device
        for n, (s, t) in want.items():
            b = buffers.get(n)
            _need(b is not None or n == "k_bounds", f"{n} is missing")
            if b is not None:
                self._tensor(b, n, t, s)
            setattr(self, n, b)
        self._c = _Cache(P, H, D, *(None if (b := getattr(self, n)) is None else b.data_ptr()
                                    for n in want))
        self._cp = ctypes.byref(self._c)
        self._ws = {}
        self._types = {torch.float16: 0, torch.bfloat16: 1}

    # ---- marshalling ---------------------------------------------------------------------
    def _tensor(self, t, name, dtype, shape=None):
        _need(t.dtype == dtype and t.device == self.device and t.is_contiguous()
              and (shape is None or t.shape == shape),
              f"{name}: a contiguous {dtype} tensor{'' if shape is None else ' of ' + str(tuple(shape))}"
              f" on {self.device} is wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _seqs(self, table):
        p = self._tensor(table, "table", self.torch.int32)
        _need(table.dim() == 2, "table: [n_seq, columns] is wanted")
        return _Seqs(table.shape[0], table.shape[1], p)

    def _per_seq(self, t, name, n):
        return None if t is None else self._tensor(t, name, self.torch.int32, (n,))

    def _rows(self, t, name, shape, dtype):
        _need(t.dtype == dtype and t.shape == shape and t.device == self.device
              and t.stride(3) == 1,
              f"{name}: {dtype} rows {tuple(shape)} with a contiguous last dimension on "
              f"{self.device} are wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
        s = t.stride()
        return _Rows(t.data_ptr(), s[0], s[1], s[2])

    def _scratch(self, stream, need):
        """The stream's scratch, allocated on that stream so that its reuse is ordered there."""
        ws = self._ws.get(stream.cuda_stream)
        if ws is None or ws.numel() < need:
            with self.torch.cuda.stream(stream):
                ws = self.torch.empty((need,), dtype=self.torch.uint8, device=self.device)
            self._ws[stream.cuda_stream] = ws
        return ws.data_ptr(), ws.numel()

    def _stream(self, stream):
        return self.torch.cuda.current_stream(self.device) if stream is None else stream

    # ---- rows in and out -----------------------------------------------------------------
    def store(self, k, v, table, starts, counts=None, status=None, stream=None):
        """Rows k, v [n_seq, n_tokens, n_heads, head_dim] become the sequences' tokens from
        ``starts`` on (``counts``: how many of each; default all). ``status``: an int32 tensor of
        one element that receives 0, or non-zero for NaN / Inf."""
        s = self._seqs(table)
        _need(k.dtype in self._types, "k: float16 or bfloat16 is wanted")
        shape = (s.n_seq, k.shape[1], self.n_heads, self.head_dim)
        kr, vr = self._rows(k, "k", shape, k.dtype), self._rows(v, "v", shape, k.dtype)
        _need(starts is not None, "starts is missing")
        st = None if status is None else self._tensor(status, "status", self.torch.int32, (1,))
        _check(_lib().cg_kv8_store(self._cp, s, self._per_seq(starts, "starts", s.n_seq),
                                   self._per_seq(counts, "counts", s.n_seq), shape[1],
                                   self._types[k.dtype], kr, vr, st,
                                   self._stream(stream).cuda_stream), "cg_kv8_store")

    def load(self, table, starts, n_tokens, counts=None, dtype=None, k=None, v=None, stream=None):
        """(k, v) [n_seq, n_tokens, n_heads, head_dim]: the sequences' tokens from ``starts`` on,
        zeros behind ``counts``. ``k``, ``v``: tensors to write into."""
        s = self._seqs(table)
        shape = (s.n_seq, int(n_tokens), self.n_heads, self.head_dim)
        stream = self._stream(stream)
        if k is None or v is None:
            dtype = dtype or self.torch.float16
            with self.torch.cuda.stream(stream):
                k = self.torch.empty(shape, dtype=dtype, device=self.device) if k is None else k
                v = self.torch.empty(shape, dtype=dtype, device=self.device) if v is None else v
        _need(k.dtype in self._types, "k: float16 or bfloat16 is wanted")
        _need(starts is not None, "starts is missing")
        _check(_lib().cg_kv8_load(self._cp, s, self._per_seq(starts, "starts", s.n_seq),
                                  self._per_seq(counts, "counts", s.n_seq), shape[1],
                                  self._types[k.dtype], self._rows(k, "k", shape, k.dtype),
                                  self._rows(v, "v", shape, k.dtype), stream.cuda_stream),
               "cg_kv8_load")
        return k, v

    # ---- attention -----------------------------------------------------------------------
    def _attn(self, q, s, lengths, q_lens, max_len):
        _need(q.dim() == 4 and q.dtype in self._types, "q: float16 or bfloat16 "
              "[n_seq, n_q, n_q_heads, head_dim] is wanted")
        _need(lengths is not None, "lengths is missing")
        a = _Attn()
        a.n_q, a.n_q_heads, a.dtype = q.shape[1], q.shape[2], self._types[q.dtype]
        a.lengths = self._per_seq(lengths, "lengths", s.n_seq)
        a.max_len = s.max_pages * PAGE if max_len is None else max_len
        a.q_lens = self._per_seq(q_lens, "q_lens", s.n_seq)
        a.q = self._rows(q, "q", (s.n_seq, a.n_q, a.n_q_heads, self.head_dim), q.dtype)
        return a

    def attend(self, q, table, lengths, scale=None, q_lens=None, max_len=None, out=None, lse=None,
               picks=None, mass=None, mass_out=None, decay=1.0, stream=None):
        """Causal attention of the queries q [n_seq, n_q, n_q_heads, head_dim], the last tokens of
        the sequences (``q_lens``: how many of each), over the sequences' pages; returns ``out``.

        scale     of q . k, default 1 / sqrt(head_dim).
        max_len   a bound of the lengths that the host knows (default: the table's width); the
                  work is laid out for it.
        lse       float32 [n_seq, n_q, n_q_heads] that receives the log-sum-exp.
        picks     int32 [n_seq, n_q, n_heads, n] from ``select``: only these pages are read.
        mass_out  float32 [n_pages, n_heads, 64] that receives decay * mass + the weight each
                  token got (``mass`` may be None, or the same tensor; given alone it is updated
                  in place)."""
        s = self._seqs(table)
        a = self._attn(q, s, lengths, q_lens, max_len)
        stream = self._stream(stream)
        f32 = self.torch.float32
        a.scale = 1.0 / math.sqrt(self.head_dim) if scale is None else scale
        if out is None:
            with self.torch.cuda.stream(stream):
                out = self.torch.empty(q.shape, dtype=q.dtype, device=self.device)
        a.out = self._rows(out, "out", q.shape, q.dtype)
        if lse is not None:
            a.lse = self._tensor(lse, "lse", f32, q.shape[:3])
        if picks is not None:
            _need(picks.dim() == 4, "picks: [n_seq, n_q, n_heads, n] is wanted")
            a.n_picks = picks.shape[3]
            a.picks = self._tensor(picks, "picks", self.torch.int32,
                                   (s.n_seq, a.n_q, self.n_heads, a.n_picks))
        if mass is not None or mass_out is not None:
            shape = (self.n_pages, self.n_heads, PAGE)
            mass_out = mass if mass_out is None else mass_out
            a.mass_in = None if mass is None else self._tensor(mass, "mass", f32, shape)
            a.mass_out = self._tensor(mass_out, "mass_out", f32, shape)
            a.decay = decay
        L = _lib()
        need = L.cg_kv8_attend_workspace_bytes(self._cp, s, a)
        ws, size = self._scratch(stream, need) if need else (None, 0)
        _check(L.cg_kv8_attend(self._cp, s, a, ws, size, stream.cuda_stream), "cg_kv8_attend")
        return out

    def select(self, q, table, lengths, n_picks, recent=1, q_lens=None, max_len=None, out=None,
               stream=None):
        """Table columns [n_seq, n_q, n_heads, n_picks] (int32, ascending, -1 behind the last) of
        the pages that each query token should read: the ``recent`` last ones it sees and the best
        of the others by the bound of their q . k."""
        s = self._seqs(table)
        a = self._attn(q, s, lengths, q_lens, max_len)
        stream = self._stream(stream)
        a.n_picks = int(n_picks)
        shape = (s.n_seq, a.n_q, self.n_heads, max(0, a.n_picks))
        if out is None:
            with self.torch.cuda.stream(stream):
                out = self.torch.empty(shape, dtype=self.torch.int32, device=self.device)
        L = _lib()
        need = L.cg_kv8_select_workspace_bytes(self._cp, s, a)
        ws, size = self._scratch(stream, need) if need else (None, 0)
        _check(L.cg_kv8_select(self._cp, s, a, int(recent),
                               self._tensor(out, "out", self.torch.int32, shape), ws, size,
                               stream.cuda_stream), "cg_kv8_select")
        return out

    # ---- eviction ------------------------------------------------------------------------
    def evict(self, table, lengths, mass, keep, recent, new_table, max_len=None, stream=None):
        """Cuts every sequence to ``keep`` tokens in the pages of ``new_table`` (pages of no
        sequence of the call): the last ``recent`` stay and the heaviest of the others by ``mass``
        [n_pages, n_heads, 64], which moves along. Returns (kept [n_seq, n_heads, keep],
        new_lengths [n_seq])."""
        s, to = self._seqs(table), self._seqs(new_table)
        stream = self._stream(stream)
        t = self.torch
        with t.cuda.stream(stream):
            kept = t.empty((s.n_seq, self.n_heads, max(0, int(keep))), dtype=t.int32,
                           device=self.device)
            new_lengths = t.empty((s.n_seq,), dtype=t.int32, device=self.device)
        _need(lengths is not None and mass is not None, "lengths and mass are wanted")
        _check(_lib().cg_kv8_evict(
            self._cp, s, self._per_seq(lengths, "lengths", s.n_seq),
            s.max_pages * PAGE if max_len is None else int(max_len),
            self._tensor(mass, "mass", t.float32, (self.n_pages, self.n_heads, PAGE)), int(keep),
            int(recent), to, kept.data_ptr(), new_lengths.data_ptr(), stream.cuda_stream),
            "cg_kv8_evict")
        return kept, new_lengths
