"""Python binding of the 8-bit serving cache (include/cachegen.h, cg_kv8_*): a pool of 64-token
pages that holds decoded contexts as int8 codes under a scale per page and head, and the operators
on it — rows in and out (``store``, ``load``), attention of one or many query tokens
(``attend``), eviction by accumulated weight (``evict``) and the choice of the pages a query reads
(``select``); and what requests that share a context need: pages shared, handed out, given back,
copied and moved together (``fork``, ``reserve``, ``release``, ``copy``, ``compact``), attention that
reads a shared context once (``attend_shared``), drafted tokens accepted or not (``verify``).

Argument marshalling only, as in ``cachegen``: every step runs in the HIP kernels of
``libcachegen.so``, torch supplies buffers and the stream handle, and there is no CPU fallback.
Tensors are checked for type, shape and device before their addresses are passed on.
"""
from __future__ import annotations

import ctypes
import math
import struct
import threading

from .cachegen import CodecError, _check, lib

PAGE = 64
ZEROED = 4096                      # CG_KV8_WORKSPACE_ZEROED
_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_I32 = ctypes.c_int32


class _Cache(ctypes.Structure):
    _fields_ = [("n_pages", _I32), ("n_heads", _I32), ("head_dim", _I32), ("k_codes", _P),
                ("v_codes", _P), ("k_scale", _P), ("v_scale", _P), ("k_bounds", _P), ("mass", _P)]


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


class _Contexts(ctypes.Structure):
    _fields_ = [("seqs", _Seqs), ("lengths", _P), ("max_len", _I32), ("firsts", _P),
                ("max_users", _I32)]


class _Verify(ctypes.Structure):
    _fields_ = [("n_seq", _I32), ("n_drafts", _I32), ("vocab", _I32), ("dtype", _I32),
                ("target", _P), ("t_seq_stride", _I64), ("t_row_stride", _I64), ("draft", _P),
                ("d_seq_stride", _I64), ("d_row_stride", _I64), ("drafts", _P), ("counts", _P),
                ("u", _P), ("tokens", _P), ("accepted", _P), ("lengths", _P), ("new_lengths", _P)]


# The same structures as bytes: a call of one token takes a few microseconds on the GPU, and packing
# a structure at once takes a fraction of setting it field by field.
_SEQS = struct.Struct("@iiP")
_ROWS = struct.Struct("@Pqqq")
_ATTN = struct.Struct("@iiifPiPPqqqPqqqPPiPPf0P")
_CONTEXTS = struct.Struct("@iiPPiPi0P")
_VERIFY = struct.Struct("@iiiiPqqPqqPPPPPPP")
assert (_SEQS.size, _ROWS.size, _ATTN.size, _CONTEXTS.size, _VERIFY.size) == tuple(
    map(ctypes.sizeof, (_Seqs, _Rows, _Attn, _Contexts, _Verify)))

_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        L = lib()
        U64 = ctypes.c_uint64
        L.cg_kv8_store.argtypes = [_P, _P, _P, _P, _I32, _I32, _P, _P, _P, _P]
        L.cg_kv8_load.argtypes = [_P, _P, _P, _P, _I32, _I32, _P, _P, _P]
        L.cg_kv8_attend_workspace_bytes.argtypes = [_P, _P, _P]
        L.cg_kv8_attend_workspace_bytes.restype = U64
        L.cg_kv8_attend.argtypes = [_P, _P, _P, _P, U64, _P]
        L.cg_kv8_select_workspace_bytes.argtypes = [_P, _P, _P]
        L.cg_kv8_select_workspace_bytes.restype = U64
        L.cg_kv8_select.argtypes = [_P, _P, _P, _I32, _P, _P, U64, _P]
        L.cg_kv8_evict.argtypes = [_P, _P, _P, _I32, _P, _I32, _I32, _P, _P, _P, _P]
        L.cg_kv8_attend_shared_workspace_bytes.argtypes = [_P, _P, _P, _P]
        L.cg_kv8_attend_shared_workspace_bytes.restype = U64
        L.cg_kv8_attend_shared.argtypes = [_P, _P, _P, _P, _P, U64, _P]
        L.cg_kv8_fork.argtypes = [_P, _P, _P, _P, _P, _P, _P, _P, _P]
        L.cg_kv8_reserve_workspace_bytes.argtypes = [_P, _P]
        L.cg_kv8_reserve_workspace_bytes.restype = U64
        L.cg_kv8_reserve.argtypes = [_P, _P, _P, _P, _P, _P, _P, U64, _P]
        L.cg_kv8_reserve_granted.argtypes = [_P, _P, _P, _P, _P, _P, _P, _P, U64, _P]
        L.cg_kv8_release.argtypes = [_P, _P, _P, _P, _P]
        L.cg_kv8_copy.argtypes = [_P, _P, _P, _I32, _P]
        L.cg_kv8_compact_workspace_bytes.argtypes = [_P]
        L.cg_kv8_compact_workspace_bytes.restype = U64
        L.cg_kv8_compact.argtypes = [_P, _P, _P, _P, _P, _P, _P, _P, U64, _P]
        L.cg_verify_workspace_bytes.argtypes = [_P]
        L.cg_verify_workspace_bytes.restype = U64
        L.cg_verify_drafts.argtypes = [_P, _P, U64, _P]
        L.cg_verify_drafts.restype = ctypes.c_int
        L.hipStreamIsCapturing.argtypes = [_P, _P]        # of the runtime that the library links
        L.hipStreamIsCapturing.restype = ctypes.c_int
        for n in ("store", "load", "attend", "select", "evict", "attend_shared", "fork", "reserve",
                  "reserve_granted", "release", "copy", "compact"):
            getattr(L, "cg_kv8_" + n).restype = ctypes.c_int
        _LIB = L
    return _LIB


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _bound(max_len, width):
    """The bound of the lengths: the caller's, or what the table's row holds."""
    return min(width * PAGE, 0x7fffffff) if max_len is None else max_len


class Kv8Cache:
    """A pool of pages on one GPU and the operators on it.

    Sequences are given by ``table`` [n_seq, columns] (int32 page numbers) and the number of
    tokens they hold. Lengths, starts and counts are int32 [n_seq]; everything is a contiguous
    tensor on the cache's device except rows of K, V, queries and outputs, which may have any
    strides as long as the head dimension is contiguous. Calls are asynchronous on ``stream``
    (default: the current one). Scratch is kept per stream and grows as needed; calls captured with
    ``torch.cuda.graph`` take theirs from the graph's pool. Threads may share a cache and a stream.

    ``buffers``: tensors ``k_codes``, ``v_codes``, ``k_scale``, ``v_scale`` and (or None)
    ``k_bounds`` to use as the pool; without it they are allocated, zeroed.
    """

    def __init__(self, n_pages, n_heads, head_dim, device="cuda", buffers=None):
        import torch
        self.torch = torch
        self._i32, self._f32 = torch.int32, torch.float32
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
        self._index = self.device.index or 0
        for n, (s, t) in want.items():
            b = buffers.get(n)
            _need(b is not None or n == "k_bounds", f"{n} is missing")
            if b is not None:
                self._tensor(b, n, t, s)
            setattr(self, n, b)
        self._c = _Cache(P, H, D, *(None if (b := getattr(self, n)) is None else b.data_ptr()
                                    for n in want))
        self._cp = ctypes.addressof(self._c)
        self._raw_stream = torch._C._cuda_getCurrentRawStream
        self._on_gpu = self.device.type == "cuda"
        self._current = torch._C._cuda_getDevice if self._on_gpu else lambda: self._index
        self._ws, self._lock = {}, threading.Lock()
        self._ints = torch.empty(0, dtype=torch.int32, device=self.device)
        self._reserve_bytes = {}           # (n_seq, columns) -> bytes
        self._status = _I32()
        self._status_p = ctypes.addressof(self._status)
        self._types = {torch.float16: 0, torch.bfloat16: 1}
        self._scale = 1.0 / math.sqrt(D)

    # ---- marshalling (no message is put together and no stream object made until needed) ----
    def _tensor(self, t, name, dtype, shape=None):
        if (t.dtype is dtype and t.device == self.device and t.is_contiguous()
                and (shape is None or t.shape == shape)):
            return t.data_ptr()
        raise ValueError(f"{name}: a contiguous {dtype} tensor"
                         f"{'' if shape is None else ' of ' + str(tuple(shape))} on {self.device} "
                         f"is wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")

    def _seqs(self, table):
        """(cg_kv8_seqs, n_seq, columns)"""
        p = self._tensor(table, "table", self._i32)
        if table.dim() != 2:
            raise ValueError("table: [n_seq, columns] is wanted")
        n, width = table.shape
        return _SEQS.pack(n, width, p), n, width

    def _per_seq(self, t, name, n):
        return 0 if t is None else self._tensor(t, name, self._i32, (n,))

    def _strided(self, t, name, shape, dtype):
        """The fields of cg_kv8_rows."""
        if t.dtype is dtype and t.shape == shape and t.device == self.device:
            a, b, c, d = t.stride()
            if d == 1:
                return t.data_ptr(), a, b, c
        raise ValueError(f"{name}: {dtype} rows {tuple(shape)} with a contiguous last dimension "
                         f"on {self.device} are wanted, got {t.dtype} {tuple(t.shape)} on "
                         f"{t.device}")

    def _rows(self, t, name, shape, dtype):
        return _ROWS.pack(*self._strided(t, name, shape, dtype))

    def _handle(self, stream):
        """The HIP stream's handle: the caller's, or torch's current one; of the cache's GPU."""
        if stream is None:
            if self._on_gpu:
                return self._raw_stream(self._index)
        elif getattr(stream, "device", self.device) == self.device:
            return stream.cuda_stream
        raise ValueError(f"the cache is on {self.device}: a GPU is wanted, and a stream of it")

    def _launch(self, name, fn, stream, *args, need=None, cache=None):
        """fn(cache, *args, stream), or with `need` bytes of scratch fn(cache, *args, scratch, its
        bytes, stream); with the cache's GPU as the current one, where a launch goes. Launches that
        share scratch are made in one piece: another thread's on the same stream would find it half
        used, or replace it."""
        handle = self._handle(stream)
        if self._current() != self._index:
            with self.torch.cuda.device(self._index):
                return self._launch(name, fn, stream, *args, need=need, cache=cache)
        if need is None:
            rc = fn(cache or self._cp, *args, handle)
        elif need == 0:
            rc = fn(cache or self._cp, *args, None, 0, handle)
        else:
            with self._lock:
                ws = self._scratch(stream, handle, need)
                rc = fn(cache or self._cp, *args, ws[0], ws[1], handle)
        _check(rc, name)

    def _new(self, make, shape, dtype, stream):
        """A tensor whose memory's reuse is ordered on the stream."""
        if stream is None:
            return make(shape, dtype=dtype, device=self.device)
        with self.torch.cuda.stream(stream):
            return make(shape, dtype=dtype, device=self.device)

    def _empty(self, shape, dtype, stream):
        return self._new(self.torch.empty, shape, dtype, stream)

    def _int_out(self, t, name, shape, stream):
        """(tensor, address) of an int32 output: the caller's, or a new one."""
        if t is not None:
            return t, self._tensor(t, name, self._i32, shape)
        t = self._ints.new_empty(shape) if stream is None else self._empty(shape, self._i32, stream)
        return t, t.data_ptr()

    def _scratch(self, stream, handle, need):
        """The stream's own scratch (address, bytes, tensor), its counters cleared once. Every call
        of a captured stream has scratch of its own instead: what eager calls use is replaced when
        one needs more, and may be at work when the graph is replayed. It comes from the graph's
        memory pool, which lives as long as the graph (and may give it to a later call of the same
        capture, which runs behind this one); the graph clears its counters."""
        if self._capturing(handle):
            return self._cleared(need, stream)
        ws = self._ws.get(handle)
        if ws is None or ws[1] < need:
            # (a quarter more: a decode's need grows with every page)
            ws = self._ws[handle] = self._cleared(need + need // 4, stream)
        return ws

    def _cleared(self, need, stream):
        """Scratch of `need` bytes, of which the counters at its front have to be zero."""
        t = self._empty((need,), self.torch.uint8, stream)
        if stream is None:
            t[:ZEROED].zero_()
        else:
            with self.torch.cuda.stream(stream):
                t[:ZEROED].zero_()
        return t.data_ptr(), need, t

    def _capturing(self, handle):
        """Whether the stream is being captured (the null stream cannot be); under the lock."""
        return handle != 0 and (_lib().hipStreamIsCapturing(handle, self._status_p) != 0
                                or self._status.value != 0)

    def _mass(self, mass):
        return self._tensor(mass, "mass", self._f32, (self.n_pages, self.n_heads, PAGE))

    def _with(self, mass):
        """The cache with these weights, for a call that clears or moves them; None without."""
        if mass is None:
            return None
        c = _Cache.from_buffer_copy(self._c)
        c.mass = self._mass(mass)
        return ctypes.byref(c)

    # ---- rows in and out -----------------------------------------------------------------
    def store(self, k, v, table, starts, counts=None, status=None, stream=None, mass=None):
        """Rows k, v [n_seq, n_tokens, n_heads, head_dim] become the sequences' tokens from
        ``starts`` on (``counts``: how many of each; default all). ``status``: an int32 tensor of
        one element that receives 0, or non-zero for NaN / Inf. ``mass``: the weights of ``attend``
        and ``evict``, in which the new tokens start from 0; without it what their places held
        stays, the weights of the pages' last owner as a rule."""
        s, n, _ = self._seqs(table)
        kind = self._types.get(k.dtype)
        _need(kind is not None and k.dim() == 4, "k: float16 or bfloat16 [n_seq, n_tokens, "
              "n_heads, head_dim] is wanted")
        _need(starts is not None, "starts is missing")
        shape = (n, k.shape[1], self.n_heads, self.head_dim)
        self._launch(
            "cg_kv8_store", _lib().cg_kv8_store, stream, s, self._per_seq(starts, "starts", n),
            self._per_seq(counts, "counts", n), shape[1], kind, self._rows(k, "k", shape, k.dtype),
            self._rows(v, "v", shape, k.dtype),
            None if status is None else self._tensor(status, "status", self._i32, (1,)),
            cache=self._with(mass))

    def load(self, table, starts, n_tokens, counts=None, dtype=None, k=None, v=None, stream=None):
        """(k, v) [n_seq, n_tokens, n_heads, head_dim]: the sequences' tokens from ``starts`` on,
        zeros behind ``counts``. ``k``, ``v``: tensors to write into."""
        s, n, _ = self._seqs(table)
        T, H, D = int(n_tokens), self.n_heads, self.head_dim
        shape = (n, T, H, D)
        if k is None and v is None:
            dtype = dtype or self.torch.float16
            k, v = self._empty(shape, dtype, stream), self._empty(shape, dtype, stream)
            kind = self._types.get(dtype)
            rows = [_ROWS.pack(x.data_ptr(), T * H * D, H * D, D) for x in (k, v)]
        else:
            dtype = dtype or (v if k is None else k).dtype
            k = self._empty(shape, dtype, stream) if k is None else k
            v = self._empty(shape, dtype, stream) if v is None else v
            kind = self._types.get(k.dtype)
            rows = self._rows(k, "k", shape, k.dtype), self._rows(v, "v", shape, k.dtype)
        _need(kind is not None, "k: float16 or bfloat16 is wanted")
        _need(starts is not None, "starts is missing")
        self._launch("cg_kv8_load", _lib().cg_kv8_load, stream, s,
                     self._per_seq(starts, "starts", n), self._per_seq(counts, "counts", n), T,
                     kind, *rows)
        return k, v

    # ---- attention -----------------------------------------------------------------------
    def _queries(self, q, n):
        kind = self._types.get(q.dtype)
        _need(q.dim() == 4 and kind is not None, "q: float16 or bfloat16 "
              "[n_seq, n_q, n_q_heads, head_dim] is wanted")
        _, nq, heads, _ = q.shape
        return kind, nq, heads, (n, nq, heads, self.head_dim)

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
        s, n, width = self._seqs(table)
        kind, nq, heads, shape = self._queries(q, n)
        _need(lengths is not None, "lengths is missing")
        if out is None:
            out = self._empty(q.shape, q.dtype, stream)
        n_picks = picks_p = mass_p = mass_out_p = 0
        if picks is not None:
            _need(picks.dim() == 4, "picks: [n_seq, n_q, n_heads, n] is wanted")
            n_picks = picks.shape[3]
            picks_p = self._tensor(picks, "picks", self._i32, (n, nq, self.n_heads, n_picks))
        if mass is not None or mass_out is not None:
            mass_out = mass if mass_out is None else mass_out
            mass_p = 0 if mass is None else self._mass(mass)
            mass_out_p = self._tensor(mass_out, "mass_out", self._f32,
                                      (self.n_pages, self.n_heads, PAGE))
        a = _ATTN.pack(nq, heads, kind, self._scale if scale is None else scale,
                       self._per_seq(lengths, "lengths", n),
                       _bound(max_len, width),
                       self._per_seq(q_lens, "q_lens", n), *self._strided(q, "q", shape, q.dtype),
                       *self._strided(out, "out", shape, q.dtype),
                       0 if lse is None else self._tensor(lse, "lse", self._f32, shape[:3]),
                       picks_p, n_picks, mass_p, mass_out_p, decay)
        L = _lib()
        self._launch("cg_kv8_attend", L.cg_kv8_attend, stream, s, a,
                     need=L.cg_kv8_attend_workspace_bytes(self._cp, s, a))
        return out

    def select(self, q, table, lengths, n_picks, recent=1, q_lens=None, max_len=None, out=None,
               stream=None):
        """Table columns [n_seq, n_q, n_heads, n_picks] (int32, ascending, -1 behind the last) of
        the pages that each query token should read: the ``recent`` last ones it sees and the best
        of the others by the bound of their q . k."""
        s, n, width = self._seqs(table)
        kind, nq, heads, shape = self._queries(q, n)
        _need(lengths is not None, "lengths is missing")
        want = (n, nq, self.n_heads, max(0, n_picks))
        if out is None:
            out = self._empty(want, self._i32, stream)
        rows = self._strided(q, "q", shape, q.dtype)
        a = _ATTN.pack(nq, heads, kind, 0.0, self._per_seq(lengths, "lengths", n),
                       _bound(max_len, width),
                       self._per_seq(q_lens, "q_lens", n), *rows, *rows, 0, 0, n_picks, 0, 0, 0.0)
        L = _lib()
        self._launch("cg_kv8_select", L.cg_kv8_select, stream, s, a, recent,
                     self._tensor(out, "out", self._i32, want),
                     need=L.cg_kv8_select_workspace_bytes(self._cp, s, a))
        return out

    # ---- eviction ------------------------------------------------------------------------
    def evict(self, table, lengths, mass, keep, recent, new_table, max_len=None, stream=None):
        """Cuts every sequence to ``keep`` tokens in the pages of ``new_table`` (pages of no
        sequence of the call): the last ``recent`` stay and the heaviest of the others by ``mass``
        [n_pages, n_heads, 64], which moves along. Returns (kept [n_seq, n_heads, keep],
        new_lengths [n_seq])."""
        s, n, width = self._seqs(table)
        to = self._seqs(new_table)[0]
        _need(lengths is not None and mass is not None, "lengths and mass are wanted")
        kept = self._empty((n, self.n_heads, max(0, keep)), self._i32, stream)
        new_lengths = self._empty((n,), self._i32, stream)
        self._launch(
            "cg_kv8_evict", _lib().cg_kv8_evict, stream, s, self._per_seq(lengths, "lengths", n),
            _bound(max_len, width),
            self._mass(mass), keep, recent, to, kept.data_ptr(), new_lengths.data_ptr())
        return kept, new_lengths

    # ---- requests that share a context -----------------------------------------------------
    def _refs(self, refs):
        return self._tensor(refs, "refs", self._i32, (self.n_pages,))

    def fork(self, table, lengths, parents, refs, ends=None, new_table=None, stream=None):
        """Children of the table's sequences, which share their pages: child i holds the first
        ``ends[i]`` tokens (default: all) of sequence ``parents[i]``. Returns (new_table, new_lengths).

        refs       int32 [n_pages]: how many table rows hold each page (0: it is free), kept by the
                   caller and brought up to date by the calls that take it.
        new_table  int32 [children, columns] to write into, at least as wide as ``table`` and none
                   of its memory a parent's row; what it held is not released. Default: a new one,
                   as wide as ``table``. A child that will outgrow its parent's row wants a wider
                   one."""
        s, n, width = self._seqs(table)
        _need(lengths is not None and parents is not None, "lengths and parents are wanted")
        _need(parents.dim() == 1, "parents: [children] is wanted")
        m = parents.shape[0]
        if new_table is None:
            new_table = self._int_out(None, "new_table", (m, width), stream)[0]
        to, rows, _ = self._seqs(new_table)
        _need(rows == m, f"new_table: {m} rows are wanted")
        new_lengths, new_p = self._int_out(None, "new_lengths", (m,), stream)
        self._launch("cg_kv8_fork", _lib().cg_kv8_fork, stream, s,
                     self._per_seq(lengths, "lengths", n), self._per_seq(parents, "parents", m),
                     self._per_seq(ends, "ends", m), to, new_p, self._refs(refs))
        return new_table, new_lengths

    def reserve(self, table, lengths, counts, refs, mass=None, missing=None, granted=None,
                stream=None):
        """Pages for ``counts[i]`` tokens behind the ``lengths[i]`` that sequence i holds, for a
        ``store`` that follows: free ones (lowest number first) where its row of ``table`` has none
        of its own, and a copy of a page that it shares and would write to. ``table`` and ``refs``
        are updated. Returns ``missing`` (int32 [1]): 0, or how many free pages too few there are;
        then nothing has changed, and the sequences must not be written to: their pages may be
        others' too. ``mass``: weights that go with a copied page.

        granted  int32 [n_seq] to write into (may be ``counts``): the tokens of ``counts`` that may be
                 stored, as far as the row of ``table`` goes, and none where pages were missing. A
                 ``store`` with these counts, and lengths that grow by them, are right either way,
                 in a captured step too."""
        s, n, width = self._seqs(table)
        _need(lengths is not None and counts is not None, "lengths and counts are wanted")
        missing, missing_p = self._int_out(missing, "missing", (1,), stream)
        L, cache = _lib(), self._with(mass)
        need = self._reserve_bytes.get((n, width))
        if need is None:
            need = L.cg_kv8_reserve_workspace_bytes(self._cp, s)
            self._reserve_bytes[n, width] = need
        self._launch("cg_kv8_reserve", L.cg_kv8_reserve_granted, stream, s,
                     self._per_seq(lengths, "lengths", n), self._per_seq(counts, "counts", n),
                     self._refs(refs), missing_p, self._per_seq(granted, "granted", n), need=need,
                     cache=cache)
        return missing

    def release(self, table, refs, keep=None, stream=None):
        """Gives back the pages of the table's sequences, or those that lie behind the first
        ``keep[i]`` tokens of sequence i; their entries become -1."""
        s, n, _ = self._seqs(table)
        self._launch("cg_kv8_release", _lib().cg_kv8_release, stream, s,
                     self._per_seq(keep, "keep", n), self._refs(refs))

    def copy(self, src, dst, mass=None, stream=None):
        """Page ``src[i]`` to page ``dst[i]`` (int32 [n]; no page twice in ``dst``, nor in both),
        with its weights if ``mass`` is given."""
        _need(src.dim() == 1, "src: [n] is wanted")
        n = src.shape[0]
        pages = self._tensor(src, "src", self._i32), self._tensor(dst, "dst", self._i32, (n,))
        cache = self._with(mass)
        if n:
            self._launch("cg_kv8_copy", _lib().cg_kv8_copy, stream, *pages, n, cache=cache)

    def compact(self, table, refs, mass=None, stream=None):
        """Moves the pages in use to the front of the pool. Returns (new_table, new_refs, moved,
        n_live): the table and the counts as the pages lie now, the new number of each page (int32
        [n_pages], -1 of a free one) for other tables, and how many are in use (int32 [1]).
        ``table`` and ``refs`` are left as they were."""
        s, n, width = self._seqs(table)
        new_table, table_p = self._int_out(None, "new_table", (n, width), stream)
        new_refs, refs_p = self._int_out(None, "new_refs", (self.n_pages,), stream)
        moved, moved_p = self._int_out(None, "moved", (self.n_pages,), stream)
        live, live_p = self._int_out(None, "live", (1,), stream)
        L, cache = _lib(), self._with(mass)
        self._launch("cg_kv8_compact", L.cg_kv8_compact, stream, s, self._refs(refs), table_p, refs_p,
                     moved_p, live_p, need=L.cg_kv8_compact_workspace_bytes(self._cp), cache=cache)
        return new_table, new_refs, moved, live

    def attend_shared(self, q, shared, shared_lengths, firsts, table=None, lengths=None, scale=None,
                      q_lens=None, max_shared=None, max_len=None, max_users=None, out=None,
                      lse=None, stream=None):
        """Attention of the queries q [n_seq, n_q, n_q_heads, head_dim] over contexts that sequences
        share, read once for all of them, and over the sequences' own tokens behind; returns ``out``.

        shared         int32 [contexts, columns]: the contexts' pages; ``shared_lengths`` [contexts].
        firsts         int32 [contexts + 1], ascending: context p is that of sequences firsts[p] ..
                       firsts[p + 1] - 1. Every query token sees all of its sequence's context.
        table, lengths the sequences' own pages and tokens, seen causally as in ``attend`` (the
                       queries are the last of them). Without: attention over the contexts alone,
                       as over an encoder's states.
        max_shared, max_len, max_users  bounds that the host knows of shared_lengths, of lengths and
                       of the sequences that share a context (default: the tables' widths, n_seq);
                       the work is laid out for them, but for no more rows than the sequences have.
        scale, q_lens, lse  as in ``attend``."""
        x, contexts, x_width = self._seqs(shared)
        _need(q.dim() == 4, "q: [n_seq, n_q, n_q_heads, head_dim] is wanted")
        n = q.shape[0]
        kind, nq, heads, shape = self._queries(q, n)
        _need(shared_lengths is not None and firsts is not None,
              "shared_lengths and firsts are wanted")
        _need((table is None) == (lengths is None), "table and lengths go together")
        if table is None:
            s, width = _SEQS.pack(n, 0, 0), 0
        else:
            s, rows, width = self._seqs(table)
            _need(rows == n, f"table: {n} rows are wanted")
        if out is None:
            out = self._empty(q.shape, q.dtype, stream)
        c = _CONTEXTS.pack(contexts, x_width, shared.data_ptr(),
                           self._per_seq(shared_lengths, "shared_lengths", contexts),
                           _bound(max_shared, x_width),
                           self._per_seq(firsts, "firsts", contexts + 1),
                           n if max_users is None else max_users)
        a = _ATTN.pack(nq, heads, kind, self._scale if scale is None else scale,
                       self._per_seq(lengths, "lengths", n), _bound(max_len, width),
                       self._per_seq(q_lens, "q_lens", n), *self._strided(q, "q", shape, q.dtype),
                       *self._strided(out, "out", shape, q.dtype),
                       0 if lse is None else self._tensor(lse, "lse", self._f32, shape[:3]),
                       0, 0, 0, 0, 1.0)
        L = _lib()
        self._launch("cg_kv8_attend_shared", L.cg_kv8_attend_shared, stream, c, s, a,
                     need=L.cg_kv8_attend_shared_workspace_bytes(self._cp, c, s, a))
        return out

    # ---- drafted tokens --------------------------------------------------------------------
    def _probabilities(self, t, name, shape, dtype):
        """(address, strides of sequences and rows)"""
        if t.dtype is dtype and t.shape == shape and t.device == self.device:
            a, b, c = t.stride()
            if c == 1:
                return t.data_ptr(), a, b
        raise ValueError(f"{name}: {dtype} probabilities {tuple(shape)} with a contiguous last "
                         f"dimension on {self.device} are wanted, got {t.dtype} {tuple(t.shape)} "
                         f"on {t.device}")

    def verify(self, target, drafts, u, draft=None, counts=None, lengths=None, tokens=None,
               accepted=None, new_lengths=None, stream=None):
        """Drafted tokens accepted by the target's probabilities, and the token behind them.
        Returns (tokens, accepted) or, with ``lengths``, (tokens, accepted, new_lengths).

        target   [n_seq, n_drafts + 1, vocab] float32, float16 or bfloat16 probabilities of the
                 target: row j for draft j, the last behind all drafts.
        drafts   int32 [n_seq, n_drafts]; ``counts`` int32 [n_seq]: how many of each sequence
                 (default: all; below 0: the sequence sits out).
        draft    [n_seq, n_drafts, vocab] of the same type: the probabilities that the drafts were
                 drawn from, or None: each draft was sure.
        u        float32 [n_seq, n_drafts + 1] random numbers in [0, 1): one for each draft, the
                 last for the token that is drawn.
        lengths  int32 [n_seq] tokens that the cache holds, the drafts among them.
        tokens   int32 [n_seq, n_drafts + 1]: the accepted drafts, the token drawn behind them, -1.
        accepted     int32 [n_seq] drafts accepted.
        new_lengths  int32 [n_seq] lengths less the drafts not accepted (may be ``lengths``): what
                     ``release`` keeps."""
        kind = {self.torch.float32: 2, **self._types}.get(target.dtype)
        _need(target.dim() == 3 and kind is not None and target.shape[1] > 0,
              "target: float32, float16 or bfloat16 [n_seq, n_drafts + 1, vocab] is wanted")
        n, k, vocab = target.shape[0], target.shape[1] - 1, target.shape[2]
        rows = self._probabilities(target, "target", target.shape, target.dtype)
        near = (0, 0, 0) if draft is None or k == 0 else self._probabilities(
            draft, "draft", (n, k, vocab), target.dtype)
        tokens, tokens_p = self._int_out(tokens, "tokens", (n, k + 1), stream)
        accepted, accepted_p = self._int_out(accepted, "accepted", (n,), stream)
        lengths_p = new_p = 0
        _need(lengths is not None or new_lengths is None, "lengths is missing")
        if lengths is not None:
            lengths_p = self._per_seq(lengths, "lengths", n)
            new_lengths, new_p = self._int_out(new_lengths, "new_lengths", (n,), stream)
        v = _VERIFY.pack(n, k, vocab, kind, *rows, *near,
                         self._tensor(drafts, "drafts", self._i32, (n, k)),
                         self._per_seq(counts, "counts", n),
                         self._tensor(u, "u", self._f32, (n, k + 1)), tokens_p, accepted_p,
                         lengths_p, new_p)
        L = _lib()
        self._launch("cg_verify_drafts", L.cg_verify_drafts, stream,
                     need=L.cg_verify_workspace_bytes(v), cache=v)
        return (tokens, accepted) if lengths is None else (tokens, accepted, new_lengths)
