"""Timed cases of the 8-bit serving cache: what a program that answers over a loaded context does
with the KV that the codec gave back.

A context is held in pages of 64 tokens of one KV head, K and V as 8-bit codes under one scale for
each page and head (K [page][head][64][dim], V transposed [page][head][dim][64], scales fp32
[page][head], the codes' lowest and highest value for each K channel [page][head][2][dim]). A
sequence is a row of page numbers and a length.

Operations (a case's "op"):
  store    rows of fp16 or bf16 K and V go into the pages, behind what the sequences hold
           already, and come back as rows (a decoded context's way in, an evicted one's way out)
  attend   queries of one or many tokens over the sequences' pages, causal, with the log-sum-exp
           of every row and (mass) the weight that each cached token got, added to a running sum
  evict    of every sequence and head the last tokens and the heaviest of the others move into
           new pages, and come back as rows for the codec
  sparse   for every query token and KV head the pages whose channel bounds promise most, then
           attention over those

A case's other fields: seqs, q_heads, heads (KV), dim, tokens (cached tokens of the longest
sequence; for op "store" the new rows of the longest), q (query tokens), start (for "store": tokens
already held), ragged (lengths differ, the last of eight or more sequences idle), dtype of rows and
queries, mass, keep and recent (for "evict"), picks (pages, for "sparse").
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE = 64
DECAY = 0.98                    # of the running sum of weights, per call
RECENT_PAGES = 1


def _case(name, op, seqs, q_heads, heads, dim, tokens, q=1, dtype="float16", **more):
    c = {"op": op, "seqs": seqs, "q_heads": q_heads, "heads": heads, "dim": dim, "tokens": tokens,
         "q": q, "start": 0, "ragged": False, "dtype": dtype, "mass": False, "keep": 0,
         "recent": 0, "picks": 0}
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # each of eight requests appends the token it has just made: launches and latency
        _case("store_append_b8", "store", 8, 32, 8, 128, 1, start=1000, ragged=True),
        # a decoded 4K-token context of a 7B model, its 32 layers at once, and back
        _case("store_mistral7b_t4096", "store", 32, 32, 8, 128, 4096),
        # three contexts behind what they hold already, in bf16, with lengths off the page
        _case("store_ragged_b3_t2003", "store", 3, 10, 5, 64, 2003, start=777, ragged=True,
              dtype="bfloat16"),
        # one token of one request over that context: the smallest attention
        _case("token_mistral7b_t4096", "attend", 1, 32, 8, 128, 4096),
        # a batch of 32 requests of uneven length, with the weights that eviction goes by
        _case("token_b32_t2048_mass", "attend", 32, 32, 8, 128, 2048, ragged=True, mass=True),
        # multi-head attention: every query head has K and V of its own
        _case("token_llama2_7b_t8192", "attend", 4, 32, 32, 128, 8192, dtype="bfloat16"),
        # a question of 500 tokens over a loaded context, with the weights
        _case("prompt500_mistral7b_t4096_mass", "attend", 1, 32, 8, 128, 4096, q=500, mass=True),
        # the largest: 2K new tokens behind a context of a model with grouped heads
        _case("prompt2048_t8192", "attend", 2, 64, 8, 128, 8192, q=2048, dtype="bfloat16"),
        # a batch is cut to a quarter of its tokens; one long context to an eighth
        _case("evict_b32_t2048", "evict", 32, 32, 8, 128, 2048, ragged=True, keep=512, recent=128),
        _case("evict_t65536", "evict", 1, 64, 8, 128, 65536, keep=8192, recent=1024),
        # one token over 64 pages of a very long context; a batch over 16K tokens, two tokens each
        _case("sparse_t131072", "sparse", 1, 64, 8, 128, 131072, picks=64),
        _case("sparse_b16_t16384", "sparse", 16, 32, 8, 128, 16384, q=2, ragged=True, picks=32,
              dtype="bfloat16"),
    ]


OPS = ("store", "attend", "attend", "attend", "evict", "sparse")
#: (query heads, KV heads) of models of several families, and odd ones
HEADS = ((32, 8), (32, 8), (64, 8), (32, 32), (16, 16), (8, 8), (8, 1), (28, 4), (12, 4), (10, 5),
         (3, 1))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(OPS)
    q_heads, heads = rng.choice(HEADS)
    dim = rng.choice((128, 128, 128, 64, 64, 256))
    more = {"ragged": rng.random() < 0.5, "dtype": rng.choice(("float16", "bfloat16"))}
    seqs = _log(rng, 1, 48)
    if op == "store":
        tokens = _log(rng, 1, max(2, min(8192, (1 << 26) // (seqs * heads * dim))))
        return _case(None, op, seqs, q_heads, heads, dim, tokens, start=rng.choice(
            (0, _log(rng, 1, 5000))), **more)
    # tokens: up to the largest listed cache, and no more operations than the largest listed prompt
    most = min(131072, (1 << 28) // (seqs * heads * dim))
    if op == "attend":
        q = 1 if rng.random() < 0.5 else _log(rng, 2, 1024)
        q = min(q, max(1, (1 << 24) // (seqs * q_heads * 16)))
        most = min(most, (1 << 37) // (seqs * q_heads * q * dim))
        tokens = max(q, _log(rng, 1, max(2, most)))
        return _case(None, op, seqs, q_heads, heads, dim, tokens, q=q, mass=rng.random() < 0.4,
                     **more)
    tokens = _log(rng, 65, max(66, most))
    if op == "evict":
        keep = max(2, int(tokens * rng.uniform(0.05, 0.6)))
        return _case(None, op, seqs, q_heads, heads, dim, tokens, keep=keep,
                     recent=rng.randrange(0, keep), **more)
    q = rng.choice((1, 1, 2, 3))
    picks = min(_log(rng, 1, 96), max(1, (1 << 28) // (seqs * q * heads * dim * PAGE)))
    return _case(None, op, seqs, q_heads, heads, dim, tokens, q=q, picks=picks, **more)


# ---- sizes that follow from the case ----------------------------------------------------------
def _lengths(case):
    """Cached tokens of every sequence; for op "store" the new rows."""
    n, t = case["seqs"], case["tokens"]
    if not case["ragged"]:
        return [t] * n
    r = random.Random(n * 1_000_003 + t)
    got = [t] + [r.randint(max(1, t // 4), t) for _ in range(n - 1)]
    if n >= 8:
        got[-1] = 0
    return got


def _starts(case):
    r = random.Random(case["seqs"] * 7 + case["start"])
    return [r.randint(case["start"] // 2, case["start"]) if case["ragged"] else case["start"]
            for _ in range(case["seqs"])]


def _queries(case):
    """Query tokens of every sequence."""
    r = random.Random(case["q"] * 31 + case["seqs"])
    return [min(n, r.randint((case["q"] + 1) // 2, case["q"]) if case["ragged"] else case["q"])
            for n in _lengths(case)]


def _pages(n):
    return -(-n // PAGE)


# ---- inputs -----------------------------------------------------------------------------------
def _rows(shape, g, dtype):
    """Rows [..., heads, dim] with a level and a size of their own for each channel."""
    size = torch.exp(0.5 * torch.randn(shape[-2:], generator=g, device="cuda"))
    level = 0.7 * torch.randn(shape[-2:], generator=g, device="cuda")
    return (torch.randn(shape, generator=g, device="cuda") * size + level).to(dtype)


def _pool(case, n_pages, g, filled):
    """The pages' buffers; `filled`: with codes of random rows, else empty."""
    H, D = case["heads"], case["dim"]
    dev = "cuda"
    p = {"k_codes": torch.zeros((n_pages, H, PAGE, D), dtype=torch.int8, device=dev),
         "v_codes": torch.zeros((n_pages, H, D, PAGE), dtype=torch.int8, device=dev),
         "k_scale": torch.zeros((n_pages, H), dtype=torch.float32, device=dev),
         "v_scale": torch.zeros((n_pages, H), dtype=torch.float32, device=dev),
         "k_bounds": torch.zeros((n_pages, H, 2, D), dtype=torch.int8, device=dev)}
    per = max(1, (1 << 26) // (H * PAGE * D))
    for i in range(0, filled, per):
        n = min(per, filled - i)
        x = _rows((n, PAGE, H, D), g, torch.float32).permute(0, 2, 1, 3)
        s = x.abs().amax((2, 3)) / 127.0
        c = (x / s[:, :, None, None]).round()
        p["k_codes"][i:i + n], p["k_scale"][i:i + n] = c.to(torch.int8), s
        p["k_bounds"][i:i + n, :, 0] = c.amin(2).to(torch.int8)
        p["k_bounds"][i:i + n, :, 1] = c.amax(2).to(torch.int8)
        x = _rows((n, PAGE, H, D), g, torch.float32).permute(0, 2, 3, 1)
        s = x.abs().amax((2, 3)) / 127.0
        p["v_codes"][i:i + n], p["v_scale"][i:i + n] = (x / s[:, :, None, None]).round(), s
    return p


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 29)
    op, B, H, D = case["op"], case["seqs"], case["heads"], case["dim"]
    dtype = getattr(torch, case["dtype"])
    lengths, starts = _lengths(case), _starts(case)
    ends = [n + a for n, a in zip(lengths, starts)] if op == "store" else lengths
    width = max(1, _pages(max(ends)))
    new_width = _pages(case["keep"]) if op == "evict" else 0
    used = B * width
    n_pages = used + B * new_width + 3
    s = {"op": op, "case": dict(case), "n_pages": n_pages, "cache": None,
         "scale": 1.0 / math.sqrt(D)}
    # pages in no order, as a pool hands them out
    order = torch.randperm(used, generator=g, device="cuda").to(torch.int32)
    s["table"] = order.view(B, width).contiguous()
    s.update(_pool(case, n_pages, g, used if op != "store" or case["start"] else 0))
    s["lengths"] = _ints(lengths)
    if op == "store":
        s["k"] = _rows((B, case["tokens"], H, D), g, dtype)
        s["v"] = _rows((B, case["tokens"], H, D), g, dtype)
        # what comes back: everything from the start of the first page written
        # (nothing of a sequence that got no rows)
        first = [a // PAGE * PAGE for a in starts]
        back = [e - f if n else 0 for e, f, n in zip(ends, first, lengths)]
        s["starts"], s["first"] = _ints(starts), _ints(first)
        s["counts"], s["back"], s["rows"] = _ints(lengths), _ints(back), max(back)
        s["dtype"] = dtype
    if op in ("attend", "sparse"):
        s["q"] = 2.0 * torch.randn((B, case["q"], case["q_heads"], D), generator=g, device="cuda")
        s["q"] = s["q"].to(dtype)
        s["q_lens"] = _ints(_queries(case)) if case["ragged"] else None
        s["max_len"] = max(lengths)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(s["q"].shape[:3], dtype=torch.float32, device="cuda")
    if case["mass"] or op == "evict":
        # weights as they build up: a few heavy tokens, many light ones, some without any
        m = torch.randn((n_pages, H, PAGE), generator=g, device="cuda").mul_(2.0).exp_()
        m[torch.rand(m.shape, generator=g, device="cuda") < 0.1] = 0.0
        s["mass"] = m
        s["mass_out"] = torch.zeros_like(m) if op == "attend" else m
    if op == "sparse":
        s["picks"] = torch.zeros((B, case["q"], H, case["picks"]), dtype=torch.int32,
                                 device="cuda")
    if op == "evict":
        order = torch.randperm(B * new_width, generator=g, device="cuda").to(torch.int32) + used
        s["new_table"] = order.view(B, new_width).contiguous()
        s["first"] = _ints([0] * B)
        s["dtype"] = dtype
    if own:
        from paper_2310_07240_amd.kv8 import Kv8Cache
        s["cache"] = Kv8Cache(n_pages, H, D, buffers={k: s[k] for k in (
            "k_codes", "v_codes", "k_scale", "v_scale", "k_bounds")})
    return s


# ---- one pass ---------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    op, c, case = s["op"], s["cache"], s["case"]
    if op == "store":
        c.store(s["k"], s["v"], s["table"], s["starts"], counts=s["counts"])
        k, v = c.load(s["table"], s["first"], s["rows"], counts=s["back"], dtype=s["dtype"])
        return {"k": k, "v": v, "k_scale": s["k_scale"], "v_scale": s["v_scale"],
                "k_bounds": s["k_bounds"]}
    if op == "attend":
        more = {}
        if case["mass"]:
            more = {"mass": s["mass"], "mass_out": s["mass_out"], "decay": DECAY}
        c.attend(s["q"], s["table"], s["lengths"], scale=s["scale"], q_lens=s["q_lens"],
                 max_len=s["max_len"], out=s["out"], lse=s["lse"], **more)
        r = {"out": s["out"], "lse": s["lse"]}
        if case["mass"]:
            r["mass"] = s["mass_out"]
        return r
    if op == "sparse":
        c.select(s["q"], s["table"], s["lengths"], case["picks"], recent=RECENT_PAGES,
                 q_lens=s["q_lens"], max_len=s["max_len"], out=s["picks"])
        c.attend(s["q"], s["table"], s["lengths"], scale=s["scale"], q_lens=s["q_lens"],
                 max_len=s["max_len"], out=s["out"], lse=s["lse"], picks=s["picks"])
        return {"picks": s["picks"], "out": s["out"], "lse": s["lse"]}
    kept, lengths = c.evict(s["table"], s["lengths"], s["mass"], case["keep"], case["recent"],
                            s["new_table"])
    k, v = c.load(s["new_table"], s["first"], case["keep"], counts=lengths, dtype=s["dtype"])
    return {"kept": kept, "lengths": lengths, "k": k, "v": v, "mass": s["mass"],
            "k_scale": s["k_scale"], "v_scale": s["v_scale"], "k_bounds": s["k_bounds"]}


def _run_plain(s):
    return {"store": _plain_store, "attend": _plain_attend, "sparse": _plain_sparse,
            "evict": _plain_evict}[s["op"]](s)


def _scales(x):
    """Scales of pages [N, H, 64, D]: fp32 quotients (a number as divisor would be multiplied by
    its rounded reciprocal)."""
    top = x.abs().amax((2, 3))
    return top / torch.full_like(top, 127.0)


def _divided(x, s):
    """Codes: fp32 quotients rounded half to even; a page of zeros has scale 0 and codes 0."""
    q = x / torch.where(s > 0, s, torch.ones_like(s))
    return q.clamp_(-127.0, 127.0).round_()


def _write_pages(s, pages, live, name, codes, scale):
    """Codes [N, H, 64, D] and scales [N, H] into the pages numbered [N] where live [N]."""
    at = pages[live].long()
    c = codes[live].to(torch.int8)
    s[name + "_scale"][at] = scale[live]
    if name == "k":
        s["k_codes"][at] = c
    else:
        s["v_codes"][at] = c.transpose(2, 3).contiguous()


def _page_bounds(codes, valid):
    """Lowest and highest code of each channel over the valid tokens [N, 64]."""
    v = valid[:, None, :, None]
    lo = torch.where(v, codes, torch.full_like(codes, 127.0)).amin(2)
    hi = torch.where(v, codes, torch.full_like(codes, -127.0)).amax(2)
    return torch.stack([lo, hi], 2).to(torch.int8)


def _plain_store(s):
    B, T, H, D = s["k"].shape
    start, count, table = s["starts"].long(), s["counts"].long(), s["table"]
    NP = (T + 2 * PAGE - 2) // PAGE
    page = start[:, None] // PAGE + torch.arange(NP, device="cuda")              # [B, NP]
    pos = page[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")            # [B, NP, 64]
    src = pos - start[:, None, None]
    new = (src >= 0) & (src < count[:, None, None])
    live = new.any(2).reshape(-1)
    old = (src < 0).reshape(-1, PAGE)
    rows = (torch.arange(B, device="cuda")[:, None, None] * T
            + src.clamp(0, T - 1)).reshape(-1)
    ids = table.gather(1, page.clamp(max=table.shape[1] - 1)).reshape(-1).long()
    new = new.reshape(-1, PAGE)
    for_k = {}
    for name, x in (("k", s["k"]), ("v", s["v"])):
        x = x.reshape(B * T, H, D)[rows].float().view(-1, PAGE, H, D).permute(0, 2, 1, 3)
        x = torch.where(new[:, None, :, None], x, torch.zeros_like(x))           # [N, H, 64, D]
        was = s[name + "_codes"][ids].float()
        was = was if name == "k" else was.transpose(2, 3)
        s_old = torch.where(old.any(1)[:, None], s[name + "_scale"][ids],
                            torch.zeros((), device="cuda"))
        scale = torch.maximum(_scales(x), s_old)
        sc, so = scale[:, :, None, None], s_old[:, :, None, None]
        again = torch.where(sc == so, was, _divided(was * so, sc))
        codes = torch.where(new[:, None, :, None], _divided(x, sc),
                            torch.where(old[:, None, :, None], again, torch.zeros_like(x)))
        _write_pages(s, ids, live, name, codes, scale)
        for_k[name] = codes
    s["k_bounds"][ids[live]] = _page_bounds(for_k["k"], new | old)[live]
    k, v = _plain_load(s, table, s["first"], s["rows"], s["back"])
    return {"k": k, "v": v, "k_scale": s["k_scale"], "v_scale": s["v_scale"],
            "k_bounds": s["k_bounds"]}


def _plain_load(s, table, first, n, counts):
    """Rows first .. first + counts of every sequence, zeros behind them."""
    pos = first.long()[:, None] + torch.arange(n, device="cuda")                 # [B, n]
    live = (torch.arange(n, device="cuda") < counts[:, None])[:, :, None, None]
    pos = pos.clamp(max=table.shape[1] * PAGE - 1)
    ids = table.gather(1, pos // PAGE).long()
    k = s["k_codes"][ids, :, pos % PAGE].float() * s["k_scale"][ids][..., None]
    v = s["v_codes"][ids, :, :, pos % PAGE].float() * s["v_scale"][ids][..., None]
    return tuple(torch.where(live, x, torch.zeros_like(x)).to(s["dtype"]) for x in (k, v))


def _softmax(scores, visible):
    """Weights and log-sum-exp over the last axis; rows without a visible token: 0 and -inf."""
    x = scores.masked_fill(~visible, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m.isinf(), torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    lse = (m + torch.log(total)).squeeze(-1)
    return p / torch.where(total > 0, total, torch.ones_like(total)), lse


def _grouped(s):
    """Queries [B, q, H, group, D] in 32 bits, and how many tokens each of [B, q] sees."""
    B, Q, HQ, D = s["q"].shape
    H = s["k_codes"].shape[1]
    i = torch.arange(Q, device="cuda")
    n = s["lengths"][:, None]
    ql = torch.full_like(n, Q) if s["q_lens"] is None else s["q_lens"][:, None]
    seen = torch.where(i < ql, (n - ql + i + 1).clamp(min=0), torch.zeros_like(n))
    return s["q"].float().view(B, Q, H, HQ // H, D), seen


def _plain_attend(s):
    q, seen = _grouped(s)
    B, Q, H, G, D = q.shape
    ids = s["table"].long()
    T = ids.shape[1] * PAGE
    k = s["k_codes"][ids].float() * s["k_scale"][ids][..., None, None]           # [B, MP, H, 64, D]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, H, T, D)
    v = s["v_codes"][ids].float() * s["v_scale"][ids][..., None, None]           # [B, MP, H, D, 64]
    v = v.permute(0, 2, 1, 4, 3).reshape(B, H, T, D)
    x = q.permute(0, 2, 1, 3, 4).reshape(B, H, Q * G, D)
    scores = torch.matmul(x, k.transpose(2, 3)) * s["scale"]                     # [B, H, Q G, T]
    visible = torch.arange(T, device="cuda") < seen[:, :, None]                  # [B, Q, T]
    visible = visible[:, None, :, None].expand(B, 1, Q, G, T).reshape(B, 1, Q * G, T)
    p, lse = _softmax(scores, visible)
    o = torch.matmul(p, v).view(B, H, Q, G, D).permute(0, 2, 1, 3, 4)
    s["out"].copy_(o.reshape(B, Q, H * G, D))
    s["lse"].copy_(lse.view(B, H, Q, G).permute(0, 2, 1, 3).reshape(B, Q, H * G))
    r = {"out": s["out"], "lse": s["lse"]}
    if "mass" in s:
        got = p.sum(2).view(B, H, -1, PAGE).permute(0, 2, 1, 3)                  # [B, MP, H, 64]
        held = torch.arange(T, device="cuda") < s["lengths"][:, None]
        held = held.view(B, -1, 1, PAGE)
        s["mass_out"][ids] = torch.where(held, DECAY * s["mass"][ids] + got, s["mass_out"][ids])
        r["mass"] = s["mass_out"]
    return r


def _plain_select(s, q, seen):
    B, Q, H, G, D = q.shape
    top = q.abs().amax((3, 4), keepdim=True)
    e = torch.frexp(top).exponent - 1
    q8 = torch.ldexp(q, 6 - e).round().clamp(-127, 127).to(torch.int32)
    up, down = q8.clamp(min=0).sum(3), q8.clamp(max=0).sum(3)                    # [B, Q, H, D]
    ids = s["table"].long()
    lo = s["k_bounds"][ids][:, :, :, 0].to(torch.int32).permute(0, 2, 1, 3)      # [B, H, MP, D]
    hi = s["k_bounds"][ids][:, :, :, 1].to(torch.int32).permute(0, 2, 1, 3)
    score = (up[:, :, :, None] * hi[:, None] + down[:, :, :, None] * lo[:, None]).sum(
        -1, dtype=torch.int32)                                                   # [B, Q, H, MP]
    score = score.float() * s["k_scale"][ids].transpose(1, 2)[:, None]
    MP, n = ids.shape[1], s["picks"].shape[3]
    j = torch.arange(MP, device="cuda")
    pages = ((seen + PAGE - 1) // PAGE)[:, :, None, None]
    score = torch.where(j >= pages - RECENT_PAGES, math.inf, score)
    score = torch.where(j < pages, score, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :n]
    best = torch.where(best < pages, best, MP).sort(-1).values
    s["picks"].fill_(-1)
    s["picks"][..., :best.shape[-1]] = torch.where(best < MP, best, -1).to(torch.int32)
    return s["picks"].long()


def _plain_sparse(s):
    q, seen = _grouped(s)
    B, Q, H, G, D = q.shape
    picks = _plain_select(s, q, seen)                                            # [B, Q, H, n]
    n = picks.shape[3]
    ids = s["table"].long()[:, None, None].expand(B, Q, H, -1).gather(3, picks.clamp(min=0))
    h = torch.arange(H, device="cuda")[:, None]
    k = s["k_codes"][ids, h].float() * s["k_scale"][ids, h][..., None, None]     # [B,Q,H,n,64,D]
    v = s["v_codes"][ids, h].float() * s["v_scale"][ids, h][..., None, None]     # [B,Q,H,n,D,64]
    k = k.reshape(B, Q, H, n * PAGE, D)
    v = v.transpose(4, 5).reshape(B, Q, H, n * PAGE, D)
    pos = picks[..., None] * PAGE + torch.arange(PAGE, device="cuda")
    visible = (picks[..., None] >= 0) & (pos < seen[:, :, None, None, None])
    p, lse = _softmax(torch.matmul(q, k.transpose(3, 4)) * s["scale"],
                      visible.reshape(B, Q, H, 1, n * PAGE))
    s["out"].copy_(torch.matmul(p, v).reshape(B, Q, H * G, D))
    s["lse"].copy_(lse.reshape(B, Q, H * G))
    return {"picks": s["picks"], "out": s["out"], "lse": s["lse"]}


def _plain_evict(s):
    case, ids = s["case"], s["table"].long()
    B, H, D = case["seqs"], case["heads"], case["dim"]
    keep, recent = case["keep"], case["recent"]
    T = ids.shape[1] * PAGE
    n = s["lengths"].long()
    mass = s["mass"][ids].permute(0, 2, 1, 3).reshape(B, H, T)
    j = torch.arange(T, device="cuda")
    m = torch.where((j >= n[:, None] - recent)[:, None], math.inf, mass)
    m = torch.where((j < n[:, None])[:, None], m, -math.inf)
    best = torch.sort(m, dim=-1, descending=True, stable=True).indices[..., :keep]
    best = torch.where(best < n[:, None, None], best, T).sort(-1).values
    live = best < T
    width = _pages(keep)
    at = torch.full((B, H, width * PAGE), T, device="cuda")
    at[..., :best.shape[-1]] = best
    valid = (at < T).view(B, H, width, PAGE)
    at = at.clamp(max=T - 1)
    src = ids[:, None].expand(B, H, -1).gather(2, at // PAGE)                    # [B, H, n]
    h = torch.arange(H, device="cuda")[:, None]
    to = s["new_table"].long().reshape(-1)
    filled = valid.any(3)[:, 0].reshape(-1)
    codes = {}
    for name in ("k", "v"):
        c = s["k_codes"][src, h, at % PAGE] if name == "k" else s["v_codes"][src, h, :, at % PAGE]
        x = c.float() * s[name + "_scale"][src, h][..., None]
        x = x.view(B, H, width, PAGE, D) * valid[..., None]
        x = x.permute(0, 2, 1, 3, 4).reshape(B * width, H, PAGE, D)
        scale = _scales(x)
        codes[name] = _divided(x, scale[:, :, None, None])
        _write_pages(s, to, filled, name, codes[name], scale)
    tokens = valid[:, 0].reshape(-1, PAGE)
    s["k_bounds"][to[filled]] = _page_bounds(codes["k"], tokens)[filled]
    moved = (mass.gather(2, at).view(B, H, width, PAGE) * valid).permute(0, 2, 1, 3)
    s["mass"][to[filled]] = moved.reshape(-1, H, PAGE)[filled]
    kept = torch.full((B, H, keep), -1, dtype=torch.int32, device="cuda")
    kept[..., :best.shape[-1]] = torch.where(live, best, -1).to(torch.int32)
    lengths = n.clamp(max=keep).to(torch.int32)
    k, v = _plain_load(s, s["new_table"], s["first"], keep, lengths)
    return {"kept": kept, "lengths": lengths, "k": k, "v": v, "mass": s["mass"],
            "k_scale": s["k_scale"], "v_scale": s["v_scale"], "k_bounds": s["k_bounds"]}


# ---- what a pass cannot do without ------------------------------------------------------------
def work(case):
    """Bytes: every code, scale, row and weight that the pass is about, once. A stored or kept row
    is read once, coded once, read back once and written once. Operations: two products of 2 dim
    for each query row and token it sees (attend, sparse), about four for each value that is coded
    or decoded, two for each bound."""
    op, H, D, HQ = case["op"], case["heads"], case["dim"], case["q_heads"]
    lengths = _lengths(case)
    n = sum(lengths)
    if op == "store":
        rows = n * H * D * 2
        kept = sum(a % PAGE for a, m in zip(_starts(case), lengths) if m) * H * D * 2
        return {"bytes": 2 * (rows * 3 + kept * 3 / 2), "flops": 4 * (rows + kept)}
    queries = _queries(case)
    if op == "attend":
        pairs = sum(q * m - q * (q - 1) // 2 for q, m in zip(queries, lengths)) * HQ
        b = n * H * (2 * D + 8 / PAGE + (8 if case["mass"] else 0)) + sum(queries) * HQ * 4 * D
        return {"bytes": b, "flops": 4 * D * pairs}
    if op == "sparse":
        pages = sum(q * _pages(m) for q, m in zip(queries, lengths)) * H
        picked = sum(q * min(_pages(m), case["picks"]) for q, m in zip(queries, lengths)) * H
        return {"bytes": pages * (2 * D + 4) + picked * PAGE * 2 * D + sum(queries) * HQ * 4 * D,
                "flops": pages * 4 * D + picked * PAGE * 4 * D * HQ // H}
    kept = sum(min(m, case["keep"]) for m in lengths) * H
    return {"bytes": n * H * 4 + kept * (2 * D * 4 + 12), "flops": kept * 2 * D * 8 + n * H * 4}


# ---- the definition in 64 bits ------------------------------------------------------------------
def _single(x):
    """A value that the definition holds in 32 bits."""
    return x.to(torch.float32).to(torch.float64)


def _coded(x):
    """Codes and scale of one page's rows [64, D] (64-bit): both 32-bit quotients."""
    s = _single(x.abs().max() / 127.0)
    if s == 0:
        return torch.zeros_like(x), s
    return _single(x / s).round().clamp(-127, 127), s


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"store": _exact_store, "attend": _exact_attend, "sparse": _exact_sparse,
            "evict": _exact_evict}[case["op"]](case, s)


def _exact_store(case, s):
    B, H, D, T = case["seqs"], case["heads"], case["dim"], case["tokens"]
    lengths, starts = _lengths(case), _starts(case)
    if sum(_pages(n) for n in lengths) * H > 6000:
        return None
    back = {n: torch.zeros((B, s["rows"], H, D), dtype=torch.float64, device="cuda")
            for n in ("k", "v")}
    scales = {n: s[n + "_scale"].double() for n in ("k", "v")}
    for b in range(B):
        a, n = starts[b], lengths[b]
        for j in range(a // PAGE, _pages(a + n) if n else 0):
            page = int(s["table"][b, j])
            lo, hi = max(a, j * PAGE), min(a + n, (j + 1) * PAGE)
            held = max(0, a - j * PAGE)
            for h in range(H):
                for name in ("k", "v"):
                    x = s[name][b, lo - a:hi - a, h].double()
                    was = s[name + "_codes"][page, h].double()
                    was = (was if name == "k" else was.T)[:held]
                    old = s[name + "_scale"][page, h].double()
                    c = _single(x.abs().max() / 127.0)
                    c = torch.maximum(c, old) if held else c
                    if held and c != old:
                        was = _single(_single(was * old) / c).round().clamp(-127, 127)
                    new = _single(x / c).round().clamp(-127, 127) if c > 0 else torch.zeros_like(x)
                    scales[name][page, h] = c
                    r = j * PAGE - a // PAGE * PAGE
                    back[name][b, r:r + held + hi - lo, h] = torch.cat([was, new]) * c
    return {"k": back["k"], "v": back["v"], "k_scale": scales["k"], "v_scale": scales["v"],
            "k_bounds": None}


def _values(s, ids, h, name):
    """Rows [64 n, D] of one head in 64 bits from the pages numbered ids."""
    c = s[name + "_codes"][ids, h].double()
    c = (c if name == "k" else c.transpose(1, 2)) * s[name + "_scale"][ids, h].double()[:, None,
                                                                                       None]
    return c.reshape(-1, c.shape[2])


def _exact_rows(x, k, v, seen, scale):
    """Attention of rows x [R, D]; row r sees the tokens with seen[r, token]."""
    z = (x @ k.T) * scale
    z[~seen] = -math.inf
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - torch.where(lse.isinf(), 0.0, lse)[:, None])
    return p @ v, lse, p


def _exact_attend(case, s):
    B, H, Q, HQ = case["seqs"], case["heads"], case["q"], case["q_heads"]
    G, D = HQ // H, case["dim"]
    out = torch.zeros((B, Q, HQ, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Q, HQ), -math.inf, dtype=torch.float64, device="cuda")
    mass = torch.zeros(s["mass"].shape, dtype=torch.float64, device="cuda") if case["mass"] else None
    queries = _queries(case) if case["ragged"] else [Q] * B
    for b, n in enumerate(_lengths(case)):
        nq = queries[b]
        ids = s["table"][b, :_pages(n)].long()
        i = torch.arange(nq, device="cuda").repeat_interleave(G)
        seen = torch.arange(n, device="cuda") <= (n - nq + i)[:, None]
        for h in range(H if n else 0):
            k, v = _values(s, ids, h, "k")[:n], _values(s, ids, h, "v")[:n]
            x = s["q"][b, :nq, h * G:(h + 1) * G].double().reshape(nq * G, D)
            o, l, p = _exact_rows(x, k, v, seen, s["scale"])
            out[b, :nq, h * G:(h + 1) * G] = o.view(nq, G, D)
            lse[b, :nq, h * G:(h + 1) * G] = l.view(nq, G)
            if case["mass"]:
                w = torch.zeros(len(ids) * PAGE, dtype=torch.float64, device="cuda")
                w[:n] = p.sum(0) + DECAY * s["mass"][ids, h].double().reshape(-1)[:n]
                mass[ids, h] = w.view(-1, PAGE)
    r = {"out": out, "lse": lse}
    if case["mass"]:
        r["mass"] = mass
    return r


def _exact_sparse(case, s):
    B, H, Q, HQ, n = case["seqs"], case["heads"], case["q"], case["q_heads"], case["picks"]
    G, D = HQ // H, case["dim"]
    out = torch.zeros((B, Q, HQ, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Q, HQ), -math.inf, dtype=torch.float64, device="cuda")
    picks = torch.full((B, Q, H, n), -1, dtype=torch.int32, device="cuda")
    queries = _queries(case) if case["ragged"] else [Q] * B
    for b, m in enumerate(_lengths(case)):
        for i in range(queries[b]):
            sees = m - queries[b] + i + 1
            ids = s["table"][b, :_pages(sees)].long()
            for h in range(H if sees > 0 else 0):
                x = s["q"][b, i, h * G:(h + 1) * G].double()
                unit = 2.0 ** (6 - math.floor(math.log2(float(x.abs().max()))))
                q8 = (x * unit).round().clamp(-127, 127)
                lo, hi = s["k_bounds"][ids, h].double().unbind(1)
                score = torch.maximum(q8[:, None] * lo, q8[:, None] * hi).sum((0, 2))
                score = (score * s["k_scale"][ids, h].double()).to(torch.float32)
                score[-RECENT_PAGES:] = math.inf
                rank = sorted(range(len(ids)), key=lambda j, z=score.tolist(): (-z[j], j))[:n]
                rank = torch.tensor(sorted(rank), device="cuda")
                picks[b, i, h, :len(rank)] = rank.to(torch.int32)
                pos = (rank[:, None] * PAGE + torch.arange(PAGE, device="cuda")).reshape(-1)
                o, l, _ = _exact_rows(x, _values(s, ids[rank], h, "k"),
                                      _values(s, ids[rank], h, "v"),
                                      (pos < sees).expand(G, -1), s["scale"])
                out[b, i, h * G:(h + 1) * G] = o
                lse[b, i, h * G:(h + 1) * G] = l
    return {"picks": picks, "out": out, "lse": lse}


def _exact_evict(case, s):
    B, H, D, keep = case["seqs"], case["heads"], case["dim"], case["keep"]
    lengths = _lengths(case)
    if sum(_pages(min(n, keep)) for n in lengths) * H > 6000 or max(lengths) * B * H > 1 << 22:
        return None
    back = {n: torch.zeros((B, keep, H, D), dtype=torch.float64, device="cuda")
            for n in ("k", "v")}
    scales = {n: s[n + "_scale"].double() for n in ("k", "v")}
    mass = s["mass"].double()
    kept = torch.full((B, H, keep), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(lengths):
        ids = s["table"][b, :_pages(n)].long()
        for h in range(H if n else 0):
            w = s["mass"][ids, h].reshape(-1)[:n]
            z = w.tolist()
            old = n - min(n, case["recent"])
            rank = sorted(range(old), key=lambda j: (-z[j], j))[:max(0, keep - (n - old))]
            at = sorted(rank + list(range(old, n))) if n > keep else list(range(n))
            at = torch.tensor(at, device="cuda")
            kept[b, h, :len(at)] = at.to(torch.int32)
            for name in ("k", "v"):
                c = s[name + "_codes"][ids[at // PAGE], h].double()
                c = c if name == "k" else c.transpose(1, 2)
                c = c[torch.arange(len(at), device="cuda"), at % PAGE]
                x = _single(c * s[name + "_scale"][ids[at // PAGE], h].double()[:, None])
                for j in range(_pages(len(at))):
                    to = int(s["new_table"][b, j])
                    codes, scale = _coded(x[j * PAGE:(j + 1) * PAGE])
                    back[name][b, j * PAGE:j * PAGE + len(codes), h] = codes * scale
                    scales[name][to, h] = scale
                    m = torch.zeros(PAGE, dtype=torch.float64, device="cuda")
                    m[:len(codes)] = w[at[j * PAGE:(j + 1) * PAGE]].double()
                    mass[to, h] = m
    return {"kept": kept, "lengths": _ints([min(n, keep) for n in lengths]), "k": back["k"],
            "v": back["v"], "mass": mass, "k_scale": scales["k"], "v_scale": scales["v"],
            "k_bounds": None}
