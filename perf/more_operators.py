"""Timed cases of requests that share a loaded context in the 8-bit serving cache: they fork from
it, draft tokens, attend over the common pages once for all, and roll back what was not accepted.

The cache is the pool of 64-token pages of perf/operators.py (K codes [page][head][64][dim], V codes
transposed [page][head][dim][64], scales fp32 [page][head], the K codes' bounds [page][head][2][dim],
weights [page][head][64]). A sequence is a row of page numbers (-1: no page) and a length; `refs`
[page] counts the rows that hold a page, 0 marks it free.

Operations (a case's "op"):
  fork     the requests of the last pass end (their pages are released), new ones fork from the
           contexts, sharing their pages, and get pages for `new` tokens: of a page that they share
           and will write to, each gets a copy of its own. Free pages go out lowest first.
  copy     whole pages are copied to others.
  compact  the pages in use move to the pool's front: the i-th page in use behind it to the i-th
           free one in it; tables and counts follow.
  shared   queries of each request attend over its context's pages (all of them: the context lies
           before every query) and causally over its own; without pages of its own that is cross
           attention to the states of an encoder.
  verify   of the tokens drafted for each request the first ones are accepted by given random
           numbers, and the next is drawn from what the target's probabilities have over the
           draft's.

A case's other fields: heads (KV), dim, q_heads, contexts, users (requests of each context), tokens
(of a context), new (tokens of each request: reserved by "fork", held by "shared"), q (query
tokens), pool (pages), live (share of the pool in use, "compact"), mass (weights move along), ragged
(lengths and counts differ), dtype of queries or probabilities, drafts, vocab, sure (the draft is
one token, not a distribution).
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE = 64
UNITS = 42                      # probabilities count in whole multiples of 2^-42


def _case(name, op, **more):
    c = {"op": op, "heads": 8, "dim": 128, "q_heads": 32, "contexts": 1, "users": 1, "tokens": 0,
         "new": 0, "q": 1, "pool": 0, "live": 0.5, "mass": False, "ragged": False,
         "dtype": "float16", "drafts": 0, "vocab": 0, "sure": False}
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # eight samples of one answer start behind a prompt of 1000 tokens: launches and latency
        _case("fork_b8_t1000", "fork", users=8, tokens=1000, new=1, pool=256),
        # the same of every layer at once, 32 of them with 16 requests each over 4K tokens
        _case("fork_layers32_b16_t4196", "fork", contexts=32, users=16, tokens=4196, new=6,
              pool=3500, mass=True),
        # a large pool of small pages (one KV head a GPU), uneven contexts, a paragraph each
        _case("fork_pool65536", "fork", heads=1, dim=64, contexts=64, users=6, tokens=8003, new=200,
              pool=65536, ragged=True),
        # contexts of 2048 pages get pages of their own
        _case("copy_p2048", "copy", pool=4096, mass=True),
        # a small pool with odd heads, and one of half a gigabyte that requests have left in holes
        _case("compact_p300_h5_d64", "compact", heads=5, dim=64, contexts=7, pool=300, live=0.6,
              ragged=True),
        _case("compact_p4096", "compact", contexts=24, pool=4096, live=0.5, mass=True),
        # one token of each of eight requests over a prompt of 1000 tokens: the smallest
        _case("shared_b8_t1000", "shared", users=8, tokens=1000, new=40),
        # 32 requests over a context of 16K tokens, each with an answer of up to 300
        _case("shared_b32_t16384", "shared", users=32, tokens=16384, new=300, ragged=True),
        # five drafted tokens and the last one of requests over three contexts
        _case("shared_drafts_c3_b8_t8192", "shared", heads=5, q_heads=10, dim=64, contexts=3,
              users=8, tokens=8192, new=200, q=6, ragged=True, dtype="bfloat16"),
        # cross attention: 448 tokens over an encoder's 1500 states, multi-head, four at a time
        _case("cross_b4_q448_t1500", "shared", heads=16, q_heads=16, dim=64, contexts=4, users=1,
              tokens=1500, q=448),
        # four drafted tokens of one request: launches and latency
        _case("verify_b1_k4_v32000", "verify", users=1, drafts=4, vocab=32000, dtype="float32"),
        # a batch of 64 requests with a vocabulary of 128K
        _case("verify_b64_k5_v131072", "verify", users=64, drafts=5, vocab=131072, ragged=True,
              dtype="float32"),
    ]


OPS = ("fork", "fork", "copy", "compact", "compact", "shared", "shared", "shared", "verify",
       "verify")
#: (query heads, KV heads) of several families, and odd ones
HEADS = ((32, 8), (32, 8), (64, 8), (32, 32), (16, 16), (8, 1), (28, 4), (12, 4), (10, 5), (3, 1))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(OPS)
    q_heads, heads = rng.choice(HEADS)
    dim = rng.choice((128, 128, 128, 64, 64, 256))
    more = {"heads": heads, "q_heads": q_heads, "dim": dim, "ragged": rng.random() < 0.5,
            "mass": rng.random() < 0.4, "dtype": rng.choice(("float16", "bfloat16"))}
    most = (1 << 29) // (heads * dim * 2 * PAGE)               # pages of half a gigabyte
    if op == "verify":
        vocab = _log(rng, 500, 200000)
        users = min(_log(rng, 1, 64), max(1, (1 << 23) // vocab))
        return _case(None, op, users=users, drafts=rng.choice((0, 1, 2, 3, 4, 5, 7, 8)),
                     vocab=vocab, ragged=more["ragged"], sure=rng.random() < 0.3,
                     dtype=rng.choice(("float32", "float32", "bfloat16", "float16")))
    if op == "shared":
        contexts, users = _log(rng, 1, 6), _log(rng, 1, 48)
        q = 1 if rng.random() < 0.5 else _log(rng, 2, 200)
        q = min(q, max(1, 8192 // (contexts * users)))
        new = 0 if rng.random() < 0.3 else q + _log(rng, 1, 400)
        # a cache, and rows times tokens, of the largest listed ones at most
        tokens = min(16384, (1 << 24) // (contexts * heads * dim),
                     (1 << 30) // (contexts * users * q * q_heads * dim // 2))
        return _case(None, op, contexts=contexts, users=users, q=q, new=new,
                     tokens=_log(rng, 1, max(2, tokens)), **more)
    if op == "fork":
        contexts, users = _log(rng, 1, 32), _log(rng, 1, 16)
        new = _log(rng, 1, 300)
        each = users * (new // PAGE + 2)
        tokens = _log(rng, 1, max(2, min(8192, PAGE * max(0, most // contexts - each - 1))))
        pool = contexts * (tokens // PAGE + 1 + each) + _log(rng, 8, 500)
        return _case(None, op, contexts=contexts, users=users, tokens=tokens, new=new, pool=pool,
                     **more)
    return _case(None, op, pool=_log(rng, 64, max(100, min(50000, most))),
                 contexts=_log(rng, 1, 24), live=rng.choice((0.05, 0.3, 0.5, 0.7, 0.95)), **more)


# ---- sizes that follow from the case ----------------------------------------------------------
def _pages(n):
    return -(-n // PAGE)


def _spread(n, most, ragged, seed):
    r = random.Random(n * 1_000_003 + most * 31 + seed)
    return [most] + [r.randint(min(most, 1 + most // 3), most) if ragged else most for _ in range(n - 1)]


def _contexts(case):
    """Tokens of every context."""
    return _spread(case["contexts"], case["tokens"], case["ragged"], 1)


def _firsts(case):
    """Context i is read by the requests from firsts[i] on. Of eight or more uneven ones the last
    request has no context, of three or more uneven contexts the second has few requests."""
    n, users = case["contexts"], case["users"]
    at = [i * users for i in range(n + 1)]
    if case["ragged"] and n >= 3:
        at[2] = at[1] + (users + 2) // 3
    if case["ragged"] and n * users >= 8:
        at[n] -= 1
    return at


def _answers(case):
    """Tokens of each request's own, the queries' among them."""
    return _spread(case["contexts"] * case["users"], case["new"], case["ragged"], 2)


def _queries(case):
    n = case["contexts"] * case["users"]
    q = _spread(n, case["q"], case["ragged"], 3)
    return [min(a, b) for a, b in zip(q, _answers(case))] if case["new"] else q


def _drafts(case):
    """Tokens drafted for each request; of eight or more uneven ones the second sits out."""
    n, k = case["users"], case["drafts"]
    r = random.Random(n * 7 + k)
    got = [k] + [r.randint(0, k) if case["ragged"] else k for _ in range(n - 1)]
    if case["ragged"] and n >= 8:
        got[1] = -1
    return got


# ---- inputs -----------------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pool(case, n_pages, g):
    """The pages' buffers with random codes."""
    H, D = case["heads"], case["dim"]

    def codes(*shape):
        return torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)

    def scales():
        return torch.exp(0.3 * torch.randn((n_pages, H), generator=g, device="cuda")) / 40.0

    p = {"k_codes": codes(n_pages, H, PAGE, D), "v_codes": codes(n_pages, H, D, PAGE),
         "k_scale": scales(), "v_scale": scales(), "k_bounds": codes(n_pages, H, 2, D)}
    if case["mass"]:
        p["mass"] = torch.randn((n_pages, H, PAGE), generator=g, device="cuda").mul_(2.0).exp_()
    return p


def _rows(shape, g):
    """Rows [..., heads, dim] with a level and a size of their own for each channel."""
    size = torch.exp(0.5 * torch.randn(shape[-2:], generator=g, device="cuda"))
    level = 0.7 * torch.randn(shape[-2:], generator=g, device="cuda")
    return torch.randn(shape, generator=g, device="cuda") * size + level


def _filled(case, n_pages, g):
    """The pages' buffers with the codes of random rows."""
    H, D = case["heads"], case["dim"]
    p = {}
    for name, axes, shape in (("k", (0, 2, 1, 3), (PAGE, D)), ("v", (0, 2, 3, 1), (D, PAGE))):
        p[name + "_codes"] = torch.empty((n_pages, H, *shape), dtype=torch.int8, device="cuda")
        p[name + "_scale"] = torch.empty((n_pages, H), device="cuda")
        per = max(1, (1 << 26) // (H * PAGE * D))
        for i in range(0, n_pages, per):
            x = _rows((min(per, n_pages - i), PAGE, H, D), g).permute(axes)
            s = x.abs().amax((2, 3)) / 127.0
            p[name + "_codes"][i:i + per] = (x / s[:, :, None, None]).round().to(torch.int8)
            p[name + "_scale"][i:i + per] = s
    p["k_bounds"] = None
    return p


def _table(pages, counts, width):
    """A table [len(counts), width]: the next counts[i] of the page numbers for row i."""
    n = torch.tensor(counts, device="cuda")
    j = torch.arange(width, device="cuda")
    at = (n.cumsum(0) - n)[:, None] + j
    live = j < n[:, None]
    return torch.where(live, pages[at.clamp(max=len(pages) - 1)], -1).to(torch.int32)


def _refs(n_pages, table):
    t = table[table >= 0].long()
    return torch.bincount(t, minlength=n_pages).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 61)
    op, H, D, P = case["op"], case["heads"], case["dim"], case["pool"]
    s = {"op": op, "case": dict(case), "cache": None, "mass": None}
    if op == "verify":
        _prepare_verify(case, s, g)
    elif op == "shared":
        P = _prepare_shared(case, s, g)
    else:
        s.update(_pool(case, P, g))
        order = torch.randperm(P, generator=g, device="cuda")
        if op == "fork":
            tokens, users = _contexts(case), case["users"]
            counts = [_pages(n) for n in tokens]
            # (a row has room for what its request will write)
            width = max(_pages(n + case["new"]) for n in tokens)
            s["table"], s["lengths"] = _table(order, counts, width), _ints(tokens)
            s["refs"] = _refs(P, s["table"])
            n = len(tokens) * users
            s["parents"] = _ints([i // users for i in range(n)])
            s["counts"] = _ints(_spread(n, case["new"], case["ragged"], 4))
            s["kids"] = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        elif op == "copy":
            n = P // 2
            s["src"], s["dst"] = order[:n].to(torch.int32), order[n:2 * n].to(torch.int32)
        else:
            used = max(case["contexts"], int(P * case["live"]))
            share = used // case["contexts"]
            counts = _spread(case["contexts"], share, case["ragged"], 5)
            s["table"] = _table(order, counts, max(counts))
            if len(counts) > 1:                   # the last one shares pages with the first
                s["table"][-1, 0] = s["table"][0, 0]
            s["refs"] = _refs(P, s["table"])
    if own:
        from paper_2310_07240_amd.kv8 import Kv8Cache
        if op == "verify":
            s["cache"] = Kv8Cache(1, 1, 64)
        else:
            s["cache"] = Kv8Cache(P, H, D, buffers={k: s[k] for k in (
                "k_codes", "v_codes", "k_scale", "v_scale", "k_bounds")})
    return s


def _prepare_shared(case, s, g):
    H, D, HQ, Q = case["heads"], case["dim"], case["q_heads"], case["q"]
    tokens, n = _contexts(case), case["contexts"] * case["users"]
    counts = [_pages(t) for t in tokens]
    answers = _answers(case)
    mine = [_pages(t) for t in answers]
    P = sum(counts) + sum(mine) + 3
    s.update(_filled(case, P, g))
    order = torch.randperm(P, generator=g, device="cuda")
    s["shared"], s["shared_lengths"] = _table(order, counts, max(counts)), _ints(tokens)
    firsts = _firsts(case)
    s["firsts"], s["users"] = _ints(firsts), max(b - a for a, b in zip(firsts, firsts[1:]))
    s["table"] = _table(order[sum(counts):], mine, max(mine)) if case["new"] else None
    s["lengths"] = _ints(answers) if case["new"] else None
    s["q"] = 2.0 * torch.randn((n, Q, HQ, D), generator=g, device="cuda")
    s["q"] = s["q"].to(getattr(torch, case["dtype"]))
    s["q_lens"] = _ints(_queries(case)) if case["ragged"] else None
    s["scale"] = 1.0 / math.sqrt(D)
    s["max_shared"], s["max_len"] = max(tokens), max(answers)
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(s["q"].shape[:3], dtype=torch.float32, device="cuda")
    return P


def _prepare_verify(case, s, g):
    B, K, V = case["users"], case["drafts"], case["vocab"]
    dtype = getattr(torch, case["dtype"])
    logits = 2.5 * torch.randn((B, K + 1, V), generator=g, device="cuda")
    near = logits[:, :K] + 0.6 * torch.randn((B, K, V), generator=g, device="cuda")
    s["target"] = torch.softmax(logits, -1).to(dtype)
    s["draft"] = None
    if case["sure"]:
        s["drafts"] = near.argmax(-1).to(torch.int32)
    else:
        s["draft"] = torch.softmax(near, -1).to(dtype)
        noise = -torch.log(-torch.log(torch.rand(near.shape, generator=g, device="cuda")
                                      .clamp(1e-20, 1 - 1e-7)))
        s["drafts"] = (near + noise).argmax(-1).to(torch.int32)
    s["u"] = torch.rand((B, K + 1), generator=g, device="cuda")
    s["counts"] = _ints(_drafts(case)) if case["ragged"] else None
    s["lengths"] = torch.randint(K + 1, 5000, (B,), generator=g, device="cuda", dtype=torch.int32)


# ---- one pass ---------------------------------------------------------------------------------
POOL = ("k_codes", "v_codes", "k_scale", "v_scale", "k_bounds", "mass")


def _held(s, **more):
    return {**more, **{k: s[k] for k in POOL if s.get(k) is not None}}


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    op, c = s["op"], s["cache"]
    if op == "fork":
        c.release(s["kids"], s["refs"])
        kids, lengths = c.fork(s["table"], s["lengths"], s["parents"], s["refs"],
                               new_table=s["kids"])
        missing = c.reserve(kids, lengths, s["counts"], s["refs"], mass=s["mass"])
        return _held(s, table=kids, lengths=lengths, missing=missing, refs=s["refs"])
    if op == "copy":
        c.copy(s["src"], s["dst"], mass=s["mass"])
        return _held(s)
    if op == "compact":
        table, refs, moved, live = c.compact(s["table"], s["refs"], mass=s["mass"])
        return _held(s, table=table, refs=refs, moved=moved, live=live)
    if op == "shared":
        c.attend_shared(s["q"], s["shared"], s["shared_lengths"], s["firsts"], table=s["table"],
                        lengths=s["lengths"], scale=s["scale"], q_lens=s["q_lens"],
                        max_shared=s["max_shared"], max_len=s["max_len"], max_users=s["users"],
                        out=s["out"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    tokens, accepted, lengths = c.verify(s["target"], s["drafts"], s["u"], draft=s["draft"],
                                         counts=s["counts"], lengths=s["lengths"])
    return {"tokens": tokens, "accepted": accepted, "lengths": lengths}


def _run_plain(s):
    return {"fork": _plain_fork, "copy": _plain_copy, "compact": _plain_compact,
            "shared": _plain_shared, "verify": _plain_verify}[s["op"]](s)


# ---- pages ------------------------------------------------------------------------------------
def _count(refs, pages, which, by):
    """refs[pages] += by where `which`, never below 0."""
    step = by * which.to(torch.int32)
    refs.scatter_add_(0, pages.clamp(min=0).long().reshape(-1), step.reshape(-1))
    refs.clamp_(min=0)


def _move_pages(s, src, dst):
    """Pages src to dst (equal numbers: they stay); what they hold, one buffer after the other."""
    return [s[k].index_copy_(0, dst, s[k][src]) for k in POOL if s.get(k) is not None]


def _numbered(which):
    """The indices where `which`, ascending, in a tensor as long as `which` (0 behind them)."""
    n = len(which)
    rank = torch.where(which, which.cumsum(0) - 1, n)
    at = torch.zeros(n + 1, dtype=torch.long, device="cuda")
    return at.scatter_(0, rank, torch.arange(n, device="cuda"))[:n]


def _plain_fork(s):
    refs, P = s["refs"], len(s["refs"])
    # the last requests end
    gone = s["kids"] >= 0
    _count(refs, s["kids"], gone, -1)
    # new ones share the contexts' pages
    lengths = s["lengths"][s["parents"].long()]
    rows = s["table"][s["parents"].long()]
    col = torch.arange(rows.shape[1], device="cuda") * PAGE
    kids = s["kids"]
    kids.copy_(torch.where(col < lengths[:, None], rows, -1))
    _count(refs, kids, kids >= 0, 1)
    # pages for the new tokens, copies of the shared ones that keep tokens before them
    start = lengths[:, None]
    end = (start + s["counts"][:, None]).clamp(max=kids.shape[1] * PAGE)
    within = (col + PAGE > start) & (col < end) & (s["counts"][:, None] > 0)
    keeps = col < start
    users = torch.where(kids >= 0, refs[kids.clamp(min=0).long()], 0)
    need = within & torch.where(keeps, users > 1, users != 1)
    flat = need.reshape(-1)
    free = refs == 0
    missing = (flat.sum() - free.sum()).clamp(min=0)
    need = need & (missing == 0)
    pages = _numbered(free)[(flat.cumsum(0) - 1).clamp(min=0, max=P - 1)].view(need.shape)
    _count(refs, kids, need & (kids >= 0), -1)
    fresh = need.reshape(-1).to(torch.int32)
    refs.scatter_add_(0, pages.reshape(-1), fresh)
    copied = need & keeps
    # one page at most for each request; without one a context's page is copied onto itself
    some, at = copied.any(1), copied.to(torch.int32).argmax(1, keepdim=True)
    src, dst = kids.gather(1, at).squeeze(1).long(), pages.gather(1, at).squeeze(1)
    spare = s["table"][0, 0].long()
    _move_pages(s, torch.where(some, src, spare), torch.where(some, dst, spare))
    kids.copy_(torch.where(need, pages.to(torch.int32), kids))
    return _held(s, table=kids, lengths=lengths, missing=missing.to(torch.int32).view(1), refs=refs)


def _plain_copy(s):
    _move_pages(s, s["src"].long(), s["dst"].long())
    return _held(s)


def _plain_compact(s):
    refs, table, P = s["refs"], s["table"], len(s["refs"])
    used = refs > 0
    n = used.sum()
    j = torch.arange(P, device="cuda")
    late = used & (j >= n)
    src, dst = _numbered(late), _numbered(~used & (j < n))
    moved = torch.where(late, dst[(late.cumsum(0) - 1).clamp(min=0)], torch.where(used, j, -1))
    moved = moved.to(torch.int32)
    # (behind the last move the first once more, or a page onto itself)
    k = torch.arange(P // 2 + 1, device="cuda") < late.sum()
    src = torch.where(k, src[:P // 2 + 1], src[0])
    dst = torch.where(k, dst[:P // 2 + 1], torch.where(late.any(), dst[0], src[0]))
    _move_pages(s, src, dst)
    live = torch.where(table >= 0, moved[table.clamp(min=0).long()], -1)
    counts = torch.zeros(P + 1, dtype=torch.int32, device="cuda")
    counts.scatter_(0, torch.where(used, moved.long(), P), refs)
    return _held(s, table=live, refs=counts[:P], moved=moved, live=n.to(torch.int32).view(1))


# ---- attention --------------------------------------------------------------------------------
def _values(s, table):
    """Rows K, V [n, H, columns * 64, D] of a table's pages in 32 bits."""
    ids = table.clamp(min=0).long()
    k = s["k_codes"][ids].float() * s["k_scale"][ids][..., None, None]
    v = s["v_codes"][ids].float() * s["v_scale"][ids][..., None, None]
    return (k.permute(0, 2, 1, 3, 4).flatten(2, 3),
            v.permute(0, 2, 1, 4, 3).flatten(2, 3).contiguous())


def _plain_shared(s):
    B, Q, HQ, D = s["q"].shape
    H = s["k_codes"].shape[1]
    G, U, firsts = HQ // H, s["users"], s["firsts"].long()
    x = s["q"].float().view(B, Q, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, Q * G, D)
    i = torch.arange(Q, device="cuda")
    ql = torch.full((B, 1), Q, device="cuda") if s["q_lens"] is None else s["q_lens"][:, None].long()
    asks = (i < ql).repeat_interleave(G, 1)                                      # [B, Q G]
    b = torch.arange(B, device="cuda")
    of = torch.searchsorted(firsts, b, right=True) - 1
    some = of < len(firsts) - 1
    of = of.clamp(max=len(firsts) - 2)
    user = (b - firsts[of]).clamp(max=U - 1)
    rows = (firsts[:-1, None] + torch.arange(U, device="cuda")).clamp(max=B - 1)   # [contexts, U]
    k, v = _values(s, s["shared"])
    T = k.shape[2]
    xs = x[rows].permute(0, 2, 1, 3, 4).reshape(len(rows), H, U * Q * G, D)
    z = torch.matmul(xs, k.transpose(2, 3).contiguous()) * s["scale"]
    z = z.view(len(rows), H, U, Q * G, T).transpose(1, 2)[of, user]              # [B, H, Q G, T]
    see = torch.arange(T, device="cuda") < (s["shared_lengths"][of] * some)[:, None]
    z = z.masked_fill(~(see[:, None] & asks[:, :, None])[:, None], -math.inf)
    if s["table"] is not None:
        ko, vo = _values(s, s["table"])
        n = s["lengths"][:, None].long()
        seen = torch.where(i < ql, (n - ql + i + 1).clamp(min=0), 0).repeat_interleave(G, 1)
        zo = torch.matmul(x, ko.transpose(2, 3).contiguous()) * s["scale"]
        see = torch.arange(ko.shape[2], device="cuda") < seen[:, :, None]
        z = torch.cat([z, zo.masked_fill(~see[:, None], -math.inf)], -1)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m.isinf(), 0.0, m))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    # back to the contexts' requests for the products with V; a place without a request is not read
    ps = p[..., :T][rows].permute(0, 2, 1, 3, 4).reshape(len(rows), H, U * Q * G, T)
    o = torch.matmul(ps, v).view(len(rows), H, U, Q * G, D).transpose(1, 2)[of, user]
    o = torch.where(some[:, None, None, None], o, 0.0)
    if s["table"] is not None:
        o = o + torch.matmul(p[..., T:], vo)
    o = o.view(B, H, Q, G, D).permute(0, 2, 1, 3, 4).reshape(B, Q, HQ, D)
    lse = (m + torch.log(total)).view(B, H, Q, G).permute(0, 2, 1, 3).reshape(B, Q, HQ)
    s["out"].copy_(o)
    s["lse"].copy_(lse)
    return {"out": s["out"], "lse": s["lse"]}


# ---- drafted tokens ----------------------------------------------------------------------------
def _probability(x):
    """What a probability counts as: NaN and what is below 0 as 0, what is above 1 as 1."""
    return torch.nan_to_num(x.double(), 0.0, 1.0, 0.0).clamp(0.0, 1.0)


def _units(x):
    return (_probability(x) * 2.0 ** UNITS).round().long()


def _plain_verify(s):
    target, drafts = s["target"], s["drafts"].long()
    B, K, V = target.shape[0], target.shape[1] - 1, target.shape[2]
    counts = torch.full((B,), K, device="cuda") if s["counts"] is None else s["counts"].long()
    j = torch.arange(K, device="cuda")
    valid = (drafts >= 0) & (drafts < V) & (j < counts[:, None])
    at = drafts.clamp(0, V - 1)[..., None]
    p = _probability(target[:, :K].gather(2, at).squeeze(2))
    q = torch.ones_like(p) if s["draft"] is None else _probability(
        s["draft"].gather(2, at).squeeze(2))
    good = valid & (s["u"][:, :K].double() * q < p)
    accepted = good.long().cumprod(1).sum(1)
    b = torch.arange(B, device="cuda")
    have = _units(target[b, accepted])
    if K:
        last = accepted.clamp(max=K - 1)
        if s["draft"] is None:
            off = torch.zeros_like(have).scatter_(1, at[b, last], 1 << UNITS)
        else:
            off = _units(s["draft"][b, last])
        over = (have - off * (accepted < counts)[:, None]).clamp(min=0)
        have = torch.where(over.sum(1, keepdim=True) > 0, over, have)
    total = have.sum(1)
    part = (s["u"][:, K].double() * 2.0 ** 24).floor().long().clamp(0, (1 << 24) - 1)
    bar = part * (total >> 24) + (part * (total & ((1 << 24) - 1)) >> 24)
    new = (have.cumsum(1) <= bar[:, None]).sum(1)
    new = torch.where(total > 0, new, -1)
    i = torch.arange(K + 1, device="cuda")
    past = torch.cat([drafts, torch.full((B, 1), -1, device="cuda")], 1)
    tokens = torch.where(i < accepted[:, None], past, -1)
    tokens = torch.where(i == accepted[:, None], new[:, None], tokens)
    tokens = torch.where(counts[:, None] < 0, -1, tokens)
    back = counts.clamp(min=0) - accepted
    return {"tokens": tokens.to(torch.int32), "accepted": accepted.to(torch.int32),
            "lengths": (s["lengths"] - back).clamp(min=0).to(torch.int32)}


# ---- what a pass cannot do without ------------------------------------------------------------
def _page_bytes(case):
    H, D = case["heads"], case["dim"]
    return H * (2 * PAGE * D + 2 * D + 8 + (4 * PAGE if case["mass"] else 0))


def work(case):
    """Bytes: of a page that is copied its codes, scales, bounds and weights, read and written; every
    count of the pool once, and a table's entries read and written; of attention every page that any
    request reads once, queries and outputs; of a verified request one row of each distribution and
    the drafted tokens' own. Operations: two products of 2 dim for each query row and token it sees;
    four for each probability."""
    op, H, D, HQ = case["op"], case["heads"], case["dim"], case["q_heads"]
    if op == "fork":
        tokens, n = _contexts(case), case["contexts"] * case["users"]
        copies = sum(case["users"] for t in tokens if t % PAGE)
        entries = sum(_pages(t) for t in tokens) * (case["users"] + 1) + n * (2 + case["new"] // PAGE)
        return {"bytes": copies * 2 * _page_bytes(case) + case["pool"] * 4 + entries * 8,
                "flops": entries}
    if op == "copy":
        return {"bytes": case["pool"] // 2 * (2 * _page_bytes(case) + 8), "flops": 0}
    if op == "compact":
        used = max(case["contexts"], int(case["pool"] * case["live"]))
        moved = used * (1 - min(1.0, used / case["pool"]))       # on average, of random places
        return {"bytes": moved * 2 * _page_bytes(case) + case["pool"] * 12 + used * 8,
                "flops": case["pool"]}
    if op == "verify":
        size = {"float32": 4}.get(case["dtype"], 2)
        live = [k for k in _drafts(case) if k >= 0] if case["ragged"] else (
            [case["drafts"]] * case["users"])
        rows = sum(1 if case["sure"] or not k else 2 for k in live)
        return {"bytes": rows * case["vocab"] * size + sum(live) * (2 * size + 12),
                "flops": 4 * rows * case["vocab"]}
    queries, answers, tokens = _queries(case), _answers(case), _contexts(case)
    at = _firsts(case)
    pairs = sum(sum(queries[a:b]) * t for a, b, t in zip(at, at[1:], tokens))
    pairs += sum(q * n - q * (q - 1) // 2 for q, n in zip(queries, answers)) if case["new"] else 0
    held = sum(tokens) + (sum(answers) if case["new"] else 0)
    return {"bytes": held * H * (2 * D + 8 / PAGE) + sum(queries) * HQ * 4 * (D + 1),
            "flops": 4 * D * pairs * HQ}


# ---- the definition in 64 bits ------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"fork": _exact_fork, "copy": _exact_copy, "compact": _exact_compact,
            "shared": _exact_shared, "verify": _exact_verify}[case["op"]](case, s)


def _exact_pool(s, moves, **more):
    """The pool after pages moved from -> to, floating values in 64 bits."""
    src = torch.tensor([a for a, _ in moves], dtype=torch.long, device="cuda")
    dst = torch.tensor([b for _, b in moves], dtype=torch.long, device="cuda")
    out = dict(more)
    for k in POOL:
        if s.get(k) is not None:
            x = s[k].double() if s[k].is_floating_point() else s[k].clone()
            x[dst] = x[src]
            out[k] = x
    return out


def _exact_fork(case, s):
    refs, table = s["refs"].tolist(), s["table"].tolist()
    width, lengths, kids = len(table[0]), [], []
    for p in s["parents"].tolist():
        n = int(s["lengths"][p])
        lengths.append(n)
        kids.append(table[p][:_pages(n)] + [-1] * (width - _pages(n)))
        for page in table[p][:_pages(n)]:
            refs[page] += 1
    free = [i for i, r in enumerate(refs) if r == 0]
    held, moves, wanted = list(refs), [], []
    for row, (n, new) in enumerate(zip(lengths, s["counts"].tolist())):
        for j in range(n // PAGE, min(width, _pages(n + new))):
            page = kids[row][j]
            if page < 0 or held[page] > 1:
                wanted.append((row, j, j * PAGE < n))
    missing = max(0, len(wanted) - len(free))
    for (row, j, keeps), page in zip(wanted if not missing else [], free):
        was = kids[row][j]
        if was >= 0:
            refs[was] -= 1
        if keeps:
            moves.append((was, page))
        kids[row][j] = page
        refs[page] = 1
    return _exact_pool(s, moves, table=_ints(kids), lengths=_ints(lengths),
                       missing=_ints([missing]), refs=_ints(refs))


def _exact_copy(case, s):
    return _exact_pool(s, list(zip(s["src"].tolist(), s["dst"].tolist())))


def _exact_compact(case, s):
    refs = s["refs"].tolist()
    live = sum(r > 0 for r in refs)
    holes = [i for i in range(live) if refs[i] == 0]
    moves = list(zip([i for i in range(live, len(refs)) if refs[i] > 0], holes))
    moved = [i if r > 0 else -1 for i, r in enumerate(refs)]
    for a, b in moves:
        moved[a], refs[b], refs[a] = b, refs[a], 0
    table = [[moved[p] if p >= 0 else -1 for p in row] for row in s["table"].tolist()]
    return _exact_pool(s, moves, table=_ints(table), refs=_ints(refs), moved=_ints(moved),
                       live=_ints([live]))


def _exact_page_rows(s, ids, h, n):
    k = s["k_codes"][ids, h].double() * s["k_scale"][ids, h].double()[:, None, None]
    v = s["v_codes"][ids, h].double() * s["v_scale"][ids, h].double()[:, None, None]
    return k.flatten(0, 1)[:n], v.transpose(1, 2).flatten(0, 1)[:n]


def _exact_shared(case, s):
    B, Q, HQ, D = s["q"].shape
    H = case["heads"]
    G = HQ // H
    out = torch.zeros((B, Q, HQ, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Q, HQ), -math.inf, dtype=torch.float64, device="cuda")
    queries = _queries(case) if case["ragged"] else [Q] * B
    answers, tokens, at = _answers(case), _contexts(case), _firsts(case)
    if B * H > 4000:
        return None
    for h in range(H):
        held = {}
        for b in range(B):
            nq, k, v = queries[b], [], []
            of = [i for i, (x, y) in enumerate(zip(at, at[1:])) if x <= b < y]
            before = tokens[of[0]] if of else 0
            if of:
                if of[0] not in held:
                    ids = s["shared"][of[0], :_pages(before)].long()
                    held = {of[0]: _exact_page_rows(s, ids, h, before)}
                k, v = [held[of[0]][0]], [held[of[0]][1]]
            mine = answers[b] if case["new"] else 0
            if mine:
                ids = s["table"][b, :_pages(mine)].long()
                x = _exact_page_rows(s, ids, h, mine)
                k, v = k + [x[0]], v + [x[1]]
            if not k:
                continue
            k, v = torch.cat(k), torch.cat(v)
            z = s["q"][b, :nq, h * G:(h + 1) * G].double().reshape(nq * G, D) @ k.T * s["scale"]
            if mine:
                i = torch.arange(nq, device="cuda").repeat_interleave(G)
                z[torch.arange(len(k), device="cuda") > (before + mine - nq + i)[:, None]] = -math.inf
            e = torch.logsumexp(z, 1)
            out[b, :nq, h * G:(h + 1) * G] = (torch.exp(z - e[:, None]) @ v).view(nq, G, D)
            lse[b, :nq, h * G:(h + 1) * G] = e.view(nq, G)
    return {"out": out, "lse": lse}


def _exact_verify(case, s):
    import numpy as np
    B, K, V = case["users"], case["drafts"], case["vocab"]
    target = s["target"].double().cpu().numpy()
    draft = None if s["draft"] is None else s["draft"].double().cpu().numpy()
    u, drafts = s["u"].double().tolist(), s["drafts"].tolist()
    counts = _drafts(case) if case["ragged"] else [K] * B
    tokens = [[-1] * (K + 1) for _ in range(B)]
    accepted, lengths = [0] * B, s["lengths"].tolist()
    for b in range(B):
        if counts[b] < 0:
            continue
        n = 0
        while n < counts[b]:
            x = drafts[b][n]
            if not u[b][n] * (1.0 if draft is None else draft[b, n, x]) < target[b, n, x]:
                break
            tokens[b][n] = x
            n += 1
        have = np.rint(target[b, n] * 2.0 ** UNITS).astype(np.int64)
        if n < counts[b]:
            if draft is None:
                over = have.copy()
                over[drafts[b][n]] = 0
            else:
                over = np.maximum(have - np.rint(draft[b, n] * 2.0 ** UNITS).astype(np.int64), 0)
            have = over if over.any() else have
        total = int(have.sum())
        bar = math.floor(u[b][K] * 2 ** 24) * total >> 24
        tokens[b][n] = int(np.searchsorted(np.cumsum(have), bar, side="right")) if total else -1
        accepted[b] = n
        lengths[b] = max(0, lengths[b] - (counts[b] - n))
    return {"tokens": _ints(tokens), "accepted": _ints(accepted), "lengths": _ints(lengths)}
