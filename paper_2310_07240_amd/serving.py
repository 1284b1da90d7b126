"""A context's life behind the codec on one GPU: it comes back from its bitstreams (``Codec``), goes
into the 8-bit serving cache (``Kv8Cache``) with every layer at once, a question and then single
tokens attend over it, the tokens that attention passed by are evicted, and what is left goes back
to the codec (the paper measures CacheGen on top of token dropping in Sec. 7.2).

With ``--requests``, many requests answer over each context instead (``answer``): they fork from it,
draft tokens, attend over the pages that they share, take what the target accepts, and give their
pages back.

Each step is timed on the GPU (HIP events); the attention of the question (or of the requests' first
step) is compared with the same attention over the decoded fp16 cache, in 32 bits. Queries, new
tokens and probabilities are random: no model is involved.

Usage: python -m paper_2310_07240_amd.serving [--workload NAME] [--heads H] [--q-heads H]
       [--question N] [--tokens N] [--keep F] [--picks N]     (one JSON line)
       python -m paper_2310_07240_amd.serving --requests N [--drafts N] [--steps N] [--vocab N]
"""
from __future__ import annotations

import argparse
import json
import math
import sys

import numpy as np


def _timed(torch, what, times, fn):
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    r = fn()
    b.record()
    torch.cuda.synchronize()
    times.setdefault(what, []).append(a.elapsed_time(b))
    return r


def _reference(torch, q, k, v, start):
    """Attention of q [n, nq, HQ, D] over rows k, v [n, T, H, D] in 32 bits, causal from `start`."""
    n, nq, HQ, D = q.shape
    H, T = k.shape[2], k.shape[1]
    x = q.float().view(n, nq, H, HQ // H, D).permute(0, 2, 1, 3, 4).reshape(n, H, -1, D)
    s = torch.matmul(x, k.float().permute(0, 2, 3, 1).contiguous()) / math.sqrt(D)
    see = torch.arange(nq, device=q.device).repeat_interleave(HQ // H) + start
    s.masked_fill_(torch.arange(T, device=q.device) > see[:, None], -math.inf)
    o = torch.matmul(torch.softmax(s, -1), v.float().permute(0, 2, 1, 3).contiguous())
    return o.view(n, H, nq, HQ // H, D).permute(0, 2, 1, 3, 4).reshape(n, nq, HQ, D)


def run(w, kv_heads=8, q_heads=32, question=100, tokens=16, keep=0.25, picks=16, seed=0,
        device="cuda"):
    """Returns a dict of figures for workload `w` (its channels are kv_heads x head size)."""
    import torch
    from paper_2310_07240_amd import workloads as W
    from paper_2310_07240_amd.cachegen import Codec, CodecParams
    from paper_2310_07240_amd.kv8 import PAGE, Kv8Cache
    p = CodecParams.of(w)
    codec = Codec(p, device)
    times = {}
    H, D, T = kv_heads, p.n_channels // kv_heads, p.n_tokens
    n = p.n_ctx * p.n_layers                       # sequences: each layer of each context is one

    def rows(kv):
        """K and V of a codec cache as rows [n, T, H, D]: views, nothing is copied."""
        x = kv.view(torch.float16).view(n, 2, -1, H, D)
        return x[:, 0], x[:, 1]

    # the context comes back from its payload
    kv = torch.from_numpy(W.generate(w).view(np.int16)).to(device)
    levels = torch.from_numpy(w.chunk_levels()).to(device)
    ca, cd = codec.fit(kv)
    words, offsets, scales = codec.encode(kv, levels, ca, cd)
    payload = int(offsets[-1]) * 4
    kv = _timed(torch, "decode", times, lambda: codec.decode(words, offsets, scales, levels, ca, cd))

    # into pages of the serving cache, all layers in one call; room for the new tokens, and pages
    # of their own for what eviction keeps
    end = T + question + tokens
    kept_tokens = max(1, int(end * keep))
    width, new_width = -(-end // PAGE), -(-kept_tokens // PAGE)
    cache = Kv8Cache(n * (width + new_width), H, D, device)
    table = torch.arange(n * width, dtype=torch.int32, device=device).view(n, width)
    new_table = torch.arange(n * width, n * (width + new_width), dtype=torch.int32,
                             device=device).view(n, new_width)
    mass = torch.zeros((cache.n_pages, H, PAGE), dtype=torch.float32, device=device)
    lengths = torch.full((n,), T, dtype=torch.int32, device=device)
    k, v = rows(kv)
    _timed(torch, "store", times, lambda: cache.store(k, v, table, torch.zeros_like(lengths),
                                                      mass=mass))

    # the question, then token after token: new rows behind the old ones, attention with weights
    g = torch.Generator(device=device).manual_seed(seed)

    def new_rows(count, heads, scale=1.0):
        x = torch.randn((n, count, heads, D), generator=g, device=device) * scale
        return x.half()

    at = T
    error = 0.0
    for step, count in enumerate([question] + [1] * tokens):
        kn, vn, q = new_rows(count, H), new_rows(count, H), new_rows(count, q_heads, 0.5)
        what = "question" if step == 0 else "token"
        starts = lengths.clone()
        lengths += count

        def one():
            cache.store(kn, vn, table, starts, mass=mass)
            return cache.attend(q, table, lengths, max_len=at + count, mass=mass, decay=0.98)
        out = _timed(torch, what, times, one)
        if step == 0:
            l = n - 1                              # compared on one layer, which is enough to see
            ref = _reference(torch, q[l:], torch.cat([k[l:], kn[l:]], 1),
                             torch.cat([v[l:], vn[l:]], 1), T)
            error = float((out[l:].float() - ref).norm() / ref.norm())
        at += count

    # the last token once more over the pages that its bounds pick
    picked = _timed(torch, "select", times, lambda: cache.select(q, table, lengths, picks,
                                                                 max_len=at))
    sparse = _timed(torch, "sparse", times, lambda: cache.attend(q, table, lengths, max_len=at,
                                                                 picks=picked))
    near = float((sparse.float() - out.float()).norm() / out.float().norm())

    # what attention passed by goes, the rest is a codec cache again
    kept, lengths = _timed(torch, "evict", times, lambda: cache.evict(
        table, lengths, mass, kept_tokens, min(kept_tokens, question + tokens), new_table,
        max_len=at))
    small = torch.empty((p.n_ctx, p.n_layers, 2, kept_tokens, p.n_channels), dtype=torch.int16,
                        device=device)
    k2, v2 = rows(small)
    _timed(torch, "load", times, lambda: cache.load(new_table, torch.zeros_like(lengths),
                                                    kept_tokens, k=k2, v=v2))
    again = Codec(CodecParams(p.n_ctx, p.n_layers, kept_tokens, p.n_channels, p.layer_bin,
                              p.level_mult, p.group_size, p.chunk_len), device)
    level0 = torch.zeros((p.n_ctx, again.n_chunks), dtype=torch.uint8, device=device)
    ca, cd = again.fit(small)
    small_payload = int(again.encode(small, level0, ca, cd)[1][-1]) * 4
    elements = 2 * n * at * H * D
    return {
        "workload": w.name, "sequences": n, "tokens": at, "kept": kept_tokens,
        "ms": {name: round(sorted(t)[len(t) // 2], 4) for name, t in times.items()},
        "bytes": {"fp16": 2 * elements, "payload": payload,
                  "pages": n * width * H * (2 * PAGE * D + 8 + 2 * D),
                  "payload_kept": small_payload},
        "rel_error_8bit": error, "rel_error_sparse": near,
        "kept_of_context": float((kept < T).float().mean()),
    }


def answer(w, kv_heads=8, q_heads=32, requests=8, drafts=4, steps=8, vocab=32000, seed=0,
           spare=None, device="cuda"):
    """`requests` answers over every context of workload `w` at once, each `steps` times `drafts`
    drafted tokens (one at least); returns a dict of figures. `spare`: pages behind the contexts' own,
    for the answers (default: enough); a step that finds too few changes nothing."""
    import torch
    from paper_2310_07240_amd import workloads as W
    from paper_2310_07240_amd.cachegen import Codec, CodecParams
    from paper_2310_07240_amd.kv8 import PAGE, Kv8Cache
    p = CodecParams.of(w)
    codec = Codec(p, device)
    times = {}
    H, D, T = kv_heads, p.n_channels // kv_heads, p.n_tokens
    n, R = p.n_ctx * p.n_layers, requests          # contexts: each layer of each is one
    kv = torch.from_numpy(W.generate(w).view(np.int16)).to(device)
    levels = torch.from_numpy(w.chunk_levels()).to(device)
    ca, cd = codec.fit(kv)
    words, offsets, scales = codec.encode(kv, levels, ca, cd)
    kv = codec.decode(words, offsets, scales, levels, ca, cd)
    x = kv.view(torch.float16).view(n, 2, T, H, D)

    def ints(*shape, value=0):
        return torch.full(shape, value, dtype=torch.int32, device=device)

    # The contexts' pages. Whole ones are shared by all requests; the last, if the context ends in
    # it, starts every request's own tokens and is copied when the request writes behind it.
    whole, tail = T // PAGE, T % PAGE
    q = drafts + 1                                 # the last token and the drafts behind it
    own = -(-(tail + q * steps) // PAGE)
    cache = Kv8Cache(n * -(-T // PAGE) + (n * R * own if spare is None else spare), H, D, device)
    refs = ints(cache.n_pages)
    table = ints(n, whole + own, value=-1)
    start, held = ints(n), ints(n, value=T)
    missing = cache.reserve(table, start, held, refs)      # (there are as many)
    cache.store(x[:, 0], x[:, 1], table, start)
    shared, tails = table[:, :max(1, whole)].contiguous(), table[:, whole:].contiguous()
    shared_len, firsts = ints(n, value=whole * PAGE), torch.arange(
        0, n * R + 1, R, dtype=torch.int32, device=device)
    parents = torch.arange(n, dtype=torch.int32, device=device).repeat_interleave(R)
    rows, lengths = _timed(torch, "fork", times, lambda: cache.fork(
        tails, ints(n, value=tail), parents, refs))

    g = torch.Generator(device=device).manual_seed(seed)

    def random(*shape):
        return torch.randn(shape, generator=g, device=device)

    error, taken, short = 0.0, [], missing.clone()
    counts, granted = ints(n * R, value=q), ints(n * R)
    for step in range(steps):
        kn, vn, qn = random(n * R, q, H, D).half(), random(n * R, q, H, D).half(), (
            0.5 * random(n * R, q, q_heads, D)).half()
        logits = 2.5 * random(p.n_ctx * R, q, vocab)
        target = torch.softmax(logits, -1)
        draft = torch.softmax(logits[:, :drafts] + 0.6 * random(p.n_ctx * R, drafts, vocab), -1)
        tokens = torch.multinomial(draft.view(-1, vocab), 1, generator=g).view(-1, drafts).int()
        u = torch.rand((p.n_ctx * R, q), generator=g, device=device)
        starts = lengths

        def one():
            # (without pages nothing is stored, and no query is asked)
            cache.reserve(rows, starts, counts, refs, missing=missing, granted=granted)
            cache.store(kn, vn, rows, starts, counts=granted)
            return cache.attend_shared(qn, shared, shared_len, firsts, table=rows,
                                       lengths=starts + granted, q_lens=granted,
                                       max_shared=whole * PAGE, max_len=tail + q * (step + 1),
                                       max_users=R)
        out = _timed(torch, "step", times, one)
        if step == 0:                              # compared on the last request
            ref = _reference(torch, qn[-1:], torch.cat([x[-1:, 0], kn[-1:]], 1),
                             torch.cat([x[-1:, 1], vn[-1:]], 1), T)
            error = float((out[-1:].float() - ref).norm() / ref.norm())
        short = torch.maximum(short, missing)
        # a request's layers go on together (all get pages, or none): verified once, cut back alike
        there = granted.view(p.n_ctx, p.n_layers, R)[:, 0].reshape(-1)
        _, accepted = _timed(torch, "verify", times, lambda: cache.verify(target, tokens, u,
                                                                          draft=draft,
                                                                          counts=there - 1))
        taken.append(accepted)
        kept = torch.where(there > 0, accepted + 1, 0)
        lengths = starts + kept.view(p.n_ctx, 1, R).expand(-1, p.n_layers, -1).reshape(-1)
        _timed(torch, "release", times, lambda: cache.release(rows, refs, keep=lengths))
    used = int((refs > 0).sum())
    most = int(lengths.max())
    # the requests end; what is left are the contexts, moved to the pool's front
    cache.release(rows, refs)
    table, refs, _, live = _timed(torch, "compact", times, lambda: cache.compact(table, refs))
    k, _ = cache.load(table, start, T)
    loaded = float((k.float() - x[:, 0].float()).norm() / x[:, 0].float().norm())
    return {
        "workload": w.name, "contexts": n, "requests": n * R, "tokens": T,
        "ms": {name: round(sorted(t)[len(t) // 2], 4) for name, t in times.items()},
        "accepted": float(torch.stack(taken).float().mean()), "missing": int(short),
        "pages": {"used": used, "unshared": n * R * (whole + -(-most // PAGE)),
                  "after": int(live), "contexts": n * -(-T // PAGE)},
        "rel_error_8bit": error, "rel_error_after": loaded,
    }


def main(argv=None):
    from paper_2310_07240_amd import workloads as W
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--workload", default="mistral7b_gqa_t4096", choices=sorted(W.WORKLOADS))
    ap.add_argument("--heads", type=int, default=8, help="KV heads of the workload's channels")
    ap.add_argument("--q-heads", type=int, default=32)
    ap.add_argument("--question", type=int, default=100)
    ap.add_argument("--tokens", type=int, default=16)
    ap.add_argument("--keep", type=float, default=0.25)
    ap.add_argument("--picks", type=int, default=16)
    ap.add_argument("--requests", type=int, default=0, help="answers over each context")
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--vocab", type=int, default=32000)
    a = ap.parse_args(argv)
    w = W.WORKLOADS[a.workload]
    for _ in range(2):                             # the first pass loads the kernels
        if a.requests:
            r = answer(w, a.heads, a.q_heads, a.requests, a.drafts, a.steps, a.vocab)
            continue
        r = run(w, a.heads, a.q_heads, a.question, a.tokens, a.keep, a.picks)
    print(json.dumps(r), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
