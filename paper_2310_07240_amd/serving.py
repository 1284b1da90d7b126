"""A context's life behind the codec on one GPU: it comes back from its bitstreams (``Codec``), goes
into the 8-bit serving cache (``Kv8Cache``) with every layer at once, a question and then single
tokens attend over it, the tokens that attention passed by are evicted, and what is left goes back
to the codec (the paper measures CacheGen on top of token dropping in Sec. 7.2).

Each step is timed on the GPU (HIP events); the attention of the question is compared with the same
attention over the decoded fp16 cache, in 32 bits. Queries and new tokens are random: no model is
involved.

Usage: python -m paper_2310_07240_amd.serving [--workload NAME] [--heads H] [--q-heads H]
       [--question N] [--tokens N] [--keep F] [--picks N]     (one JSON line)
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
    a = ap.parse_args(argv)
    w = W.WORKLOADS[a.workload]
    for _ in range(2):                             # the first pass loads the kernels
        r = run(w, a.heads, a.q_heads, a.question, a.tokens, a.keep, a.picks)
    print(json.dumps(r), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
