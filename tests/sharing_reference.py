"""Requests that share a context of the 8-bit cache, from the definitions, in Python lists and numpy:
who holds which page, attention over a context and a request's own tokens in 64 bits, drafted tokens
accepted by whole numbers. No shared code with the HIP path."""
import math
from fractions import Fraction

import numpy as np

PAGE = 64


def pages_of(n):
    return -(-n // PAGE)


def clip(n, width):
    return max(0, min(int(n), width * PAGE))


def fork(table, lengths, parents, refs, n_pages, width, ends=None):
    """(new_table, new_lengths, refs) as lists; `table` is a list of rows."""
    refs, rows, new = list(refs), [], []
    for i, p in enumerate(parents):
        row, n = [-1] * width, 0
        if 0 <= p < len(table):
            n = clip(lengths[p], len(table[0]))
            if ends is not None:
                n = max(0, min(n, ends[i]))
            for j in range(pages_of(n)):
                page = table[p][j]
                if 0 <= page < n_pages:
                    row[j] = page
                    refs[page] += 1
        rows.append(row)
        new.append(n)
    return rows, new, refs


def release(table, refs, n_pages, keep=None):
    refs, rows = list(refs), []
    for i, row in enumerate(table):
        row = list(row)
        for j, page in enumerate(row):
            if keep is not None and j * PAGE < keep[i]:
                continue
            if 0 <= page < n_pages and refs[page] > 0:
                refs[page] -= 1
            row[j] = -1
        rows.append(row)
    return rows, refs


def reserve(table, lengths, counts, refs, n_pages):
    """(table, refs, missing, copies [(from, to)])"""
    rows, width = [list(r) for r in table], len(table[0])
    free = [i for i, r in enumerate(refs) if r <= 0]
    wanted = []
    for b, row in enumerate(rows):
        a = clip(lengths[b], width)
        end = clip(a + max(0, int(counts[b])), width)
        for j in range(a // PAGE, pages_of(end) if end > a else 0):
            held = refs[row[j]] if 0 <= row[j] < n_pages else 0
            keeps = j * PAGE < a
            if held > 1 if keeps else held != 1:
                wanted.append((b, j, keeps, held > 1))
    if len(wanted) > len(free):
        return rows, list(refs), len(wanted) - len(free), []
    after, copies = list(refs), []
    for (b, j, keeps, shared), page in zip(wanted, free):
        if shared:
            after[rows[b][j]] = max(0, after[rows[b][j]] - 1)
        if keeps:
            copies.append((rows[b][j], page))
        rows[b][j] = page
    for _, page in zip(wanted, free):
        after[page] = 1
    return rows, after, 0, copies


def compact(table, refs, n_pages):
    """(table, refs, moved, live, copies)"""
    live = sum(r > 0 for r in refs)
    holes = [i for i in range(live) if refs[i] <= 0]
    late = [i for i in range(live, n_pages) if refs[i] > 0]
    moved = [i if r > 0 else -1 for i, r in enumerate(refs)]
    after = [max(0, r) if i < live else 0 for i, r in enumerate(refs)]
    for a, b in zip(late, holes):
        moved[a], after[b] = b, refs[a]
    rows = [[moved[p] if 0 <= p < n_pages else -1 for p in row] for row in table]
    return rows, after, moved, live, list(zip(late, holes))


def attend(ref, q, shared, shared_lengths, firsts, max_users, table, lengths, q_lens, scale):
    """(out, lse, size, spread) as kv8_reference.attend; table None: the contexts alone."""
    n, Q, HQ, D = q.shape
    G = HQ // ref.H
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    lse, spread = np.full((n, Q, HQ), -np.inf), np.zeros((n, Q, HQ))
    of = {}
    for p in range(len(firsts) - 1):
        a, b = max(0, firsts[p]), min(n, firsts[p + 1])
        of.update({s: p for s in range(a, min(b, a + max_users))})
    for s in range(n):
        own = 0 if table is None else clip(lengths[s], table.shape[1])
        for h in range(ref.H):
            k0, v0, there0 = np.zeros((0, D)), np.zeros((0, D)), np.zeros(0, bool)
            if s in of:
                p = of[s]
                k0, v0, _, there0 = ref.rows(shared, p, h, clip(shared_lengths[p], shared.shape[1]))
            for i in range(min(Q, q_lens[s])):
                k, v, there = k0, v0, there0
                see = max(0, own - q_lens[s] + i + 1)
                if see:
                    k1, v1, _, there1 = ref.rows(table, s, h, see)
                    k, v = np.concatenate([k, k1]), np.concatenate([v, v1])
                    there = np.concatenate([there, there1])
                if not there.any():
                    continue
                for g in range(h * G, h * G + G):
                    x = q[s, i, g].astype(np.float64)
                    z = np.where(there, (k @ x) * scale, -np.inf)
                    m = z.max()
                    e = np.exp(z - m)
                    w = e / e.sum()
                    out[s, i, g], size[s, i, g] = w @ v, w @ np.abs(v)
                    lse[s, i, g] = m + np.log(e.sum())
                    spread[s, i, g] = (np.abs(k) @ np.abs(x)).max() * abs(scale)
    return out, lse, size, spread


def counted(x):
    x = float(x)
    return 0.0 if math.isnan(x) or x <= 0 else min(x, 1.0)


def verify(target, drafts, u, draft=None, counts=None, lengths=None):
    """(tokens, accepted, new_lengths) of float64 arrays, decided in fractions."""
    n, k, vocab = target.shape[0], target.shape[1] - 1, target.shape[2]
    tokens, accepted = np.full((n, k + 1), -1, np.int32), np.zeros(n, np.int32)
    new = None if lengths is None else np.maximum(0, np.asarray(lengths, np.int64))
    for b in range(n):
        count = k if counts is None else min(k, int(counts[b]))
        if count < 0:
            continue
        took = 0
        while took < count:
            x = int(drafts[b, took])
            if not 0 <= x < vocab or not u[b, took] < math.inf:
                break
            q = 1.0 if draft is None else counted(draft[b, took, x])
            if not Fraction(float(u[b, took])) * Fraction(q) < Fraction(
                    counted(target[b, took, x])):
                break
            took += 1

        def weights(row):
            with np.errstate(invalid="ignore"):
                row = np.where(row > 0, np.minimum(row, 1.0), 0.0)
            return np.rint(np.ldexp(row, 42)).astype(np.int64)
        have = weights(target[b, took])
        if took < count:
            over = have.copy()
            if draft is not None:
                over = np.maximum(have - weights(draft[b, took]), 0)
            elif 0 <= drafts[b, took] < vocab:
                over[drafts[b, took]] = 0
            have = over if over.any() else have
        total = int(have.sum())
        part = float(u[b, k])
        part = 0 if math.isnan(part) or part <= 0 else min(math.floor(min(part, 2.0) * 2 ** 24),
                                                           2 ** 24 - 1)
        tokens[b, :took] = drafts[b, :took]
        if total:
            bar = part * total >> 24
            tokens[b, took] = int(np.searchsorted(np.cumsum(have), bar, side="right"))
        accepted[b] = took
        if new is not None:
            new[b] = max(0, int(lengths[b]) - (count - took))
    return tokens, accepted, new
