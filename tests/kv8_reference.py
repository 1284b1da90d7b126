"""The 8-bit serving cache in numpy, from its definition: codes with their 32-bit quotients,
attention, weights and scores in 64 bits. One page, head or row at a time, no shared code with the
HIP path."""
import numpy as np

PAGE = 64
f32 = np.float32


def codes_of(x, s):
    """rint(clamp(fp32(x / s))) of fp32 values."""
    if s == 0:
        return np.zeros(x.shape, np.int8)
    with np.errstate(invalid="ignore", over="ignore"):
        q = (x.astype(f32) / f32(s)).astype(f32)
    q = np.where(np.isnan(q), f32(0), q)
    return np.rint(np.clip(q, -127, 127)).astype(np.int8)


def scale_of(x):
    a = np.abs(x[np.isfinite(x)])
    return f32(f32(a.max() if a.size else 0.0) / f32(127.0))


class Ref:
    """Host copies of a cache's buffers, K and V both [P][H][64][D]."""

    def __init__(self, cache):
        self.k = cache.k_codes.cpu().numpy().copy()
        self.v = cache.v_codes.cpu().numpy().transpose(0, 1, 3, 2).copy()
        self.ks = cache.k_scale.cpu().numpy().copy()
        self.vs = cache.v_scale.cpu().numpy().copy()
        self.bounds = None if cache.k_bounds is None else cache.k_bounds.cpu().numpy().copy()
        self.P, self.H, _, self.D = self.k.shape

    def page(self, table, b, j):
        if j >= table.shape[1]:
            return -1
        p = int(table[b, j])
        return p if 0 <= p < self.P else -1

    def put_page(self, page, h, k, v, held):
        """Rows k, v [n, D] (fp32) behind `held` tokens of the page."""
        end = held + len(k)
        for codes, scales, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
            s_old = scales[page, h] if held else f32(0)
            s = max(scale_of(x), s_old)
            was = codes[page, h, :held].copy()
            if held and s != s_old:
                was = codes_of((was.astype(f32) * s_old).astype(f32), s)
            codes[page, h] = 0
            codes[page, h, :held] = was
            codes[page, h, held:end] = codes_of(x, s)
            scales[page, h] = s
        if self.bounds is not None:
            self.bounds[page, h, 0] = self.k[page, h, :end].min(0)
            self.bounds[page, h, 1] = self.k[page, h, :end].max(0)

    def store(self, k, v, table, starts, counts):
        """k, v [n, T, H, D] as fp32 arrays."""
        for b in range(len(starts)):
            a, n = int(starts[b]), int(counts[b])
            if a < 0 or n <= 0:
                continue
            for j in range(a // PAGE, (a + n + PAGE - 1) // PAGE):
                page = self.page(table, b, j)
                if page < 0:
                    continue
                lo, hi = max(a, j * PAGE), min(a + n, (j + 1) * PAGE)
                for h in range(self.H):
                    self.put_page(page, h, k[b, lo - a:hi - a, h], v[b, lo - a:hi - a, h],
                                  lo - j * PAGE)

    def rows(self, table, b, h, n, columns=None):
        """(K, V, position, present) of the sequence's tokens in 64 bits."""
        cols = range((n + PAGE - 1) // PAGE) if columns is None else columns
        k, v, pos, there = [], [], [], []
        for j in cols:
            page = self.page(table, b, j)
            m = min(PAGE, n - j * PAGE)
            there += [page >= 0] * m
            pos += range(j * PAGE, j * PAGE + m)
            k.append(self.k[page, h, :m].astype(np.float64) * float(self.ks[page, h]))
            v.append(self.v[page, h, :m].astype(np.float64) * float(self.vs[page, h]))
        z = np.zeros((0, self.D))
        return (np.concatenate(k) if k else z, np.concatenate(v) if v else z,
                np.array(pos, np.int64), np.array(there, bool))


def visible(n, q_len, i):
    return max(0, n - q_len + i + 1) if i < q_len else 0


def attend(ref, q, table, lengths, q_lens, scale, picks=None):
    """(out, lse, mass [P, H, 64], size, spread): `size` is sum p |v| per output value and
    `spread` the largest sum |q k| * |scale| of a row, which the error bounds go by."""
    B, Q, HQ, D = q.shape
    G = HQ // ref.H
    out = np.zeros(q.shape)
    size = np.zeros(q.shape)
    lse = np.full((B, Q, HQ), -np.inf)
    spread = np.zeros((B, Q, HQ))
    mass = np.zeros((ref.P, ref.H, PAGE))
    for b in range(B):
        n = max(0, min(int(lengths[b]), table.shape[1] * PAGE))
        for i in range(Q):
            see = visible(n, int(q_lens[b]), i)
            if not see:
                continue
            for h in range(ref.H):
                cols = None
                if picks is not None:
                    cols = [int(j) for j in picks[b, i, h] if 0 <= j and j * PAGE < see]
                k, v, pos, there = ref.rows(table, b, h, see, cols)
                if not there.any():
                    continue
                for g in range(h * G, h * G + G):
                    x = q[b, i, g].astype(np.float64)
                    z = np.where(there, (k @ x) * scale, -np.inf)
                    m = z.max()
                    p = np.exp(z - m)
                    l = p.sum()
                    p /= l
                    out[b, i, g] = p @ v
                    size[b, i, g] = p @ np.abs(v)
                    lse[b, i, g] = m + np.log(l)
                    spread[b, i, g] = (np.abs(k) @ np.abs(x)).max() * abs(scale)
                    for t in np.nonzero(there)[0]:
                        page = ref.page(table, b, int(pos[t]) // PAGE)
                        mass[page, h, int(pos[t]) % PAGE] += p[t]
    return out, lse, mass, size, spread


def select(ref, q, table, lengths, q_lens, n_picks, recent):
    B, Q, HQ, D = q.shape
    G = HQ // ref.H
    picks = np.full((B, Q, ref.H, n_picks), -1, np.int32)
    for b in range(B):
        n = max(0, min(int(lengths[b]), table.shape[1] * PAGE))
        for i in range(Q):
            see = visible(n, int(q_lens[b]), i)
            pages = (see + PAGE - 1) // PAGE
            for h in range(ref.H):
                x = q[b, i, h * G:(h + 1) * G].astype(np.float64)
                top = np.abs(x).max()
                e = np.frexp(top)[1] - 1 if top > 0 else 0
                q8 = np.rint(np.clip(np.ldexp(x, 6 - e), -127, 127))
                score = []
                for j in range(pages):
                    page = ref.page(table, b, j)
                    if page < 0:
                        score.append(-np.inf)
                        continue
                    lo, hi = ref.bounds[page, h].astype(np.float64)
                    w = int(np.maximum(q8 * lo, q8 * hi).sum())
                    score.append(float(f32(f32(w) * ref.ks[page, h])))
                last = min(recent, n_picks, pages)
                old = pages - last
                best = sorted(range(old), key=lambda j: (-score[j], j))[:n_picks - last]
                best = sorted(best + list(range(old, pages)))
                picks[b, i, h, :len(best)] = best
    return picks


def kept_tokens(weights, n, keep, recent):
    """Ascending places that stay, of the first n weights."""
    if n <= keep:
        return list(range(n))
    last = min(recent, keep)
    old = n - last
    w = [(-np.inf if np.isnan(x) else x) for x in weights[:old]]
    nan = [bool(np.isnan(x)) for x in weights[:old]]
    best = sorted(range(old), key=lambda j: (nan[j], -w[j], j))[:keep - last]
    return sorted(best) + list(range(old, n))


def evict(ref, table, lengths, mass, keep, recent, to):
    """Moves the kept tokens within `ref` and `mass` (both changed); (kept, lengths)."""
    B = table.shape[0]
    kept = np.full((B, ref.H, keep), -1, np.int32)
    new = np.zeros(B, np.int32)
    for b in range(B):
        n = max(0, min(int(lengths[b]), table.shape[1] * PAGE))
        new[b] = min(n, keep)
        for h in range(ref.H):
            w = [mass[ref.page(table, b, t // PAGE), h, t % PAGE] for t in range(n)]
            at = kept_tokens(w, n, keep, recent)
            kept[b, h, :len(at)] = at
            for j in range((len(at) + PAGE - 1) // PAGE):
                some = at[j * PAGE:(j + 1) * PAGE]
                src = [(ref.page(table, b, t // PAGE), t % PAGE) for t in some]
                k = np.stack([ref.k[p, h, s].astype(f32) * ref.ks[p, h] for p, s in src])
                v = np.stack([ref.v[p, h, s].astype(f32) * ref.vs[p, h] for p, s in src])
                page = ref.page(to, b, j)
                ref.put_page(page, h, k.astype(f32), v.astype(f32), 0)
                mass[page, h] = 0
                mass[page, h, :len(some)] = [w[t] for t in some]
    return kept, new
