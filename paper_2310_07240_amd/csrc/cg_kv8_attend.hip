// cg_kv8_attend.hip — attention over the pages of the 8-bit cache (cg_kv8_attend).
//
// For each (sequence, KV head) the queries of its group are the rows of two matrix products,
// S = q K^T and O = P V, with the softmax carried along: running maximum m, running sum l, and O
// under the reference m, all in 32 bits. The codes go into the matrix units as fp16 (exact), the
// scales of the page are applied to S and to the page's share of O in 32 bits, and P is rounded
// to fp16 for the second product, the rounding that the fp16 result gets anyway (attend_kernel:
// relative 2^-11 of a weight down to 2^-29 of the page's largest; prompt_kernel, whose reference is
// the row's: down to 2^-25 of the heaviest; l sums the unrounded weights).
//
// Operand layout (v_mfma_f32_16x16x32_f16; lane = 16 g + m): both products are taken transposed,
// S^T = K q^T and O^T = V^T P^T, so a lane's results belong to one query row (m) throughout and
// the softmax needs only the four lanes of equal m. The order of the contracted index is free as
// long as both operands agree: row m of K tile t is token 16 (m >> 2) + 4 t + (m & 3), which makes
// the 16 tokens whose S a lane gets the consecutive 16 g .. 16 g + 15, exactly the k slots that it
// supplies for the second product, and the V operand 16 consecutive bytes of a channel.
#include <math.h>

#include <type_traits>

#include "cg_kv8.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ float quad_max(float x) {   // over the lanes of equal m
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// N sums over N neighbouring lanes at once: afterwards lane i of the N holds the sum of v[i].
template <int N, int LEN>
__device__ __forceinline__ float sum_across(float (&v)[LEN]) {
  if constexpr (N > 1) {
    const bool upper = threadIdx.x & (N / 2);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float mine = upper ? v[i + N / 2] : v[i], other = upper ? v[i] : v[i + N / 2];
      v[i] = mine + __shfl_xor(other, N / 2);
    }
    return sum_across<N / 2>(v);
  } else {
    return v[0];
  }
}

// Eight row elements; `wide`: rows lie on 16-byte boundaries.
__device__ __forceinline__ uint4v load8(const uint16_t* p, bool wide) {
  if (wide) return *reinterpret_cast<const uint4v*>(p);
  uint16_t u[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) u[c] = p[c];
  return *reinterpret_cast<uint4v*>(u);
}

// One 16-row tile's queries as B operands, and what a row needs of them.
template <int D>
struct QTile {
  half8 q[D / 32];
  float unit;        // times the page's K scale: S in units of log2
  int visible;       // tokens that the lane's row sees
};

// A value that is the same in every lane, in a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Where the rows of a (virtual) sequence come from. With picks every query token is a sequence
// of its own, whose rows are the heads of the group.
struct RowsOf {
  int seq, i0, nq;   // sequence, first query token, query tokens
  int len, q_len;

  // Tokens that query token i sees: those up to its own place, the last q_len tokens being the
  // queries' own.
  __device__ __forceinline__ int visible(int i) const {
    if (i >= q_len) return 0;
    const int64_t n = (int64_t)len - q_len + i + 1;
    return n > 0 ? (int)n : 0;
  }
  // Tokens that any of the query tokens first .. last sees.
  __device__ __forceinline__ int most(int first, int last) const {
    return q_len > 0 ? visible(last < q_len ? last : q_len - 1) : 0;
  }
  __device__ __forceinline__ int64_t at(const KvRows& r, int i) const {
    return seq * r.seq + (int64_t)i * r.tok;
  }
  // Index of query token i among all sequences' (of A.nq each), and whether it is one.
  __device__ __forceinline__ int64_t token(int nq_all, int i) const {
    return (int64_t)seq * nq_all + i;
  }
  __device__ __forceinline__ bool exists(int) const { return true; }
};

__device__ __forceinline__ RowsOf rows_of(const KvSeqs& S, const KvAttn& A, int vseq) {
  RowsOf r;
  const bool sparse = A.picks != nullptr;
  r.seq = sparse ? vseq / A.nq : vseq;
  r.i0 = sparse ? vseq % A.nq : 0;
  r.nq = sparse ? 1 : A.nq;
  int len = A.lengths[r.seq];
  const int64_t room = (int64_t)S.width * kPage;
  if (len > A.max_len) len = A.max_len;
  if (len > room) len = (int)room;
  r.len = len > 0 ? len : 0;
  const int ql = A.q_lens ? A.q_lens[r.seq] : A.nq;
  r.q_len = ql < A.nq ? ql : A.nq;
  return r;
}

// The requests of a shared context, as one sequence whose query tokens are theirs one after the
// other: token i is token i % per of request first + i / per. All of them see the whole context.
struct SharedRows {
  int seq;           // the context, whose pages are read
  int nq, i0;        // query tokens that there is room for; 0
  int len, q_len;    // the context's tokens; query tokens of the requests that there are
  int first, per;
  const int32_t* q_lens;

  __device__ __forceinline__ int visible(int i) const {
    if (i >= q_len) return 0;
    return !q_lens || i % per < q_lens[first + i / per] ? len : 0;
  }
  __device__ __forceinline__ int most(int from, int) const { return from < q_len ? len : 0; }
  __device__ __forceinline__ int64_t at(const KvRows& r, int i) const {
    return (int64_t)(first + i / per) * r.seq + (int64_t)(i % per) * r.tok;
  }
  __device__ __forceinline__ int64_t token(int, int i) const {
    return (int64_t)first * per + i;
  }
  __device__ __forceinline__ bool exists(int i) const { return i < q_len; }
};

// Requests first .. first + count - 1 read context p: what `firsts` says, cut to the requests that
// exist and to the bound of them.
struct Requests {
  int first, count;
};

__device__ __forceinline__ Requests requests_of(const KvUsers& U, int p) {
  int a = U.firsts[p], b = U.firsts[p + 1];
  a = a < 0 ? 0 : a < U.n_seq ? a : U.n_seq;
  b = b < a ? a : b < U.n_seq ? b : U.n_seq;
  return Requests{a, b - a < U.most ? b - a : U.most};
}

__device__ __forceinline__ SharedRows rows_of(const KvSeqs& S, const KvAttn& A, const KvUsers& U,
                                              int p) {
  SharedRows r;
  const Requests q = requests_of(U, p);
  r.seq = p;
  r.i0 = 0;
  r.nq = A.nq;
  r.per = U.per;
  r.first = q.first;
  r.q_len = q.count * U.per;
  r.q_lens = A.q_lens;
  int len = A.lengths[p];
  const int64_t room = (int64_t)S.width * kPage;
  if (len > A.max_len) len = A.max_len;
  if (len > room) len = (int)room;
  r.len = len > 0 ? len : 0;
  return r;
}

// Where a context's tiles start (see KvTiles); `first`: its first request.
__device__ __forceinline__ int tiles_before(const KvTiles& T, const KvUsers& U, int p, int first) {
  // (all rows of a head are below 2^30)
  return T.each ? p * T.each : p + ((first * U.rows) >> __builtin_ctz(T.size));
}

// The context that tile t is of, or -1, and which of its tiles (below 0 if firsts is in no order).
// A wave looks at 64 contexts at once.
__device__ __forceinline__ int context_at(const KvTiles& T, const KvUsers& U, int t, int& tile) {
  int p;
  if (T.each) {
    p = t / T.each;
    tile = t - p * T.each;
    return p;
  }
  int lo = 0, hi = U.contexts;                         // contexts from lo on may start behind t
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64;
    const int64_t at = lo + (int64_t)(threadIdx.x & 63) * step;
    bool before = false;
    if (at < hi) before = tiles_before(T, U, (int)at, requests_of(U, (int)at).first) <= t;
    const int c = __popcll(__ballot(before));
    if (c == 0) break;
    const int64_t end = lo + (int64_t)c * step;
    lo += (c - 1) * step + 1;
    hi = end < hi ? (int)end : hi;
  }
  p = uniform(lo - 1);
  tile = p < 0 ? 0 : t - tiles_before(T, U, p, uniform(requests_of(U, p).first));
  return p;
}

// The same of either kind.
template <class Rows>
__device__ __forceinline__ Rows rows_in(const KvSeqs& S, const KvAttn& A, const KvUsers& U, int i) {
  if constexpr (__is_same(Rows, SharedRows)) return rows_of(S, A, U, i);
  else return rows_of(S, A, i);
}

// Rows 16 tile .. 16 tile + 15 of the group's queries; rows past the last one see nothing.
// bf16 rows are scaled by a power of two to [1, 2) at their largest, so that fp16 holds them to
// 2^-25 of it; fp16 rows go as they are.
template <int D, bool BF16, class Rows>
__device__ __forceinline__ void load_q(const KvAttn& A, const Rows& R, int h, int tile,
                                       QTile<D>& Q) {
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int row = tile * 16 + m;
  const int i = R.i0 + row / A.group, head = h * A.group + row % A.group;
  // (there is room for more requests of a context than it has: those have no queries to read)
  const bool live = row < R.nq * A.group && R.exists(i);
  Q.visible = live ? R.visible(i) : 0;
  const uint16_t* src = static_cast<const uint16_t*>(A.q.p) + R.at(A.q, i) +
                        (int64_t)head * A.q.head;
  uint16_t u[D / 32][8];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) *reinterpret_cast<uint4v*>(u[s]) = uint4v{0, 0, 0, 0};
  if (live && A.wide_q) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      *reinterpret_cast<uint4v*>(u[s]) =
          *reinterpret_cast<const uint4v*>(src + (s >> 1) * 64 + g * 16 + (s & 1) * 8);
  } else if (live) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      *reinterpret_cast<uint4v*>(u[s]) = load8(src + (s >> 1) * 64 + g * 16 + (s & 1) * 8, false);
  }
  int e = 0;
  if (BF16) {
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t a = u[s][c] & 0x7fffu;
        top = a > top && a < 0x7f80u ? a : top;
      }
    uint32_t o = __shfl_xor(top, 16);
    top = o > top ? o : top;
    o = __shfl_xor(top, 32);
    top = o > top ? o : top;
    e = (int)(top >> 7) - 127;
    if (e < -126) e = -126;
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
      for (int c = 0; c < 8; ++c)
        Q.q[s][c] = (_Float16)__builtin_ldexpf(kv_widen<true>(u[s][c]), -e);
  } else {
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
      for (int c = 0; c < 8; ++c) Q.q[s][c] = __builtin_bit_cast(_Float16, u[s][c]);
  }
  Q.unit = __builtin_ldexpf(A.scale * kLog2e, e);
}

// The page's K codes as the lane's operands: piece s of row 16 (m >> 2) + 4 t + (m & 3).
template <int D>
struct KRegs {
  uint4v c[4][D / 64];
};
template <int D>
struct VRegs {
  uint4v c[D / 16];
};

template <int D>
__device__ __forceinline__ void load_k(const int8_t* k, KRegs<D>& K) {
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int8_t* row = k + (16 * (m >> 2) + (m & 3)) * D + 16 * g;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int s = 0; s < D / 64; ++s)
      K.c[t][s] = *reinterpret_cast<const uint4v*>(row + 4 * t * D + 64 * s);
}

template <int D>
__device__ __forceinline__ void load_v(const int8_t* v, VRegs<D>& V) {
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt)
    V.c[dt] = *reinterpret_cast<const uint4v*>(v + (16 * dt + m) * kPage + 16 * g);
}

// S^T of one page: x[4 t + i] is token 16 g + 4 t + i against the lane's row, unscaled.
template <int D>
__device__ __forceinline__ void page_scores(const KRegs<D>& K, const QTile<D>& Q, float x[16]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    float4v acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < D / 64; ++s) {
      const uint4v c = K.c[t][s];
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_widen8(c[0], c[1]), Q.q[2 * s], acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_widen8(c[2], c[3]), Q.q[2 * s + 1], acc, 0, 0,
                                                   0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[4 * t + i] = acc[i];
  }
}

// A wave's state for one 16-row tile: O^T (row m of the lane, channels 16 dt + 4 g + i), m and l.
template <int D>
struct Acc {
  float4v o[D / 16];
  float m, l;
};

// The softmax of one page's scores (left at `kept`, if given, as the lane's row has them): P as
// operands in p, m and l moved on; `keep` brings O to the new reference, the return value (times
// the V scale) the page's share.
template <int D>
__device__ __forceinline__ float page_softmax(float x[16], float ks, int pos0, const QTile<D>& Q,
                                              Acc<D>& S, half8 p[2], float& keep, float* kept) {
  const int g = (threadIdx.x & 63) >> 4;
  const float f = Q.unit * ks;
  float top = kNegInf;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    x[j] = pos0 + 16 * g + j < Q.visible ? x[j] * f : kNegInf;
    top = fmaxf(top, x[j]);
  }
  if (kept) {
#pragma unroll
    for (int j = 0; j < 16; j += 4)
      *reinterpret_cast<float4v*>(kept + 16 * g + j) = float4v{x[j], x[j + 1], x[j + 2], x[j + 3]};
  }
  // P is taken relative to the page's own maximum, so that fp16 loses no light page beside a heavy
  // one, and that is 2^15, so that a token of a light weight keeps its bits beside the heaviest one
  // (which may have nothing in a channel); w brings the page to the running reference.
  top = quad_max(top);
  const float mine = top == kNegInf ? 0.0f : top - 15.0f;    // (nothing of the page is visible)
  const float both = fmaxf(S.m, top);
  const float ref = both == kNegInf ? 0.0f : both;
  keep = __builtin_amdgcn_exp2f(S.m - ref);
  const float w = __builtin_amdgcn_exp2f(top - ref - 15.0f);
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    x[j] = __builtin_amdgcn_exp2f(x[j] - mine);
    sum += x[j];
    p[j >> 3][j & 7] = (_Float16)x[j];
  }
  S.l = __builtin_fmaf(S.l, keep, sum * w);
  S.m = both;
  return w;
}

template <int D>
__device__ __forceinline__ void page_values(const VRegs<D>& V, const half8 p[2], float keep,
                                            float vw, Acc<D>& S) {
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    const uint4v c = V.c[dt];
    float4v acc = {0.0f, 0.0f, 0.0f, 0.0f};
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_widen8(c[0], c[1]), p[0], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_widen8(c[2], c[3]), p[1], acc, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      S.o[dt][i] = __builtin_fmaf(acc[i], vw, S.o[dt][i] * keep);
  }
}

template <int D, bool BF16, class Rows>
__device__ __forceinline__ void put_out(const KvAttn& A, const Rows& R, int h, int row, int d,
                                        const float* o, int n) {
  const int i = R.i0 + row / A.group, head = h * A.group + row % A.group;
  if (!R.exists(i)) return;
  uint16_t* p = static_cast<uint16_t*>(A.out.p) + R.at(A.out, i) + (int64_t)head * A.out.head + d;
  for (int c = 0; c < n; ++c) p[c] = kv_narrow<BF16>(o[c]);
}

template <class Rows>
__device__ __forceinline__ int64_t lse_at(const KvAttn& A, const Rows& R, int H, int h, int row) {
  const int i = R.i0 + row / A.group, head = h * A.group + row % A.group;
  return R.token(A.nq, i) * ((int64_t)H * A.group) + head;
}

template <class Rows>
__device__ __forceinline__ void put_lse(const KvAttn& A, const Rows& R, int H, int h, int row,
                                        float* lse, float x) {
  if (lse && R.exists(R.i0 + row / A.group)) lse[lse_at(A, R, H, h, row)] = x;
}

// Partial states of one 16-row tile in 32 bits: O [16][D], then (m, l) [16].
template <int D>
constexpr int kPart = 16 * (D + 2);
constexpr int kMostSplits = 128;

// Pairs of floats past this XCD's caches.
__device__ __forceinline__ void put_pair(float* p, float a, float b) {
  const uint64_t w = (uint64_t)__builtin_bit_cast(uint32_t, b) << 32 |
                     __builtin_bit_cast(uint32_t, a);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), w, __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
template <bool FAR>
__device__ __forceinline__ void get_pair(const float* p, float& a, float& b) {
  const uint64_t* q = reinterpret_cast<const uint64_t*>(p);
  const uint64_t w = FAR ? __hip_atomic_load(const_cast<uint64_t*>(q), __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT)
                         : *q;
  a = __builtin_bit_cast(float, (uint32_t)w);
  b = __builtin_bit_cast(float, (uint32_t)(w >> 32));
}

// The rows of one 16-row tile from n partial states kPart apart, in the order of the states, and
// out: the 256 threads first fetch every state's (m, l) at once, then each takes pairs of channels
// through all states. FAR: written by other workgroups of this launch. w [n][16]: LDS. rows0: rows
// of the tile that exist.
template <int D, bool BF16, bool FAR, int kAhead, class Rows>
__device__ __forceinline__ void join_tile(const KvAttn& A, const Rows& R, int H, int h, int tile,
                                          int rows0, const float* p, int n, float* w, float* lse) {
  const int tid = threadIdx.x;
  const int row = tid >> 4, sub = tid & 15;            // 16 threads a row
  // the first states' channels are on their way while the factors are found
  float2 ahead[kAhead];
  const int e0 = tid < rows0 * (D / 2) ? tid : 0;
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    get_pair<FAR>(p + (i < n ? i : 0) * kPart<D> + e0 / (D / 2) * D + e0 % (D / 2) * 2, ahead[i].x,
                  ahead[i].y);
  float top = kNegInf, l = 0.0f;
  if (row < rows0) {
    for (int i = sub; i < n; i += 16) {
      float m, x;
      get_pair<FAR>(p + i * kPart<D> + 16 * D + 2 * row, m, x);
      w[i * 16 + row] = m;
      const float both = fmaxf(top, m), ref = both == kNegInf ? 0.0f : both;
      l = l * __builtin_amdgcn_exp2f(top - ref) + x * __builtin_amdgcn_exp2f(m - ref);
      top = both;
    }
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    const float m = __shfl_xor(top, o), x = __shfl_xor(l, o);
    const float both = fmaxf(top, m), ref = both == kNegInf ? 0.0f : both;
    l = l * __builtin_amdgcn_exp2f(top - ref) + x * __builtin_amdgcn_exp2f(m - ref);
    top = both;
  }
  const float ref = top == kNegInf ? 0.0f : top;
  if (row < rows0) {
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    for (int i = sub; i < n; i += 16)
      w[i * 16 + row] = __builtin_amdgcn_exp2f(w[i * 16 + row] - ref) * inv;
    if (sub == 0) put_lse(A, R, H, h, tile * 16 + row, lse, (top + __builtin_amdgcn_logf(l)) * kLn2);
  }
  __syncthreads();
  for (int e = tid; e < rows0 * (D / 2); e += 256) {
    const int r = e / (D / 2), d = e % (D / 2) * 2;
    float o[2] = {0.0f, 0.0f};
    const float* q = p + r * D + d;
    // kAhead states at a time, all their loads on their way together
    for (int i0 = 0; i0 < n; i0 += kAhead) {
      if (e != tid || i0 > 0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
          get_pair<FAR>(q + (i0 + i < n ? i0 + i : 0) * kPart<D>, ahead[i].x, ahead[i].y);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (i0 + i < n) {
          const float f = w[(i0 + i) * 16 + r];
          o[0] = __builtin_fmaf(ahead[i].x, f, o[0]);
          o[1] = __builtin_fmaf(ahead[i].y, f, o[1]);
        }
      }
    }
    put_out<D, BF16>(A, R, h, tile * 16 + r, d, o, 2);
  }
}

// One joined row's channels to `out`, and its log-sum-exp.
template <int D, bool BF16, int N, class Rows>
__device__ __forceinline__ void finish_row(const KvAttn& A, const Rows& R, int H, int h, int row,
                                           int d0, float* o, float top, float l, float* lse) {
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
#pragma unroll
  for (int c = 0; c < N; ++c) o[c] *= inv;
  put_out<D, BF16>(A, R, h, row, d0, o, N);
  if (d0 == 0) put_lse(A, R, H, h, row, lse, (top + __builtin_amdgcn_logf(l)) * kLn2);
}

// Up to 16 rows of one head from n partial states each, in the order of the states, and for each row
// one state more (top, l: 16 threads a row, the first of them has it). state(i, x, in): where state i
// of row x lies, and which row of it that is; scaled(f): this thread's row takes the additional state
// times f; done(x, d, o): the other states' sum of four channels of row x. 256 threads: 16 a row find
// the factors, then a thread takes four channels of a row, and where there are threads left they share
// the states, whose sums meet in LDS. top and l leave as those of the row.
template <int D, class State, class Scaled, class Done>
__device__ __forceinline__ void join_rows(int rows, int n, float* w, float4v* sums, float& top,
                                          float& l, State state, Scaled scaled, Done done) {
  constexpr int kAhead = 8;
  const int tid = threadIdx.x, row = tid >> 4, sub = tid & 15;
  const float top0 = top;
  if (row < rows) {
    for (int i = sub; i < n; i += 16) {
      int in;
      const float* const s = state(i, row, in);
      const float2v ml = *reinterpret_cast<const float2v*>(s + 16 * D + 2 * in);
      w[i * 16 + row] = ml[0];
      const float both = fmaxf(top, ml[0]), ref = both == kNegInf ? 0.0f : both;
      l = l * __builtin_amdgcn_exp2f(top - ref) + ml[1] * __builtin_amdgcn_exp2f(ml[0] - ref);
      top = both;
    }
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    const float m = __shfl_xor(top, o), x = __shfl_xor(l, o);
    const float both = fmaxf(top, m), ref = both == kNegInf ? 0.0f : both;
    l = l * __builtin_amdgcn_exp2f(top - ref) + x * __builtin_amdgcn_exp2f(m - ref);
    top = both;
  }
  const float first = __shfl(top0, (int)(threadIdx.x & 48));
  if (row < rows) {
    const float ref = top == kNegInf ? 0.0f : top, inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    for (int i = sub; i < n; i += 16)
      w[i * 16 + row] = __builtin_amdgcn_exp2f(w[i * 16 + row] - ref) * inv;
    scaled(__builtin_amdgcn_exp2f(first - ref) * inv);
  }
  __syncthreads();
  const int units = rows * (D / 4);                    // four channels of a row
  const int shares = units < 256 ? 256 / units : 1;
  for (int e = tid; e < units * shares; e += 256) {
    const int share = e / units, u = e - share * units, x = u / (D / 4), d = u % (D / 4) * 4;
    float4v o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = share; i0 < n; i0 += kAhead * shares) {
      float4v v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k * shares;
        int in;
        const float* const s = state(i < n ? i : n - 1, x, in);
        v[k] = *reinterpret_cast<const float4v*>(s + in * D + d);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k * shares;
        const float f = i < n ? w[i * 16 + x] : 0.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = __builtin_fmaf(v[k][c], f, o[c]);
      }
    }
    if (shares == 1) done(x, d, o);
    else sums[e] = o;
  }
  if (shares > 1) {
    __syncthreads();
    if (tid < units) {
      float4v o = sums[tid];
      for (int s = 1; s < shares; ++s) o += sums[s * units + tid];
      done(tid / (D / 4), tid % (D / 4) * 4, o);
    }
  }
}

// Which context request `b` reads and its place among that one's, and where its tiles start; or -1.
__device__ __forceinline__ int context_of(const KvUsers& U, const KvTiles& T, int b, int& place,
                                          int& tile0) {
  int lo = 0, hi = U.contexts;                         // firsts[lo - 1] <= b < firsts[hi]
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (U.firsts[mid] <= b) lo = mid + 1;
    else hi = mid;
  }
  if (lo == 0) return -1;
  const Requests q = requests_of(U, lo - 1);
  place = b - q.first;
  tile0 = tiles_before(T, U, lo - 1, q.first);
  return place >= 0 && place < q.count ? lo - 1 : -1;
}

// Contexts' tiles of 16 rows, and the states of them that a launch before has left, for the requests'
// own tokens to join: for every tile and head those of its splits, `step` of them a tile. (Heads next to
// each other, in the order of the requests' own workgroups: of eight heads those of one then run on one
// XCD. 2 contexts of 75 tokens and 3 requests each 16.5 us, 17.3 with a head's tiles together.)
struct ContextStates {
  KvTiles tiles;
  int splits;
  int64_t step;
  const float* part;

  template <int D>
  __device__ __forceinline__ const float* from(int h, int tile) const {
    return part + (tile * step + h * splits) * kPart<D>;
  }
};

// Requests that have no context see nothing: those before the first context's, between the bound of
// a context's requests and the next one's, and behind the last. Context p's workgroups fill in those
// behind p's own, of which this is one of `shares`, a row a wave (4095 such requests of 32 heads of 128
// channels and one with a context: 5.9 ms by one workgroup, 175 us by one of each head).
template <int NT>
__device__ __forceinline__ void fill_without(const KvAttn& A, const KvUsers& U, int contexts, int p,
                                             int H, int D, int share, int shares, float* lse) {
  const Requests q = requests_of(U, p);
  int to = U.firsts[p + 1];
  to = to < U.n_seq && p + 1 < contexts ? to : U.n_seq;
  const int before = p == 0 ? q.first : 0;               // [0, before) and [q.first + q.count, to)
  const int from = q.first + q.count, n = before + (to > from ? to - from : 0);
  const int heads = H * A.group, each = U.per * heads, lane = threadIdx.x & 63;
  const int64_t rows = (int64_t)n * each;
  for (int64_t r = share * (NT / 64) + uniform(threadIdx.x >> 6); r < rows; r += shares * (NT / 64)) {
    const int k = (int)(r / each), row = (int)(r - (int64_t)k * each);
    const int64_t b = k < before ? k : from + (k - before);
    const int i = row / heads, head = row - i * heads;
    uint16_t* const to =
        static_cast<uint16_t*>(A.out.p) + b * A.out.seq + i * A.out.tok + head * A.out.head;
    for (int d = lane; d < D; d += 64) to[d] = 0;
    if (lse && lane == 0) lse[(b * U.per + i) * heads + head] = kNegInf;
  }
}

// Workgroup = (virtual sequence, KV head, 16-row tile, split of the pages); its four waves take
// the split's pages in turn and meet in LDS. A page's K is requested as soon as the scores have
// used the last one's, its V as soon as the second product has: each wave has a page in flight all
// the time, which is what carries the memory's rate at 8 waves a CU. With splits, the workgroup
// leaves its partial state in memory and counts itself in; the last of a tile joins them all, in
// the order of the splits, and clears the counter for the next call. The states are written and
// read past the XCDs' own caches (agent scope), and counted when they have arrived: a release
// fence instead writes back the whole L2 for every workgroup (25 -> 197 us for 32 sequences of 2K).
// Bound by the codes' bytes where there are many: 4 sequences of 8K on 32 heads, 269 MB in 51 us, 5.3
// TB/s (a copy of 1 GiB: 5.1); one sequence of 4K on 8 heads, 8 MB, 11 us, is a chain of dependent
// reads (length, table, codes) and the join, 6 us with a single page.
// With SharedRows the sequences are contexts that requests share. Its result is `out`, or (kParts)
// every split's state stays in memory for a launch behind it to join, or (kJoin) the only split joins
// what the launch before has left of the sequence's context: 32 requests of 300 tokens behind one of
// 16K 11 us for 17 with a launch for the own tokens and one for the join.
enum Result { kOut, kParts, kJoin };

template <int D, bool BF16, class Rows, Result TO>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void attend_kernel(KvPool pool, KvSeqs S, KvAttn A,
                                                        KvUsers U, int tiles, int splits,
                                                        int64_t items, float* part,
                                                        uint32_t* arrived, float* lse,
                                                        float* scores, int np, ContextStates C) {
  __shared__ float os[4][16][D + 4];
  __shared__ float ml[4][32];
  __shared__ uint32_t others;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int split = (int)(it % splits);
    const int64_t unit = it / splits;
    constexpr bool kShared = __is_same(Rows, SharedRows);
    int tile, h, vseq;
    if constexpr (kShared) {
      h = (int)(unit % pool.H);
      vseq = context_at(C.tiles, U, (int)(unit / pool.H), tile);
      if (vseq < 0 || tile < 0) continue;
    } else {
      tile = (int)(unit % tiles);
      h = (int)(unit / tiles % pool.H);
      vseq = (int)(unit / tiles / pool.H);
    }
    const Rows R = rows_in<Rows>(S, A, U, vseq);
    if constexpr (kShared && TO == kOut)
      if (tile == 0)
        fill_without<256>(A, U, S.n, vseq, pool.H, D, h * splits + split, pool.H * splits, lse);
    // the pages that any row of the tile sees
    const int rows = R.nq * A.group;
    const int last = tile * 16 + 15 < rows ? tile * 16 + 15 : rows - 1;
    const int most = R.most(R.i0 + tile * 16 / A.group, R.i0 + last / A.group);
    const int n = A.picks ? A.n_picks : (most + kPage - 1) / kPage;
    const int per = (n + splits - 1) / splits;
    const int j0 = split * per, j1 = j0 + per < n ? j0 + per : n;
    const int32_t* picks = A.picks ? A.picks + ((int64_t)vseq * pool.H + h) * A.n_picks : nullptr;
    // the next page of this wave from column j on, or -1; j moves behind it
    int at = 0;
    const auto next_page = [&](int& j) -> int64_t {
      while (j < j1) {
        at = picks ? picks[j] : j;
        j += 4;
        if (at < 0 || (int64_t)at * kPage >= most) continue;
        const int page = kv_page(S, pool.P, R.seq, at);
        if (page >= 0) return (int64_t)page * pool.H + h;
      }
      return -1;
    };
    int j = j0 + __builtin_amdgcn_readfirstlane(wave);
    int64_t b = next_page(j);
    KRegs<D> K;
    VRegs<D> V;
    if (b >= 0) {
      load_k<D>(pool.k + b * (kPage * D), K);
      load_v<D>(pool.v + b * (kPage * D), V);
    }
    QTile<D> Q;
    load_q<D, BF16>(A, R, h, tile, Q);
    int place = 0, tile0 = 0, context = -1;      // (looked up beside the first page's codes)
    if constexpr (TO == kJoin) context = uniform(context_of(U, C.tiles, R.seq, place, tile0));
    Acc<D> acc;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc.o[dt] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    acc.m = kNegInf;
    acc.l = 0.0f;
    float* const kept = scores && tile * 16 + m < rows
        ? scores + (((int64_t)R.seq * pool.H + h) * rows + tile * 16 + m) * np * kPage : nullptr;
    while (b >= 0) {
      const float ks = pool.ks[b], vs = pool.vs[b];
      const int pos0 = at * kPage;
      float x[16], keep;
      half8 p[2];
      const int64_t bn = next_page(j);
      page_scores<D>(K, Q, x);
      if (bn >= 0) load_k<D>(pool.k + bn * (kPage * D), K);
      const float w = page_softmax<D>(x, ks, pos0, Q, acc, p, keep, kept ? kept + pos0 : nullptr);
      // (a row that sees nothing of the page takes nothing of its scale, whatever that is)
      page_values<D>(V, p, keep, w == 0.0f ? 0.0f : w * vs, acc);
      if (bn >= 0) load_v<D>(pool.v + bn * (kPage * D), V);
      b = bn;
    }
    acc.l = quad_sum(acc.l);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
      *reinterpret_cast<float4v*>(&os[wave][m][16 * dt + 4 * g]) = acc.o[dt];
    if (g == 0) {
      ml[wave][m] = acc.m;
      ml[wave][16 + m] = acc.l;
    }
    __syncthreads();
    // 16 threads a row, D / 16 channels each
    constexpr int N = D / 16;
    const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * N;
    const bool live = tile * 16 + row < rows;
    float o[N], top, l;
    if (live) {
      // the waves' states are 16 (D + 4) apart in os and 32 in ml: joined in wave order
      top = kNegInf;
#pragma unroll
      for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w][row]);
      const float ref = top == kNegInf ? 0.0f : top;
      l = 0.0f;
#pragma unroll
      for (int c = 0; c < N; ++c) o[c] = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[w][row] - ref);
        l = __builtin_fmaf(ml[w][16 + row], f, l);
#pragma unroll
        for (int c = 0; c < N; ++c) o[c] = __builtin_fmaf(os[w][row][d0 + c], f, o[c]);
      }
    }
    if constexpr (TO == kJoin) {
      // (os has room for the factors, the sums and this row's own share; its readers come first)
      static_assert(sizeof(os) >= (kMostSplits * 16 + 1024 + 16 * D) * sizeof(float), "room in os");
      float* const w = &os[0][0][0];
      float4v* const sums = reinterpret_cast<float4v*>(w + kMostSplits * 16);
      float* const own = w + kMostSplits * 16 + 1024;
      const int n0 = context >= 0 ? C.splits : 0, from = place * rows + tile * 16;
      const float* const s0 = C.from<D>(h, uniform(tile0));
      const bool first = d0 == 0 && live;
      float t0 = first ? top : kNegInf, l0 = first ? l : 0.0f;
      __syncthreads();
      join_rows<D>(rows - tile * 16 < 16 ? rows - tile * 16 : 16, n0, w, sums, t0, l0,
                   [&](int i, int x, int& in) {
                     in = (from + x) & 15;
                     return s0 + (((from + x) >> 4) * C.step + i) * kPart<D>;
                   },
                   [&](float f) {
#pragma unroll
                     for (int c = 0; c < N; ++c) own[row * D + d0 + c] = o[c] * f;
                   },
                   [&](int x, int d, float4v y) {
#pragma unroll
                     for (int c = 0; c < 4; ++c) y[c] += own[x * D + d + c];
                     put_out<D, BF16>(A, R, h, tile * 16 + x, d,
                                      reinterpret_cast<const float*>(&y), 4);
                   });
      if (first) put_lse(A, R, pool.H, h, tile * 16 + row, lse,
                         (t0 + __builtin_amdgcn_logf(l0)) * kLn2);
    } else if constexpr (TO == kParts) {
      float* mine = part + it * kPart<D>;
      if (live) {
#pragma unroll
        for (int c = 0; c < N; c += 2)
          *reinterpret_cast<float2v*>(mine + row * D + d0 + c) = float2v{o[c], o[c + 1]};
        if (d0 == 0)
          *reinterpret_cast<float2v*>(mine + 16 * D + 2 * row) = float2v{top, l};
      }
    } else if (splits == 1) {
      if (live) finish_row<D, BF16, N>(A, R, pool.H, h, tile * 16 + row, d0, o, top, l, lse);
    } else {
      float* mine = part + it * kPart<D>;
      if (live) {
#pragma unroll
        for (int c = 0; c < N; c += 2) put_pair(mine + row * D + d0 + c, o[c], o[c + 1]);
        if (d0 == 0) put_pair(mine + 16 * D + 2 * row, top, l);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's part has arrived
      __syncthreads();
      if (threadIdx.x == 0)
        others = __hip_atomic_fetch_add(&arrived[unit], 1u, __ATOMIC_RELAXED,
                                        __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      if (others == (uint32_t)splits - 1) {
        if (threadIdx.x == 0)
          __hip_atomic_store(&arrived[unit], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // (os has room for the factors of 128 states; its readers have passed two barriers)
        join_tile<D, BF16, true, 16>(A, R, pool.H, h, tile, rows - tile * 16 < 16 ? rows - tile * 16 : 16,
                                 part + unit * splits * kPart<D>, splits, &os[0][0][0], lse);
      }
    }
    __syncthreads();
  }
}

// The splits of prompt_kernel joined: a workgroup a 16-row tile. Bound by the states' bytes: 33 MB of
// 2000 rows of 8 heads in 4 splits, 9 us, 3.7 TB/s.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void join_kernel(KvPool pool, KvSeqs S, KvAttn A, int tiles,
                                                   int splits, int64_t items, const float* part,
                                                   float* lse) {
  __shared__ float w[kMostSplits * 16];
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int tile = (int)(it % tiles);
    const int64_t r = it / tiles;
    const int h = (int)(r % pool.H);
    const RowsOf R = rows_of(S, A, (int)(r / pool.H));
    const int rows = R.nq * A.group - tile * 16;
    join_tile<D, BF16, false, 4>(A, R, pool.H, h, tile, rows < 16 ? rows : 16,
                              part + it * splits * kPart<D>, splits, w, lse);
    __syncthreads();
  }
}

// What every cached token got: decay * mass_in + the sum over the rows of exp(S - lse). One wave
// per (sequence, KV head, page) walks the row tiles; the sum over the 16 rows of a tile is taken
// once at the end, so no result depends on any order of arrival. Bound by reading K again, at one
// page a wave: 4 sequences of 8K, 8 heads, 16 rows each, 34 MB in 13.4 us.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void mass_kernel(KvPool pool, KvSeqs S, KvAttn A, int tiles,
                                                   int np, int64_t items, const float* lse) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  for (int64_t it = (int64_t)blockIdx.x * 4 + wave; it < items; it += (int64_t)gridDim.x * 4) {
    const int j = (int)(it % np);
    const int64_t r = it / np;
    const int h = (int)(r % pool.H), seq = (int)(r / pool.H);
    const RowsOf R = rows_of(S, A, seq);
    if (j * (int64_t)kPage >= R.len) continue;
    const int page = kv_page(S, pool.P, seq, j);
    if (page < 0) continue;
    const int64_t b = (int64_t)page * pool.H + h;
    const float ks = pool.ks[b];
    KRegs<D> K;
    load_k<D>(pool.k + b * (kPage * D), K);
    float sum[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[e] = 0.0f;
    for (int tile = 0; tile < tiles; ++tile) {
      QTile<D> Q;
      load_q<D, BF16>(A, R, h, tile, Q);
      if (!__any(Q.visible > j * kPage)) continue;
      const int row = tile * 16 + m;
      const float z = row < R.nq * A.group ? lse[lse_at(A, R, pool.H, h, row)] * kLog2e : 0.0f;
      float x[16];
      page_scores<D>(K, Q, x);
      const float f = Q.unit * ks;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (j * kPage + 16 * g + e < Q.visible)
          sum[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], f, -z));
    }
    const float mine = sum_across<16>(sum);
    const int t = 16 * g + m;
    if (j * kPage + t < R.len) {
      const int64_t at = b * kPage + t;
      A.mass_out[at] = A.mass_in ? __builtin_fmaf(A.decay, A.mass_in[at], mine) : mine;
    }
  }
}

// The same from scores that attend_kernel has kept: a lane a token, one wave a page. Bound by the
// scores' bytes and a launch: 6 MB of 32 sequences, 44K tokens together, 4 rows a head, 7.4 us.
__global__ __launch_bounds__(256) void mass_scores_kernel(KvPool pool, KvSeqs S, KvAttn A, int np,
                                                          int64_t items, const float* scores,
                                                          const float* lse) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t it = (int64_t)blockIdx.x * 4 + wave; it < items; it += (int64_t)gridDim.x * 4) {
    const int j = (int)(it % np);
    const int64_t r = it / np;
    const int h = (int)(r % pool.H), seq = (int)(r / pool.H);
    const RowsOf R = rows_of(S, A, seq);
    const int t = j * kPage + lane;
    if (t - lane >= R.len) continue;
    const int page = kv_page(S, pool.P, seq, j);
    if (page < 0) continue;
    const int rows = R.nq * A.group;
    const float* x = scores + r * rows * np * kPage + t;
    float sum = 0.0f;
#pragma unroll 4
    for (int row = 0; row < rows; ++row) {
      const int see = R.visible(row / A.group);
      const float z = lse[lse_at(A, R, pool.H, h, row)] * kLog2e;
      if (t < see) sum += __builtin_amdgcn_exp2f(x[(int64_t)row * np * kPage] - z);
    }
    if (t < R.len) {
      const int64_t at = ((int64_t)page * pool.H + h) * kPage + lane;
      A.mass_out[at] = A.mass_in ? __builtin_fmaf(A.decay, A.mass_in[at], sum) : sum;
    }
  }
}

// ---- many rows ------------------------------------------------------------------------------
// Where a KV head has many rows, the matrix units bound: v_mfma_f32_32x32x16_f16, transposed as
// above (lane = 32 half + m, results of row m), 32 rows a wave. The workgroup's waves share each
// page through LDS: it is loaded as codes ahead of its turn, widened to fp16 once, and read as
// operands by every wave. Row m of a 32-token K tile is the token whose place makes a lane's 16
// results the consecutive tokens 16 half .. 16 half + 15 (`tile_row`), the k slots it supplies for
// P V.
//
// The weights of a page enter the second product times the page's V scale, relative to a running
// reference of that product (`ref`, log2), so O needs no further factor, and l sums them without
// the scale. No maximum is taken: the weights go by the reference that is there, and only where
// 16 of them sum to more than fp16 holds a tile's maximum is found, the accumulators move to it, and
// the weights are taken again; a row's first tile does that. Behind a move the heaviest weight is
// 2^kLift, so that 16 as heavy still pass and nothing moves before one is 2^(16 - kLift) times as
// heavy; below, a weight keeps 11 bits down to 2^-(14 + kLift) of the heaviest and is off by
// 2^-(25 + kLift) of it under that. What a light weight keeps shows in the channels where the heavy
// ones have nothing, so kLift is the largest that equal weights pass.
constexpr int kLift = 11;
constexpr float kMost = 65504.0f;

__device__ __forceinline__ int tile_row(int t) {       // of token t of 32: its row in the K tile
  return 8 * ((t & 15) >> 2) + 4 * (t >> 4) + (t & 3);
}

// A value and that of the lane with the other half. The copy is made opaque: given one value as
// both operands of the swap, the compiler takes its two results to be equal.
__device__ __forceinline__ void both_halves(uint32_t u, uint32_t& lo, uint32_t& hi) {
  uint32_t w = u;
  asm("" : "+v"(w));
  const auto r = __builtin_amdgcn_permlane32_swap(u, w, false, false);
  lo = r[0];
  hi = r[1];
}
// The larger of two in one instruction: fmaxf of a product's result costs a second one that quiets
// NaNs. (Not through inline assembly, whose reads of a matrix result the compiler does not pad.)
__device__ __forceinline__ float max2(float a, float b) {
  return __builtin_amdgcn_fmed3f(a, b, __builtin_inff());
}
__device__ __forceinline__ float half_max(float x) {   // over the lanes of equal m
  uint32_t lo, hi;
  both_halves(__builtin_bit_cast(uint32_t, x), lo, hi);
  return fmaxf(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
}
__device__ __forceinline__ float half_sum(float x) {
  uint32_t lo, hi;
  both_halves(__builtin_bit_cast(uint32_t, x), lo, hi);
  return __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
}

// One row's queries as B operands of the 32-row products: q[s] holds channels 16 s + 8 half ..
// + 7. Returns what S is multiplied by (bf16 rows scaled as in load_q, the scale's sign taken
// into the queries so that a row's largest product is its largest S).
template <int D, bool BF16>
__device__ __forceinline__ float load_row32(const KvAttn& A, const uint16_t* src, bool live,
                                            half8* q) {
  const int half = (threadIdx.x & 63) >> 5;
  uint16_t u[D / 16][8];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) *reinterpret_cast<uint4v*>(u[s]) = uint4v{0, 0, 0, 0};
  if (live && A.wide_q) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      *reinterpret_cast<uint4v*>(u[s]) =
          *reinterpret_cast<const uint4v*>(src + 16 * s + 8 * half);
  } else if (live) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      *reinterpret_cast<uint4v*>(u[s]) = load8(src + 16 * s + 8 * half, false);
  }
  int e = 0;
  const uint16_t flip = A.scale < 0.0f ? 0x8000u : 0;
  if (BF16) {
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t a = u[s][c] & 0x7fffu;
        top = a > top && a < 0x7f80u ? a : top;
      }
    uint32_t lo, hi;
    both_halves(top, lo, hi);
    top = lo > hi ? lo : hi;
    e = (int)(top >> 7) - 127;
    if (e < -126) e = -126;
  }
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint16_t w = u[s][c] ^ flip;
      q[s][c] = BF16 ? (_Float16)__builtin_ldexpf(kv_widen<true>(w), -e)
                     : __builtin_bit_cast(_Float16, w);
    }
  return __builtin_ldexpf(__builtin_fabsf(A.scale) * kLog2e, e);
}

// K pages in LDS: with three a page takes one barrier, with two (all that 256 channels leave room
// for) it takes two.
template <int D>
constexpr int kPagesK = D == 256 ? 2 : 3;

template <int D>
struct PromptLds {
  _Float16 k[kPagesK<D>][kPage][D + 8];   // rows in the order of tile_row; 16 bytes of padding a
  _Float16 v[2][D][kPage + 8];            // row keep the lanes' 16-byte reads off one another's
};                                        // banks

// Codes of one page's K or V on their way to LDS: 16 bytes a thread and step.
template <int D, int NT>
constexpr int kPieces = (4 * D + NT - 1) / NT;         // of the page's 4 D, a thread
template <int D, int NT>
constexpr bool kWhole = 4 * D % NT == 0;
template <int D, int NT>
struct PageRegs {
  uint4v c[kPieces<D, NT>];
};

template <int D, int NT>
__device__ __forceinline__ void page_fetch(const int8_t* codes, PageRegs<D, NT>& r) {
  const uint4v* p = reinterpret_cast<const uint4v*>(codes);
#pragma unroll
  for (int i = 0; i < kPieces<D, NT>; ++i)
    if (kWhole<D, NT> || threadIdx.x < 4 * D) r.c[i] = p[i * NT + threadIdx.x];
}

template <int D, int NT>
__device__ __forceinline__ void widen_k(const PageRegs<D, NT>& r, _Float16 (*k)[D + 8]) {
#pragma unroll
  for (int i = 0; i < kPieces<D, NT>; ++i) {
    const int n = i * NT + threadIdx.x;
    if (!kWhole<D, NT> && n >= 4 * D) break;
    const int t = n / (D / 16), d = n % (D / 16) * 16;
    _Float16* to = &k[(t & 32) + tile_row(t & 31)][d];
    *reinterpret_cast<half8*>(to) = kv_widen8(r.c[i][0], r.c[i][1]);
    *reinterpret_cast<half8*>(to + 8) = kv_widen8(r.c[i][2], r.c[i][3]);
  }
}

template <int D, int NT>
__device__ __forceinline__ void widen_v(const PageRegs<D, NT>& r, _Float16 (*v)[kPage + 8]) {
#pragma unroll
  for (int i = 0; i < kPieces<D, NT>; ++i) {
    const int n = i * NT + threadIdx.x;
    if (!kWhole<D, NT> && n >= 4 * D) break;
    _Float16* to = &v[n >> 2][(n & 3) * 16];
    *reinterpret_cast<half8*>(to) = kv_widen8(r.c[i][0], r.c[i][1]);
    *reinterpret_cast<half8*>(to + 8) = kv_widen8(r.c[i][2], r.c[i][3]);
  }
}

// S^T of 32 tokens (rows k of the K tile) against the wave's rows.
template <int D>
__device__ __forceinline__ float16v tile_scores(const _Float16 (*k)[D + 8],
                                                const half8 (&q)[D / 16]) {
  const int m = threadIdx.x & 31, half = (threadIdx.x & 63) >> 5;
  float16v x;
#pragma unroll
  for (int e = 0; e < 16; ++e) x[e] = 0.0f;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const half8 a = *reinterpret_cast<const half8*>(&k[m][16 * s + 8 * half]);
    x = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, q[s], x, 0, 0, 0);
  }
  return x;
}

// Waves of a workgroup: with 256 channels a wave's registers leave room for one on a SIMD.
template <int D>
constexpr int kPromptWaves = D == 256 ? 4 : 8;

// Workgroup = (sequence, KV head, tile of 32 rows a wave, split of the pages). `it0`: where this
// launch starts (see in_launches). Bound by the matrix units and the vector instructions of the
// softmax (32 exponentials a lane and page), which two waves on a SIMD overlap in part: 2 sequences
// of 8K, 64 heads, 2048 queries, 962 GFLOP in 0.92 to 1.07 ms as the clock goes, 0.90 to 1.05
// PFLOP/s (a library product of 8192 cubed: 1.23); 500 queries of 32 heads over 4K, 33 GFLOP, 51 us.
// `part`: where the splits' states go; null: there is one, and it is the result.
template <int D, bool BF16>
__global__ __launch_bounds__(64 * kPromptWaves<D>, kPromptWaves<D> / 4)
void prompt_kernel(KvPool pool, KvSeqs S, KvAttn A, int tiles, int splits, int64_t it0,
                   float* part, float* lse) {
  constexpr int NT = 64 * kPromptWaves<D>;
  __shared__ PromptLds<D> L;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 31, half = lane >> 5;
  const int64_t it = it0 + blockIdx.x;
  const int h = uniform((int)(it % pool.H));
  int64_t r = it / pool.H;
  const int split = uniform((int)(r % splits));
  r /= splits;
  const int tile = uniform(tiles - 1 - (int)(r % tiles));   // the tiles that see most go first
  const int seq = uniform((int)(r / tiles));
  RowsOf R = rows_of(S, A, seq);
  R.len = uniform(R.len);
  R.q_len = uniform(R.q_len);
  const int rows = R.nq * A.group, row = (tile * kPromptWaves<D> + wave) * 32 + m;

  half8 q[D / 16];
  // a row that sees nothing is not masked tile by tile: it is written as empty at the end
  const int i_row = row / A.group, head = h * A.group + row % A.group;
  const int see = row < rows ? R.visible(i_row) : 0;
  const int visible = see > 0 ? see : 0x7fffffff;
  const float unit = load_row32<D, BF16>(
      A, static_cast<const uint16_t*>(A.q.p) + R.at(A.q, i_row) + (int64_t)head * A.q.head, see > 0,
      q);
  int low = visible;                                   // what every row of the wave sees
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_xor(low, o);
    low = v < low ? v : low;
  }
  low = __builtin_amdgcn_readfirstlane(low);
  // the workgroup's pages: up to what its last live row sees
  int last = (tile + 1) * (32 * kPromptWaves<D>) - 1;
  last = last < rows ? last : rows - 1;
  const int most = R.most(tile * (32 * kPromptWaves<D>) / A.group, last / A.group);
  const int n = (most + kPage - 1) / kPage;
  const int per = (n + splits - 1) / splits;
  const int j0 = split * per, j1 = j0 + per < n ? j0 + per : n;

  float16v o[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.0f;
  float ref = -1e30f, l = 0.0f;      // O and l in units of 2^(ref - kLift)
  float ref0 = -1e30f, l0 = 0.0f;    // l of the pages without V, in units of 2^ref0
  // l has no V scale in it: where all of them are tiny it is kept 2^64 times smaller, or it would
  // overflow.
  bool tiny = false;
  float l_unit = 1.0f;
  float v_top = 0x1p-40f;            // the largest V scale so far; what is 2^-60 of it counts as none

  // The pages in turn, those that do not exist left out.
  int jn = j0;
  const auto next_page = [&](int& j) -> int64_t {
    while (jn < j1) {
      j = jn++;
      const int page = uniform(kv_page(S, pool.P, seq, j));
      if (page >= 0) return (int64_t)page * pool.H + h;
    }
    return -1;
  };
  // One tile of 32 tokens: its scores x become weights and go into O, while the scores of the
  // tile after it (the return value) are computed from `next` and `put` widens codes for later
  // ones. k, v: the tile's own operands.
  const auto tile_step = [&](float16v x, const _Float16 (*k)[D + 8], const _Float16 (*next)[D + 8],
                             const _Float16 (*v)[kPage + 8], int pos0, float ks, float vs,
                             auto put) -> float16v {
    // What a row does not see is taken out behind the exponentials: then neither its scores nor
    // the page's scales reach the row, whatever they are.
    const bool cut = pos0 + 32 > low;                  // the tile ends beyond what some row sees
    const int seen_here = visible - pos0 - 16 * half;  // of the lane's 16 tokens
    const auto mask = [&](float16v& z, float to) {
      if (cut) {
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = e < seen_here ? z[e] : to;
      }
    };
    const float f = unit * ks;
    // a V scale 2^60 below an earlier one (or none) adds nothing to O, only its weights to a sum of
    // their own: they must not move the reference that the others are rounded by
    const bool with_v = !(vs <= v_top * 0x1p-60f);
    const float lv = with_v ? __builtin_amdgcn_logf(vs) + (float)kLift : 0.0f;
    const float c = with_v ? lv - ref : kNegInf;
    const float16v y = tile_scores<D>(next, q);
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], f, c));
    mask(x, 0.0f);
#pragma unroll
    for (int e = 0; e < 16; ++e) sum += x[e];
    if (__builtin_expect(__any(!(sum <= kMost)) || !with_v, 0)) {
      float g;
      if (with_v && !__any(!(sum < __builtin_inff()))) {
        // weights that 32 bits hold move by a power of two
        float t = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) t = max2(t, x[e]);
        const int up = __builtin_amdgcn_frexp_expf(half_max(t)) - kLift;
        const int by = up > 0 ? up : 0;
        g = __builtin_ldexpf(1.0f, -by);
        ref += (float)by;
        sum *= g;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= g;
      } else {
        x = tile_scores<D>(k, q);
        float t = kNegInf;
#pragma unroll
        for (int e = 0; e < 16; ++e) t = max2(t, !cut || e < seen_here ? x[e] : kNegInf);
        t = half_max(t);
        t = t == kNegInf ? t : t * f;
        const float was = with_v ? ref : ref0;
        const float now = fmaxf(was, with_v ? t + lv - (float)kLift : t);
        g = __builtin_amdgcn_exp2f(was - now);
        const float by = with_v ? lv - now : -now;
        sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], f, by));
        mask(x, 0.0f);
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += x[e];
        if (with_v) {
          ref = now;
        } else {
          ref0 = now;
          l0 = __builtin_fmaf(l0, g, sum);
          g = 1.0f;
          sum = 0.0f;
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = 0.0f;
        }
      }
      l *= g;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= g;
    }
    half8 a[D / 32][2];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        a[dt][e] = *reinterpret_cast<const half8*>(&v[32 * dt + m][16 * half + 8 * e]);
    l = sum == 0.0f ? l : __builtin_fmaf(sum, __builtin_amdgcn_rcpf(vs) * l_unit, l);
    half8 p[2];
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const half2v h2 = __builtin_convertvector((float2v{x[e], x[e + 1]}), half2v);
      p[e >> 3][e & 7] = h2[0];
      p[e >> 3][(e & 7) + 1] = h2[1];
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[dt][e], p[e], o[dt], 0, 0, 0);
    put();
    return y;
  };

  // What page i's turn does besides its own two tiles: K of page i + kAhead is widened into LDS
  // beside the first and V of page i + 1 beside the second, and the registers they leave take the
  // codes of the page after. With kAhead = 2 the first scores of page i + 1, which come with the
  // second tile, find K there since the last barrier; with 1 they need one of their own. (Behind
  // the last page registers, buffers and scores are stale, and nobody uses them.)
  constexpr int kAhead = kPagesK<D> - 1;
  PageRegs<D, NT> kr, vr;
  float16v x;
  int pos[4];
  int64_t at[4];                     // this page and the next three
  float ks = 0.0f, vs = 0.0f, ks_n = 0.0f, vs_n = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    pos[i] = 0;
    at[i] = i && at[i ? i - 1 : 0] < 0 ? -1 : next_page(pos[i]);
  }
  const auto fetch_k = [&](int64_t a) {
    if (a >= 0) page_fetch<D, NT>(pool.k + a * (kPage * D), kr);
  };
  const auto fetch_v = [&](int64_t a) {
    if (a < 0) return;
    page_fetch<D, NT>(pool.v + a * (kPage * D), vr);
    ks_n = pool.ks[a];
    vs_n = pool.vs[a];
  };
  if (at[0] >= 0) {
    fetch_k(at[0]);
    fetch_v(at[0]);
    float v_most = 0.0f;
    for (int jb = j0; jb < j1; jb += 64) {
      const int page = jb + lane < j1 ? kv_page(S, pool.P, seq, jb + lane) : -1;
      const float v = page >= 0 ? pool.vs[(int64_t)page * pool.H + h] : 0.0f;
      v_most = v < __builtin_inff() ? fmaxf(v_most, v) : v_most;
    }
    tiny = !__any(v_most >= 0x1p-40f);
    if (tiny) {
      l_unit = 0x1p-64f;
      v_top = 0x1p-66f;
    }
    ks = ks_n;
    vs = vs_n;
    widen_k<D, NT>(kr, L.k[0]);
    widen_v<D, NT>(vr, L.v[0]);
    fetch_k(at[1]);
    fetch_v(at[1]);
    if (kAhead == 2 && at[1] >= 0) {
      widen_k<D, NT>(kr, L.k[1]);
      fetch_k(at[2]);
    }
    __syncthreads();
    x = tile_scores<D>(L.k[0], q);
  }
  int k0 = 0, k1 = 1;                // K buffers of this page and the next
  for (int buf = 0; at[0] >= 0; buf ^= 1) {
    v_top = vs < __builtin_inff() ? fmaxf(v_top, vs) : v_top;
    const int k2 = kAhead == 2 ? 3 - k0 - k1 : k0;
    const int pos0 = pos[0] * kPage;
    x = tile_step(x, L.k[k0], L.k[k0] + 32, L.v[buf], pos0, ks, vs,
                  [&] { widen_k<D, NT>(kr, L.k[kAhead == 2 ? k2 : k1]); });
    fetch_k(at[kAhead + 1]);
    if (kAhead == 1) __syncthreads();
    x = tile_step(x, L.k[k0] + 32, L.k[k1],
                  reinterpret_cast<const _Float16 (*)[kPage + 8]>(&L.v[buf][0][32]), pos0 + 32, ks,
                  vs, [&] { widen_v<D, NT>(vr, L.v[buf ^ 1]); });
    ks = ks_n;
    vs = vs_n;
    fetch_v(at[2]);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      at[i] = at[i + 1];
      pos[i] = pos[i + 1];
    }
    at[3] = at[2] < 0 ? -1 : next_page(pos[3]);
    k0 = k1;
    k1 = k2;
    __syncthreads();
  }

  // lane (m, half) has row m, channels 32 dt + 8 a + 4 half + 0 .. 3
  l = half_sum(l);
  l0 = half_sum(l0);
  if (row >= rows) return;
  // both sums to one reference, and O with them
  const float l_ref = ref - (float)kLift + (tiny ? 64.0f : 0.0f);
  const bool some = l > 0.0f || l != l, some0 = l0 > 0.0f || l0 != l0;
  const bool empty = see <= 0 || !(some || some0);
  const float top = fmaxf(some ? l_ref : -1e30f, some0 ? ref0 : -1e30f);
  const float to_top = some ? __builtin_amdgcn_exp2f(l_ref - top) : 0.0f;
  const float sum = l * to_top + (some0 ? l0 * __builtin_amdgcn_exp2f(ref0 - top) : 0.0f);
  const float g = empty ? 0.0f : (part ? to_top : to_top / sum) * l_unit;
  const int64_t u16 = ((int64_t)seq * pool.H + h) * ((rows + 15) / 16) + row / 16;
  float* dst = part ? part + (u16 * splits + split) * kPart<D> : nullptr;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      float4v w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = empty ? 0.0f : o[dt][4 * a + e] * g;
      const int d = 32 * dt + 8 * a + 4 * half;
      if (dst)
        *reinterpret_cast<float4v*>(dst + (row & 15) * D + d) = w;
      else
        put_out<D, BF16>(A, R, h, row, d, reinterpret_cast<const float*>(&w), 4);
    }
  if (half != 0) return;
  if (dst) {
    dst[16 * D + 2 * (row & 15)] = empty ? kNegInf : top;
    dst[16 * D + 2 * (row & 15) + 1] = empty ? 0.0f : sum;
  } else {
    put_lse(A, R, pool.H, h, row, lse,
            empty ? kNegInf : (top + __builtin_amdgcn_logf(sum)) * kLn2);
  }
}

// ---- weights of many rows -------------------------------------------------------------------
// The same sum as mass_kernel where there are many rows: a wave keeps one page's K as operands in
// registers (in the queries' own type: the codes are exact in either) and adds up its 64 tokens'
// weights row tile by row tile. A tile's queries are read as whole rows, since a load whose lanes
// lie in different rows takes a cache access for each of them, and turned through LDS of the
// wave's own, without barriers: the two waves of a SIMD drift apart, and one's products run beside
// the other's exponentials. The waves of a workgroup are pages x `shares` shares of the row tiles
// (every shares-th), whose sums meet in LDS at the end in a fixed order. Bound by a wave's chain
// from a tile's queries through LDS to its products and exponentials, at two waves a SIMD: 500
// queries of 32 heads over 4K, 16 GFLOP and 65 M exponentials, 31.5 us. (Two tiles ahead instead of
// one takes the registers over 256: 3 us more.)
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));

// Eight codes in the queries' type.
template <bool BF16>
__device__ __forceinline__ uint4v widen_as(uint32_t a, uint32_t b) {
  if (!BF16) return __builtin_bit_cast(uint4v, kv_widen8(a, b));
  uint4v w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t c = i < 2 ? a : b;
    const uint32_t lo = __builtin_bit_cast(uint32_t, (float)(int8_t)(c >> (16 * (i & 1))));
    const uint32_t hi = __builtin_bit_cast(uint32_t, (float)(int8_t)(c >> (16 * (i & 1) + 8)));
    w[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);   // the upper halves: exact for 8 bits
  }
  return w;
}

template <bool BF16>
__device__ __forceinline__ float16v mfma32(uint4v a, uint4v b, float16v c) {
  if (BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bhalf8, a),
                                                   __builtin_bit_cast(bhalf8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a),
                                                __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

template <int D, bool BF16, bool EVEN>
__global__ __launch_bounds__(64 * kPromptWaves<D>, kPromptWaves<D> / 4)
void mass_rows_kernel(KvPool pool, KvSeqs S, KvAttn A, int np, int shares, int64_t it0,
                      const float* lse) {
  constexpr int LR = D / 8, RC = 64 / LR;      // lanes a row, rows a load
  __shared__ __align__(16) uint16_t rows_of_wave[kPromptWaves<D>][32][D + 8];
  __shared__ float sums[kPromptWaves<D>][kPage];
  const int lane = threadIdx.x & 63, m = lane & 31, half = lane >> 5;
  const int wave = uniform(threadIdx.x >> 6), pages = kPromptWaves<D> / shares;
  const int share = wave / pages;
  const int64_t it = it0 + blockIdx.x;
  const int h = uniform((int)(it % pool.H));
  const int64_t r0 = it / pool.H;
  const int groups = (np + pages - 1) / pages;
  const int j = uniform((int)(r0 % groups) * pages + wave % pages), seq = uniform((int)(r0 / groups));
  const int pos0 = j * kPage;
  const RowsOf R = rows_of(S, A, seq);
  const int page = j < np && pos0 < R.len ? uniform(kv_page(S, pool.P, seq, j)) : -1;
  const int64_t at = (int64_t)page * pool.H + h;
  float sum[32];                     // 16 results of each 32-token tile
#pragma unroll
  for (int e = 0; e < 32; ++e) sum[e] = 0.0f;
  if (page >= 0) {
    const float f = A.scale * kLog2e * pool.ks[at];
    uint4v k[2][D / 16];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int8_t* row = pool.k + at * (kPage * D) + (32 * u + m) * D + 16 * half;
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        const uint4v c = *reinterpret_cast<const uint4v*>(row + 32 * s);
        k[u][2 * s] = widen_as<BF16>(c[0], c[1]);
        k[u][2 * s + 1] = widen_as<BF16>(c[2], c[3]);
      }
    }
    const int rows = (R.q_len > 0 ? R.q_len : 0) * A.group;
    // the tile of the first query token that sees the page
    const int64_t first = (int64_t)pos0 - R.len + R.q_len;
    int tile = first > 0 ? uniform((int)(first * A.group / 32)) : 0;
    tile += (share - tile % shares + shares) % shares;
    // Rows are moved on without divisions and products: `off` elements into the queries and place g
    // in the group. A lane loads its first row of the tile and those RC apart from it, and has the
    // results of row m.
    struct Place {
      int64_t off;
      int g;
      __device__ __forceinline__ void move(int64_t by, int dg, int group, int64_t wrap) {
        off += by;
        g += dg;
        const bool over = g >= group;
        off += over ? wrap : 0;
        g -= over ? group : 0;
      }
    };
    const int64_t wrap = A.q.tok - A.group * A.q.head, lse_tok = (int64_t)pool.H * A.group;
    const int step = 32 * shares, step_i = uniform(step / A.group), step_g = step - step_i * A.group;
    const int near_i = uniform(RC / A.group), near_g = RC - near_i * A.group;
    const int64_t step_off = step_i * A.q.tok + step_g * A.q.head;
    const int64_t near_off = near_i * A.q.tok + near_g * A.q.head;
    const int row_l = 32 * tile + lane / LR, row_m = 32 * tile + m;
    Place from = {(int64_t)(row_l / A.group) * A.q.tok + (int64_t)(row_l % A.group) * A.q.head,
                  row_l % A.group};
    int own_i = row_m / A.group, own_g = row_m % A.group;
    const uint16_t* const q0 = static_cast<const uint16_t*>(A.q.p) + R.seq * A.q.seq +
                               (int64_t)h * A.group * A.q.head + lane % LR * 8;
    const float* const lse0 = lse + (int64_t)R.seq * A.nq * lse_tok + h * A.group;
    constexpr int CH = 32 / RC;
    uint4v u[CH];
    float z;
    int see;
    // EVEN: a step is whole tokens, so the lane's offsets from the tile's first token stay
    const int step_first = EVEN ? uniform(32 * tile / A.group) : 0;
    const char* tile_q = reinterpret_cast<const char*>(q0 - lane % LR * 8 + step_first * A.q.tok);
    const float* tile_lse = lse0 + step_first * lse_tok;
    uint32_t q_off[CH], lse_off = 0;
    if constexpr (EVEN) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int row = row_l + c * RC, i = row / A.group;
        q_off[c] = (uint32_t)(((i - step_first) * A.q.tok + (row - i * A.group) * A.q.head +
                               lane % LR * 8) * 2);
      }
      lse_off = (uint32_t)((own_i - step_first) * lse_tok + own_g);
    }
    const auto fetch = [&](int t) {
      if constexpr (EVEN) {
        if (32 * t + 32 <= rows) {
#pragma unroll
          for (int c = 0; c < CH; ++c) u[c] = *reinterpret_cast<const uint4v*>(tile_q + q_off[c]);
          see = R.visible(own_i);
          z = tile_lse[lse_off];
        } else {                     // (behind the last row the tile's first, of no use)
#pragma unroll
          for (int c = 0; c < CH; ++c)
            u[c] = *reinterpret_cast<const uint4v*>(
                tile_q + (32 * t + c * RC + lane / LR < rows ? q_off[c] : 0u));
          const bool live = 32 * t + m < rows;
          see = live ? R.visible(own_i) : 0;
          z = tile_lse[live ? lse_off : 0u];
        }
        tile_q += step_off * 2;
        tile_lse += step_i * lse_tok;
        own_i += step_i;
        return;
      }
      const uint16_t* src[CH];
      Place p = from;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        // (behind the last row the first one, whose results are not used)
        src[c] = q0 + (32 * t + c * RC + lane / LR < rows ? p.off : 0);
        p.move(near_off, near_g, A.group, wrap);
      }
      if (A.wide_q) {
#pragma unroll
        for (int c = 0; c < CH; ++c) u[c] = load8(src[c], true);
      } else {
#pragma unroll
        for (int c = 0; c < CH; ++c) u[c] = load8(src[c], false);
      }
      const bool live = 32 * t + m < rows;
      see = live ? R.visible(own_i) : 0;
      z = lse0[live ? own_i * lse_tok + own_g : 0];
      from.move(step_off, step_g, A.group, wrap);
      own_i += step_i;
      own_g += step_g;
      if (own_g >= A.group) {
        own_g -= A.group;
        ++own_i;
      }
    };
    uint16_t(*const mine)[D + 8] = rows_of_wave[wave];
    if (32 * tile < rows) fetch(tile);
    for (; 32 * tile < rows; tile += shares) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
        *reinterpret_cast<uint4v*>(&mine[c * RC + lane / LR][lane % LR * 8]) = u[c];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // the other lanes' rows are read
      const float c0 = -z * kLog2e;
      const int seen = see;
      if (32 * (tile + shares) < rows) fetch(tile + shares);
      float16v x[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[t][e] = 0.0f;
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        const uint4v q = *reinterpret_cast<const uint4v*>(
            &mine[m][32 * (s >> 1) + 16 * half + 8 * (s & 1)]);
#pragma unroll
        for (int t = 0; t < 2; ++t) x[t] = mfma32<BF16>(k[t][s], q, x[t]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // before the next tile's overwrite them
      if (__any(seen < pos0 + kPage)) {          // some row sees the page in part or not at all
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][e], f, c0));
            sum[16 * t + e] += pos0 + 32 * t + 8 * (e >> 2) + 4 * half + (e & 3) < seen ? w : 0.0f;
          }
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            sum[16 * t + e] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][e], f, c0));
      }
    }
  }
  // over the 32 rows of a tile (lane m has result 16 t + e = m), then over the shares
  const float total = sum_across<32>(sum);
  sums[wave][32 * (m >> 4) + 8 * (m >> 2 & 3) + 4 * half + (m & 3)] = total;
  __syncthreads();
  if (share == 0 && page >= 0 && pos0 + lane < R.len) {
    float s = 0.0f;
    for (int w = 0; w < shares; ++w) s += sums[w * pages + wave][lane];
    const int64_t to = at * kPage + lane;
    A.mass_out[to] = A.mass_in ? __builtin_fmaf(A.decay, A.mass_in[to], s) : s;
  }
}

// ---- a shared context of many rows ----------------------------------------------------------------
// The rows of all requests of a context against its pages: prompt_kernel's products and weights, but
// no row sees less than the others, so only the context's last page is masked, and the V scales are
// taken relative to the power of two at the largest of the workgroup's pages (what is 2^-60 of it
// counts as none: its weights are summed apart, and must not move the reference that the others are
// rounded by).
//
// RW of the workgroup's waves have 32 rows each. With half of them the others take the same rows, and
// of every page the first tile of 32 tokens goes to the first half and the second to the other (32
// requests of four heads a group, 16K tokens: 29.5 -> 27.9 us); the halves' states meet in LDS. A split's
// pages are listed in LDS first, a column a thread, with their scales: a chain of lookups would be as
// long as a page's products. (So a split has at most a column a thread.)
//
// Weights go to V's product as fp16, 2^-11 of a weight, and bf16 rows to K's under a power of two each:
// the codes have 8 bits, and products of 32-bit operands a sixteenth of the rate. Sums are 32-bit.
//
// Those 32 requests take 25 us now: 6 until the first products, 1.4 for each of a workgroup's 8 pages, 3
// for the halves and the states' way out. Of a page's 3360 cycles the two waves of a SIMD take half to
// issue their vector instructions (142 each, 4 cycles, and 16 exponentials, 16 cycles); the rest is the
// order of its steps: products, weights, products, a barrier. 448 queries over four times 1500 tokens, 16
// heads of 64 channels: 29 us, 380 TFLOP/s; a page of shorter products takes 0.75 us, 1800 cycles, of
// which those instructions (140 and 16) are 1630, a third of them the exponentials; 10 us are its ends.
template <int D>
struct PageList {
  static constexpr int kColumns = 64 * kPromptWaves<D>;
  int page[kColumns], column[kColumns];
  float ks[kColumns], vs[kColumns];
  int count[kPromptWaves<D>];
  float top[kPromptWaves<D>];
};

template <int D, bool BF16, int RW>
__global__ __launch_bounds__(64 * kPromptWaves<D>, kPromptWaves<D> / 4)
void shared_kernel(KvPool pool, KvSeqs S, KvAttn A, KvUsers U, KvTiles T, KvTiles small, int splits,
                   int tile0, int p0, float* part, float* lse) {
  constexpr int W = kPromptWaves<D>, NT = 64 * W, TW = W / RW;
  constexpr int kAhead = kPagesK<D> - 1;
  static_assert(TW == 1 || (TW == 2 && kAhead == 2), "a tile of every page for each half");
  __shared__ PromptLds<D> L;
  __shared__ PageList<D> list;
  const int lane = threadIdx.x & 63, m = lane & 31, half = lane >> 5;
  const int wave = uniform(threadIdx.x >> 6), side = wave / RW;
  // Which 32 rows: the halves' waves of the same rows lie on different SIMDs, so that 64 rows keep all
  // four busy (two contexts of 16K, 64 rows of 8 heads, kernels' us: 41.7 -> 39.0; four of 8K, 40 rows
  // 37.8 -> 35.0).
  const int band = (wave + side * (RW / 2)) % RW;
  const int split = blockIdx.x / pool.H, h = blockIdx.x - split * pool.H;
  int tile = tile0 + blockIdx.y, p = p0 + blockIdx.z;
  if (T.each == 0) {
    p = context_at(T, U, tile, tile);
    if (p < 0) return;
  }

  const Requests req = requests_of(U, p);
  int len = A.lengths[p];
  len = len < A.max_len ? len : A.max_len;
  len = uniform(len > 0 ? len : 0);
  const int first = uniform(req.first), count = uniform(req.count);
  if (!part && tile == 0) fill_without<NT>(A, U, S.n, p, pool.H, D, blockIdx.x, gridDim.x, lse);
  const int per_user = U.rows, rows = count * per_user, r0 = tile * (32 * RW);
  if (tile < 0 || r0 >= rows) return;                  // (nobody's rows)
  // this split's state of the context's first tile, and those of the next tiles behind it
  const int64_t step = (int64_t)pool.H * splits;
  const int64_t u16 = tiles_before(small, U, p, first) * step + h * splits + split;
  const int columns = (int)(((int64_t)len + kPage - 1) / kPage);
  const int per = (columns + splits - 1) / splits;
  const int j0 = split * per, j1 = j0 + per < columns ? j0 + per : columns;

  // the split's pages, a column a thread
  int n = 0;
  float v_most = 0.0f;
  {
    const int j = j0 + (int)threadIdx.x;
    const int page = j < j1 ? kv_page(S, pool.P, p, j) : -1;
    const int64_t at = (int64_t)(page >= 0 ? page : 0) * pool.H + h;
    const float ks = pool.ks[at], vs = pool.vs[at];
    const uint64_t there = __ballot(page >= 0);
    float top = page >= 0 && vs < __builtin_inff() ? vs : 0.0f;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) {
      list.count[wave] = __popcll(there);
      list.top[wave] = top;
    }
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int c = list.count[w];
      before += w < wave ? c : 0;
      n += c;
      v_most = fmaxf(v_most, list.top[w]);
    }
    if (page >= 0) {
      const int i = before + __popcll(there & ((1ull << lane) - 1));
      list.page[i] = page;
      list.column[i] = j;
      list.ks[i] = ks;
      list.vs[i] = vs;
    }
    __syncthreads();
    n = uniform(n);
    v_most = __builtin_bit_cast(float, uniform(__builtin_bit_cast(int, v_most)));
  }

  // the first pages' codes are on their way while the rows are read
  PageRegs<D, NT> kr, vr, k_first, v_first, k_second;
  const auto fetch = [&](const int8_t* codes, int i, PageRegs<D, NT>& r) {
    if (i < n) page_fetch<D, NT>(codes + ((int64_t)uniform(list.page[i]) * pool.H + h) * (kPage * D), r);
  };
  fetch(pool.k, 0, k_first);
  fetch(pool.v, 0, v_first);
  if (kAhead == 2) fetch(pool.k, 1, k_second);
  fetch(pool.v, 1, vr);
  fetch(pool.k, kAhead, kr);

  // this lane's row
  const int row = r0 + band * 32 + m;
  const int user = row / per_user, of_user = row - user * per_user;
  const int i_row = of_user / A.group, head = h * A.group + of_user - i_row * A.group;
  const int64_t b = first + user;
  bool alive = user < count && len > 0;
  if (alive && A.q_lens) alive = i_row < A.q_lens[b];
  half8 q[D / 16];
  const float unit = load_row32<D, BF16>(
      A, static_cast<const uint16_t*>(A.q.p) + b * A.q.seq + (int64_t)i_row * A.q.tok +
             (int64_t)head * A.q.head, alive, q);

  float16v o[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.0f;
  float ref = -1e30f, l = 0.0f;      // O and l in units of 2^(ref - kLift), O also of 2^v_exp
  float ref0 = -1e30f, l0 = 0.0f;    // l of the pages without V, in units of 2^ref0
  const int v_exp = __builtin_amdgcn_frexp_expf(v_most);         // (0 of 0)

  // One tile of 32 tokens: see prompt_kernel.
  const auto tile_step = [&](float16v x, const _Float16 (*k)[D + 8], const _Float16 (*next)[D + 8],
                             const _Float16 (*v)[kPage + 8], int pos0, float ks, float vs,
                             auto put) -> float16v {
    const bool cut = pos0 + 32 > len;
    const int seen_here = len - pos0 - 16 * half;
    const auto mask = [&](float16v& z, float to) {
      if (cut) {
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = e < seen_here ? z[e] : to;
      }
    };
    const float f = unit * ks, ratio = __builtin_ldexpf(vs, -v_exp);
    const bool with_v = !(ratio <= 0x1p-60f);
    const float lv = with_v ? __builtin_amdgcn_logf(ratio) + (float)kLift : 0.0f;
    const float c = with_v ? lv - ref : kNegInf;
    const float16v y = tile_scores<D>(next, q);
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], f, c));
    mask(x, 0.0f);
#pragma unroll
    for (int e = 0; e < 16; ++e) sum += x[e];
    if (__builtin_expect(__any(!(sum <= kMost)) || !with_v, 0)) {
      float g;
      if (with_v && !__any(!(sum < __builtin_inff()))) {
        float t = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) t = max2(t, x[e]);
        const int up = __builtin_amdgcn_frexp_expf(half_max(t)) - kLift;
        const int by = up > 0 ? up : 0;
        g = __builtin_ldexpf(1.0f, -by);
        ref += (float)by;
        sum *= g;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= g;
      } else {
        x = tile_scores<D>(k, q);
        float t = kNegInf;
#pragma unroll
        for (int e = 0; e < 16; ++e) t = max2(t, !cut || e < seen_here ? x[e] : kNegInf);
        t = half_max(t);
        t = t == kNegInf ? t : t * f;
        const float was = with_v ? ref : ref0;
        const float now = fmaxf(was, with_v ? t + lv - (float)kLift : t);
        g = __builtin_amdgcn_exp2f(was - now);
        const float by = with_v ? lv - now : -now;
        sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], f, by));
        mask(x, 0.0f);
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += x[e];
        if (with_v) {
          ref = now;
        } else {
          ref0 = now;
          l0 = __builtin_fmaf(l0, g, sum);
          g = 1.0f;
          sum = 0.0f;
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = 0.0f;
        }
      }
      l *= g;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= g;
    }
    half8 a[D / 32][2];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        a[dt][e] = *reinterpret_cast<const half8*>(&v[32 * dt + m][16 * half + 8 * e]);
    l = sum == 0.0f ? l : __builtin_fmaf(sum, __builtin_amdgcn_rcpf(ratio), l);
    half8 w[2];
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const half2v h2 = __builtin_convertvector((float2v{x[e], x[e + 1]}), half2v);
      w[e >> 3][e & 7] = h2[0];
      w[e >> 3][(e & 7) + 1] = h2[1];
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[dt][e], w[e], o[dt], 0, 0, 0);
    put();
    return y;
  };

  // The listed pages in turn; what a page's turn does besides its tiles is prompt_kernel's. A wave
  // without a live row only helps with the pages.
  const auto walk = [&](auto busy) {
    constexpr bool kBusy = decltype(busy)::value;
    float16v x;
    const auto step = [&](const _Float16 (*k)[D + 8], const _Float16 (*next)[D + 8],
                          const _Float16 (*v)[kPage + 8], int pos0, float ks, float vs, auto put) {
      if constexpr (kBusy) x = tile_step(x, k, next, v, pos0, ks, vs, put);
      else put();
    };
    const auto second = [&](int buf) {
      return reinterpret_cast<const _Float16 (*)[kPage + 8]>(&L.v[buf][0][32]);
    };
    // (behind the last page the registers and buffers hold anything, and nobody uses it)
    widen_k<D, NT>(k_first, L.k[0]);
    widen_v<D, NT>(v_first, L.v[0]);
    if (kAhead == 2) widen_k<D, NT>(k_second, L.k[1]);
    __syncthreads();
    if constexpr (kBusy) {
      // the first tile's largest score is the first reference (with a V scale that counts)
      x = tile_scores<D>(L.k[0] + 32 * side, q);
      const float ratio = __builtin_ldexpf(list.vs[0], -v_exp);
      const int seen = len - uniform(list.column[0]) * kPage - 32 * side - 16 * half;
      float t = kNegInf;
#pragma unroll
      for (int e = 0; e < 16; ++e) t = max2(t, e < seen ? x[e] : kNegInf);
      t = half_max(t) * (unit * list.ks[0]) + __builtin_amdgcn_logf(ratio);
      if (ratio > 0x1p-60f && t > -1e30f && t < 1e30f) ref = t;
    }
    int k0 = 0, k1 = 1;                // K buffers of this page and the next
    for (int i = 0; i < n; ++i) {
      const int buf = i & 1, k2 = kAhead == 2 ? 3 - k0 - k1 : k0;
      const int pos0 = uniform(list.column[i]) * kPage;
      const float ks = list.ks[i], vs = list.vs[i];
      if constexpr (TW == 2) {
        step(L.k[k0] + 32 * side, L.k[k1] + 32 * side, side ? second(buf) : L.v[buf],
             pos0 + 32 * side, ks, vs, [&] {
               widen_k<D, NT>(kr, L.k[k2]);
               widen_v<D, NT>(vr, L.v[buf ^ 1]);
             });
        fetch(pool.k, i + 3, kr);
      } else {
        step(L.k[k0], L.k[k0] + 32, L.v[buf], pos0, ks, vs,
             [&] { widen_k<D, NT>(kr, L.k[kAhead == 2 ? k2 : k1]); });
        fetch(pool.k, i + kAhead + 1, kr);
        if (kAhead == 1) __syncthreads();
        step(L.k[k0] + 32, L.k[k1], second(buf), pos0 + 32, ks, vs,
             [&] { widen_v<D, NT>(vr, L.v[buf ^ 1]); });
      }
      fetch(pool.v, i + 2, vr);
      k0 = k1;
      k1 = k2;
      __syncthreads();
    }
  };
  if (n > 0) {
    if (__any(alive)) walk(std::true_type{});
    else walk(std::false_type{});
  }

  // Both sums to one reference, and O with them; then the halves' states to one.
  l = half_sum(l);
  l0 = half_sum(l0);
  const float l_ref = ref - (float)kLift;
  const bool some = l > 0.0f || l != l, some0 = l0 > 0.0f || l0 != l0;
  bool empty = !alive || !(some || some0);
  float top = fmaxf(some ? l_ref : -1e30f, some0 ? ref0 : -1e30f);
  const float to_top = some ? __builtin_amdgcn_exp2f(l_ref - top) : 0.0f;
  float sum = l * to_top + (some0 ? l0 * __builtin_amdgcn_exp2f(ref0 - top) : 0.0f);
  top = empty ? kNegInf : top;
  sum = empty ? 0.0f : sum;
  // The sum goes to [1/2, 1) by a power of two before O gets the V scales' own: then O is at most the
  // largest |V|, and a number wherever the result is one. (The weights' unit is 2^-kLift, and there are
  // as many as tokens: of V at 1e33 their sum would pass 32 bits.)
  const int by = __builtin_amdgcn_frexp_expf(sum);               // (0 of 0)
  top += (float)by;
  sum = __builtin_ldexpf(sum, -by);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e)
      o[dt][e] = empty ? 0.0f : __builtin_ldexpf(o[dt][e] * to_top, v_exp - by);
  float* const space = reinterpret_cast<float*>(&L);
  float (*const all)[D + 4] = reinterpret_cast<float (*)[D + 4]>(space);       // halves: [32 RW]
  if constexpr (TW == 2) {
    float (*const os)[D + 4] = all + band * 32;
    float2v* const ml = reinterpret_cast<float2v*>(space + 32 * RW * (D + 4)) + band * 32;
    static_assert(sizeof(PromptLds<D>) >= 32 * RW * (D + 6) * sizeof(float), "a half's rows");
    if (side) {
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int a = 0; a < 4; ++a)
          *reinterpret_cast<float4v*>(&os[m][32 * dt + 8 * a + 4 * half]) =
              float4v{o[dt][4 * a], o[dt][4 * a + 1], o[dt][4 * a + 2], o[dt][4 * a + 3]};
      if (half == 0) ml[m] = float2v{top, sum};
    }
    __syncthreads();
    if (!side) {
      const float2v other = ml[m];
      const float both = fmaxf(top, other[0]), base = both == kNegInf ? 0.0f : both;
      // (halved, so that the sum stays below 1)
      float f0 = 0.5f * __builtin_amdgcn_exp2f(top - base);
      float f1 = 0.5f * __builtin_amdgcn_exp2f(other[0] - base);
      sum = sum * f0 + other[1] * f1;
      top = both + 1.0f;
      if (!part) {
        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
        f0 *= inv;
        f1 *= inv;
      }
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          float4v* const w = reinterpret_cast<float4v*>(&os[m][32 * dt + 8 * a + 4 * half]);
          float4v y = *w;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = o[dt][4 * a + e] * f0 + y[e] * f1;
          *w = y;
        }
    }
  }
  if (TW == 2 && side) {
    // (the first half's)
  } else if (part) {
    if (half == 0 && row < rows) {
      *reinterpret_cast<float2v*>(part + (u16 + row / 16 * step) * kPart<D> + 16 * D +
                                  2 * (row & 15)) = float2v{top, sum};
    }
  } else {
    if constexpr (TW == 1) {
      const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= inv;
    }
    if (lse && half == 0 && user < count)
      lse[(b * U.per + i_row) * ((int64_t)pool.H * A.group) + head] =
          (top + __builtin_amdgcn_logf(sum)) * kLn2;
  }
  // the rows leave by way of LDS: a lane has pieces of one row, and a store should have whole ones
  const auto leave = [&](int to, int d, const float4v& w) {
    if (part) {
      if (to >= rows) return;
      *reinterpret_cast<float4v*>(part + (u16 + to / 16 * step) * kPart<D> + (to & 15) * D + d) =
          w;
    } else {
      const int user_to = to / per_user, of = to - user_to * per_user;
      if (user_to >= count) return;
      const int i_to = of / A.group, head_to = h * A.group + of - i_to * A.group;
      uint16_t* const dst = static_cast<uint16_t*>(A.out.p) +
                            (int64_t)(first + user_to) * A.out.seq + (int64_t)i_to * A.out.tok +
                            (int64_t)head_to * A.out.head + d;
#pragma unroll
      for (int e = 0; e < 4; ++e) dst[e] = kv_narrow<BF16>(w[e]);
    }
  };
  if constexpr (TW == 2) {
    __syncthreads();
    constexpr int LR = D / 4;                            // threads a row
#pragma unroll 2
    for (int in = threadIdx.x / LR; in < 32 * RW; in += NT / LR) {
      const int d = threadIdx.x % LR * 4;
      leave(r0 + in, d, *reinterpret_cast<const float4v*>(&all[in][d]));
    }
  } else {
    // (a wave's own rows, half of the channels at a time: there is no more room)
    constexpr int C = D / 2, LR = C / 4, RC = 64 / LR;   // channels; lanes a row, rows a store
    float (*const mine)[C + 4] = reinterpret_cast<float (*)[C + 4]>(space) + wave * 32;
    static_assert(sizeof(PromptLds<D>) >= W * 32 * (C + 4) * sizeof(float), "all waves' rows");
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int dt = 0; dt < D / 64; ++dt)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const float16v& from = o[c * (D / 64) + dt];
          *reinterpret_cast<float4v*>(&mine[m][32 * dt + 8 * a + 4 * half]) =
              float4v{from[4 * a], from[4 * a + 1], from[4 * a + 2], from[4 * a + 3]};
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
      for (int in = lane / LR; in < 32; in += RC) {
        const int d = lane % LR * 4;
        leave(r0 + wave * 32 + in, c * C + d, *reinterpret_cast<const float4v*>(&mine[in][d]));
      }
    }
  }
}

// ---- states joined ----------------------------------------------------------------------------
struct JoinLds {
  float w[2 * kMostSplits * 16];
  float4v sums[256];
};

// kJoin of attend_kernel by a single wave: of a short answer three waves of four would have no page, and
// hold their registers all the same (see one_wave).
template <int D, bool BF16>
__global__ __launch_bounds__(64, D == 256 ? 1 : 2) void own_join_kernel(KvPool pool, KvSeqs S, KvAttn A,
                                                       KvUsers U, int tiles, int64_t items,
                                                       ContextStates C, float* lse) {
  __shared__ float os[16][D + 4];
  __shared__ float ml[32], own_f[16], w[kMostSplits * 16];
  const int lane = threadIdx.x, m = lane & 15, g = lane >> 4;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int tile = (int)(it % tiles);
    const int64_t r = it / tiles;
    const int h = (int)(r % pool.H);
    const RowsOf R = rows_of(S, A, (int)(r / pool.H));
    const int all = R.nq * A.group, rows = all - tile * 16 < 16 ? all - tile * 16 : 16;
    const int most = R.most(tile * 16 / A.group, (tile * 16 + rows - 1) / A.group);
    const int n = (most + kPage - 1) / kPage;
    int at = 0;
    const auto next_page = [&](int& j) -> int64_t {
      while (j < n) {
        at = j++;
        const int page = kv_page(S, pool.P, R.seq, at);
        if (page >= 0) return (int64_t)page * pool.H + h;
      }
      return -1;
    };
    int j = 0;
    int64_t b = next_page(j);
    KRegs<D> K;
    VRegs<D> V;
    if (b >= 0) {
      load_k<D>(pool.k + b * (kPage * D), K);
      load_v<D>(pool.v + b * (kPage * D), V);
    }
    QTile<D> Q;
    load_q<D, BF16>(A, R, h, tile, Q);
    int place = 0, tile0 = 0;
    const int context = uniform(context_of(U, C.tiles, R.seq, place, tile0));
    Acc<D> acc;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc.o[dt] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    acc.m = kNegInf;
    acc.l = 0.0f;
    while (b >= 0) {
      const float ks = pool.ks[b], vs = pool.vs[b];
      const int pos0 = at * kPage;
      float x[16], keep;
      half8 p[2];
      const int64_t bn = next_page(j);
      page_scores<D>(K, Q, x);
      if (bn >= 0) load_k<D>(pool.k + bn * (kPage * D), K);
      const float f = page_softmax<D>(x, ks, pos0, Q, acc, p, keep, nullptr);
      page_values<D>(V, p, keep, f == 0.0f ? 0.0f : f * vs, acc);
      if (bn >= 0) load_v<D>(pool.v + bn * (kPage * D), V);
      b = bn;
    }
    acc.l = quad_sum(acc.l);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
      *reinterpret_cast<float4v*>(&os[m][16 * dt + 4 * g]) = acc.o[dt];
    if (g == 0) {
      ml[m] = acc.m;
      ml[16 + m] = acc.l;
    }
    __syncthreads();
    // four lanes a row find the factors of the context's states and of the own one
    const int n0 = context >= 0 ? C.splits : 0, from = place * all + tile * 16;
    const float* const s0 = C.from<D>(h, uniform(tile0));
    const auto state = [&](int i, int x, int& in) -> const float* {
      in = (from + x) & 15;
      return s0 + (((from + x) >> 4) * C.step + i) * kPart<D>;
    };
    const int row = lane >> 2, sub = lane & 3;
    float top = sub == 0 ? ml[row] : kNegInf, l = sub == 0 ? ml[16 + row] : 0.0f;
    if (row < rows) {
      for (int i = sub; i < n0; i += 4) {
        int in;
        const float* const s = state(i, row, in);
        const float2v x = *reinterpret_cast<const float2v*>(s + 16 * D + 2 * in);
        w[i * 16 + row] = x[0];
        const float both = fmaxf(top, x[0]), ref = both == kNegInf ? 0.0f : both;
        l = l * __builtin_amdgcn_exp2f(top - ref) + x[1] * __builtin_amdgcn_exp2f(x[0] - ref);
        top = both;
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      const float y = __shfl_xor(top, o), x = __shfl_xor(l, o);
      const float both = fmaxf(top, y), ref = both == kNegInf ? 0.0f : both;
      l = l * __builtin_amdgcn_exp2f(top - ref) + x * __builtin_amdgcn_exp2f(y - ref);
      top = both;
    }
    if (row < rows) {
      const float ref = top == kNegInf ? 0.0f : top, inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
      for (int i = sub; i < n0; i += 4)
        w[i * 16 + row] = __builtin_amdgcn_exp2f(w[i * 16 + row] - ref) * inv;
      if (sub == 0) {
        own_f[row] = __builtin_amdgcn_exp2f(ml[row] - ref) * inv;
        put_lse(A, R, pool.H, h, tile * 16 + row, lse, (top + __builtin_amdgcn_logf(l)) * kLn2);
      }
    }
    __syncthreads();
    constexpr int kAhead = 4;
    for (int e = lane; e < rows * (D / 4); e += 64) {
      const int x = e / (D / 4), d = e % (D / 4) * 4;
      float4v o = *reinterpret_cast<const float4v*>(&os[x][d]);
      const float f0 = own_f[x];
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] *= f0;
      for (int i0 = 0; i0 < n0; i0 += kAhead) {
        float4v v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          int in;
          const float* const s = state(i0 + k < n0 ? i0 + k : n0 - 1, x, in);
          v[k] = *reinterpret_cast<const float4v*>(s + in * D + d);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const float f = i0 + k < n0 ? w[(i0 + k) * 16 + x] : 0.0f;
#pragma unroll
          for (int c = 0; c < 4; ++c) o[c] = __builtin_fmaf(v[k][c], f, o[c]);
        }
      }
      put_out<D, BF16>(A, R, h, tile * 16 + x, d, reinterpret_cast<const float*>(&o), 4);
    }
    __syncthreads();
  }
}

// A context's states alone: a tile of T (a few rows) a workgroup. Bound by the states' bytes.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void contexts_join_kernel(KvPool pool, KvSeqs S, KvAttn A, KvUsers U,
                                                            KvTiles T, int64_t items,
                                                            ContextStates C, float* lse) {
  __shared__ JoinLds L;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int h = (int)(it % pool.H);
    int tile;
    const int p = context_at(T, U, (int)(it / pool.H), tile);
    if (p < 0 || tile < 0) continue;
    const SharedRows R = rows_of(S, A, U, p);
    const int first = tile * T.size, left = R.q_len * A.group - first;
    const int rows = left < T.size ? left : T.size;
    if (rows <= 0) continue;
    const float* const s0 = C.from<D>(h, tiles_before(C.tiles, U, p, R.first));
    float top = kNegInf, l = 0.0f;
    join_rows<D>(rows, C.splits, L.w, L.sums, top, l, [&](int i, int x, int& in) {
      in = (first + x) & 15;
      return s0 + (((first + x) >> 4) * C.step + i) * kPart<D>;
    }, [](float) {}, [&](int x, int d, const float4v& o) {
      put_out<D, BF16>(A, R, h, first + x, d, reinterpret_cast<const float*>(&o), 4);
    });
    if ((threadIdx.x & 15) == 0 && (int)(threadIdx.x >> 4) < rows)
      put_lse(A, R, pool.H, h, first + (threadIdx.x >> 4), lse,
              (top + __builtin_amdgcn_logf(l)) * kLn2);
    __syncthreads();
  }
  // requests without a context
  for (int64_t e = blockIdx.x; e < (int64_t)S.n * pool.H; e += gridDim.x)
    fill_without<256>(A, U, S.n, (int)(e / pool.H), pool.H, D, (int)(e % pool.H), pool.H, lse);
}

// A context's states and those of a request's own tokens: a workgroup a request's 16-row tile. The
// context's states of the tile lie in rows of its own tiles, from the request's first on.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void shared_join_kernel(KvPool pool, KvSeqs S, KvAttn A, KvUsers U,
                                                          int tiles, int splits, int64_t items,
                                                          ContextStates C, const float* part,
                                                          float* lse) {
  __shared__ JoinLds L;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int tile = (int)(it % tiles);
    const int64_t r = it / tiles;
    const int h = (int)(r % pool.H);
    const RowsOf R = rows_of(S, A, (int)(r / pool.H));
    const int all = R.nq * A.group, rows = all - tile * 16 < 16 ? all - tile * 16 : 16;
    int place = 0, tile0 = 0;
    const int p = context_of(U, C.tiles, R.seq, place, tile0);
    const int n0 = p >= 0 ? C.splits : 0, from = place * all + tile * 16;
    const float* const s0 = C.from<D>(h, uniform(tile0));
    float top = kNegInf, l = 0.0f;
    join_rows<D>(rows, n0 + splits, L.w, L.sums, top, l, [&](int i, int x, int& in) {
      if (i < n0) {
        in = (from + x) & 15;
        return s0 + (((from + x) >> 4) * C.step + i) * kPart<D>;
      }
      in = x;
      return part + (it * splits + (i - n0)) * kPart<D>;
    }, [](float) {}, [&](int x, int d, const float4v& o) {
      put_out<D, BF16>(A, R, h, tile * 16 + x, d, reinterpret_cast<const float*>(&o), 4);
    });
    if ((threadIdx.x & 15) == 0 && (int)(threadIdx.x >> 4) < rows)
      put_lse(A, R, pool.H, h, tile * 16 + (threadIdx.x >> 4), lse,
              (top + __builtin_amdgcn_logf(l)) * kLn2);
    __syncthreads();
  }
}

unsigned grid_of(int64_t items) { return (unsigned)(items < (1 << 22) ? items : (1 << 22)); }

// Kernels of one workgroup per item: as many launches as keep each below 2^32 threads.
template <class Launch>
void in_launches(int64_t items, Launch launch) {
  constexpr int64_t kMost = 1 << 22;
  for (int64_t it0 = 0; it0 < items; it0 += kMost)
    launch(it0, (unsigned)(items - it0 < kMost ? items - it0 : kMost));
}

template <int D, bool BF16>
void prompt_d(const KvPool& pool, const KvSeqs& S, const KvAttn& A, const KvAttnPlan& P,
              float* part, float* lse, hipStream_t st) {
  in_launches((int64_t)S.n * pool.H * P.big * P.splits, [&](int64_t it0, unsigned n) {
    hipLaunchKernelGGL((prompt_kernel<D, BF16>), dim3(n), dim3(64 * kPromptWaves<D>), 0, st, pool,
                       S, A, P.big, P.splits, it0, part, lse);
  });
}

template <int D, bool BF16>
void mass_rows_d(const KvPool& pool, const KvSeqs& S, const KvAttn& A, int np, const float* lse,
                 hipStream_t st) {
  // a wave a page where that makes two for every SIMD, else several share a page's rows (whole calls of
  // 500 queries, 32 heads on 8 of 128 channels, us with 1, 2, 4 and 8 shares: 2K tokens, 256 items, 119
  // 83 66 58; 4K 130 95 81 84; 8K 160 130 135 143; 16K 234 236 249 266; of 100 queries 4K 56 47 45 51)
  const int64_t items = (int64_t)S.n * pool.H * np;
  int shares = items >= 2048 ? 1 : items >= 1024 ? 2 : items >= 512 ? 4 : 8;
  if (shares > kPromptWaves<D>) shares = kPromptWaves<D>;
  const int pages = kPromptWaves<D> / shares;
  // Where a wave's step from tile to tile is whole tokens, it moves on by one addition of a uniform
  // base and its loads need no addresses of their own: 500 queries of 32 heads over 4K 31.5 us, 34.9
  // with every row's place followed. (Offsets within a tile fit 32 bits.)
  const bool even = 32 * shares % A.group == 0 && A.wide_q && A.q.tok >= 0 && A.q.head >= 0 &&
                    A.q.tok < 1 << 24 && A.q.head < (1 << 30) / A.group;
  in_launches((int64_t)S.n * pool.H * ((np + pages - 1) / pages), [&](int64_t it0, unsigned n) {
    if (even)
      hipLaunchKernelGGL((mass_rows_kernel<D, BF16, true>), dim3(n), dim3(64 * kPromptWaves<D>), 0,
                         st, pool, S, A, np, shares, it0, lse);
    else
      hipLaunchKernelGGL((mass_rows_kernel<D, BF16, false>), dim3(n), dim3(64 * kPromptWaves<D>), 0,
                         st, pool, S, A, np, shares, it0, lse);
  });
}

template <int D, bool BF16>
hipError_t attend_d(const KvPool& pool, const KvSeqs& S, const KvAttn& A, void* ws,
                    hipStream_t st) {
  const KvAttnPlan P = cg_kv8_plan(pool, S, A, D);
  char* base = static_cast<char*>(ws);
  float* part = reinterpret_cast<float*>(base + P.part_off);
  float* lse = A.lse ? A.lse : A.mass_out ? reinterpret_cast<float*>(base + P.lse_off) : nullptr;
  float* scores = P.keep_scores ? reinterpret_cast<float*>(base + P.score_off) : nullptr;
  const int np = (int)(((int64_t)A.max_len + kPage - 1) / kPage);
  const int vseqs = A.picks ? S.n * A.nq : S.n;
  const int64_t units = (int64_t)vseqs * pool.H * P.tiles;
  if (P.big)
    prompt_d<D, BF16>(pool, S, A, P, P.splits > 1 ? part : nullptr, lse, st);
  else
    hipLaunchKernelGGL((attend_kernel<D, BF16, RowsOf, kOut>), dim3(grid_of(units * P.splits)),
                       dim3(256), 0, st, pool, S, A, KvUsers{}, P.tiles, P.splits,
                       units * P.splits, part, reinterpret_cast<uint32_t*>(base), lse, scores, np,
                       ContextStates{});
  if (P.splits > 1 && P.big)
    hipLaunchKernelGGL((join_kernel<D, BF16>), dim3(grid_of(units)), dim3(256), 0, st, pool, S, A,
                       P.tiles, P.splits, units, part, lse);
  if (A.mass_out && np) {
    const int64_t items = (int64_t)S.n * pool.H * np;
    if (P.many)
      mass_rows_d<D, BF16>(pool, S, A, np, lse, st);
    else if (P.keep_scores)
      hipLaunchKernelGGL(mass_scores_kernel, dim3(grid_of((items + 3) / 4)), dim3(256), 0, st, pool,
                         S, A, np, items, scores, lse);
    else
      hipLaunchKernelGGL((mass_kernel<D, BF16>), dim3(grid_of((items + 3) / 4)), dim3(256), 0, st,
                         pool, S, A, P.tiles, np, items, lse);
  }
  return hipGetLastError();
}

// shared_kernel over all contexts and tiles, in launches below 2^32 threads and inside the grid's
// limits. part null: the result.
template <int D, bool BF16>
void shared_rows_d(const KvPool& pool, const KvSeqs& C, const KvAttn& CA, const KvUsers& U,
                   const KvSharedPlan& P, float* part, float* lse, hipStream_t st) {
  constexpr int W = kPromptWaves<D>, kMost = 1 << 22, kSide = 65535;
  const int splits = P.shared.splits, x = pool.H * splits;
  // (tiles of contexts one after the other: one dimension for them all)
  const int all_y = P.big.each ? P.big.each : P.big.all, all_z = P.big.each ? C.n : 1;
  const auto at_most = [](int n, int most) { return n < most ? n : most < 1 ? 1 : most; };
  const int tiles = at_most(all_y, kMost / x < kSide ? kMost / x : kSide);
  const int contexts = at_most(all_z, kMost / x / tiles < kSide ? kMost / x / tiles : kSide);
  for (int p0 = 0; p0 < all_z; p0 += contexts)
    for (int tile0 = 0; tile0 < all_y; tile0 += tiles) {
      const dim3 grid((unsigned)x, (unsigned)at_most(all_y - tile0, tiles),
                      (unsigned)at_most(all_z - p0, contexts));
      if constexpr (D < 256)
        if (P.shared.halves) {
          hipLaunchKernelGGL((shared_kernel<D, BF16, W / 2>), grid, dim3(64 * W), 0, st, pool, C, CA,
                             U, P.big, P.small, splits, tile0, p0, part, lse);
          continue;
        }
      hipLaunchKernelGGL((shared_kernel<D, BF16, W>), grid, dim3(64 * W), 0, st, pool, C, CA, U,
                         P.big, P.small, splits, tile0, p0, part, lse);
    }
}

// (see KvTiles)
KvTiles tiles_of(const KvUsers& U, int size) {
  const int64_t each = ((int64_t)U.most * U.rows + size - 1) / size, even = each * U.contexts;
  const int64_t all = (int64_t)U.n_seq * U.rows / size + U.contexts;
  return even <= all ? KvTiles{size, (int32_t)each, (int32_t)even} : KvTiles{size, 0, (int32_t)all};
}

// Whether a wave alone takes a request's own tokens: few pages, or requests enough (one wave / four,
// us, 8 heads of 128 channels, behind a context of 1000: 32 requests of a page 6.9 / 8.6, 128 8.9 / 17.7;
// of 5 pages 64 requests 17.8 / 17.2, 128 21.4 / 30.6; of 16 pages 64 41 / 30, 128 50 / 57, 256 101 / 121;
// 512 requests of 20 rows and a page 56 / 150. 64 channels, 4 pages: 64 10.2 / 9.8, 128 11.7 / 18.3; 256:
// 64 23 / 27).
bool one_wave(int64_t units, int max_len) { return max_len <= 2 * kPage || units >= 768; }

template <int D, bool BF16>
hipError_t shared_d(const KvPool& pool, const KvSeqs& C, const KvAttn& CA, const KvUsers& U,
                    const KvSeqs& S, const KvAttn& A, void* ws, hipStream_t st) {
  const KvSharedPlan P = cg_kv8_shared_plan(pool, C, CA, U, S, A, D);
  char* base = static_cast<char*>(ws);
  float* const part0 = reinterpret_cast<float*>(base + P.shared_off);
  const int64_t units0 = (int64_t)pool.H * P.small.all;
  const int splits0 = P.shared.splits;
  const ContextStates states = {P.small, splits0, (int64_t)pool.H * splits0, part0};
  if (P.own.tiles == 0) {
    // the context alone
    if (P.shared.big) {
      shared_rows_d<D, BF16>(pool, C, CA, U, P, splits0 > 1 ? part0 : nullptr, A.lse, st);
      if (splits0 > 1) {
        // (16 rows a workgroup where that makes enough of them; 4 rows / 16, us with shared_kernel: 128
        // rows of 8 heads in 32 splits 32.2 / 34.6, 200 of 32 heads and two contexts 52.8 / 49.0)
        const KvTiles few = tiles_of(U, units0 < 512 ? 4 : 16);
        const int64_t items = (int64_t)pool.H * few.all;
        hipLaunchKernelGGL((contexts_join_kernel<D, BF16>), dim3(grid_of(items)), dim3(256), 0, st,
                           pool, C, CA, U, few, items, states, A.lse);
      }
    } else {
      hipLaunchKernelGGL((attend_kernel<D, BF16, SharedRows, kOut>),
                         dim3(grid_of(units0 * splits0)), dim3(256), 0, st, pool, C, CA, U,
                         0, splits0, units0 * splits0, part0, reinterpret_cast<uint32_t*>(base),
                         A.lse, nullptr, 0, states);
    }
    return hipGetLastError();
  }
  if (P.shared.big)
    shared_rows_d<D, BF16>(pool, C, CA, U, P, part0, nullptr, st);
  else
    hipLaunchKernelGGL((attend_kernel<D, BF16, SharedRows, kParts>), dim3(grid_of(units0 * splits0)),
                       dim3(256), 0, st, pool, C, CA, U, 0, splits0, units0 * splits0, part0, nullptr,
                       nullptr, nullptr, 0, states);
  float* const part = reinterpret_cast<float*>(base + P.own_off);
  const int64_t units = (int64_t)S.n * pool.H * P.own.tiles;
  if (P.joins && one_wave(units, A.max_len)) {
    hipLaunchKernelGGL((own_join_kernel<D, BF16>), dim3(grid_of(units)), dim3(64), 0, st, pool, S, A,
                       U, P.own.tiles, units, states, A.lse);
    return hipGetLastError();
  }
  if (P.joins) {
    hipLaunchKernelGGL((attend_kernel<D, BF16, RowsOf, kJoin>), dim3(grid_of(units)), dim3(256), 0,
                       st, pool, S, A, U, P.own.tiles, 1, units, nullptr, nullptr, A.lse, nullptr, 0,
                       states);
    return hipGetLastError();
  }
  if (P.own.big)
    prompt_d<D, BF16>(pool, S, A, P.own, part, nullptr, st);
  else
    hipLaunchKernelGGL((attend_kernel<D, BF16, RowsOf, kParts>), dim3(grid_of(units * P.own.splits)),
                       dim3(256), 0, st, pool, S, A, KvUsers{}, P.own.tiles, P.own.splits,
                       units * P.own.splits, part, nullptr, nullptr, nullptr, 0, ContextStates{});
  hipLaunchKernelGGL((shared_join_kernel<D, BF16>), dim3(grid_of(units)), dim3(256), 0, st, pool, S,
                     A, U, P.own.tiles, P.own.splits, units, states, part, A.lse);
  return hipGetLastError();
}

}  // namespace

KvSharedPlan cg_kv8_shared_plan(const KvPool& pool, const KvSeqs& C, const KvAttn& CA,
                                const KvUsers& U, const KvSeqs& S, const KvAttn& A, int D) {
  KvSharedPlan P = {};
  P.shared = cg_kv8_plan(pool, C, CA, D, &U);
  P.small = tiles_of(U, 16);
  P.big = tiles_of(U, 32 * (D == 256 ? kPromptWaves<256> : kPromptWaves<128>) /
                          (P.shared.halves ? 2 : 1));
  const uint64_t state = 16ull * (D + 2) * 4;
  const bool own = S.table != nullptr;
  uint64_t at = own || P.shared.splits > 1 ? kKv8Front : 0;
  P.shared_off = at;
  if (own || P.shared.splits > 1)
    at += (uint64_t)pool.H * P.small.all * P.shared.splits * state;
  at = (at + 255) & ~255ull;
  P.own_off = at;
  if (own) {
    P.own = cg_kv8_plan(pool, S, A, D);
    // One launch for the own tokens and the join, where a wave has two pages of them at most or there
    // would be one split anyway (kernels' us with it / without, which costs another launch's 2; 8 heads
    // of 128 channels behind a context of 1000: 8 requests of 5 pages 18.6 / 17.9, of 16 24.5 / 18.6, of
    // 32 38.0 / 24.6; 32 requests of 5 pages behind 16K tokens 39.2 / 43.9).
    P.joins = !P.own.big &&
              (P.own.splits == 1 || ((int64_t)A.max_len + kPage - 1) / kPage <= 8);
    if (P.joins) P.own.splits = 0;     // (no states)
    at += (uint64_t)S.n * pool.H * P.own.tiles * P.own.splits * state;
  }
  P.total = (at + 255) & ~255ull;
  return P;
}

hipError_t cg_launch_kv8_shared(const KvPool& pool, const KvSeqs& C, const KvAttn& CA,
                                const KvUsers& U, const KvSeqs& S, const KvAttn& A, int D, bool bf16,
                                void* ws, hipStream_t st) {
  switch (D) {
    case 64: return (bf16 ? shared_d<64, true> : shared_d<64, false>)(pool, C, CA, U, S, A, ws, st);
    case 128: return (bf16 ? shared_d<128, true> : shared_d<128, false>)(pool, C, CA, U, S, A, ws, st);
    default: return (bf16 ? shared_d<256, true> : shared_d<256, false>)(pool, C, CA, U, S, A, ws, st);
  }
}

KvAttnPlan cg_kv8_plan(const KvPool& pool, const KvSeqs& S, const KvAttn& A, int D,
                       const KvUsers* shared) {
  KvAttnPlan P;
  int64_t rows = (int64_t)(A.picks ? 1 : A.nq) * A.group;
  if (shared) {
    // the rows of a context as if all requests had one, alike: the bound of a context's requests may be
    // as many as there are, and only the device knows who reads what
    const int64_t users = ((int64_t)shared->n_seq + shared->contexts - 1) / shared->contexts;
    rows = (users < shared->most ? users : shared->most) * shared->rows;
  }
  P.tiles = (int)((rows + 15) / 16);
  const int64_t vseqs = A.picks ? (int64_t)S.n * A.nq : S.n;
  // tiles of all contexts, or of all sequences
  const auto all_tiles = [&](int size) -> int64_t {
    return shared ? tiles_of(*shared, size).all : vseqs * ((rows + size - 1) / size);
  };
  const int64_t units = pool.H * all_tiles(16);
  const int64_t pages = A.picks ? A.n_picks : ((int64_t)A.max_len + kPage - 1) / kPage;
  // From three 16-row tiles on, the rows share the pages through LDS (prompt_kernel), but not where
  // there is little to do: a call that attend_kernel's workgroups hold at once, of at most 8192
  // (tile, page)s or 2048 of 256 channels, is bound by latency, and theirs is shorter. (Both, us; 8
  // heads, group 4, 128 channels: 1K tokens, 64 queries 19.0 / 23.4; 4K, 64 30.6 / 33.8, 128 45.5 /
  // 36.6; 32 sequences of 2K, 8 queries 46.6 / 60.7, 12 69.4 / 63.3; 16 of 256 tokens, 16 queries
  // 11.5 / 14.0, 24 17.8 / 14.3. 4 heads, group 8, 256 channels, 2K: 32 32.7 / 34.7, 48 38.8 / 36.8.)
  // Every query token with pages of its own is a tile or more to itself.
  const int64_t at_once = D == 64 ? 768 : D == 128 ? 512 : 256;
  // Of a shared context of 128 channels 64 rows or fewer leave shared_kernel a wave's work on each SIMD;
  // where its splits of four pages fill the card, it is ahead in such calls too (both, kernels' us with
  // the own tokens; 8 heads: 48 rows of two contexts of 4K 27.4 / 23.0, of one of 16K 37.3 / 34.7, 64
  // rows of 8K 26.0 / 24.6, 60 of 16 heads and two of 4K 33.2 / 28.8; 80 rows of 8K 30.4 / 32.5, 128
  // 34.3 / 41.3; of 64 channels, 64 rows of 8K 21.8 / 19.2, 48 of four of 2K 15.2 / 16.5, of 30K 30.4 /
  // 32.3).
  const bool fills = shared && D == 128 && rows <= 64 && vseqs * pool.H * (pages / 4) >= 256;
  const bool little = !fills && units <= at_once && units * pages <= (D == 256 ? 2048 : 8192);
  // Of contexts that leave room for unequal numbers of requests (see KvTiles) some have more rows than the
  // average, and attend_kernel's tiles without rows take places of others: there two tiles are enough
  // (three / two, us of calls that bound the requests of a context by all; 8 heads, group 4, 128
  // channels: 4 contexts of 8K and 8 requests each 44.9 / 28.8, 32 of 2K 66.2 / 47.0, 40 requests of one of
  // 4K and 9 of nine more 46.8 / 46.1, 256 channels, 4 of 4K and 4 each 55.9 / 37.2; 64 channels 21.3 /
  // 22.9 and 25.1 / 36.5).
  const bool uneven = shared && D > 64 && tiles_of(*shared, 16).each == 0;
  P.big = 0;
  P.halves = false;
  int64_t s, most, at_least = 1;
  const int64_t listed = D == 256 ? PageList<256>::kColumns : PageList<128>::kColumns;
  if (P.tiles > (uneven ? 1 : 2) && !little && !A.picks && (!shared || pages <= listed * kMostSplits)) {
    int per = D == 256 ? 32 * kPromptWaves<256> : 32 * kPromptWaves<128>;
    // Of a shared context tiles of 128 rows by half of the waves, where those of all of them would not
    // fill the card (128 / 256 rows, us: 448 queries over 4 x 1500 tokens, 16 heads of 64, 32.2 / 39.8 with
    // the join that two splits need; 512 rows of 8 heads over 8K 44.2 / 47.8; 160 rows of 8 contexts and 32
    // heads 168 / 131).
    P.halves = shared && D < 256 && pool.H * all_tiles(per) < 256;
    if (P.halves) per /= 2;
    // (shared_kernel lists a split's columns, one a thread)
    if (shared) at_least = (pages + listed - 1) / listed;
    P.big = (int)((rows + per - 1) / per);
    const int64_t groups = pool.H * all_tiles(per);
    // Splits of a shared context: as many as the CUs hold at once, a workgroup each; one round more
    // costs another prologue (rounded down / up, kernels' us: 3 contexts of 8K with 48 rows of 5 heads
    // of 64 channels 28 / 37, 5 of 8K with 128 rows of 8 heads of 128 54 / 75, 20 of 4K 118 / 130).
    s = shared ? 256 / groups : (256 + groups - 1) / groups;
    // a split has four pages at least (us with one, two, four and eight; 64 queries, 32 heads on 8 of
    // 128 channels: 5K tokens 41.2 40.9 38.7 36.9, twice 2.5K 32.2 32.2 33.1 34.2; of 64 channels, 5K
    // 28.5 28.5 24.9 25.4; of 256, 32 queries over 5K 55.0 54.9 47.4 48.1, 64 over 3K 44.9 44.9 43.8
    // 48.7)
    most = pages / 4;
  } else {
    // As many workgroups as the registers let the card hold at once (3, 2 or 1 a CU), each wave
    // with a page of its own at least: a second round of half-filled CUs costs more than longer
    // splits do (4 sequences of 8K, 32 heads: 50 us with 512 workgroups, 64 with 768, 58 with
    // 1024; 32 of 2K, 8 heads: 26, 34 and 33). A long sequence on few heads gains a page's step of
    // a wave with every split less of it and pays for joining one more, a tenth of that: at most
    // twice the root of the pages (8 heads, one sequence: 16K tokens 17 us with 32 splits, 21 with
    // 64; 4K 11 us with 16, 13 with 8).
    s = at_once / units;
    most = (pages + 3) / 4;
    const int64_t root = (int64_t)sqrt(4.0 * (double)pages);
    if (most > root) most = root;
  }
  if (most > kMostSplits) most = kMostSplits;
  if (s > most) s = most;
  if (s < at_least) s = at_least;
  if (s < 1) s = 1;
  P.splits = (int)s;
  // Weights of few rows: their scores are kept for the second launch (8 bytes a row and token to
  // write and read again) where that is at most half of reading K again (D bytes a token), and of 8
  // rows at most (both, us; 128 channels: 32 sequences of 2K, 1 row 35.2 / 48.5, 4 38.8 / 48.9, 8
  // 42.9 / 51.0; 64: 16 of 2K, 4 rows 21.6 / 22.5, 8 24.5 / 22.5; 256: 8 of 4K, 8 rows 28.2 / 28.4,
  // 16 39.5 / 36.7). Of three tiles or more mass_rows_kernel takes them (a question of 64 tokens over
  // 2K: 7 us; mass_kernel, whose waves walk the tiles alone, 17; of 12 tokens 6 and 6).
  P.keep_scores = A.mass_out && rows * 16 <= D && rows <= 8;
  P.many = P.tiles > 2 && !A.picks;
  const bool parts = s > 1, weights = A.mass_out && !A.lse;
  uint64_t at = parts || weights || P.keep_scores ? kKv8Front : 0;
  P.part_off = at;
  if (parts) at += (uint64_t)units * (uint64_t)s * (16ull * (D + 2)) * 4ull;
  at = (at + 255) & ~255ull;
  P.lse_off = at;
  if (weights) at += (uint64_t)S.n * A.nq * pool.H * A.group * 4ull;
  at = (at + 255) & ~255ull;
  P.score_off = at;
  if (P.keep_scores) at += (uint64_t)S.n * pool.H * rows * pages * kPage * 4ull;
  P.total = (at + 255) & ~255ull;
  return P;
}

hipError_t cg_launch_kv8_attend(const KvPool& pool, const KvSeqs& S, int D, bool bf16,
                                const KvAttn& A, void* ws, hipStream_t st) {
  switch (D) {
    case 64: return (bf16 ? attend_d<64, true> : attend_d<64, false>)(pool, S, A, ws, st);
    case 128: return (bf16 ? attend_d<128, true> : attend_d<128, false>)(pool, S, A, ws, st);
    default: return (bf16 ? attend_d<256, true> : attend_d<256, false>)(pool, S, A, ws, st);
  }
}
