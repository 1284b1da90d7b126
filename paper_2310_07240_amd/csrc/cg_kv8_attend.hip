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

// Tokens that query token i sees: those up to its own place, the last q_len tokens being the
// queries' own.
__device__ __forceinline__ int visible_of(const RowsOf& r, int i) {
  if (i >= r.q_len) return 0;
  const int64_t n = (int64_t)r.len - r.q_len + i + 1;
  return n > 0 ? (int)n : 0;
}

// Rows 16 tile .. 16 tile + 15 of the group's queries; rows past the last one see nothing.
// bf16 rows are scaled by a power of two to [1, 2) at their largest, so that fp16 holds them to
// 2^-25 of it; fp16 rows go as they are.
template <int D, bool BF16>
__device__ __forceinline__ void load_q(const KvAttn& A, const RowsOf& R, int h, int tile,
                                       QTile<D>& Q) {
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int row = tile * 16 + m;
  const int i = R.i0 + row / A.group, head = h * A.group + row % A.group;
  const bool live = row < R.nq * A.group;
  Q.visible = live ? visible_of(R, i) : 0;
  const uint16_t* src = static_cast<const uint16_t*>(A.q.p) + R.seq * A.q.seq +
                        (int64_t)i * A.q.tok + (int64_t)head * A.q.head;
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

template <int D, bool BF16>
__device__ __forceinline__ void put_out(const KvAttn& A, const RowsOf& R, int h, int row, int d,
                                        const float* o, int n) {
  const int i = R.i0 + row / A.group, head = h * A.group + row % A.group;
  uint16_t* p = static_cast<uint16_t*>(A.out.p) + R.seq * A.out.seq + (int64_t)i * A.out.tok +
                (int64_t)head * A.out.head + d;
  for (int c = 0; c < n; ++c) p[c] = kv_narrow<BF16>(o[c]);
}

__device__ __forceinline__ int64_t lse_at(const KvAttn& A, const RowsOf& R, int H, int h,
                                          int row) {
  const int i = R.i0 + row / A.group, head = h * A.group + row % A.group;
  return ((int64_t)R.seq * A.nq + i) * ((int64_t)H * A.group) + head;
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
template <int D, bool BF16, bool FAR, int kAhead>
__device__ __forceinline__ void join_tile(const KvAttn& A, const RowsOf& R, int H, int h, int tile,
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
    if (lse && sub == 0)
      lse[lse_at(A, R, H, h, tile * 16 + row)] = (top + __builtin_amdgcn_logf(l)) * kLn2;
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
template <int D, bool BF16, int N>
__device__ __forceinline__ void finish_row(const KvAttn& A, const RowsOf& R, int H, int h, int row,
                                           int d0, float* o, float top, float l, float* lse) {
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
#pragma unroll
  for (int c = 0; c < N; ++c) o[c] *= inv;
  put_out<D, BF16>(A, R, h, row, d0, o, N);
  if (lse && d0 == 0)
    lse[lse_at(A, R, H, h, row)] = (top + __builtin_amdgcn_logf(l)) * kLn2;
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
template <int D, bool BF16>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void attend_kernel(KvPool pool, KvSeqs S, KvAttn A, int tiles,
                                                        int splits, int64_t items, float* part,
                                                        uint32_t* arrived, float* lse,
                                                        float* scores, int np) {
  __shared__ float os[4][16][D + 4];
  __shared__ float ml[4][32];
  __shared__ uint32_t others;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int split = (int)(it % splits);
    const int64_t unit = it / splits;
    const int tile = (int)(unit % tiles);
    const int h = (int)(unit / tiles % pool.H);
    const int vseq = (int)(unit / tiles / pool.H);
    const RowsOf R = rows_of(S, A, vseq);
    // the pages that any row of the tile sees
    const int rows = R.nq * A.group;
    int last = tile * 16 + 15 < rows ? tile * 16 + 15 : rows - 1;
    last = R.i0 + last / A.group;
    const int most = R.q_len > 0 ? visible_of(R, last < R.q_len ? last : R.q_len - 1) : 0;
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
    if (splits == 1) {
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
      const int see = visible_of(R, row / A.group);
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
  const int see = row < rows ? visible_of(R, i_row) : 0;
  const int visible = see > 0 ? see : 0x7fffffff;
  const float unit = load_row32<D, BF16>(
      A, static_cast<const uint16_t*>(A.q.p) + R.seq * A.q.seq + (int64_t)i_row * A.q.tok +
             (int64_t)head * A.q.head, see > 0, q);
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
  int top_token = last / A.group;
  if (top_token >= R.q_len) top_token = R.q_len - 1;
  const int most = top_token >= 0 ? visible_of(R, top_token) : 0;
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
  const float g = empty ? 0.0f : (splits > 1 ? to_top : to_top / sum) * l_unit;
  const int64_t u16 = ((int64_t)seq * pool.H + h) * ((rows + 15) / 16) + row / 16;
  float* dst = splits > 1 ? part + (u16 * splits + split) * kPart<D> : nullptr;
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
  } else if (lse) {
    lse[lse_at(A, R, pool.H, h, row)] =
        empty ? kNegInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
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
          see = visible_of(R, own_i);
          z = tile_lse[lse_off];
        } else {                     // (behind the last row the tile's first, of no use)
#pragma unroll
          for (int c = 0; c < CH; ++c)
            u[c] = *reinterpret_cast<const uint4v*>(
                tile_q + (32 * t + c * RC + lane / LR < rows ? q_off[c] : 0u));
          const bool live = 32 * t + m < rows;
          see = live ? visible_of(R, own_i) : 0;
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
      see = live ? visible_of(R, own_i) : 0;
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
    prompt_d<D, BF16>(pool, S, A, P, part, lse, st);
  else
    hipLaunchKernelGGL((attend_kernel<D, BF16>), dim3(grid_of(units * P.splits)), dim3(256), 0,
                       st, pool, S, A, P.tiles, P.splits, units * P.splits, part,
                       reinterpret_cast<uint32_t*>(base), lse, scores, np);
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

}  // namespace

KvAttnPlan cg_kv8_plan(const KvPool& pool, const KvSeqs& S, const KvAttn& A, int D) {
  KvAttnPlan P;
  const int64_t rows = (int64_t)(A.picks ? 1 : A.nq) * A.group;
  P.tiles = (int)((rows + 15) / 16);
  const int64_t vseqs = A.picks ? (int64_t)S.n * A.nq : S.n;
  const int64_t units = vseqs * pool.H * P.tiles;
  const int64_t pages = A.picks ? A.n_picks : ((int64_t)A.max_len + kPage - 1) / kPage;
  // From three 16-row tiles on, the rows share the pages through LDS (prompt_kernel), but not where
  // there is little to do: a call that attend_kernel's workgroups hold at once, of at most 8192
  // (tile, page)s or 2048 of 256 channels, is bound by latency, and theirs is shorter. (Both, us; 8
  // heads, group 4, 128 channels: 1K tokens, 64 queries 19.0 / 23.4; 4K, 64 30.6 / 33.8, 128 45.5 /
  // 36.6; 32 sequences of 2K, 8 queries 46.6 / 60.7, 12 69.4 / 63.3; 16 of 256 tokens, 16 queries
  // 11.5 / 14.0, 24 17.8 / 14.3. 4 heads, group 8, 256 channels, 2K: 32 32.7 / 34.7, 48 38.8 / 36.8.)
  // Every query token with pages of its own is a tile or more to itself.
  const int64_t at_once = D == 64 ? 768 : D == 128 ? 512 : 256;
  const bool little = units <= at_once && units * pages <= (D == 256 ? 2048 : 8192);
  P.big = 0;
  int64_t s, most;
  if (P.tiles > 2 && !little && !A.picks) {
    const int per = D == 256 ? 32 * kPromptWaves<256> : 32 * kPromptWaves<128>;
    P.big = (int)((rows + per - 1) / per);
    const int64_t groups = vseqs * pool.H * P.big;
    s = (256 + groups - 1) / groups;
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
