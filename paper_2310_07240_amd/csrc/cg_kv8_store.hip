// cg_kv8_store.hip — rows of K and V into the pages of the 8-bit cache, and back (cg_kv8_store,
// cg_kv8_load).
//
// One workgroup per (sequence, page it touches, KV head): 2 D threads, thread (rg, cg) holding
// rows 4 rg .. 4 rg + 3 of channels 8 cg .. 8 cg + 7, so a wave's load of one row index is whole
// 2 D-byte rows and four tokens of a channel meet in one lane, as the transposed V codes want
// them. The scale is the page's absolute maximum over 127, and the page is held in registers from
// its maximum to its codes: one read of the rows, one write of the codes. Bound by those bytes.
// Store: 537 MB of fp16 rows in and 268 MB of codes out in 176 us, 4.6 TB/s; load, the other way
// round, 149 us, 5.4 TB/s (a copy of 1 GiB: 5.1). A call of one token for each of 8 requests is a
// chain of dependent reads: start, table, rows and codes; 8.4 us and 5.9.
#include "cg_kv8.h"

namespace {

typedef uint16_t ushort2v __attribute__((ext_vector_type(2)));

// Row elements at p: 8 of them, in one 16-byte load where VEC.
template <bool VEC>
__device__ __forceinline__ uint4v get8(const uint16_t* p) {
  if (VEC) return *reinterpret_cast<const uint4v*>(p);
  uint16_t u[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) u[c] = p[c];
  return *reinterpret_cast<uint4v*>(u);
}

// Largest magnitude bits of a thread's rows, the two 16-bit halves apart.
__device__ __forceinline__ ushort2v top_bits(const uint4v u[4]) {
  ushort2v m = {0, 0};
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      m = __builtin_elementwise_max(m, __builtin_bit_cast(ushort2v, u[r][c] & 0x7fff7fffu));
  return m;
}

// A thread's rows as values (what put_plain takes).
template <bool BF16>
struct NewRows {
  const uint4v* u;
  __device__ __forceinline__ float value(int r, int c) const {
    return kv_widen<BF16>((uint16_t)(u[r][c >> 1] >> (16 * (c & 1))));
  }
};

// The same where the first `old` rows are the page's own, as codes under its last scale: K's row
// by row, V's (KEPT_V) channel by channel.
template <bool BF16, bool KEPT_V>
struct KeptRows {
  const uint4v* u;
  const uint32_t* codes;
  int old;
  float scale;
  __device__ __forceinline__ float value(int r, int c) const {
    return r < old ? (float)kept_code<KEPT_V>(codes, r, c) * scale
                   : kv_widen<BF16>((uint16_t)(u[r][c >> 1] >> (16 * (c & 1))));
  }
};

// Whether put_plain may code a page of scale `old` on under max(old, fresh): both plain and one not
// zero, and no product of a code and `old` overflows.
__device__ __forceinline__ bool kept_plain(float old, float fresh) {
  return plain_scale(old) && old <= 0x1p120f && plain_scale(fresh) && fmaxf(old, fresh) > 0.0f;
}

// One page of a head: rows `held` .. last - 1 from k, v, which point at the page's first row.
// KEPT: the page keeps `held` > 0 tokens, whose codes and scales are requested with the rows: one
// token behind the tokens of 8 requests takes 8.4 us, and 12.0 where they are read after the rows'
// maximum, K's and V's in turn. Returns whether all rows are finite.
template <int D, bool BF16, bool VEC, bool KEPT>
__device__ __forceinline__ bool store_page(const KvPool& pool, int page, int h, const uint16_t* k,
                                           int64_t k_tok, const uint16_t* v, int64_t v_tok,
                                           int held, int last, ushort2v* tops, StoreLds<D>& L) {
  const int tid = threadIdx.x, cg = tid % (D / 8), rg = tid / (D / 8);
  const int64_t at = (int64_t)page * pool.H + h;
  uint4v x[4], y[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = 4 * rg + r;
    x[r] = y[r] = uint4v{0, 0, 0, 0};
    if (t >= held && t < last) {
      x[r] = get8<VEC>(k + t * k_tok + 8 * cg);
      y[r] = get8<VEC>(v + t * v_tok + 8 * cg);
    }
  }
  const int old = held - 4 * rg;                      // of this thread's rows (0 or less: none)
  uint32_t kc[8], vc[8];
  float ks_old = 0.0f, vs_old = 0.0f;
  if constexpr (KEPT) {
    ks_old = pool.ks[at];
    vs_old = pool.vs[at];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      uint2v w = {0, 0};
      if (r < old)
        w = *reinterpret_cast<const uint2v*>(pool.k + at * (kPage * D) + (4 * rg + r) * D + 8 * cg);
      kc[2 * r] = w[0];
      kc[2 * r + 1] = w[1];
    }
#pragma unroll
    for (int c = 0; c < 8; ++c)
      vc[c] = old > 0 ? *reinterpret_cast<const uint32_t*>(pool.v + at * (kPage * D) +
                                                           (8 * cg + c) * kPage + 4 * rg)
                      : 0u;
  }
  // the maxima of both, K's in the high half: magnitude bits are ordered as the magnitudes are
  const ushort2v mx = top_bits(x), my = top_bits(y);
  ushort2v m = {my[0] > my[1] ? my[0] : my[1], mx[0] > mx[1] ? mx[0] : mx[1]};
#pragma unroll
  for (int o = 32; o; o >>= 1)
    m = __builtin_elementwise_max(
        m, __builtin_bit_cast(ushort2v, __shfl_xor(__builtin_bit_cast(int, m), o)));
  __syncthreads();                   // the last page's LDS is read
  if ((tid & 63) == 0) tops[tid >> 6] = m;
  __syncthreads();
  m = tops[0];
#pragma unroll
  for (int w = 1; w < 2 * D / 64; ++w) m = __builtin_elementwise_max(m, tops[w]);
  constexpr uint16_t kInf = BF16 ? 0x7f80 : 0x7c00;
  const bool finite = m[0] < kInf && m[1] < kInf;
  float ks = kv_widen<BF16>(m[1]) / 127.0f, vs = kv_widen<BF16>(m[0]) / 127.0f;
  if (!KEPT && finite && plain_scale(ks) && plain_scale(vs)) {
    put_plain<D>(pool, at, NewRows<BF16>{x}, NewRows<BF16>{y}, last, ks, vs, L);
  } else if (KEPT && finite && kept_plain(ks_old, ks) && kept_plain(vs_old, vs)) {
    ks = fmaxf(ks, ks_old);
    vs = fmaxf(vs, vs_old);
    put_plain<D>(pool, at, KeptRows<BF16, false>{x, kc, old, ks_old},
                 KeptRows<BF16, true>{y, vc, old, vs_old}, last, ks, vs, L);
  } else {
    put_any<D, KEPT>(pool, page, h, NewRows<BF16>{x}, NewRows<BF16>{y}, held, last, L, kc, ks_old,
                     vc, vs_old);
  }
  return finite;
}

// Which pages a launch is for: those that keep tokens (a sequence's first, if any), those that do
// not, or both. Keeping takes 187 registers where coding new rows takes 128, so one kernel for both
// leaves two waves on a SIMD: 217 us for 805 MB of rows and codes, against 176 (4.6 TB/s) and 5 for
// the second launch with one for each. Up to kFewPages pages (of heads) all run at once anyway, and
// one launch for both is the shorter. (One / two, us, 8 heads of 128 channels. Rows behind 100
// tokens: 8192 of one sequence, 1032 pages, 17.6 / 22.3; 16384, 2056, 27.5 / 29.8; 32768, 4104, 47.2 /
// 43.3. 4096 rows from a sequence's start: of 4, 2080 pages, 27.2 / 24.0; of 8, 4160, 47.3 / 37.4. One
// row behind 100 tokens of 256 sequences, 2048 pages, 33.8 / 36.9, of 512, 4096, 62.5 / 67.8: where
// nearly all pages keep tokens the second launch never pays.)
enum Pages { kBoth, kNew, kKept };

template <int D, bool BF16, bool VEC, Pages WHICH>
__global__ __launch_bounds__(2 * D, WHICH == kNew ? 4 : 2) void store_kernel(KvPool pool, KvSeqs S,
                                                      const int32_t* __restrict__ starts,
                                                      const int32_t* __restrict__ counts,
                                                      int n_tokens, int np, int64_t items,
                                                      KvRows k, KvRows v, uint32_t* status) {
  __shared__ StoreLds<D> L;
  __shared__ ushort2v tops[2 * D / 64];
  const int tid = threadIdx.x;
  uint32_t bad = 0;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int h = (int)(it % pool.H);
    const int64_t r0 = it / pool.H;
    const int seq = (int)(r0 / np);
    const int start = starts[seq];
    int count = counts ? counts[seq] : n_tokens;
    count = count < n_tokens ? count : n_tokens;
    if (start < 0 || count <= 0) continue;
    const int64_t j = start / kPage + r0 % np;        // the sequence's page
    const int64_t end = (int64_t)start + count;
    if (j * kPage >= end) continue;
    const int held = start > j * kPage ? (int)(start - j * kPage) : 0;
    if (WHICH != kBoth && (held > 0) != (WHICH == kKept)) continue;
    const int page = j < S.width ? kv_page(S, pool.P, seq, (int)j) : -1;
    if (page < 0) continue;                           // no such page: nothing is written
    const int last = end - j * kPage < kPage ? (int)(end - j * kPage) : kPage;
    if (pool.mass && tid >= held && tid < kPage)
      pool.mass[((int64_t)page * pool.H + h) * kPage + tid] = 0.0f;
    const int64_t row0 = j * kPage - start;           // row of the page's first token
    const uint16_t* kp = static_cast<const uint16_t*>(k.p) + seq * k.seq + row0 * k.tok + h * k.head;
    const uint16_t* vp = static_cast<const uint16_t*>(v.p) + seq * v.seq + row0 * v.tok + h * v.head;
    bool finite;
    if (WHICH != kNew && held > 0)
      finite = store_page<D, BF16, VEC, true>(pool, page, h, kp, k.tok, vp, v.tok, held, last, tops,
                                              L);
    else if (WHICH != kKept)
      finite = store_page<D, BF16, VEC, false>(pool, page, h, kp, k.tok, vp, v.tok, 0, last, tops,
                                               L);
    bad |= finite ? 0u : 1u;
  }
  if (status && __any(bad) && (tid & 63) == 0) atomicOr(status, 1u);
}

__global__ void kv_zero_word(uint32_t* p) { *p = 0u; }

// code * scale in 32 bits. The value is made opaque: the compiler would fuse the product with its
// rounding to fp16 and round once, which differs from the definition in about one of 20000 values.
__device__ __forceinline__ float product(int code, float scale) {
  float p = (float)code * scale;
  asm("" : "+v"(p));
  return p;
}

template <int D, bool BF16, bool VEC>
__global__ __launch_bounds__(2 * D) void load_kernel(KvPool pool, KvSeqs S,
                                                     const int32_t* __restrict__ starts,
                                                     const int32_t* __restrict__ counts,
                                                     int n_tokens, int np, int64_t items,
                                                     KvRows k, KvRows v) {
  __shared__ uint32_t vt[D * 17];
  constexpr int NT = 2 * D;
  const int tid = threadIdx.x, cg = tid % (D / 8), rg = tid / (D / 8);
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int h = (int)(it % pool.H);
    const int64_t r0 = it / pool.H;
    const int seq = (int)(r0 / np);
    int start = starts[seq];
    int count = counts ? counts[seq] : n_tokens;
    count = count < n_tokens ? count : n_tokens;
    if (start < 0) start = count = 0;
    const int64_t j = start / kPage + r0 % np;
    const int64_t row0 = j * kPage - start;           // row of the page's first token
    const int page = j * kPage < (int64_t)start + count && j < S.width
                         ? kv_page(S, pool.P, seq, (int)j) : -1;
    const int64_t at = (int64_t)page * pool.H + h;
    float ks = 0.0f, vs = 0.0f;
    if (page >= 0) {
      ks = pool.ks[at];
      vs = pool.vs[at];
      const int8_t* src = pool.v + at * (kPage * D);
#pragma unroll
      for (int i = tid; i < D * 4; i += NT) {
        const int d = i >> 2, q = i & 3;
        const uint4v o = *reinterpret_cast<const uint4v*>(src + d * kPage + 16 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) vt[d * 17 + 4 * q + e] = o[e];
      }
    }
    __syncthreads();
    uint32_t w[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) w[c] = vt[(8 * cg + c) * 17 + rg];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t row = row0 + 4 * rg + r;
      if (row < 0 || row >= n_tokens) continue;
      const bool live = page >= 0 && row < count;
      uint16_t a[8], b[8];
      uint2v kc = {0, 0};
      if (live)
        kc = *reinterpret_cast<const uint2v*>(pool.k + at * (kPage * D) + (4 * rg + r) * D +
                                              8 * cg);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const int qk = (int8_t)(kc[c >> 2] >> (8 * (c & 3)));
        const int qv = (int8_t)(w[c] >> (8 * r));
        a[c] = live ? kv_narrow<BF16>(product(qk, ks)) : 0;
        b[c] = live ? kv_narrow<BF16>(product(qv, vs)) : 0;
      }
      uint16_t* ka = static_cast<uint16_t*>(k.p) + seq * k.seq + row * k.tok + h * k.head + 8 * cg;
      uint16_t* va = static_cast<uint16_t*>(v.p) + seq * v.seq + row * v.tok + h * v.head + 8 * cg;
      if (VEC) {
        *reinterpret_cast<uint4v*>(ka) = *reinterpret_cast<uint4v*>(a);
        *reinterpret_cast<uint4v*>(va) = *reinterpret_cast<uint4v*>(b);
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          ka[c] = a[c];
          va[c] = b[c];
        }
      }
    }
    __syncthreads();
  }
}

bool wide(const KvRows& r) {
  return ((uintptr_t)r.p & 15) == 0 && ((r.seq | r.tok | r.head) & 7) == 0;
}

// Pages that n tokens can touch, wherever in a page they start.
int touched(int n) { return (int)(((int64_t)n + 2 * kPage - 2) / kPage); }

// Workgroups for `items`: all at once, below 2^32 threads and well inside the grid's limit; the
// kernels walk on where there are more.
unsigned grid_of(int64_t items) { return (unsigned)(items < (1 << 22) ? items : (1 << 22)); }

constexpr int64_t kFewPages = 2048;

template <int D, bool BF16, bool VEC>
hipError_t store_d(const KvPool& pool, const KvSeqs& S, const int32_t* starts,
                   const int32_t* counts, int n, const KvRows& k, const KvRows& v,
                   uint32_t* status, hipStream_t st) {
  const int np = touched(n);
  const int64_t items = (int64_t)S.n * np * pool.H, first = (int64_t)S.n * pool.H;
  if (items <= kFewPages) {
    hipLaunchKernelGGL((store_kernel<D, BF16, VEC, kBoth>), dim3(grid_of(items)), dim3(2 * D), 0, st,
                       pool, S, starts, counts, n, np, items, k, v, status);
  } else {
    hipLaunchKernelGGL((store_kernel<D, BF16, VEC, kNew>), dim3(grid_of(items)), dim3(2 * D), 0, st,
                       pool, S, starts, counts, n, np, items, k, v, status);
    hipLaunchKernelGGL((store_kernel<D, BF16, VEC, kKept>), dim3(grid_of(first)), dim3(2 * D), 0, st,
                       pool, S, starts, counts, n, 1, first, k, v, status);
  }
  return hipGetLastError();
}

template <int D, bool BF16>
hipError_t store_w(const KvPool& pool, const KvSeqs& S, const int32_t* starts,
                   const int32_t* counts, int n, const KvRows& k, const KvRows& v,
                   uint32_t* status, hipStream_t st) {
  return (wide(k) && wide(v) ? store_d<D, BF16, true> : store_d<D, BF16, false>)(
      pool, S, starts, counts, n, k, v, status, st);
}

template <int D, bool BF16>
hipError_t load_d(const KvPool& pool, const KvSeqs& S, const int32_t* starts,
                  const int32_t* counts, int n, const KvRows& k, const KvRows& v,
                  hipStream_t st) {
  const int np = touched(n);
  const int64_t items = (int64_t)S.n * np * pool.H;
  if (wide(k) && wide(v))
    hipLaunchKernelGGL((load_kernel<D, BF16, true>), dim3(grid_of(items)), dim3(2 * D), 0, st,
                       pool, S, starts, counts, n, np, items, k, v);
  else
    hipLaunchKernelGGL((load_kernel<D, BF16, false>), dim3(grid_of(items)), dim3(2 * D), 0, st,
                       pool, S, starts, counts, n, np, items, k, v);
  return hipGetLastError();
}

}  // namespace

hipError_t cg_launch_kv8_store(const KvPool& pool, const KvSeqs& S, int D, bool bf16,
                               const int32_t* starts, const int32_t* counts, int n,
                               const KvRows& k, const KvRows& v, uint32_t* status,
                               hipStream_t st) {
  if (status) hipLaunchKernelGGL(kv_zero_word, dim3(1), dim3(1), 0, st, status);
  if (n <= 0) return hipGetLastError();
  switch (D) {
    case 64: return (bf16 ? store_w<64, true> : store_w<64, false>)(pool, S, starts, counts, n, k, v, status, st);
    case 128: return (bf16 ? store_w<128, true> : store_w<128, false>)(pool, S, starts, counts, n, k, v, status, st);
    default: return (bf16 ? store_w<256, true> : store_w<256, false>)(pool, S, starts, counts, n, k, v, status, st);
  }
}

hipError_t cg_launch_kv8_load(const KvPool& pool, const KvSeqs& S, int D, bool bf16,
                              const int32_t* starts, const int32_t* counts, int n,
                              const KvRows& k, const KvRows& v, hipStream_t st) {
  switch (D) {
    case 64: return (bf16 ? load_d<64, true> : load_d<64, false>)(pool, S, starts, counts, n, k, v, st);
    case 128: return (bf16 ? load_d<128, true> : load_d<128, false>)(pool, S, starts, counts, n, k, v, st);
    default: return (bf16 ? load_d<256, true> : load_d<256, false>)(pool, S, starts, counts, n, k, v, st);
  }
}
