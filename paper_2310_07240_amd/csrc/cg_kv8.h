// cg_kv8.h — what the kernels of the 8-bit serving cache share: the page's layout, the views of
// the caller's rows, the int8 -> fp16 widening, and the launchers the C ABI calls.
//
// A page holds 64 tokens of one KV head. K codes lie token by token ([64][D]), V codes channel by
// channel ([D][64]): the two matrix products of attention contract over K's channels and V's
// tokens, and each layout puts the contracted index innermost, so a lane of either product finds
// its operand in 16 consecutive bytes of the page and nothing is transposed on the way.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/cachegen.h"
#include "cg_device.h"

constexpr int kPage = CG_KV8_PAGE;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));

// The cache and one set of sequences, as the kernels see them.
struct KvPool {
  int32_t P, H;                 // pages, KV heads
  int8_t* k;
  int8_t* v;
  float* ks;
  float* vs;
  int8_t* bounds;               // may be null
  float* mass;                  // weights that store clears; may be null
};

struct KvSeqs {
  int32_t n, width;             // sequences, table columns
  const int32_t* table;
};

struct KvRows {
  void* p;
  int64_t seq, tok, head;       // strides in elements
};

// A page number from the table, or -1 where it names no page of the pool.
__device__ __forceinline__ int kv_page(const KvSeqs& S, int P, int seq, int j) {
  const int p = S.table[(int64_t)seq * S.width + j];
  return p >= 0 && p < P ? p : -1;
}

// How pick_best's waves share the blocks of 64 keys: a wave has `mine` (0 for the last ones, maybe)
// from `first` on, and lane l looks up where block pick_block(run, l) lies (-1: none, nothing is read).
struct PickRun {
  int first, mine;
};

__host__ __device__ inline PickRun pick_run(int n, int waves, int wave) {
  const int blocks = (n + 63) / 64, per = (blocks + waves - 1) / waves, first = wave * per;
  return PickRun{first, first + per < blocks ? per : blocks > first ? blocks - first : 0};
}

__host__ __device__ inline int pick_block(const PickRun& r, int lane) {
  return r.mine == 0 ? -1 : r.first + (lane < r.mine ? lane : 0);
}

// Rows of either 16-bit type, widened exactly.
template <bool BF16>
__device__ __forceinline__ float kv_widen(uint16_t u) {
  if (BF16) return __builtin_bit_cast(float, (uint32_t)u << 16);
  return cg_h2f(u);
}

// fp32 to either 16-bit type, to nearest even; a NaN stays one.
template <bool BF16>
__device__ __forceinline__ uint16_t kv_narrow(float f) {
  if (!BF16) return cg_f2h(f);
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}

// Four codes to fp16, exactly: code + 128 (the sign bit flipped) becomes the low byte of
// 0x64xx = 1024 + xx, and 1152 is taken off again. 5 instructions for 4 values.
__device__ __forceinline__ uint2v kv_widen4(uint32_t c) {
  const uint32_t b = c ^ 0x80808080u;
  const half2v off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
  const half2v lo = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u));
  const half2v hi = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u));
  return uint2v{__builtin_bit_cast(uint32_t, lo + off), __builtin_bit_cast(uint32_t, hi + off)};
}

__device__ __forceinline__ half8 kv_widen8(uint32_t a, uint32_t b) {
  const uint2v x = kv_widen4(a), y = kv_widen4(b);
  return __builtin_bit_cast(half8, uint4v{x[0], x[1], y[0], y[1]});
}

// ---- rows into a page (store and eviction) --------------------------------------------------
// Code of x at scale s > 0 (inv = 1 / s, correctly rounded): rint(clamp(x / s)), 0 for a NaN. tiny:
// s may be subnormal, where 1 / s overflows, and the division is taken itself.
__device__ __forceinline__ int kv_code(float x, float s, float inv, bool tiny) {
  if (x != x) return 0;
  return tiny ? cg_quant(x, s) : cg_quant_inv(x, s, inv);
}

// Largest over the workgroup of NT threads, through LDS `red` (one word per wave).
template <int NT>
__device__ __forceinline__ float wg_max(float m, float* red) {
#pragma unroll
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if (NT == 64) return m;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  m = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) m = fmaxf(m, red[w]);
  return m;
}

// Four codes of one row or column as a dword, the first lowest.
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 |
         (uint32_t)d << 24;
}

template <int D>
struct StoreLds {
  float red[2 * D / 64];
  uint32_t vt[D * 17];               // V codes [D][64 + 4]
  uint32_t lo[16 * D / 4], hi[16 * D / 4];   // per row group: bounds of each channel
};

// V codes [D][64] from L.vt, a quarter of a channel's tokens (16 bytes) a thread and step.
template <int D>
__device__ __forceinline__ void write_v(int8_t* codes, const StoreLds<D>& L) {
#pragma unroll
  for (int i = threadIdx.x; i < D * 4; i += 2 * D) {
    const int d = i >> 2, j = i & 3;
    const uint4v o = {L.vt[d * 17 + 4 * j], L.vt[d * 17 + 4 * j + 1], L.vt[d * 17 + 4 * j + 2],
                      L.vt[d * 17 + 4 * j + 3]};
    *reinterpret_cast<uint4v*>(codes + d * kPage + 16 * j) = o;
  }
}

// Bounds [2][D] from the 16 row groups': thread d the lowest of channel d, thread D + d the
// highest.
template <int D>
__device__ __forceinline__ void write_bounds(int8_t* bounds, const StoreLds<D>& L) {
  const int tid = threadIdx.x;
  const int8_t* src = reinterpret_cast<const int8_t*>(tid < D ? L.lo : L.hi) + tid % D;
  int b = src[0];
#pragma unroll
  for (int g = 1; g < 16; ++g) {
    const int o = src[g * D];
    b = tid < D ? (o < b ? o : b) : (o > b ? o : b);
  }
  bounds[tid] = (int8_t)b;
}

// Code (r, c) of a thread's four rows and eight channels: K's words hold four channels of a row,
// V's the four rows of a channel.
template <bool IS_V>
__device__ __forceinline__ int8_t kept_code(const uint32_t* w, int r, int c) {
  return (int8_t)(IS_V ? w[c] >> (8 * r) : w[2 * r + (c >> 2)] >> (8 * (c & 3)));
}

// Writes one page of a head from the 2 D threads' rows x[4][8]: thread (rg, cg) = (tid / (D / 8),
// tid % (D / 8)) has rows 4 rg .. 4 rg + 3 of channels 8 cg .. 8 cg + 7. Rows held .. end - 1 are
// new, the `held` before them (KEPT: the page's codes `was` under its scale s_old) keep their codes,
// re-coded where the scale grows; rows from `end` on become zero codes. Codes, scale and, for K,
// the channels' bounds go to memory.
template <int D, bool IS_V, bool KEPT>
__device__ __forceinline__ void put_page(const KvPool& pool, int page, int h, const float x[4][8],
                                         const uint32_t* was, float s_old, int held, int end,
                                         StoreLds<D>& L) {
  constexpr int NT = 2 * D;
  const int tid = threadIdx.x, cg = tid % (D / 8), rg = tid / (D / 8);
  const int64_t at = (int64_t)page * pool.H + h;
  int8_t* codes = (IS_V ? pool.v : pool.k) + at * (kPage * D);
  float* scale = (IS_V ? pool.vs : pool.ks) + at;
  float m = 0.0f;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (4 * rg + r >= held && 4 * rg + r < end)
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float a = __builtin_fabsf(x[r][c]);
        m = a <= 3.4028234e38f ? fmaxf(m, a) : m;     // NaN and Inf set no scale
      }
  m = wg_max<NT>(m, L.red);
  float s = m / 127.0f;
  if (KEPT) s = fmaxf(s, s_old);
  const float inv = s > 0.0f ? 1.0f / s : 0.0f;
  const bool tiny = s < 0x1p-100f;
  int q[4][8];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = 4 * rg + r;
    if (KEPT && t < held) {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const int code = kept_code<IS_V>(was, r, c);
        q[r][c] = s == s_old ? code : kv_code((float)code * s_old, s, inv, tiny);
      }
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c)
        q[r][c] = t < end && s > 0.0f ? kv_code(x[r][c], s, inv, tiny) : 0;
    }
  }
  __syncthreads();                   // all that the page held is read
  if (tid == 0) *scale = s;
  if (IS_V) {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      L.vt[(8 * cg + c) * 17 + rg] = pack4(q[0][c], q[1][c], q[2][c], q[3][c]);
    __syncthreads();
    write_v<D>(codes, L);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *reinterpret_cast<uint2v*>(codes + (4 * rg + r) * D + 8 * cg) =
          uint2v{pack4(q[r][0], q[r][1], q[r][2], q[r][3]),
                 pack4(q[r][4], q[r][5], q[r][6], q[r][7])};
    if (pool.bounds) {
      int lo[8], hi[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        lo[c] = 127;
        hi[c] = -127;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (4 * rg + r < end) {
            lo[c] = q[r][c] < lo[c] ? q[r][c] : lo[c];
            hi[c] = q[r][c] > hi[c] ? q[r][c] : hi[c];
          }
      }
      const int w = rg * (D / 4) + 2 * cg;
      L.lo[w] = pack4(lo[0], lo[1], lo[2], lo[3]);
      L.lo[w + 1] = pack4(lo[4], lo[5], lo[6], lo[7]);
      L.hi[w] = pack4(hi[0], hi[1], hi[2], hi[3]);
      L.hi[w + 1] = pack4(hi[4], hi[5], hi[6], hi[7]);
      __syncthreads();
      write_bounds<D>(pool.bounds + at * (2 * D), L);
    }
  }
  __syncthreads();                   // the LDS may be used again
}

// Codes of a thread's rows at scale s, as floats whose low byte is the code: v / s rounded to a
// whole number by adding 1.5 2^23. The quotient is taken as v * inv, which below 127.0001 is
// within 2.3e-5 of the correctly rounded v / s; only where it comes within 2^-15 of a half-integer
// could the two round apart, and there (one row of 64 x 8 values in 30) the wave divides. No clamp:
// |v| <= 127 s (1 + 2^-23).
template <class Rows>
__device__ __forceinline__ void fast_codes(const Rows& rows, float s, float inv, float q[4][8]) {
  constexpr float kMagic = 12582912.0f;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float x[8], far = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      x[c] = rows.value(r, c);
      const float v = __builtin_fmaf(x[c], inv, 0.0f);
      q[r][c] = v + kMagic;
      far = fmaxf(far, __builtin_fabsf(v - (q[r][c] - kMagic)));
    }
    if (__builtin_expect(__any(far >= 0.5f - 0x1p-15f), 0)) {
#pragma unroll
      for (int c = 0; c < 8; ++c) q[r][c] = (s > 0.0f ? x[c] / s : 0.0f) + kMagic;
    }
  }
}

__device__ __forceinline__ uint32_t low_bytes(float a, float b, float c, float d) {
  const uint32_t ab = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b),
                                            __builtin_bit_cast(uint32_t, a), 0x0c0c0400u);
  const uint32_t cd = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, d),
                                            __builtin_bit_cast(uint32_t, c), 0x04000c0cu);
  return ab | cd;
}

// A page of finite rows and scales far from the subnormals: put_page's result for K and V together,
// under the scales ks, vs, with one barrier. Rows that stay in place are given as codes times
// their scale, which return to their codes where the scale is the same.
template <int D, class KRows, class VRows>
__device__ __forceinline__ void put_plain(const KvPool& pool, int64_t at, const KRows& k,
                                          const VRows& v, int end, float ks, float vs,
                                          StoreLds<D>& L) {
  const int tid = threadIdx.x, cg = tid % (D / 8), rg = tid / (D / 8);
  float q[4][8];
  fast_codes(v, vs, vs > 0.0f ? 1.0f / vs : 0.0f, q);
#pragma unroll
  for (int c = 0; c < 8; ++c)
    L.vt[(8 * cg + c) * 17 + rg] = low_bytes(q[0][c], q[1][c], q[2][c], q[3][c]);
  fast_codes(k, ks, ks > 0.0f ? 1.0f / ks : 0.0f, q);
  int8_t* kc = pool.k + at * (kPage * D);
#pragma unroll
  for (int r = 0; r < 4; ++r)
    *reinterpret_cast<uint2v*>(kc + (4 * rg + r) * D + 8 * cg) =
        uint2v{low_bytes(q[r][0], q[r][1], q[r][2], q[r][3]),
               low_bytes(q[r][4], q[r][5], q[r][6], q[r][7])};
  if (pool.bounds) {
    float lo[8], hi[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      lo[c] = 12582912.0f + 127.0f;
      hi[c] = 12582912.0f - 127.0f;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * rg + r < end) {
          lo[c] = fminf(lo[c], q[r][c]);
          hi[c] = fmaxf(hi[c], q[r][c]);
        }
    }
    const int w = rg * (D / 4) + 2 * cg;
    L.lo[w] = low_bytes(lo[0], lo[1], lo[2], lo[3]);
    L.lo[w + 1] = low_bytes(lo[4], lo[5], lo[6], lo[7]);
    L.hi[w] = low_bytes(hi[0], hi[1], hi[2], hi[3]);
    L.hi[w + 1] = low_bytes(hi[4], hi[5], hi[6], hi[7]);
  }
  __syncthreads();                   // all that the page held is read, its scales too
  if (tid == 0) {
    pool.ks[at] = ks;
    pool.vs[at] = vs;
  }
  write_v<D>(pool.v + at * (kPage * D), L);
  if (pool.bounds) write_bounds<D>(pool.bounds + at * (2 * D), L);
}

// put_page for K and V of any page; of one that keeps tokens, kc and vc are their codes.
template <int D, bool KEPT, class KRows, class VRows>
__device__ __forceinline__ void put_any(const KvPool& pool, int page, int h, const KRows& k,
                                        const VRows& v, int held, int end, StoreLds<D>& L,
                                        const uint32_t* kc = nullptr, float ks_old = 0.0f,
                                        const uint32_t* vc = nullptr, float vs_old = 0.0f) {
  float x[4][8];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < 8; ++c) x[r][c] = k.value(r, c);
  put_page<D, false, KEPT>(pool, page, h, x, kc, ks_old, held, end, L);
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < 8; ++c) x[r][c] = v.value(r, c);
  put_page<D, true, KEPT>(pool, page, h, x, vc, vs_old, held, end, L);
}

// Whether put_plain may code under this scale.
__device__ __forceinline__ bool plain_scale(float s) { return s == 0.0f || s >= 0x1p-100f; }

// Launchers; arguments are checked by the C ABI.
struct KvAttn {
  const int32_t* lengths;
  const int32_t* q_lens;        // may be null
  const int32_t* picks;         // may be null
  const float* mass_in;
  float* mass_out;              // null: no weights wanted
  float* lse;                   // may be null
  KvRows q, out;
  int32_t max_len, nq, group, n_picks;
  float scale, decay;
  bool wide_q;                  // q's rows on 16-byte boundaries
};

// The workspaces' first bytes: a counter for each tile whose pages are split, zero between calls
// (a tile is split only where there are fewer than kKv8Counters of them).
constexpr int kKv8Counters = 1024;
constexpr uint64_t kKv8Front = CG_KV8_WORKSPACE_ZEROED;
static_assert(kKv8Front == kKv8Counters * 4, "one 32-bit counter a tile");

struct KvAttnPlan {
  int32_t tiles, splits;        // 16-row tiles and splits of the pages for each (sequence, KV head)
  int32_t big;                  // prompt_kernel's row tiles; 0: attend_kernel
  bool keep_scores, many;       // for the weights (see cg_kv8_plan)
  uint64_t part_off, lse_off, score_off, total;   // workspace, in bytes
};

KvAttnPlan cg_kv8_plan(const KvPool& pool, const KvSeqs& seqs, const KvAttn& a, int D);
hipError_t cg_launch_kv8_store(const KvPool&, const KvSeqs&, int D, bool bf16,
                               const int32_t* starts, const int32_t* counts, int n_tokens,
                               const KvRows& k, const KvRows& v, uint32_t* status, hipStream_t);
hipError_t cg_launch_kv8_load(const KvPool&, const KvSeqs&, int D, bool bf16,
                              const int32_t* starts, const int32_t* counts, int n_tokens,
                              const KvRows& k, const KvRows& v, hipStream_t);
hipError_t cg_launch_kv8_attend(const KvPool&, const KvSeqs&, int D, bool bf16, const KvAttn&,
                                void* ws, hipStream_t);
uint64_t cg_kv8_select_ws(const KvSeqs&, int H, int nq, int max_len);
hipError_t cg_launch_kv8_select(const KvPool&, const KvSeqs&, int D, bool bf16, const KvAttn&,
                                int recent, int32_t* picks, void* ws, hipStream_t);
hipError_t cg_launch_kv8_evict(const KvPool&, const KvSeqs&, int D, const int32_t* lengths,
                               int max_len, float* mass, int keep, int recent,
                               const KvSeqs& to, int32_t* kept, int32_t* new_lengths,
                               hipStream_t);
