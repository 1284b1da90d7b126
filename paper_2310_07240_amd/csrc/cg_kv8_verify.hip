// cg_kv8_verify.hip — drafted tokens against the target's probabilities (cg_verify_drafts).
//
// A sequence's drafts are accepted while u q(x) < p(x), and the next token is drawn from the row of
// the first one that is not: from max(p - q, 0), or from p behind the last. Probabilities count in
// whole multiples of 2^-42, so a row's weights sum up exactly, in any order, and the drawn token is
// that of the definition, whichever workgroups shared the row. A multiple comes from one addition:
// p + 1536 in 64 bits is rounded to 2^-42, and lies in the low bits of the sum.
//
// Workgroup = (sequence, slice of 4096 probabilities of its row): each finds the row by itself (a
// wave's lanes take a draft each), sums its slice, and the last of a sequence to arrive finds the
// slice of the drawn token, reads it again, and the token in it. Bound by the row's bytes of p and q
// where there are many sequences; a single one is a chain of dependent reads: count and drafts,
// their probabilities, the row, the other slices' sums, the slice.
#include "cg_kv8.h"

namespace {

constexpr int kSlice = 4096;           // probabilities of a workgroup
constexpr int kMostSlices = CG_VERIFY_MAX_VOCAB / kSlice;

// 16 bytes of a row, which need no alignment but an element's.
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Sixteen {
  T x[16 / sizeof(T)];
};

enum Kind { kF16, kBF16, kF32 };

template <Kind K>
struct Prob {
  typedef uint16_t Raw;
  static __device__ __forceinline__ float value(Raw r) { return kv_widen<K == kBF16>(r); }
};
template <>
struct Prob<kF32> {
  typedef float Raw;
  static __device__ __forceinline__ float value(Raw r) { return r; }
};

// What a probability counts as: a NaN and what is below 0 as 0, what is above 1 as 1.
__device__ __forceinline__ float counted(float x) {
  x = x > 0.0f ? x : 0.0f;
  return x < 1.0f ? x : 1.0f;
}

// Multiples of 2^-42, to the nearest (halves to even).
__device__ __forceinline__ int64_t units(float x) {
  return __builtin_bit_cast(int64_t, (double)counted(x) + 1536.0) -
         __builtin_bit_cast(int64_t, 1536.0);
}

__device__ __forceinline__ uint64_t lane_value(uint64_t x, int lane) {
  const uint32_t lo = __shfl((uint32_t)x, lane), hi = __shfl((uint32_t)(x >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += (uint64_t)__shfl_xor((unsigned long long)x, o);
  return x;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {       // inclusive
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = (uint64_t)__shfl_up((unsigned long long)x, o);
    x += (int)(threadIdx.x & 63) >= o ? y : 0;
  }
  return x;
}

struct VerifyLds {
  uint64_t part[2][16];              // per (chunk, wave) or wave: sums of the residual and of p
  uint32_t order;
  int32_t token;
};

// The first draft of the sequence that is not accepted, or `count`.
template <Kind K>
__device__ __forceinline__ int accepted_of(const CgVerify& A, int b, int count) {
  typedef typename Prob<K>::Raw Raw;
  const int lane = threadIdx.x & 63;
  for (int j0 = 0; j0 < count; j0 += 64) {
    const int j = j0 + lane;
    bool good = true;
    if (j < count) {
      const int x = A.drafts[(int64_t)b * A.n_drafts + j];
      const float u = A.u[(int64_t)b * (A.n_drafts + 1) + j];
      good = x >= 0 && x < A.vocab;
      if (good) {
        const Raw* t = static_cast<const Raw*>(A.target) + b * A.t_seq + j * A.t_row + x;
        float q = 1.0f;
        if (A.draft)
          q = counted(Prob<K>::value(
              static_cast<const Raw*>(A.draft)[b * A.d_seq + j * A.d_row + x]));
        // (24 by 24 bits: the product is exact)
        good = (double)u * (double)q < (double)counted(Prob<K>::value(*t));
      }
    }
    const uint64_t bad = __ballot(!good);
    if (bad) return j0 + __builtin_ctzll(bad);
  }
  return count;
}

// A thread's probabilities of a slice: N = 16 / size in each chunk, chunk c's at c 256 N + N thread.
template <Kind K>
struct SliceRegs {
  typedef typename Prob<K>::Raw Raw;
  static constexpr int N = 16 / sizeof(Raw), C = kSlice / (256 * N);
  Sixteen<Raw> p[C], q[C];
};

template <Kind K>
__device__ __forceinline__ void read_slice(const typename Prob<K>::Raw* p,
                                           const typename Prob<K>::Raw* q, int at, int vocab,
                                           SliceRegs<K>& r) {
  typedef typename Prob<K>::Raw Raw;
  constexpr int N = SliceRegs<K>::N;
#pragma unroll
  for (int c = 0; c < SliceRegs<K>::C; ++c) {
    const int e = at + (c * 256 + (int)threadIdx.x) * N;
    if (e + N <= vocab) {
      r.p[c] = *reinterpret_cast<const Sixteen<Raw>*>(p + e);
      if (q) r.q[c] = *reinterpret_cast<const Sixteen<Raw>*>(q + e);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        r.p[c].x[i] = e + i < vocab ? p[e + i] : Raw(0);
        r.q[c].x[i] = q && e + i < vocab ? q[e + i] : Raw(0);
      }
    }
  }
}

// Weights of chunk c: of p, or (residual) of p over q, or without the token `skip`.
template <Kind K>
__device__ __forceinline__ uint64_t weight(const SliceRegs<K>& r, int c, int i, bool with_q,
                                           int at, int skip) {
  const int64_t p = units(Prob<K>::value(r.p[c].x[i]));
  if (with_q) {
    const int64_t d = p - units(Prob<K>::value(r.q[c].x[i]));
    return d > 0 ? d : 0;
  }
  return at + (c * 256 + (int)threadIdx.x) * SliceRegs<K>::N + i == skip ? 0 : p;
}

template <Kind K>
__global__ __launch_bounds__(256) void verify_kernel(CgVerify A, int b0, int slices, uint64_t* parts,
                                                     uint32_t* arrived) {
  typedef typename Prob<K>::Raw Raw;
  constexpr int N = SliceRegs<K>::N, C = SliceRegs<K>::C;
  __shared__ VerifyLds L;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x / slices, slice = blockIdx.x % slices, b = b0 + row;
  int count = A.counts ? A.counts[b] : A.n_drafts;
  if (count > A.n_drafts) count = A.n_drafts;
  int32_t* const tokens = A.tokens + (int64_t)b * (A.n_drafts + 1);
  if (count < 0) {                   // the sequence sits out
    if (slice != 0) return;
    for (int j = threadIdx.x; j <= A.n_drafts; j += 256) tokens[j] = -1;
    if (threadIdx.x == 0) {
      A.accepted[b] = 0;
      if (A.new_lengths) A.new_lengths[b] = A.lengths[b] > 0 ? A.lengths[b] : 0;
    }
    return;
  }
  const int took = accepted_of<K>(A, b, count);
  const Raw* const p = static_cast<const Raw*>(A.target) + b * A.t_seq + took * A.t_row;
  const Raw* q = nullptr;
  int skip = -1;
  if (took < count) {
    if (A.draft) q = static_cast<const Raw*>(A.draft) + b * A.d_seq + took * A.d_row;
    else skip = A.drafts[(int64_t)b * A.n_drafts + took];
  }

  // the slice's weights, and those of p alone
  SliceRegs<K> r;
  read_slice<K>(p, q, slice * kSlice, A.vocab, r);
  uint64_t over = 0, plain = 0;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      over += weight<K>(r, c, i, q != nullptr, slice * kSlice, skip);
      plain += units(Prob<K>::value(r.p[c].x[i]));
    }
  over = wave_sum(over);
  plain = wave_sum(plain);
  if (lane == 0) {
    L.part[0][wave] = over;
    L.part[1][wave] = plain;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    uint64_t* const mine = parts + 2 * ((int64_t)row * slices + slice);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      __hip_atomic_store(mine + k, L.part[k][0] + L.part[k][1] + L.part[k][2] + L.part[k][3],
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // they have arrived
    L.order = __hip_atomic_fetch_add(&arrived[row], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (L.order == (uint32_t)slices - 1)
      __hip_atomic_store(&arrived[row], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    L.token = -1;
  }
  __syncthreads();
  if (L.order != (uint32_t)slices - 1) return;

  // the last one: every wave finds the drawn token's slice, four slices a lane
  uint64_t s[2][kMostSlices / 64], sum[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < kMostSlices / 64; ++i) {
      const int at = lane * (kMostSlices / 64) + i;
      s[k][i] = at < slices ? __hip_atomic_load(parts + 2 * ((int64_t)row * slices + at) + k,
                                                __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)
                            : 0;
      sum[k] += s[k][i];
    }
  uint64_t before[2], total[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    before[k] = wave_scan(sum[k]);
    total[k] = lane_value(before[k], 63);
    before[k] -= sum[k];
  }
  // nothing of p is over q (or nothing but the draft has weight): from p itself
  const int k = total[0] > 0 ? 0 : 1;
  const uint64_t all = k == 0 ? total[0] : total[1];
  if (all > 0) {
    const float u = A.u[(int64_t)b * (A.n_drafts + 1) + A.n_drafts];
    uint32_t part = 0;                                  // floor(u 2^24), below 2^24
    if (u > 0.0f) part = u < 1.0f ? (uint32_t)(u * 16777216.0f) : 16777215u;
    uint64_t bar = part * (all >> 24) + (part * (all & 0xffffff) >> 24);
    // the slice that holds the bar: before <= bar < before + its sum
    uint64_t run = k == 0 ? before[0] : before[1];
    int found = -1;
    uint64_t left = 0;
#pragma unroll
    for (int i = 0; i < kMostSlices / 64; ++i) {
      const uint64_t x = k == 0 ? s[0][i] : s[1][i];
      if (bar >= run && bar < run + x) {
        found = lane * (kMostSlices / 64) + i;
        left = bar - run;
      }
      run += x;
    }
    const int who = __builtin_ctzll(__ballot(found >= 0));
    const int at = __shfl(found, who) * kSlice;
    left = lane_value(left, who);
    const bool with_q = k == 0 && q != nullptr;
    const int without = k == 0 ? skip : -1;
    read_slice<K>(p, with_q ? q : nullptr, at, A.vocab, r);
    // sums of the chunks' waves, in the order of the tokens
    uint64_t mine[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      mine[c] = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) mine[c] += weight<K>(r, c, i, with_q, at, without);
      mine[c] = wave_scan(mine[c]);
      if (lane == 63) L.part[0][c * 4 + wave] = mine[c];
    }
    __syncthreads();
    uint64_t base = 0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint64_t x = L.part[0][c * 4 + w];
        if (w == wave && left >= base && left < base + x) {
          // this wave's chunk c: the lane, then the token
          uint64_t from = base + lane_value(mine[c], lane > 0 ? lane - 1 : 0);
          if (lane == 0) from = base;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const uint64_t y = weight<K>(r, c, i, with_q, at, without);
            if (left >= from && left < from + y)
              L.token = at + (c * 256 + (int)threadIdx.x) * N + i;
            from += y;
          }
        }
        base += x;
      }
    __syncthreads();
  }
  const int token = L.token;
  for (int j = threadIdx.x; j <= A.n_drafts; j += 256)
    tokens[j] = j < took ? A.drafts[(int64_t)b * A.n_drafts + j] : j == took ? token : -1;
  if (threadIdx.x == 0) {
    A.accepted[b] = took;
    if (A.new_lengths) {
      const int64_t n = (int64_t)A.lengths[b] - (count - took);
      A.new_lengths[b] = n > 0 ? (int32_t)n : 0;
    }
  }
}

int slices_of(int vocab) { return (vocab + kSlice - 1) / kSlice; }

template <Kind K>
void launch(const CgVerify& A, void* ws, hipStream_t st) {
  const int slices = slices_of(A.vocab);
  uint64_t* const parts = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + kKv8Front);
  // (a counter a sequence: as many sequences a launch as there are counters)
  for (int b0 = 0; b0 < A.n; b0 += kKv8Counters) {
    const int n = A.n - b0 < kKv8Counters ? A.n - b0 : kKv8Counters;
    hipLaunchKernelGGL((verify_kernel<K>), dim3((unsigned)(n * slices)), dim3(256), 0, st, A, b0,
                       slices, parts, static_cast<uint32_t*>(ws));
  }
}

}  // namespace

uint64_t cg_verify_ws(int n, int vocab) {
  const int rows = n < kKv8Counters ? n : kKv8Counters;
  return kKv8Front + (uint64_t)rows * slices_of(vocab) * 16;
}

hipError_t cg_launch_verify(const CgVerify& A, int dtype, void* ws, hipStream_t st) {
  switch (dtype) {
    case CG_KV8_F16: launch<kF16>(A, ws, st); break;
    case CG_KV8_BF16: launch<kBF16>(A, ws, st); break;
    default: launch<kF32>(A, ws, st); break;
  }
  return hipGetLastError();
}
