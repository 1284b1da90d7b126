// cg_kv8_verify.hip — drafted tokens against the target's probabilities (cg_verify_drafts).
//
// A sequence's drafts are accepted while u q(x) < p(x), and the next token is drawn from the row of
// the first one that is not: from max(p - q, 0), or from p behind the last. Probabilities count in
// whole multiples of 2^-42, so a row's weights sum up exactly, in any order, and the drawn token is
// that of the definition, whichever workgroups shared the row. A multiple comes from one addition:
// p + 1536 in 64 bits is rounded to 2^-42, and lies in the low bits of the sum; the differences of two
// such sums, and a wave's 1024 of them added up, fit a 64-bit float as they are.
//
// Workgroup = (sequence, slices of 4096 probabilities of its row): each finds the row by itself (a
// wave's lanes take a draft each), sums its slices, and the last of a sequence to arrive finds the
// slice of the drawn token, reads it again, and the token in it. Bound by the row's bytes of p and q
// where there are many sequences: 64 of 131072 tokens, 62 MB in 20.0 us, 3.1 TB/s; a single one is a
// chain of dependent reads: count and drafts, their probabilities, the row, the other slices' sums,
// the slice (8.8 us of 32000 tokens).
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
__device__ __forceinline__ float counted(float x) { return fminf(fmaxf(x, 0.0f), 1.0f); }

// A probability as 1536 + its multiple of 2^-42, to the nearest (halves to even).
__device__ __forceinline__ double lifted(float x) { return (double)counted(x) + 1536.0; }

// Its number of them.
__device__ __forceinline__ int64_t units(float x) {
  return __builtin_bit_cast(int64_t, lifted(x)) - __builtin_bit_cast(int64_t, 1536.0);
}

__device__ __forceinline__ uint64_t lane_value(uint64_t x, int lane) {
  const uint32_t lo = __shfl((uint32_t)x, lane), hi = __shfl((uint32_t)(x >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}
// The whole number of multiples of 2^-42 in the wave's sum of x, which is exact.
__device__ __forceinline__ uint64_t wave_units(double x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return (uint64_t)(x * 0x1p42);
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
  uint64_t part[2][16];              // sums of each wave, or of each (chunk, wave)
  uint32_t order;
  int32_t token;
};

// The first draft of the sequence that is not accepted, or `count`.
template <Kind K>
__device__ __forceinline__ int accepted_of(const CgVerify& A, int b, int count) {
  typedef typename Prob<K>::Raw Raw;
  const int lane = threadIdx.x & 63;
  for (int j0 = 0; j0 < A.n_drafts; j0 += 64) {
    // (all drafts that there is room for, whatever `count` says: it may not have arrived yet)
    const int j = j0 + lane;
    bool good = true;
    if (j < A.n_drafts) {
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
    if (bad) {
      const int first = j0 + __builtin_ctzll(bad);
      return first < count ? first : count;
    }
    if (j0 + 64 >= count) break;
  }
  return count;
}

// A thread's probabilities of a slice: N = 16 / size in each of C chunks, chunk c's at c 256 N + N
// thread.
template <Kind K>
struct SliceRegs {
  typedef typename Prob<K>::Raw Raw;
  static constexpr int N = 16 / sizeof(Raw), C = kSlice / (256 * N);
  Sixteen<Raw> p[C], q[C];
};

template <class Raw>
__device__ __forceinline__ void read_some(const Raw* row, int e, int vocab, Sixteen<Raw>& to) {
  constexpr int N = 16 / sizeof(Raw);
  if (e + N <= vocab) {
    to = *reinterpret_cast<const Sixteen<Raw>*>(row + e);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) to.x[i] = e + i < vocab ? row[e + i] : Raw(0);
  }
}

template <Kind K>
__device__ __forceinline__ void read_slice(const typename Prob<K>::Raw* p,
                                           const typename Prob<K>::Raw* q, int at, int vocab,
                                           SliceRegs<K>& r) {
  typedef typename Prob<K>::Raw Raw;
  constexpr int N = SliceRegs<K>::N, C = SliceRegs<K>::C;
  const int e = at + (int)threadIdx.x * N;
  if (at + kSlice <= vocab) {        // (the whole workgroup's: the loads go out together)
#pragma unroll
    for (int c = 0; c < C; ++c)
      r.p[c] = *reinterpret_cast<const Sixteen<Raw>*>(p + e + c * 256 * N);
    if (q) {
#pragma unroll
      for (int c = 0; c < C; ++c)
        r.q[c] = *reinterpret_cast<const Sixteen<Raw>*>(q + e + c * 256 * N);
    }
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      read_some(p, e + c * 256 * N, vocab, r.p[c]);
      if (q) read_some(q, e + c * 256 * N, vocab, r.q[c]);
    }
  }
}

// This thread's weights of a chunk, or of the slice, together: of p over q, or of p.
template <Kind K>
__device__ __forceinline__ double sum_chunk(const SliceRegs<K>& r, int c, bool with_q) {
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < SliceRegs<K>::N; ++i) {
    const double p = lifted(Prob<K>::value(r.p[c].x[i]));
    if (with_q) {
      const double d = p - lifted(Prob<K>::value(r.q[c].x[i]));
      sum += d > 0.0 ? d : 0.0;
    } else {
      sum += p - 1536.0;
    }
  }
  return sum;
}

template <Kind K>
__device__ __forceinline__ double sum_slice(const SliceRegs<K>& r, bool with_q) {
  double sum = 0.0;
#pragma unroll
  for (int c = 0; c < SliceRegs<K>::C; ++c) sum += sum_chunk<K>(r, c, with_q);
  return sum;
}

// A thread's weights of chunk c, whose first probability is e: of p over q, or of p, of which the token
// `skip` has none.
template <Kind K>
struct ChunkWeights {
  static constexpr int N = SliceRegs<K>::N;
  uint64_t w[N], sum;

  __device__ __forceinline__ ChunkWeights(const SliceRegs<K>& r, int c, bool with_q, int e, int skip) {
    sum = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int64_t d = units(Prob<K>::value(r.p[c].x[i]));
      if (with_q) d -= units(Prob<K>::value(r.q[c].x[i]));
      w[i] = d > 0 && e + i != skip ? d : 0;
      sum += w[i];
    }
  }
};

// The workgroup's sum in multiples of 2^-42; every wave adds up to 1024 weights. `turn`: another one
// than the last call's, whose sums may still be read.
__device__ __forceinline__ uint64_t wg_units(double x, VerifyLds& L, int turn) {
  const uint64_t s = wave_units(x);
  if ((threadIdx.x & 63) == 0) L.part[turn & 1][threadIdx.x >> 6] = s;
  __syncthreads();
  const uint64_t* const p = L.part[turn & 1];
  return p[0] + p[1] + p[2] + p[3];
}

__device__ __forceinline__ void put_part(uint64_t* p, uint64_t x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <Kind K>
__global__ __launch_bounds__(256) void verify_kernel(CgVerify A, int b0, int slices, int per,
                                                     uint64_t* parts, uint32_t* arrived) {
  typedef typename Prob<K>::Raw Raw;
  constexpr int N = SliceRegs<K>::N, C = SliceRegs<K>::C;
  __shared__ VerifyLds L;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int groups = (slices + per - 1) / per;          // workgroups of a sequence
  const int row = blockIdx.x / groups, group = blockIdx.x % groups, b = b0 + row;
  int count = A.counts ? A.counts[b] : A.n_drafts;
  if (count > A.n_drafts) count = A.n_drafts;
  int32_t* const tokens = A.tokens + (int64_t)b * (A.n_drafts + 1);
  if (count < 0) {                   // the sequence sits out
    if (group != 0) return;
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

  // the weights of the slices
  SliceRegs<K> r;
  uint64_t* const parts_of = parts + (int64_t)row * slices;
  for (int i = group * per; i < (group + 1) * per && i < slices; ++i) {
    const int at = i * kSlice;
    read_slice<K>(p, q, at, A.vocab, r);
    double sum = q ? sum_slice<K>(r, true) : sum_slice<K>(r, false);
    // (the thread whose sum has it: a wave's sum is never below 0)
    if (skip >= at && skip < at + kSlice && skip < A.vocab &&
        (skip - at) / N % 256 == (int)threadIdx.x)
      sum -= lifted(Prob<K>::value(p[skip])) - 1536.0;
    const uint64_t part = wg_units(sum, L, i);
    if (threadIdx.x == 0) put_part(parts_of + i, part);
  }
  if (threadIdx.x == 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // they have arrived
    L.order = __hip_atomic_fetch_add(&arrived[row], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (L.order == (uint32_t)groups - 1)
      __hip_atomic_store(&arrived[row], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    L.token = -1;
  }
  __syncthreads();
  if (L.order != (uint32_t)groups - 1) return;

  // the last one: every wave finds the drawn token's slice, four slices a lane
  uint64_t s[kMostSlices / 64], before, all;
  const auto sum_up = [&] {
    uint64_t x = 0;
#pragma unroll
    for (int i = 0; i < kMostSlices / 64; ++i) {
      const int at = lane * (kMostSlices / 64) + i;
      s[i] = at < slices ? __hip_atomic_load(parts_of + at, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT)
                         : 0;
      x += s[i];
    }
    before = wave_scan(x);
    all = lane_value(before, 63);
    before -= x;
  };
  sum_up();
  if (all == 0 && (q || skip >= 0)) {
    // nothing of p is over q (or only the sure draft has weight): the token is drawn from p itself,
    // whose slices are summed here, which is rare
    q = nullptr;
    skip = -1;
    for (int i = 0; i < slices; ++i) {
      read_slice<K>(p, nullptr, i * kSlice, A.vocab, r);
      const uint64_t part = wg_units(sum_slice<K>(r, false), L, i);
      if (threadIdx.x == 0) put_part(parts_of + i, part);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    sum_up();
  }
  if (all > 0) {
    const float u = A.u[(int64_t)b * (A.n_drafts + 1) + A.n_drafts];
    uint32_t share = 0;                                 // floor(u 2^24), below 2^24
    if (u > 0.0f) share = u < 1.0f ? (uint32_t)(u * 16777216.0f) : 16777215u;
    const uint64_t bar = share * (all >> 24) + (share * (all & 0xffffff) >> 24);
    // the slice that holds the bar: before <= bar < before + its sum
    uint64_t run = before, left = 0;
    int found = -1;
#pragma unroll
    for (int i = 0; i < kMostSlices / 64; ++i) {
      if (bar >= run && bar < run + s[i]) {
        found = lane * (kMostSlices / 64) + i;
        left = bar - run;
      }
      run += s[i];
    }
    const int who = __builtin_ctzll(__ballot(found >= 0));
    const int at = __shfl(found, who) * kSlice;
    left = lane_value(left, who);
    // sums of the chunks' waves, in the order of the tokens
    read_slice<K>(p, q, at, A.vocab, r);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int e = at + (c * 256 + (int)threadIdx.x) * N;
      double sum = q ? sum_chunk<K>(r, c, true) : sum_chunk<K>(r, c, false);
      if (skip >= e && skip < e + N && skip < A.vocab)
        sum -= lifted(Prob<K>::value(p[skip])) - 1536.0;
      const uint64_t total = wave_units(sum);
      if (lane == 0) L.part[0][c * 4 + wave] = total;
    }
    __syncthreads();
    uint64_t base = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      uint64_t of_wave = 0, mine = 0;              // this wave's sum, and those before it
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint64_t total = L.part[0][c * 4 + w];
        if (w == wave) {
          mine = base;
          of_wave = total;
        }
        base += total;
      }
      if (left >= mine && left < mine + of_wave) {
        // (chunk, wave) has it: the lane, then the token
        const int e = at + (c * 256 + (int)threadIdx.x) * N;
        const ChunkWeights<K> x(r, c, q != nullptr, e, skip);
        uint64_t from = mine + wave_scan(x.sum) - x.sum;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if (left >= from && left < from + x.w[i]) L.token = e + i;
          from += x.w[i];
        }
      }
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

// Workgroups that the card holds at once, five a CU (64 sequences of 32 slices: 2048 workgroups 28 us,
// 1024 of two slices each 20.5).
constexpr int kAtOnce = 5 * 256;

int slices_of(int vocab) { return (vocab + kSlice - 1) / kSlice; }

template <Kind K>
void launch(const CgVerify& A, void* ws, hipStream_t st) {
  const int slices = slices_of(A.vocab);
  uint64_t* const parts = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + kKv8Front);
  // (a counter a sequence: as many sequences a launch as there are counters)
  for (int b0 = 0; b0 < A.n; b0 += kKv8Counters) {
    const int n = A.n - b0 < kKv8Counters ? A.n - b0 : kKv8Counters;
    // as many workgroups as the card holds at once, of several slices where there are more
    const int per = (n * slices + kAtOnce - 1) / kAtOnce;
    const int groups = (slices + per - 1) / per;
    hipLaunchKernelGGL((verify_kernel<K>), dim3((unsigned)(n * groups)), dim3(256), 0, st, A, b0,
                       slices, per, parts, static_cast<uint32_t*>(ws));
  }
}

}  // namespace

uint64_t cg_verify_ws(int n, int vocab) {
  const int rows = n < kKv8Counters ? n : kKv8Counters;
  return kKv8Front + (uint64_t)rows * slices_of(vocab) * 8;
}

hipError_t cg_launch_verify(const CgVerify& A, int dtype, void* ws, hipStream_t st) {
  switch (dtype) {
    case CG_KV8_F16: launch<kF16>(A, ws, st); break;
    case CG_KV8_BF16: launch<kBF16>(A, ws, st); break;
    default: launch<kF32>(A, ws, st); break;
  }
  return hipGetLastError();
}
