// cg_kv8_pick.hip — which tokens stay (cg_kv8_evict) and which pages a query reads
// (cg_kv8_select): the best `need` of a row of 32-bit keys, ties to the lowest index, in
// ascending order of index; and the move of the kept tokens into new pages.
#include "cg_kv8.h"

namespace {

// Keys in the order of the values: a larger value has a larger key, -0 and +0 the same, a NaN the
// lowest of all. 0 is no value's key.
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, f + 0.0f);
  const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return f != f ? 1u : k;
}

// How many lanes below this one are in the mask.
__device__ __forceinline__ uint32_t lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                   __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// f over the lanes up to this one (lane 63: over all): steps within rows of 16 lanes, then lane 15's
// result into the second and fourth row's and lane 31's into the upper half's. `none` is f's
// identity. (Moves between lanes in the vector unit itself; __shfl_up goes through the LDS.)
template <class F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, uint32_t none, F f) {
  v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x111, 0xf, 0xf, false));
  v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x112, 0xf, 0xf, false));
  v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x114, 0xf, 0xf, false));
  v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x118, 0xf, 0xf, false));
  v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x142, 0xa, 0xf, false));
  return f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x143, 0xc, 0xf, false));
}

constexpr int kBins = 2048;          // of a pass: 11 bits

// Each counted in copies that the lanes of a wave take in turn: weights crowd into a few octaves and
// may be equal, and lanes that meet on one word wait for each other.
template <int NT>
constexpr int kCopies = NT / 256;

template <int NT>
struct PickLds {
  __align__(16) uint32_t hist[kBins * kCopies<NT>];
  uint32_t above[NT / 64], equal[NT / 64];
  uint32_t digit, rest, whole;
};

// The best `need` (1 <= need < n) of n keys: emit(position, index) for each, positions ascending
// with the index. Of a block j of 64 keys, place(j) says where it lies (below 0: nowhere, its keys
// are the lowest), raw() loads and key() makes the key of index 64 j + lane; they are called apart
// so that no load waits for another. Places from n on get 0, which is no key. Every wave has a run
// of whole blocks, the first kHeld of them in registers, so the keys are read once. Passes over the
// keys, 11 bits of their distance from the lowest positive one at a time, narrow them to the smallest
// key that is taken and the number of its equals that are: over the range that the keys do take,
// two passes are enough as a rule, since a bin taken whole ends them. Then each wave counts and emits
// its run by ballots. Counts are whole numbers, so no order of the LDS additions changes anything.
// 65536 keys of one workgroup: 20 us at 2.3 GHz, of which the loads take 7 (what one CU gets from
// memory), the first pass 4.5, the second 2.7, the rest is ballots and barriers.
template <int NT, int kHeld, class Keys, class Emit>
__device__ __forceinline__ void pick_best(int n, int need, PickLds<NT>& L, const Keys& keys,
                                          Emit emit) {
  constexpr int NW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PickRun run = pick_run(n, NW, wave);
  const int first = run.first, mine = run.mine;
  uint32_t held[kHeld];
  // a lane finds a block's place, then all blocks are on their way at once
  const int block = pick_block(run, lane), place = block < 0 ? -1 : keys.place(block);
  int lost = 0;
#pragma unroll
  for (int r = 0; r < kHeld; r += 8)
    if (r < mine) {
#pragma unroll
      for (int i = r; i < r + 8; ++i) {
        const int at = __builtin_amdgcn_readlane(place, i);
        lost |= at;
        held[i] = keys.raw(at, first + (i < mine ? i : 0), lane);
      }
    }
#pragma unroll
  for (int r = 0; r < kHeld; r += 8)
    if (r < mine) {
#pragma unroll
      for (int i = r; i < r + 8; ++i) held[i] = keys.key(held[i]);
      // blocks that lie nowhere, and the end of the run or of the keys
      if (lost < 0) {
#pragma unroll
        for (int i = r; i < r + 8; ++i)
          held[i] = __builtin_amdgcn_readlane(place, i) < 0 ? 1u : held[i];
      }
      if (r + 8 >= mine) {
#pragma unroll
        for (int i = r; i < r + 8; ++i)
          held[i] = i < mine && (first + i) * 64 + lane < n ? held[i] : 0u;
      }
    }
  // f(block, key) for the wave's keys, eight blocks of registers a branch
  const auto each = [&](auto f) {
#pragma unroll
    for (int r = 0; r < kHeld; r += 8)
      if (r < mine) {
#pragma unroll
        for (int i = r; i < r + 8; ++i) f(first + i, held[i]);
      }
    for (int r = kHeld; r < mine; ++r) {
      const int at = keys.place(first + r);
      const uint32_t k = at < 0 ? 1u : keys.key(keys.raw(at, first + r, lane));
      f(first + r, (first + r) * 64 + lane < n ? k : 0u);
    }
  };

  constexpr uint32_t kZero = 0x80000000u;              // the key of 0
  uint32_t low = ~0u, high = 0;      // the lowest key above kZero, less kZero + 1, and the highest
  each([&](int, uint32_t k) {
    low = k - kZero - 1 < low ? k - kZero - 1 : low;
    high = k > high ? k : high;
  });
  low = over_lanes(low, ~0u, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
  high = over_lanes(high, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
  if (lane == 63) {
    L.above[wave] = low;
    L.equal[wave] = high;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    low = L.above[w] < low ? L.above[w] : low;
    high = L.equal[w] > high ? L.equal[w] : high;
  }
  low = __builtin_amdgcn_readfirstlane(low);
  high = __builtin_amdgcn_readfirstlane(high);
  // The last key taken lies in prefix .. prefix + span - 1, or, before the first pass, below that.
  uint32_t prefix = low < kZero ? low + kZero + 1 : 1, span = high - prefix + 1;
  uint32_t rest = (uint32_t)need;
  bool first_pass = true;
  do {
    const int bits = span > 1 ? 32 - __builtin_clz(span - 1) : 0;
    const int shift = bits > 11 ? bits - 11 : 0;
    uint4v* bins = reinterpret_cast<uint4v*>(L.hist);
#pragma unroll
    for (int i = 0; i < kBins * kCopies<NT> / 4 / NT; ++i) bins[i * NT + tid] = uint4v{0, 0, 0, 0};
    __syncthreads();
    // digits from 1 up, digit d in bin d - 1: the lowest needs no count
    const uint32_t from = prefix + (1u << shift), to = span - (1u << shift);
    each([&](int, uint32_t k) {
      const uint32_t d = k - from;
      if (d < to) atomicAdd(&L.hist[(d >> shift) * kCopies<NT> + lane % kCopies<NT>], 1u);
    });
    __syncthreads();
    // the bins from the highest down, kBins / NT a thread
    constexpr int BT = kBins / NT;
    uint32_t c[BT], s = 0;
#pragma unroll
    for (int i = 0; i < BT; ++i) {
      c[i] = 0;
#pragma unroll
      for (int j = 0; j < kCopies<NT>; ++j)
        c[i] += L.hist[(kBins - 1 - (tid * BT + i)) * kCopies<NT> + j];
      s += c[i];
    }
    uint32_t before = over_lanes(s, 0u, [](uint32_t a, uint32_t b) { return a + b; });
    if (lane == 63) L.above[wave] = before;
    __syncthreads();
    before -= s;
#pragma unroll
    for (int w = 0; w < NW; ++w) before += w < wave ? L.above[w] : 0u;
#pragma unroll
    for (int i = 0; i < BT; ++i) {
      const int digit = kBins - (tid * BT + i);
      if (before < rest && rest <= before + c[i]) {    // true for one digit, or for none but 0
        L.digit = (uint32_t)digit;
        L.rest = rest - before;
        L.whole = rest == before + c[i];
      }
      before += c[i];
    }
    if (tid == NT - 1 && before < rest) {
      L.digit = L.whole = 0;
      L.rest = rest - before;
    }
    __syncthreads();
    rest = __builtin_amdgcn_readfirstlane(L.rest);
    const uint32_t digit = __builtin_amdgcn_readfirstlane(L.digit);
    if (__builtin_amdgcn_readfirstlane(L.whole)) {     // the whole bin is taken
      prefix += (digit << shift) - 1;
      rest = 0;
      span = 1;
    } else if (first_pass && digit == 0) {             // or something below the first pass's range
      span = prefix + (1u << shift) - 1;
      prefix = 1;
    } else {
      prefix += digit << shift;
      span = 1u << shift;
    }
    first_pass = false;
  } while (span > 1);

  uint32_t na = 0, ne = 0;           // of the wave's run: taken for sure, and equal to the last
  each([&](int, uint32_t k) {
    na += (uint32_t)__popcll(__ballot(k > prefix));
    ne += (uint32_t)__popcll(__ballot(k == prefix));
  });
  __syncthreads();
  if (lane == 0) {
    L.above[wave] = na;
    L.equal[wave] = ne;
  }
  __syncthreads();
  na = ne = 0;
  for (int w = 0; w < wave; ++w) {
    na += L.above[w];
    ne += L.equal[w];
  }
  na = __builtin_amdgcn_readfirstlane(na);
  ne = __builtin_amdgcn_readfirstlane(ne);
  each([&](int j, uint32_t k) {
    const uint64_t ba = __ballot(k > prefix), be = __ballot(k == prefix);
    const uint32_t before = na + (ne < rest ? ne : rest);
    if (be) {
      const uint32_t re = ne + lanes_below(be);
      const uint32_t at = na + lanes_below(ba) + (re < rest ? re : rest);
      if (k > prefix || (k == prefix && re < rest)) emit((int)at, j * 64 + lane);
      ne += (uint32_t)__popcll(be);
    } else if (k > prefix) {
      emit((int)(before + lanes_below(ba)), j * 64 + lane);
    }
    na += (uint32_t)__popcll(ba);
  });
}

__device__ __forceinline__ int held_tokens(const KvSeqs& S, const int32_t* lengths, int max_len,
                                           int seq) {
  int n = lengths[seq];
  const int64_t room = (int64_t)S.width * kPage;
  if (n > max_len) n = max_len;
  if (n > room) n = (int)room;
  return n > 0 ? n : 0;
}


// The weights of one sequence and head as keys: a block is a page.
struct MassKeys {
  const KvPool& pool;
  const KvSeqs& S;
  const float* mass;
  int seq, h;
  __device__ __forceinline__ int place(int j) const { return kv_page(S, pool.P, seq, j); }
  __device__ __forceinline__ uint32_t raw(int page, int, int lane) const {
    return __builtin_bit_cast(
        uint32_t, mass[((int64_t)(page < 0 ? 0 : page) * pool.H + h) * kPage + lane]);
  }
  __device__ __forceinline__ uint32_t key(uint32_t raw) const {
    return order_key(__builtin_bit_cast(float, raw));
  }
};

constexpr int kKeepThreads = 1024;

// One workgroup per (sequence, KV head): the tokens that stay. The passes over a row's weights need
// all of them at once, so a row is one CU's: 27 us for 65536 tokens of 8 heads, 11 for 32 sequences
// of 2048. (Several workgroups a row would need a launch for every pass.)
__global__ __launch_bounds__(kKeepThreads) void keep_kernel(KvPool pool, KvSeqs S,
                                                            const int32_t* __restrict__ lengths,
                                                            int max_len,
                                                            const float* __restrict__ mass,
                                                            int keep, int recent, int32_t* kept,
                                                            int32_t* new_lengths) {
  __shared__ PickLds<kKeepThreads> L;
  const int h = blockIdx.x % pool.H, seq = blockIdx.x / pool.H, tid = threadIdx.x;
  const int n = held_tokens(S, lengths, max_len, seq);
  int32_t* out = kept + (int64_t)blockIdx.x * keep;
  if (h == 0 && tid == 0) new_lengths[seq] = n < keep ? n : keep;
  if (n <= keep) {
    for (int i = tid; i < keep; i += kKeepThreads) out[i] = i < n ? i : -1;
    return;
  }
  const int last = recent < keep ? recent : keep;
  const int need = keep - last, old = n - last;
  for (int i = tid; i < last; i += kKeepThreads) out[need + i] = old + i;
  if (need == 0) return;
  pick_best<kKeepThreads, 64>(
      old, need, L, MassKeys{pool, S, mass, seq, h},
      [&](int at, int i) { out[at] = i; });
}

// A thread's rows of moved tokens: codes times their own pages' scales.
struct MovedK {
  const uint2v* c;                             // row r, channels 0 .. 7
  const float* s;
  __device__ __forceinline__ float value(int r, int i) const {
    return (float)(int8_t)(c[r][i >> 2] >> (8 * (i & 3))) * s[r];
  }
};
struct MovedV {
  const uint32_t* w;                           // channel i, rows 0 .. 3
  const float* s;
  __device__ __forceinline__ float value(int r, int i) const {
    return (float)(int8_t)(w[i] >> (8 * r)) * s[r];
  }
};

__device__ __forceinline__ int code_size(int c) { return c < 0 ? -c : c; }

// One workgroup of 2 D threads per (sequence, new page, KV head): gathers the page's tokens,
// codes them under the scale of their own largest value, and moves their weights along. K is read
// row by row; V (whose tokens lie a byte apart) with a token a lane, so that a wave's load is one
// channel of neighbouring slots, and turned in LDS. The largest value of a token is its largest
// code times its scale. Bound by the chain from lengths and kept over the table to the codes, at 4
// workgroups a CU, and by V's lines, of which most bytes are not kept: 32 sequences of 8 heads keep
// 512 tokens each in 29 us, 107 MB read and written, 67 of them kept (3.7 TB/s).
template <int D>
__global__ __launch_bounds__(2 * D, 4) void move_kernel(KvPool pool, KvSeqs S, KvSeqs to,
                                                     const int32_t* __restrict__ lengths,
                                                     int max_len, float* mass, int keep,
                                                     const int32_t* __restrict__ kept,
                                                     int64_t items) {
  constexpr int NT = 2 * D, NW = NT / 64;
  __shared__ StoreLds<D> L;
  __shared__ int64_t from[kPage];              // (page, head) of a slot's token, or -1
  __shared__ int32_t slot[kPage];
  __shared__ float k_scale[kPage], v_scale[kPage];
  __shared__ uint32_t vt[D * 17];              // V codes [D][64 + 4]
  __shared__ uint32_t tops[NW][2];
  const int tid = threadIdx.x, cg = tid % (D / 8), rg = tid / (D / 8);
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int h = (int)(it % pool.H);
    const int64_t r = it / pool.H;
    const int j = (int)(r % to.width), seq = (int)(r / to.width);
    const int n = held_tokens(S, lengths, max_len, seq);
    const int total = n < keep ? n : keep;
    if (j * (int64_t)kPage >= total) continue;
    const int page = kv_page(to, pool.P, seq, j);
    if (page < 0) continue;
    const int64_t at = (int64_t)page * pool.H + h;
    const int end = total - j * kPage < kPage ? total - j * kPage : kPage;
    if (tid < kPage) {
      int64_t f = -1;
      int t = 0;
      if (tid < end) {
        t = kept[((int64_t)seq * pool.H + h) * keep + j * kPage + tid];
        const int p = kv_page(S, pool.P, seq, t / kPage);
        if (p >= 0) f = (int64_t)p * pool.H + h;
      }
      from[tid] = f;
      slot[tid] = t % kPage;
      k_scale[tid] = f >= 0 ? pool.ks[f] : 0.0f;
      v_scale[tid] = f >= 0 ? pool.vs[f] : 0.0f;
      mass[at * kPage + tid] = f >= 0 ? mass[f * kPage + t % kPage] : 0.0f;
    }
    __syncthreads();
    uint2v kc[4];
    float ks[4], vs[4];
    uint32_t k_top = 0, v_top = 0;             // magnitude bits: ordered as the magnitudes are
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = 4 * rg + e;
      const int64_t f = from[t];
      kc[e] = *reinterpret_cast<const uint2v*>(pool.k + (f < 0 ? 0 : f) * (kPage * D) +
                                               slot[t] * D + 8 * cg);
      ks[e] = k_scale[t];
      vs[e] = v_scale[t];
    }
    {
      constexpr int kSteps = D / NW;
      const int t = tid % kPage, d0 = tid / kPage;
      const int64_t f = from[t];
      const int8_t* src = pool.v + (f < 0 ? 0 : f) * (kPage * D) + slot[t];
      int8_t c[kSteps];
#pragma unroll
      for (int i = 0; i < kSteps; ++i) c[i] = src[(d0 + i * NW) * kPage];
      int top = 0;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int v = f >= 0 ? c[i] : 0;
        top = code_size(v) > top ? code_size(v) : top;
        reinterpret_cast<uint8_t*>(vt)[(d0 + i * NW) * 68 + t] = (uint8_t)v;
      }
      v_top = __builtin_bit_cast(uint32_t, (float)top * v_scale[t]) & 0x7fffffffu;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      int top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = code_size((int8_t)(kc[e][i >> 2] >> (8 * (i & 3))));
        top = c > top ? c : top;
      }
      const uint32_t b = __builtin_bit_cast(uint32_t, (float)top * ks[e]) & 0x7fffffffu;
      k_top = b > k_top ? b : k_top;           // (rows of no token have scale 0)
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
      const uint32_t a = __shfl_xor(k_top, o), b = __shfl_xor(v_top, o);
      k_top = a > k_top ? a : k_top;
      v_top = b > v_top ? b : v_top;
    }
    if ((tid & 63) == 0) {
      tops[tid >> 6][0] = k_top;
      tops[tid >> 6][1] = v_top;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      k_top = tops[w][0] > k_top ? tops[w][0] : k_top;
      v_top = tops[w][1] > v_top ? tops[w][1] : v_top;
    }
    uint32_t vw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) vw[i] = vt[(8 * cg + i) * 17 + rg];
    const float k_new = __builtin_bit_cast(float, k_top) / 127.0f;
    const float v_new = __builtin_bit_cast(float, v_top) / 127.0f;
    const bool finite = k_top < 0x7f800000u && v_top < 0x7f800000u;
    if (finite && plain_scale(k_new) && plain_scale(v_new))
      put_plain<D>(pool, at, MovedK{kc, ks}, MovedV{vw, vs}, end, k_new, v_new, L);
    else
      put_any<D, false>(pool, page, h, MovedK{kc, ks}, MovedV{vw, vs}, 0, end, L);
    __syncthreads();
  }
}

// Keys that other workgroups of the launch have left in memory.
struct LeftKeys {
  uint32_t* keys;
  int n;
  __device__ __forceinline__ int place(int) const { return 0; }
  __device__ __forceinline__ uint32_t raw(int, int j, int lane) const {
    const int e = j * 64 + lane;
    return __hip_atomic_load(keys + (e < n ? e : 0), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ uint32_t key(uint32_t raw) const { return raw; }
};

constexpr int kSelectThreads = 256;
constexpr int kScoreRounds = 4;      // pages a lane group scores at once

// One workgroup per (sequence, query token, KV head) and split of its pages: scores of the pages,
// then the best ones. The group's queries are taken at 8 bits under one power of two, so a score is
// a whole number times the page's K scale, and the same on any machine. max(q8 lo, q8 hi) is q8 hi
// where q8 > 0 and q8 lo where it is not, so the sum over the group's heads goes into the weights
// first: one weight per channel and bound, at most 127 group in size, taken as 128 w1 + w0 for the
// 8-bit dot products. Bound by latency, the chain of table, bounds, keys and the pick's passes: 12.7 us
// for 2048 pages of 8 heads (4 MB), 14.0 for 16 sequences of 256 pages and two queries each.
// With splits, the last workgroup of a row to leave its keys picks (as attend_kernel joins).
template <int D, bool BF16>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(KvPool pool, KvSeqs S, KvAttn A,
                                                                int recent, int splits,
                                                                int32_t* out, uint32_t* keys,
                                                                int np, uint32_t* arrived) {
  __shared__ PickLds<kSelectThreads> L;
  __shared__ float red[kSelectThreads / 64];
  __shared__ uint32_t w0[2 * D / 4], w1[2 * D / 4];    // of the lowest codes, then the highest
  __shared__ uint32_t others;
  const int tid = threadIdx.x;
  const int split = blockIdx.x % splits;
  const int64_t row = blockIdx.x / splits;
  const int h = (int)(row % pool.H), vseq = (int)(row / pool.H);
  const int seq = vseq / A.nq, i = vseq % A.nq;
  int32_t* picks = out + row * A.n_picks;
  const int len = held_tokens(S, A.lengths, A.max_len, seq);
  int ql = A.q_lens ? A.q_lens[seq] : A.nq;
  if (ql > A.nq) ql = A.nq;
  const int64_t sees = i < ql ? (int64_t)len - ql + i + 1 : 0;
  const int seen = sees > 0 ? (int)sees : 0;
  const int pages = (seen + kPage - 1) / kPage;
  const int last = recent < A.n_picks ? recent : A.n_picks;
  const int need = A.n_picks - last, old = pages - last;
  if (pages <= A.n_picks) {
    if (split == 0)
      for (int e = tid; e < A.n_picks; e += kSelectThreads) picks[e] = e < pages ? e : -1;
    return;
  }
  if (split == 0)
    for (int e = tid; e < last; e += kSelectThreads) picks[need + e] = old + e;
  if (need == 0) return;

  const uint16_t* q = static_cast<const uint16_t*>(A.q.p) + seq * A.q.seq +
                      (int64_t)i * A.q.tok + (int64_t)h * A.group * A.q.head;
  float top = 0.0f;
  for (int e = tid; e < A.group * D; e += kSelectThreads) {
    const float a = __builtin_fabsf(kv_widen<BF16>(q[(int64_t)(e / D) * A.q.head + e % D]));
    top = a <= 3.4028234e38f ? fmaxf(top, a) : top;
  }
  top = wg_max<kSelectThreads>(top, red);
  const int shift = 6 - (top > 0.0f ? __builtin_amdgcn_frexp_expf(top) - 1 : 0);
  // D / 8 lanes a page, 16 bytes of its bounds each: the lowest codes, then the highest. Groups
  // past 128 heads are taken 128 heads at a time, whose weights fit two 8-bit digits.
  constexpr int LP = D / 8, PG = kSelectThreads / LP;
  const int per = (old + splits - 1) / splits;
  const int a0 = split * per, a1 = a0 + per < old ? a0 + per : old;
  uint32_t* mine = keys + row * np;
  const int sub = tid % LP;
  for (int g0 = 0; g0 < A.group; g0 += 128) {
    const int g1 = g0 + 128 < A.group ? g0 + 128 : A.group;
    __syncthreads();
    for (int d = tid; d < D; d += kSelectThreads) {
      int up = 0, down = 0;
      for (int g = g0; g < g1; ++g) {
        const float f = __builtin_ldexpf(kv_widen<BF16>(q[(int64_t)g * A.q.head + d]), shift);
        const int c = f != f ? 0 : (int)__builtin_rintf(fminf(fmaxf(f, -127.0f), 127.0f));
        up += c > 0 ? c : 0;
        down -= c < 0 ? c : 0;
      }
      reinterpret_cast<uint8_t*>(w0)[d] = (uint8_t)(down & 127);
      reinterpret_cast<uint8_t*>(w1)[d] = (uint8_t)(down >> 7);
      reinterpret_cast<uint8_t*>(w0)[D + d] = (uint8_t)(up & 127);
      reinterpret_cast<uint8_t*>(w1)[D + d] = (uint8_t)(up >> 7);
    }
    __syncthreads();
    int v0[4], v1[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v0[e] = (int)w0[4 * sub + e];
      v1[e] = (int)w1[4 * sub + e];
    }
    for (int j0 = a0 + tid / LP; j0 < a1; j0 += kScoreRounds * PG) {
      uint4v c[kScoreRounds];
      int page[kScoreRounds];
      float ks[kScoreRounds];
#pragma unroll
      for (int r = 0; r < kScoreRounds; ++r) {
        const int j = j0 + r * PG;
        page[r] = j < a1 ? kv_page(S, pool.P, seq, j) : -1;
      }
#pragma unroll
      for (int r = 0; r < kScoreRounds; ++r) {
        const int64_t at = (int64_t)(page[r] < 0 ? 0 : page[r]) * pool.H + h;
        c[r] = *reinterpret_cast<const uint4v*>(pool.bounds + at * (2 * D) + 16 * sub);
        ks[r] = pool.ks[at];
      }
#pragma unroll
      for (int r = 0; r < kScoreRounds; ++r) {
        int lo = 0, hi = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo = __builtin_amdgcn_sdot4((int)c[r][e], v0[e], lo, false);
          hi = __builtin_amdgcn_sdot4((int)c[r][e], v1[e], hi, false);
        }
        int sum = hi * 128 + lo;
        sum = sub < LP / 2 ? -sum : sum;               // the lowest codes' weights are negative
#pragma unroll
        for (int o = 1; o < LP; o <<= 1) sum += __shfl_xor(sum, o);
        const int j = j0 + r * PG;
        if (sub == 0 && j < a1) {
          // whole numbers until the last head is in
          if (g0 > 0)
            sum += (int)__hip_atomic_load(&mine[j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          const uint32_t k = g1 < A.group ? (uint32_t)sum
                             : page[r] < 0 ? 1u : order_key((float)sum * ks[r]);
          __hip_atomic_store(&mine[j], k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
      }
    }
  }
  if (splits > 1) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // this wave's keys have arrived
    __syncthreads();
    if (tid == 0)
      others = __hip_atomic_fetch_add(&arrived[row], 1u, __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (others != (uint32_t)splits - 1) return;
    if (tid == 0)
      __hip_atomic_store(&arrived[row], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  pick_best<kSelectThreads, 8>(
      old, need, L, LeftKeys{mine, old},
      [&](int at, int j) { picks[at] = j; });
}

unsigned grid_of(int64_t items) { return (unsigned)(items < (1 << 22) ? items : (1 << 22)); }

template <int D>
void move_d(const KvPool& pool, const KvSeqs& S, const KvSeqs& to, const int32_t* lengths,
            int max_len, float* mass, int keep, const int32_t* kept, hipStream_t st) {
  const int64_t items = (int64_t)S.n * to.width * pool.H;
  hipLaunchKernelGGL((move_kernel<D>), dim3(grid_of(items)), dim3(2 * D), 0, st, pool, S, to,
                     lengths, max_len, mass, keep, kept, items);
}

template <int D, bool BF16>
void select_d(const KvPool& pool, const KvSeqs& S, const KvAttn& A, int recent, int32_t* picks,
              char* ws, hipStream_t st) {
  const int np = (int)(((int64_t)A.max_len + kPage - 1) / kPage);
  const int64_t rows = (int64_t)S.n * A.nq * pool.H;
  // a page needs D / 8 lanes: kScoreRounds rounds of the workgroup's lanes a split, and no more
  // splits than two workgroups a CU (one query over 2048 pages: 75 us without splits, 15 with; 16
  // sequences of 256 pages, two queries: 16.8 without, 16.6 with two, 18.4 with four)
  const int round = kScoreRounds * kSelectThreads / (D / 8);
  int64_t splits = rows < kKv8Counters ? (512 + rows - 1) / rows : 1;
  if (splits > (np + round - 1) / round) splits = (np + round - 1) / round;
  if (splits < 1) splits = 1;
  uint32_t* keys = reinterpret_cast<uint32_t*>(ws + kKv8Front);
  // (the C ABI takes at most 2^23 rows: below 2^32 threads)
  hipLaunchKernelGGL((select_kernel<D, BF16>), dim3((unsigned)(rows * splits)),
                     dim3(kSelectThreads), 0, st, pool, S, A, recent, (int)splits, picks, keys, np,
                     reinterpret_cast<uint32_t*>(ws));
}

}  // namespace

uint64_t cg_kv8_select_ws(const KvSeqs& S, int H, int nq, int max_len) {
  return ((uint64_t)S.n * nq * H * (((uint64_t)max_len + kPage - 1) / kPage) * 4ull + kKv8Front + 255) &
         ~255ull;
}

hipError_t cg_launch_kv8_select(const KvPool& pool, const KvSeqs& S, int D, bool bf16,
                                const KvAttn& A, int recent, int32_t* picks, void* ws,
                                hipStream_t st) {
  char* keys = static_cast<char*>(ws);
  switch (D) {
    case 64: (bf16 ? select_d<64, true> : select_d<64, false>)(pool, S, A, recent, picks, keys, st); break;
    case 128: (bf16 ? select_d<128, true> : select_d<128, false>)(pool, S, A, recent, picks, keys, st); break;
    default: (bf16 ? select_d<256, true> : select_d<256, false>)(pool, S, A, recent, picks, keys, st);
  }
  return hipGetLastError();
}

hipError_t cg_launch_kv8_evict(const KvPool& pool, const KvSeqs& S, int D, const int32_t* lengths,
                               int max_len, float* mass, int keep, int recent, const KvSeqs& to,
                               int32_t* kept, int32_t* new_lengths, hipStream_t st) {
  hipLaunchKernelGGL(keep_kernel, dim3((unsigned)(S.n * pool.H)), dim3(kKeepThreads), 0, st, pool,
                     S, lengths, max_len, mass, keep, recent, kept, new_lengths);
  switch (D) {
    case 64: move_d<64>(pool, S, to, lengths, max_len, mass, keep, kept, st); break;
    case 128: move_d<128>(pool, S, to, lengths, max_len, mass, keep, kept, st); break;
    default: move_d<256>(pool, S, to, lengths, max_len, mass, keep, kept, st);
  }
  return hipGetLastError();
}
