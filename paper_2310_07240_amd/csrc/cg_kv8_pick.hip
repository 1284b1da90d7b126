// cg_kv8_pick.hip — which tokens stay (cg_kv8_evict) and which pages a query reads
// (cg_kv8_select): the best `need` of a row of 32-bit keys, ties to the lowest index, in
// ascending order of index; and the move of the kept tokens into new pages.
#include "cg_kv8.h"

namespace {

// Keys in the order of the values: a larger value has a larger key, -0 and +0 the same, a NaN the
// lowest of all.
__device__ __forceinline__ uint32_t order_key(float f) {
  if (f != f) return 0u;
  const uint32_t u = __builtin_bit_cast(uint32_t, f + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int NT>
struct PickLds {
  uint32_t hist[256];
  uint32_t above[NT / 64], equal[NT / 64];
  uint32_t digit, rest;
};

// The best `need` (1 <= need < n) of key(0 .. n - 1): emit(position, index) for each, positions
// ascending with the index. Four passes over the keys' bytes, highest first, narrow them to the
// smallest key that is taken and the number of its equals that are; a fifth pass emits. Counts are
// whole numbers, so no order of the LDS additions changes anything.
template <int NT, class Key, class Emit>
__device__ __forceinline__ void pick_best(int n, int need, PickLds<NT>& L, Key key, Emit emit) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t prefix = 0, mask = 0;
  uint32_t rest = (uint32_t)need;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += NT) L.hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
      const uint32_t k = key(i);
      if ((k & mask) == prefix) atomicAdd(&L.hist[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (wave == 0) {
      // lane l holds bins 255 - 4 l .. 252 - 4 l, the highest first
      uint32_t c[4], s = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = L.hist[255 - 4 * lane - i];
        s += c[i];
      }
      uint32_t before = s;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(before, o);
        if (lane >= o) before += v;
      }
      before -= s;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < rest && rest <= before + c[i]) {   // true in one lane, for one bin
          L.digit = (uint32_t)(255 - 4 * lane - i);
          L.rest = rest - before;
        }
        before += c[i];
      }
    }
    __syncthreads();
    prefix |= L.digit << shift;
    mask |= 255u << shift;
    rest = L.rest;
  }
  uint32_t above = 0, equal = 0;     // taken or equal before this round
  for (int i0 = 0; i0 < n; i0 += NT) {
    const int i = i0 + tid;
    const uint32_t k = i < n ? key(i) : 0u;
    const bool a = i < n && k > prefix, e = i < n && k == prefix;
    const uint64_t ba = __ballot(a), be = __ballot(e);
    if (lane == 0) {
      L.above[wave] = (uint32_t)__popcll(ba);
      L.equal[wave] = (uint32_t)__popcll(be);
    }
    __syncthreads();
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    uint32_t na = above + (uint32_t)__popcll(ba & below), ne = equal + (uint32_t)__popcll(be & below);
    for (int w = 0; w < NT / 64; ++w) {
      if (w < wave) {
        na += L.above[w];
        ne += L.equal[w];
      }
      above += L.above[w];
      equal += L.equal[w];
    }
    if (a || (e && ne < rest)) emit((int)(na + (ne < rest ? ne : rest)), i);
    __syncthreads();
  }
}

__device__ __forceinline__ int held_tokens(const KvSeqs& S, const int32_t* lengths, int max_len,
                                           int seq) {
  int n = lengths[seq];
  const int64_t room = (int64_t)S.width * kPage;
  if (n > max_len) n = max_len;
  if (n > room) n = (int)room;
  return n > 0 ? n : 0;
}

constexpr int kKeepThreads = 1024;

// One workgroup per (sequence, KV head): the tokens that stay.
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
  pick_best<kKeepThreads>(
      old, need, L,
      [&](int i) {
        const int page = kv_page(S, pool.P, seq, i / kPage);
        if (page < 0) return 0u;
        return order_key(mass[((int64_t)page * pool.H + h) * kPage + i % kPage]);
      },
      [&](int at, int i) { out[at] = i; });
}

// One workgroup of 2 D threads per (sequence, new page, KV head): gathers the page's tokens,
// codes them under the scale of their own largest value, and moves their weights along.
template <int D>
__global__ __launch_bounds__(2 * D) void move_kernel(KvPool pool, KvSeqs S, KvSeqs to,
                                                     const int32_t* __restrict__ lengths,
                                                     int max_len, float* mass, int keep,
                                                     const int32_t* __restrict__ kept,
                                                     int64_t items) {
  __shared__ StoreLds<D> L;
  __shared__ int64_t from[kPage];              // (page, head) of a slot's token, or -1
  __shared__ int32_t slot[kPage];
  __shared__ uint8_t vt[D * (kPage + 4)];
  constexpr int NT = 2 * D;
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
      mass[((int64_t)page * pool.H + h) * kPage + tid] =
          f >= 0 ? mass[f * kPage + t % kPage] : 0.0f;
    }
    __syncthreads();
    float x[4][8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = 4 * rg + e;
      const int64_t f = from[t];
      uint2v c = {0, 0};
      float s = 0.0f;
      if (f >= 0) {
        c = *reinterpret_cast<const uint2v*>(pool.k + f * (kPage * D) + slot[t] * D + 8 * cg);
        s = pool.ks[f];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[e][i] = (float)(int8_t)(c[i >> 2] >> (8 * (i & 3))) * s;
    }
    // V: a lane is a token, so a wave reads one channel of neighbouring slots
    for (int d = tid / kPage; d < D; d += NT / kPage) {
      const int t = tid % kPage;
      const int64_t f = from[t];
      vt[d * (kPage + 4) + t] =
          f >= 0 ? (uint8_t)pool.v[f * (kPage * D) + (int64_t)d * kPage + slot[t]] : 0;
    }
    put_page<D, false>(pool, page, h, x, 0, end, L);   // its barriers cover vt
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = 4 * rg + e;
      const int64_t f = from[t];
      const float s = f >= 0 ? pool.vs[f] : 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[e][i] = (float)(int8_t)vt[(8 * cg + i) * (kPage + 4) + t] * s;
    }
    put_page<D, true>(pool, page, h, x, 0, end, L);
  }
}

constexpr int kSelectThreads = 256;

// One workgroup per (sequence, query token, KV head): scores of the pages, then the best ones.
// The group's queries are taken at 8 bits under one power of two, so a score is a whole number
// times the page's K scale, and the same on any machine.
template <int D, bool BF16>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(KvPool pool, KvSeqs S, KvAttn A,
                                                                int recent, int32_t* out,
                                                                uint32_t* keys, int np) {
  __shared__ PickLds<kSelectThreads> L;
  __shared__ float red[kSelectThreads / 64];
  __shared__ int up[D], down[D];
  const int tid = threadIdx.x;
  const int h = blockIdx.x % pool.H, vseq = blockIdx.x / pool.H;
  const int seq = vseq / A.nq, i = vseq % A.nq;
  int32_t* picks = out + (int64_t)blockIdx.x * A.n_picks;
  const int len = held_tokens(S, A.lengths, A.max_len, seq);
  int ql = A.q_lens ? A.q_lens[seq] : A.nq;
  if (ql > A.nq) ql = A.nq;
  const int seen = i < ql && len - ql + i + 1 > 0 ? len - ql + i + 1 : 0;
  const int pages = (seen + kPage - 1) / kPage;
  if (pages <= A.n_picks) {
    for (int e = tid; e < A.n_picks; e += kSelectThreads) picks[e] = e < pages ? e : -1;
    return;
  }
  const int last = recent < A.n_picks ? recent : A.n_picks;
  const int need = A.n_picks - last, old = pages - last;
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
  for (int d = tid; d < D; d += kSelectThreads) {
    int u = 0, w = 0;
    for (int g = 0; g < A.group; ++g) {
      const float f = __builtin_ldexpf(kv_widen<BF16>(q[(int64_t)g * A.q.head + d]), shift);
      const int c = f != f ? 0
                           : (int)__builtin_rintf(fminf(fmaxf(f, -127.0f), 127.0f));
      u += c > 0 ? c : 0;
      w += c < 0 ? c : 0;
    }
    up[d] = u;
    down[d] = w;
  }
  __syncthreads();
  // D / 8 lanes a page, 16 bytes of its bounds each: the lowest codes, then the highest
  constexpr int LP = D / 8;
  uint32_t* mine = keys + (int64_t)blockIdx.x * np;
  const int sub = tid % LP;
  for (int j = tid / LP; j < old; j += kSelectThreads / LP) {
    const int page = kv_page(S, pool.P, seq, j);
    int sum = 0;
    if (page >= 0) {
      const uint4v c = *reinterpret_cast<const uint4v*>(
          pool.bounds + ((int64_t)page * pool.H + h) * (2 * D) + 16 * sub);
      const int* w = sub < LP / 2 ? down + 16 * sub : up + 16 * sub - D;
#pragma unroll
      for (int e = 0; e < 16; ++e) sum += w[e] * (int)(int8_t)(c[e >> 2] >> (8 * (e & 3)));
    }
#pragma unroll
    for (int o = 1; o < LP; o <<= 1) sum += __shfl_xor(sum, o);
    if (sub == 0)
      mine[j] = page < 0 ? 0u : order_key((float)sum * pool.ks[(int64_t)page * pool.H + h]);
  }
  __syncthreads();
  pick_best<kSelectThreads>(
      old, need, L, [&](int j) { return mine[j]; }, [&](int at, int j) { picks[at] = j; });
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
              uint32_t* keys, hipStream_t st) {
  const int np = (int)(((int64_t)A.max_len + kPage - 1) / kPage);
  hipLaunchKernelGGL((select_kernel<D, BF16>), dim3((unsigned)(S.n * A.nq * pool.H)),
                     dim3(kSelectThreads), 0, st, pool, S, A, recent, picks, keys, np);
}

}  // namespace

uint64_t cg_kv8_select_ws(const KvSeqs& S, int H, int nq, int max_len) {
  return ((uint64_t)S.n * nq * H * (((uint64_t)max_len + kPage - 1) / kPage) * 4ull + 255) & ~255ull;
}

hipError_t cg_launch_kv8_select(const KvPool& pool, const KvSeqs& S, int D, bool bf16,
                                const KvAttn& A, int recent, int32_t* picks, void* ws,
                                hipStream_t st) {
  uint32_t* keys = static_cast<uint32_t*>(ws);
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
