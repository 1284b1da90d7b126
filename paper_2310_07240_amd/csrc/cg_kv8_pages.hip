// cg_kv8_pages.hip — who holds which page of the 8-bit cache: sequences that share another's pages
// (cg_kv8_fork), pages for what comes (cg_kv8_reserve), pages given back (cg_kv8_release), moved
// together (cg_kv8_compact) and copied (cg_kv8_copy).
//
// Free pages are found by rank: sums over the pages' counts give each page its place among the free
// ones (or those in use), so the i-th page wanted gets the i-th free one, and no result depends on
// an order of arrival. Up to some tens of thousands of pages one workgroup does it all: a second one
// would have to hand its sums over, which takes longer than the pages do. Of larger pools a workgroup
// counts 4096 pages, and the last to arrive sums up; what workgroups of one launch hand to each other
// is written and read past the XCDs' own caches (agent scope).
#include "cg_kv8.h"

#include <type_traits>

namespace {

constexpr int kRounds = 16, kChunk = 256 * kRounds;   // (of a workgroup of 256)

__device__ __forceinline__ void put_far(int32_t* p, int32_t v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ int32_t get_far(const int32_t* p) {
  return __hip_atomic_load(const_cast<int32_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ int below(uint64_t mask) {     // set bits under the lane's own
  return __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1));
}

// Whether this workgroup is the last of the launch to come here; all that it wrote has arrived
// before it counts itself in. The counter is left at zero.
__device__ __forceinline__ bool last_here(uint32_t* counter, uint32_t* lds) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    *lds = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (*lds == gridDim.x - 1)
      __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return *lds == gridDim.x - 1;
}

// Exclusive sum over the workgroup's NT threads; `total` receives the whole. lds: a word a wave.
template <int NT, class T>
__device__ __forceinline__ T scan_wg(T x, T* lds, T& total) {
  T s = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(s, o);
    s += (int)(threadIdx.x & 63) >= o ? y : 0;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  T before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const T y = lds[w];
    before += w < (int)(threadIdx.x >> 6) ? y : 0;
    total += y;
  }
  return before + s - x;
}

// In place: values [n] another workgroup of the launch wrote become their exclusive sums. Returns
// the whole. (Sums past 32 bits are of no use to anyone: more pages than a pool can have.)
__device__ __forceinline__ int64_t scan_far(int32_t* v, int n, int64_t* lds) {
  constexpr int N = 8;
  int64_t run = 0;
  for (int64_t i0 = 0; i0 < n; i0 += 256 * N) {
    int32_t x[N];
    int64_t sum = 0, total;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int64_t i = i0 + threadIdx.x * N + k;
      x[k] = i < n ? get_far(v + i) : 0;
      sum += x[k];
    }
    int64_t at = run + scan_wg<256>(sum, lds, total);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int64_t i = i0 + threadIdx.x * N + k;
      if (i < n) v[i] = (int32_t)at;
      at += x[k];
    }
    run += total;
  }
  return run;
}

template <int NT>
struct ChunkLds {
  int32_t at[kRounds * NT / 64];     // pages in use before round k's wave w: [k][w]
  int32_t total;
};

// The pages of a chunk of 16 NT, a thread each in 16 rounds. Held: the counts, then f(page, count,
// pages of the chunk in use before it) for every page.
template <int NT>
struct Chunk {
  int32_t r[kRounds];
  int64_t p0;

  __device__ __forceinline__ void load(const int32_t* refs, int P, int chunk) {
    p0 = (int64_t)chunk * (kRounds * NT) + threadIdx.x;
#pragma unroll
    for (int k = 0; k < kRounds; ++k) r[k] = p0 + k * NT < P ? refs[p0 + k * NT] : 0;
  }
  __device__ __forceinline__ bool past(int P, int k) const {   // no page of round k, in any lane
    return p0 - threadIdx.x + k * NT >= P;
  }
  // Returns the chunk's pages in use.
  __device__ __forceinline__ int count(int P, ChunkLds<NT>& L) const {
    constexpr int W = NT / 64, E = kRounds * W / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();                 // the LDS may have been used
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      const uint64_t mask = __ballot(r[k] > 0);
      if (lane == 0) L.at[k * W + wave] = __popcll(mask);
    }
    __syncthreads();
    if (wave == 0) {
      int x[E], sum = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x[e] = sum;
        sum += L.at[lane * E + e];
      }
      int s = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(s, o);
        s += lane >= o ? y : 0;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) L.at[lane * E + e] = s - sum + x[e];
      if (lane == 63) L.total = s;
    }
    __syncthreads();
    return L.total;
  }
  template <class F>
  __device__ __forceinline__ void each(int P, const ChunkLds<NT>& L, F f) const {
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      if (past(P, k)) break;
      const int before = L.at[k * (NT / 64) + (threadIdx.x >> 6)] + below(__ballot(r[k] > 0));
      if (p0 + k * NT < P) f((int)(p0 + k * NT), r[k], before);
    }
  }
};

// ---- copies -----------------------------------------------------------------------------------
// A page is copied in pieces of 16 KB of its codes, K's and then V's, a workgroup each, with four
// 16-byte loads of a thread on their way together; the pieces share its scales, bounds and weights.
// Bound by those bytes: 2048 pages of 8 heads of 128 channels, 554 MB read and written in 113 us, 4.9
// TB/s (a copy of 1 GiB: 5.1); 96 us where the Infinity Cache has a part of them from the call before.
constexpr int kUnits = 1024;           // of 16 bytes, a piece

__host__ __device__ inline int pieces_of(int H, int D) {
  return (int)(((int64_t)8 * H * D + kUnits - 1) / kUnits);
}

// More of them than the L2s hold are read and written past the caches (without / with, whole calls, us:
// 2048 pages 115.3 / 113.5, 1024 of a compaction 67.9 / 60.0; with few it is slower, 70 pages of 40 KB
// 7.5 / 8.4). Copies of a shared page are only written past them, however few: its readers then find it
// there (512 copies of 32 pages, with the calls around them, 45.2 / 35.6; read past them too 49.6). With the
// store and the attention that come next both are alike: 8 requests 38.1 / 38.9, 64 50.1 / 49.4, 512
// 155.8 / 157.0.
__device__ __forceinline__ bool past_caches(int64_t items) {
  return items > (32 << 20) / (16 * kUnits);
}

// loads_past, stores_past: nontemporal accesses to the codes.
__device__ __forceinline__ void copy_piece(const KvPool& pool, int D, int src, int dst, int piece,
                                           int pieces, bool loads_past, bool stores_past) {
  const int64_t half = (int64_t)4 * pool.H * D;                // 16-byte units of K (and of V)
  const uint4v* k = reinterpret_cast<const uint4v*>(pool.k);
  const uint4v* v = reinterpret_cast<const uint4v*>(pool.v);
  uint4v x[kUnits / 256];
  const int64_t u0 = (int64_t)piece * kUnits + threadIdx.x;
  const auto read = [&](auto past) {
#pragma unroll
    for (int i = 0; i < kUnits / 256; ++i) {
      const int64_t u = u0 + 256 * i;
      if (u >= 2 * half) continue;
      const uint4v* const from = u < half ? k + src * half + u : v + src * half + u - half;
      x[i] = decltype(past)::value ? __builtin_nontemporal_load(from) : *from;
    }
  };
  if (loads_past) read(std::true_type{});
  else read(std::false_type{});
  // words of the scales, the bounds and the weights
  const int H = pool.H, nb = pool.bounds ? H * (D / 2) : 0, nm = pool.mass ? H * kPage : 0;
  uint32_t* const bounds = reinterpret_cast<uint32_t*>(pool.bounds);
  for (int i = piece * 256 + threadIdx.x; i < 2 * H + nb + nm; i += pieces * 256) {
    if (i < H) {
      pool.ks[(int64_t)dst * H + i] = pool.ks[(int64_t)src * H + i];
    } else if (i < 2 * H) {
      pool.vs[(int64_t)dst * H + i - H] = pool.vs[(int64_t)src * H + i - H];
    } else if (i < 2 * H + nb) {
      const int64_t w = i - 2 * H, n = H * (D / 2);
      bounds[dst * n + w] = bounds[src * n + w];
    } else {
      const int64_t w = i - 2 * H - nb, n = H * kPage;
      pool.mass[dst * n + w] = pool.mass[src * n + w];
    }
  }
  uint4v* const k_to = reinterpret_cast<uint4v*>(pool.k);
  uint4v* const v_to = reinterpret_cast<uint4v*>(pool.v);
  const auto write = [&](auto past) {
#pragma unroll
    for (int i = 0; i < kUnits / 256; ++i) {
      const int64_t u = u0 + 256 * i;
      if (u >= 2 * half) continue;
      uint4v* const to = u < half ? k_to + dst * half + u : v_to + dst * half + u - half;
      if (decltype(past)::value) __builtin_nontemporal_store(x[i], to);
      else *to = x[i];
    }
  };
  if (stores_past) write(std::true_type{});
  else write(std::false_type{});
}

__global__ __launch_bounds__(256) void copy_kernel(KvPool pool, int D, const int32_t* src,
                                                   const int32_t* dst, int pieces, int64_t items) {
  const bool past = past_caches(items);
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t i = it / pieces;
    const int a = src[i], b = dst[i];
    if (a >= 0 && a < pool.P && b >= 0 && b < pool.P && a != b)
      copy_piece(pool, D, a, b, (int)(it % pieces), pieces, past, past);
  }
}

// ---- sharing and giving back --------------------------------------------------------------------
__device__ __forceinline__ bool names_page(int32_t p, int P) { return p >= 0 && p < P; }

// One holder less; a count that is 0 stays. (However many threads do so at once, the count ends at
// what it was less the holders, or 0.)
__device__ __forceinline__ void drop(int32_t* refs, int p) {
  if (atomicSub(refs + p, 1) <= 0) atomicAdd(refs + p, 1);
}

__device__ __forceinline__ int clamp_len(int64_t n, int width) {
  const int64_t room = (int64_t)width * kPage;
  n = n < room ? n : room;
  n = n < INT32_MAX ? n : INT32_MAX;
  return n > 0 ? (int)n : 0;
}

// A workgroup = 256 columns of a row. Bound by the counts' additions (sharers of a page meet on it): 512
// children of 66 pages 5.5 us, 8 of 16 2.9.
__global__ __launch_bounds__(256) void fork_kernel(int P, KvSeqs S, const int32_t* lengths,
                                                   const int32_t* parents, const int32_t* ends,
                                                   int width, int per_row, int32_t* table,
                                                   int32_t* new_lengths, int32_t* refs) {
  const int row = blockIdx.x / per_row, j = blockIdx.x % per_row * 256 + threadIdx.x;
  const int p = parents[row];
  int len = 0;
  if (p >= 0 && p < S.n) {
    len = clamp_len(lengths[p], S.width);
    if (ends) len = ends[row] < len ? (ends[row] > 0 ? ends[row] : 0) : len;
  }
  if (j == 0) new_lengths[row] = len;
  if (j >= width) return;
  int32_t page = -1;
  if ((int64_t)j * kPage < len) page = kv_page(S, P, p, j);
  table[(int64_t)row * width + j] = page;
  if (page >= 0) atomicAdd(refs + page, 1);
}

__global__ __launch_bounds__(256) void release_kernel(int P, int width, int per_row, int32_t* table,
                                                      const int32_t* keep, int32_t* refs) {
  const int row = blockIdx.x / per_row, j = blockIdx.x % per_row * 256 + threadIdx.x;
  if (j >= width || (keep && (int64_t)j * kPage < keep[row])) return;
  int32_t* const at = table + (int64_t)row * width + j;
  const int32_t p = *at;
  if (names_page(p, P)) drop(refs, p);
  if (p != -1) *at = -1;
}

// ---- pages for what comes -----------------------------------------------------------------------
// The workspace of reserve behind the counters.
struct Reserve {
  int32_t* chunks;                   // [chunks] free pages of each, then before each
  int32_t* need;                     // [n] pages that each sequence wants, then those before it
  int32_t* source;                   // [n] the page that a sequence's first wanted one copies, or -1
  uint64_t* wants;                   // [n][words] bits: the columns that want a page, by sequence,
  uint64_t* drops;                   // and those that name a page which others hold too
  int64_t* bits;                     // [n] where a sequence's first column lies in them
  int32_t* state;                    // pages wanted by all, or -1: there are not as many
  int32_t* list;                     // [at most P] the free pages in order
};

struct Span {                        // columns that a sequence will write to, and tokens
  int first, last, start, end;       // (last, end: one behind)
};

__device__ __forceinline__ Span span_of(const int32_t* lengths, const int32_t* counts, int width,
                                        int b) {
  const int start = clamp_len(lengths[b], width);
  const int64_t end = clamp_len((int64_t)start + (counts[b] > 0 ? counts[b] : 0), width);
  Span s;
  s.start = start;
  s.end = (int)end;
  s.first = start / kPage;
  s.last = end > start ? (int)((end + kPage - 1) / kPage) : s.first;
  return s;
}

// Workgroups 0 .. chunks - 1 count the free pages of their chunks, the others what four sequences
// want, a wave each; the last to come sums both up.
__global__ __launch_bounds__(256) void want_kernel(int P, int n, int width, const int32_t* table,
                                                   const int32_t* lengths, const int32_t* counts,
                                                   const int32_t* refs, int chunks, int words,
                                                   Reserve R, int32_t* missing,
                                                   uint32_t* counter) {
  __shared__ ChunkLds<256> L;
  __shared__ int64_t sums[4];
  __shared__ uint32_t order;
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x < chunks) {
    const int chunk = blockIdx.x;
    Chunk<256> c;
    c.load(refs, P, chunk);
    const int used = c.count(P, L);
    const int64_t left = (int64_t)P - (int64_t)chunk * kChunk;
    if (threadIdx.x == 0) put_far(R.chunks + chunk, (int)(left < kChunk ? left : kChunk) - used);
  } else {
    const int b = ((int)blockIdx.x - chunks) * 4 + (threadIdx.x >> 6);
    if (b < n) {
      const Span s = span_of(lengths, counts, width, b);
      int need = 0, source = -1;
      for (int j0 = s.first; j0 < s.last; j0 += 64) {
        const int j = j0 + lane;
        bool want = false, drops = false;
        if (j < s.last) {
          const int32_t p = table[(int64_t)b * width + j];
          const int held = names_page(p, P) ? refs[p] : 0;
          // a page with tokens that stay is copied if others hold it too (one that is lost stays
          // so); behind them a page has to be the sequence's alone
          const bool keeps = (int64_t)j * kPage < s.start;
          want = keeps ? held > 1 : held != 1;
          drops = held > 1;
          if (keeps && want) source = p;
        }
        const uint64_t mask = __ballot(want), shared = __ballot(drops);
        if (lane == 0) {
          const int64_t w = (int64_t)b * words + (j0 - s.first) / 64;
          R.wants[w] = mask;
          R.drops[w] = shared;
        }
        need += __popcll(mask);
      }
      if (lane == 0) {                 // (a page that is copied is in the first column: lane 0's)
        R.source[b] = source;
        R.bits[b] = (int64_t)b * words * 64;
        put_far(R.need + b, need);
      }
    }
  }
  if (!last_here(counter, &order)) return;
  const int64_t free = scan_far(R.chunks, chunks, sums);
  const int64_t wanted = scan_far(R.need, n, sums);
  const bool ok = wanted <= free;
  if (threadIdx.x == 0) {
    *R.state = ok ? (int32_t)wanted : -1;
    *missing = ok ? 0 : wanted - free < INT32_MAX ? (int32_t)(wanted - free) : INT32_MAX;
  }
}

// The free pages to their places in the list, as far as they are wanted.
__global__ __launch_bounds__(256) void list_kernel(int P, const int32_t* refs, Reserve R) {
  __shared__ ChunkLds<256> L;
  const int wanted = *R.state, before = R.chunks[blockIdx.x], first = blockIdx.x * kChunk;
  if (before >= wanted) return;
  Chunk<256> c;
  c.load(refs, P, blockIdx.x);
  c.count(P, L);
  c.each(P, L, [&](int page, int held, int used_before) {
    const int64_t rank = (int64_t)before + (page - first - used_before);
    if (held <= 0 && rank < wanted) R.list[rank] = page;
  });
}

// All of the above in one workgroup. A thread takes a sequence's span of columns first; then the
// spans' columns lie one after the other, a thread each, found by a search over the spans' sums in
// LDS. Then the free pages, 16384 a step, until there are as many as wanted. Bound by a chain of
// dependent reads (lengths, table, counts) and the sums between them: 8 sequences of 256 pages 5.6 us,
// 512 of 3500 7.0, 384 of 65536 10.9.
constexpr int kPlanThreads = 1024, kPlanSeqs = 2048, kPlanPages = 16 * kPlanThreads;

struct PlanLds {
  int32_t at[kPlanSeqs + 1];           // columns before each sequence's
  int32_t first[kPlanSeqs];            // its first column
  int32_t keep[kPlanSeqs];             // tokens of its first column that stay
  int32_t sums[kPlanThreads / 64];
};

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(int P, int n, int width,
                                                            const int32_t* table,
                                                            const int32_t* lengths,
                                                            const int32_t* counts,
                                                            const int32_t* refs, Reserve R,
                                                            int32_t* missing) {
  __shared__ PlanLds L;
  __shared__ ChunkLds<kPlanThreads> C;
  const int tid = threadIdx.x, lane = tid & 63;
  Chunk<kPlanThreads> c;
  c.load(refs, P, 0);                                  // (on its way meanwhile)
  int cols = 0, total;
  for (int b0 = 0; b0 < n; b0 += kPlanThreads) {
    const int b = b0 + tid;
    Span s = {0, 0, 0, 0};
    if (b < n) s = span_of(lengths, counts, width, b);
    const int at = cols + scan_wg<kPlanThreads>(s.last - s.first, L.sums, total);
    if (b < n) {
      L.at[b] = at;
      L.first[b] = s.first;
      L.keep[b] = s.start - s.first * kPage;
      R.bits[b] = at;
      if (s.first == s.last) R.source[b] = -1;         // (the others': with their first column)
    }
    cols += total;
  }
  if (tid == 0) L.at[n] = cols;
  __syncthreads();
  // which of the columns want a page
  int wanted = 0;
  for (int i0 = 0; i0 < cols; i0 += kPlanThreads) {
    const int i = i0 + tid;
    bool want = false, drops = false;
    int b = 0, j = 0, page = -1;
    if (i < cols) {
      int lo = 0, hi = n;                              // at[lo] <= i < at[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (L.at[mid] <= i) lo = mid;
        else hi = mid;
      }
      b = lo;
      j = i - L.at[b];
      page = table[(int64_t)b * width + L.first[b] + j];
      const int held = names_page(page, P) ? refs[page] : 0;
      drops = held > 1;
      want = j == 0 && L.keep[b] > 0 ? drops : held != 1;
    }
    const uint64_t mask = __ballot(want), shared = __ballot(drops);
    if (lane == 0 && i < cols) {
      R.wants[i >> 6] = mask;
      R.drops[i >> 6] = shared;
    }
    const int rank = wanted + scan_wg<kPlanThreads>(want ? 1 : 0, L.sums, total);
    if (i < cols && j == 0) {
      R.need[b] = rank;
      R.source[b] = want && L.keep[b] > 0 ? page : -1;
    }
    wanted += total;
  }
  // the first free pages
  int free = 0;
  for (int chunk = 0; (int64_t)chunk * kPlanPages < P && (free < wanted || chunk == 0); ++chunk) {
    if (chunk) c.load(refs, P, chunk);
    const int first = chunk * kPlanPages, left = P - first, used = c.count(P, C);
    c.each(P, C, [&](int page, int held, int used_before) {
      const int rank = free + (page - first - used_before);
      if (held <= 0 && rank < wanted) R.list[rank] = page;
    });
    free += (left < kPlanPages ? left : kPlanPages) - used;
  }
  if (tid == 0) {
    const bool ok = wanted <= free;
    *R.state = ok ? wanted : -1;
    *missing = ok ? 0 : wanted - free;
  }
}

// n <= 64 bits from bit `at` on.
__device__ __forceinline__ uint64_t bits_at(const uint64_t* w, int64_t at, int n) {
  const int off = (int)(at & 63);
  uint64_t x = w[at >> 6] >> off;
  if (n > 64) n = 64;
  if (off + n > 64) x |= w[(at >> 6) + 1] << (64 - off);
  return n < 64 ? x & ((1ull << n) - 1) : x;
}

// Workgroup = (sequence, piece of a page): the first piece's first wave hands the pages out and says
// what the sequence may store, all pieces copy the sequence's shared page. 512 copies of 135 KB from 32 pages 17 us, 66 MiB written.
__global__ __launch_bounds__(256) void hand_out_kernel(KvPool pool, int D, int n, int width,
                                                       int32_t* table, const int32_t* lengths,
                                                       const int32_t* counts, int32_t* refs,
                                                       int32_t* granted, int pieces, int64_t items,
                                                       Reserve R) {
  const int lane = threadIdx.x & 63, wanted = *R.state;
  if (wanted <= 0 && !granted) return;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int b = (int)(it / pieces), piece = (int)(it % pieces);
    int rank = 0;
    if (wanted > 0) {
      const int source = R.source[b];
      rank = R.need[b];                                // (of no use where nothing is wanted)
      if (source >= 0) copy_piece(pool, D, source, R.list[rank], piece, pieces, false, true);
    }
    if (piece != 0 || threadIdx.x >= 64) continue;
    const Span s = span_of(lengths, counts, width, b);
    if (granted && lane == 0) granted[b] = wanted >= 0 ? s.end - s.start : 0;
    if (wanted <= 0) continue;
    for (int j0 = s.first; j0 < s.last; j0 += 64) {
      const int64_t at = R.bits[b] + (j0 - s.first);
      const int left = s.last - j0;
      const uint64_t mask = bits_at(R.wants, at, left);
      if (mask >> lane & 1) {
        int32_t* const entry = table + (int64_t)b * width + j0 + lane;
        const int32_t page = R.list[rank + below(mask)];
        if (bits_at(R.drops, at, left) >> lane & 1) drop(refs, *entry);
        *entry = page;
        refs[page] = 1;
      }
      rank += __popcll(mask);
    }
  }
}

// ---- pages moved together -----------------------------------------------------------------------
struct Compact {
  int32_t* chunks;                   // [chunks] pages in use of each, then before each
  int32_t* state;                    // pages in use, those of them that lie in front, moves
  int32_t* holes;                    // [P / 2 + 1] free pages in front, in order
  int32_t* late;                     // [P / 2 + 1] pages in use behind, in order
  int32_t* key;                      // [P] a page's new number, -1 (free), or -2 - i: the i-th hole
};

// What becomes of a page that `rank` pages in use lie before, of `live` in all and `front` before
// page `live`.
__device__ __forceinline__ void place(const Compact& C, int32_t* moved, int32_t* new_refs, int page,
                                      int held, int rank, int live, int front) {
  int key = held > 0 ? page : -1;
  if (page < live) {
    if (held <= 0) C.holes[page - rank] = page;
    else new_refs[page] = held;
  } else {
    if (held > 0) {
      C.late[rank - front] = page;
      key = -2 - (rank - front);
    }
    new_refs[page] = 0;
  }
  C.key[page] = key;
  if (key >= -1) moved[page] = key;
}

__global__ __launch_bounds__(256) void used_kernel(int P, const int32_t* refs, int chunks, Compact C,
                                                   int32_t* n_live, uint32_t* counter) {
  __shared__ ChunkLds<256> L;
  __shared__ int64_t sums[4];
  __shared__ uint32_t order;
  __shared__ int32_t in_front;
  Chunk<256> k;
  k.load(refs, P, blockIdx.x);
  const int used = k.count(P, L);
  if (threadIdx.x == 0) put_far(C.chunks + blockIdx.x, used);
  if (!last_here(counter, &order)) return;
  const int live = (int)scan_far(C.chunks, chunks, sums);
  __syncthreads();                   // (scan_far's writes are this workgroup's own)
  if (threadIdx.x == 0) in_front = live;               // (all of them, where live == P)
  __syncthreads();
  if (live < P) {
    // pages in use before page `live`
    const int c = live / kChunk, before = C.chunks[c];
    k.load(refs, P, c);
    k.count(P, L);
    k.each(P, L, [&](int page, int, int used_before) {
      if (page == live) in_front = before + used_before;
    });
    __syncthreads();
  }
  const int front = in_front;
  if (threadIdx.x == 0) {
    C.state[0] = live;
    C.state[1] = front;
    C.state[2] = live - front;
    *n_live = live;
  }
}

__global__ __launch_bounds__(256) void place_kernel(int P, const int32_t* refs, Compact C,
                                                    int32_t* moved, int32_t* new_refs) {
  __shared__ ChunkLds<256> L;
  const int before = C.chunks[blockIdx.x], live = C.state[0], front = C.state[1];
  Chunk<256> c;
  c.load(refs, P, blockIdx.x);
  c.count(P, L);
  c.each(P, L, [&](int page, int held, int used_before) {
    place(C, moved, new_refs, page, held, before + used_before, live, front);
  });
}

// Both in one workgroup, which holds all counts in registers.
__global__ __launch_bounds__(kPlanThreads) void places_kernel(int P, const int32_t* refs, Compact C,
                                                              int32_t* moved, int32_t* new_refs,
                                                              int32_t* n_live) {
  __shared__ ChunkLds<kPlanThreads> L;
  __shared__ int32_t in_front;
  Chunk<kPlanThreads> c;
  c.load(refs, P, 0);
  const int live = c.count(P, L);
  if (threadIdx.x == 0) in_front = live;               // (all of them, where there are no others)
  __syncthreads();
  c.each(P, L, [&](int page, int, int before) {
    if (page == live) in_front = before;
  });
  __syncthreads();
  const int front = in_front;
  c.each(P, L, [&](int page, int held, int before) {
    place(C, moved, new_refs, page, held, before, live, front);
  });
  if (threadIdx.x == 0) {
    C.state[0] = live;
    C.state[1] = front;
    C.state[2] = live - front;
    *n_live = live;
  }
}

// The moves, and the table: workgroups 0 .. movers - 1 copy, the others rewrite entries. 1024 pages of
// 8 heads of 128 channels, 266 MiB in 51 us, 5.4 TB/s.
__global__ __launch_bounds__(256) void move_kernel(KvPool pool, int D, const int32_t* refs,
                                                   int64_t entries, const int32_t* table,
                                                   int32_t* new_table, int movers, int pieces,
                                                   Compact C, int32_t* moved, int32_t* new_refs) {
  if ((int)blockIdx.x < movers) {
    const int64_t items = (int64_t)C.state[2] * pieces;
    const bool past = past_caches(items);
    for (int64_t it = blockIdx.x; it < items; it += movers) {
      const int i = (int)(it / pieces), piece = (int)(it % pieces);
      const int src = C.late[i], dst = C.holes[i];
      copy_piece(pool, D, src, dst, piece, pieces, past, past);
      if (piece == 0 && threadIdx.x == 0) {
        moved[src] = dst;
        new_refs[dst] = refs[src];
      }
    }
    return;
  }
  for (int64_t e = (int64_t)(blockIdx.x - movers) * 256 + threadIdx.x; e < entries;
       e += (int64_t)(gridDim.x - movers) * 256) {
    const int32_t p = table[e];
    int32_t to = names_page(p, pool.P) ? C.key[p] : -1;
    if (to < -1) to = C.holes[-2 - to];
    new_table[e] = to;
  }
}

unsigned grid_of(int64_t items) { return (unsigned)(items < (1 << 20) ? items : (1 << 20)); }

int chunks_of(int P) { return (int)(((int64_t)P + kChunk - 1) / kChunk); }

// Launches of a workgroup for each 256 columns of a row, of below 2^32 threads each.
template <class Launch>
void in_rows(int n, int width, Launch launch) {
  const int per_row = (int)(((int64_t)width + 255) / 256);
  const int most = per_row < (1 << 22) ? (1 << 22) / per_row : 1;
  for (int row0 = 0; row0 < n; row0 += most)
    launch(row0, n - row0 < most ? n - row0 : most, per_row);
}

// The words of `wants`: a sequence's columns from its first on, 64 a word.
int words_of(int width) { return (width + 63) / 64; }

struct Carve {                         // pieces of a workspace, each 256-byte aligned
  char* base;
  uint64_t at;
  template <class T>
  T* take(int64_t n) {
    T* p = reinterpret_cast<T*>(base + at);
    at = (at + (uint64_t)n * sizeof(T) + 255) & ~255ull;
    return p;
  }
};

Reserve reserve_of(void* ws, int P, int n, int width, uint64_t* total) {
  Carve c = {static_cast<char*>(ws), kKv8Front};
  Reserve R;
  R.chunks = c.take<int32_t>(chunks_of(P));
  R.need = c.take<int32_t>(n);
  R.source = c.take<int32_t>(n);
  R.wants = c.take<uint64_t>((int64_t)n * words_of(width));
  R.drops = c.take<uint64_t>((int64_t)n * words_of(width));
  R.bits = c.take<int64_t>(n);
  R.state = c.take<int32_t>(1);
  const int64_t most = (int64_t)n * width;
  R.list = c.take<int32_t>(most < P ? most : P);
  *total = c.at;
  return R;
}

Compact compact_of(void* ws, int P, uint64_t* total) {
  Carve c = {static_cast<char*>(ws), kKv8Front};
  Compact C;
  C.chunks = c.take<int32_t>(chunks_of(P));
  C.state = c.take<int32_t>(3);
  C.holes = c.take<int32_t>(P / 2 + 1);
  C.late = c.take<int32_t>(P / 2 + 1);
  C.key = c.take<int32_t>(P);
  *total = c.at;
  return C;
}

}  // namespace

hipError_t cg_launch_kv8_fork(const KvPool& pool, const KvSeqs& S, const int32_t* lengths,
                              const int32_t* parents, const int32_t* ends, int n, int width,
                              int32_t* table, int32_t* new_lengths, int32_t* refs, hipStream_t st) {
  in_rows(n, width, [&](int row0, int rows, int per_row) {
    hipLaunchKernelGGL(fork_kernel, dim3((unsigned)(rows * per_row)), dim3(256), 0, st, pool.P, S,
                       lengths, parents + row0, ends ? ends + row0 : nullptr, width, per_row,
                       table + (int64_t)row0 * width, new_lengths + row0, refs);
  });
  return hipGetLastError();
}

hipError_t cg_launch_kv8_release(const KvPool& pool, int n, int width, int32_t* table,
                                 const int32_t* keep, int32_t* refs, hipStream_t st) {
  in_rows(n, width, [&](int row0, int rows, int per_row) {
    hipLaunchKernelGGL(release_kernel, dim3((unsigned)(rows * per_row)), dim3(256), 0, st, pool.P,
                       width, per_row, table + (int64_t)row0 * width, keep ? keep + row0 : nullptr,
                       refs);
  });
  return hipGetLastError();
}

hipError_t cg_launch_kv8_copy(const KvPool& pool, int D, const int32_t* src, const int32_t* dst,
                              int n, hipStream_t st) {
  const int pieces = pieces_of(pool.H, D);
  const int64_t items = (int64_t)n * pieces;
  hipLaunchKernelGGL(copy_kernel, dim3(grid_of(items)), dim3(256), 0, st, pool, D, src, dst, pieces,
                     items);
  return hipGetLastError();
}

uint64_t cg_kv8_reserve_ws(int P, int n, int width) {
  uint64_t total;
  reserve_of(nullptr, P, n, width, &total);
  return total;
}

hipError_t cg_launch_kv8_reserve(const KvPool& pool, int D, int n, int width, int32_t* table,
                                 const int32_t* lengths, const int32_t* counts, int32_t* refs,
                                 int32_t* missing, int32_t* granted, void* ws, hipStream_t st) {
  uint64_t total;
  const Reserve R = reserve_of(ws, pool.P, n, width, &total);
  const int chunks = chunks_of(pool.P), words = words_of(width), pieces = pieces_of(pool.H, D);
  // (65536 pages: one workgroup 10.8 us, two launches of many 17.6; a full pool costs the one 1.2 for
  // every 16384 pages. Many columns are dear to it: whole calls that want 1024 of them 13.5 / 18.4 us,
  // 4096 18.6 / 19.8, 16384 41 / 20, 65536 145 / 22. But only the device knows how many a call touches,
  // and a step of answers touches one or two a sequence.)
  if (pool.P <= 4 * kPlanPages && n <= kPlanSeqs && (int64_t)n * width <= 1 << 30) {
    hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, pool.P, n, width, table,
                       lengths, counts, refs, R, missing);
  } else {
    hipLaunchKernelGGL(want_kernel, dim3(chunks + (n + 3) / 4), dim3(256), 0, st, pool.P, n, width,
                       table, lengths, counts, refs, chunks, words, R, missing,
                       static_cast<uint32_t*>(ws));
    hipLaunchKernelGGL(list_kernel, dim3(chunks), dim3(256), 0, st, pool.P, refs, R);
  }
  const int64_t items = (int64_t)n * pieces;
  hipLaunchKernelGGL(hand_out_kernel, dim3(grid_of(items)), dim3(256), 0, st, pool, D, n, width,
                     table, lengths, counts, refs, granted, pieces, items, R);
  return hipGetLastError();
}

uint64_t cg_kv8_compact_ws(int P) {
  uint64_t total;
  compact_of(nullptr, P, &total);
  return total;
}

hipError_t cg_launch_kv8_compact(const KvPool& pool, const KvSeqs& S, int D, const int32_t* refs,
                                 int32_t* new_table, int32_t* new_refs, int32_t* moved,
                                 int32_t* n_live, void* ws, hipStream_t st) {
  uint64_t total;
  const Compact C = compact_of(ws, pool.P, &total);
  const int chunks = chunks_of(pool.P), pieces = pieces_of(pool.H, D);
  // (as many pages as one workgroup has registers for the counts of: 4096 pages 4.9 us, 19.3 where the
  // workgroups' counts meet in memory; whole calls with nothing to move, 16384 pages 10.9 us, 16385 19.3,
  // 65536 20.1)
  if (pool.P <= kPlanPages) {
    hipLaunchKernelGGL(places_kernel, dim3(1), dim3(kPlanThreads), 0, st, pool.P, refs, C, moved,
                       new_refs, n_live);
  } else {
    hipLaunchKernelGGL(used_kernel, dim3(chunks), dim3(256), 0, st, pool.P, refs, chunks, C, n_live,
                       static_cast<uint32_t*>(ws));
    hipLaunchKernelGGL(place_kernel, dim3(chunks), dim3(256), 0, st, pool.P, refs, C, moved,
                       new_refs);
  }
  // as many copying workgroups as the card holds at once, or as there can be pieces to move
  const int64_t most = (int64_t)(pool.P / 2 + 1) * pieces, entries = (int64_t)S.n * S.width;
  const int movers = (int)(most < 2048 ? most : 2048);
  const int64_t rest = (entries + 255) / 256;
  hipLaunchKernelGGL(move_kernel, dim3(movers + (unsigned)(rest < 4096 ? rest : 4096)), dim3(256), 0,
                     st, pool, D, refs, entries, S.table, new_table, movers, pieces, C, moved,
                     new_refs);
  return hipGetLastError();
}
