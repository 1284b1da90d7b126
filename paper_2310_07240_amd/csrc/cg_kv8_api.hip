// cg_kv8_api.hip — the C ABI of the 8-bit serving cache (include/cachegen.h): arguments are
// checked on the host, then the kernels are launched on the caller's stream.
#include <math.h>

#include "cg_kv8.h"

namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

int check_cache(const cg_kv8_cache* c, KvPool* out) {
  if (!c) return CG_ERR_ARG;
  if (c->n_pages <= 0 || c->n_heads <= 0) return CG_ERR_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return CG_ERR_SHAPE;
  if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return CG_ERR_ARG;
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scale, 4) ||
      !aligned(c->v_scale, 4) || !aligned(c->k_bounds, 16) || !aligned(c->mass, 4))
    return CG_ERR_ARG;
  *out = KvPool{c->n_pages, c->n_heads, c->k_codes, c->v_codes, c->k_scale, c->v_scale,
                c->k_bounds, c->mass};
  return CG_OK;
}

int check_seqs(const cg_kv8_seqs* s, const KvPool& pool, KvSeqs* out) {
  if (!s) return CG_ERR_ARG;
  if (s->n_seq <= 0 || s->max_pages <= 0) return CG_ERR_SHAPE;
  // one workgroup per (sequence, KV head) in some launches: below 2^32 threads
  if ((int64_t)s->n_seq * pool.H > (1 << 21)) return CG_ERR_SHAPE;
  if (!s->table || !aligned(s->table, 4)) return CG_ERR_ARG;
  *out = KvSeqs{s->n_seq, s->max_pages, s->table};
  return CG_OK;
}

// The caller's bound of the lengths, or the table's row where that is the smaller: no sequence is
// longer, and work and scratch are laid out for it. (The kernels round tokens up to pages in 32 bits.)
int32_t most_tokens(int32_t max_len, const KvSeqs& S) {
  int64_t room = (int64_t)S.width * kPage;
  if (room > INT32_MAX - (kPage - 1)) room = INT32_MAX - (kPage - 1);
  return max_len < room ? max_len : (int32_t)room;
}

bool bad_rows(const cg_kv8_rows* r) { return !r || !r->data || !aligned(r->data, 2); }

KvRows rows(const cg_kv8_rows& r) {
  return KvRows{r.data, r.seq_stride, r.token_stride, r.head_stride};
}

bool wide(const cg_kv8_rows& r) {
  return aligned(r.data, 16) && ((r.seq_stride | r.token_stride | r.head_stride) & 7) == 0;
}

bool bad_dtype(int32_t d) { return d != CG_KV8_F16 && d != CG_KV8_BF16; }

// What attend and select share: shapes, queries and lengths.
int check_queries(const cg_kv8_attn* a, const KvPool& pool, const KvSeqs& S, KvAttn* out) {
  if (!a) return CG_ERR_ARG;
  if (a->n_q <= 0 || a->n_q_heads <= 0 || a->n_q_heads % pool.H || a->max_len < 0)
    return CG_ERR_SHAPE;
  if ((int64_t)S.n * a->n_q * a->n_q_heads > (1LL << 30) ||
      (int64_t)S.n * a->n_q * pool.H > (1 << 23))
    return CG_ERR_SHAPE;
  if (bad_dtype(a->dtype) || bad_rows(&a->q) || !a->lengths || !aligned(a->lengths, 4) ||
      !aligned(a->q_lens, 4))
    return CG_ERR_ARG;
  *out = KvAttn{};
  out->lengths = a->lengths;
  out->q_lens = a->q_lens;
  out->q = rows(a->q);
  out->wide_q = wide(a->q);
  out->max_len = most_tokens(a->max_len, S);
  out->nq = a->n_q;
  out->group = a->n_q_heads / pool.H;
  out->n_picks = a->n_picks;
  return CG_OK;
}

int check_attend(const cg_kv8_cache* c, const cg_kv8_seqs* s, const cg_kv8_attn* a, KvPool* pool,
                 KvSeqs* S, KvAttn* A) {
  int rc = check_cache(c, pool);
  if (rc == CG_OK) rc = check_seqs(s, *pool, S);
  if (rc == CG_OK) rc = check_queries(a, *pool, *S, A);
  if (rc != CG_OK) return rc;
  if (bad_rows(&a->out) || !aligned(a->lse, 4)) return CG_ERR_ARG;
  if (!isfinite(a->scale) || !isfinite(a->decay)) return CG_ERR_PARAM;
  if (a->picks && a->n_picks <= 0) return CG_ERR_SHAPE;
  if (!aligned(a->picks, 4) || !aligned(a->mass_in, 4) || !aligned(a->mass_out, 4))
    return CG_ERR_ARG;
  if ((a->mass_in && !a->mass_out) || (a->mass_out && a->picks)) return CG_ERR_ARG;
  A->out = rows(a->out);
  A->lse = a->lse;
  A->picks = a->picks;
  A->mass_in = a->mass_in;
  A->mass_out = a->mass_out;
  A->scale = a->scale;
  A->decay = a->decay;
  return CG_OK;
}

// A page's score is a sum over the group's channels of products of two codes, in 32 bits.
bool score_fits(int64_t group, int64_t D) { return group * D * (127 * 127) <= INT32_MAX; }

int hip_rc(hipError_t e) { return e == hipSuccess ? CG_OK : CG_ERR_HIP; }

}  // namespace

extern "C" {

int cg_kv8_store(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* starts,
                 const int32_t* counts, int32_t n_tokens, int32_t dtype, const cg_kv8_rows* k,
                 const cg_kv8_rows* v, uint32_t* status, hipStream_t stream) {
  KvPool pool;
  KvSeqs S;
  int rc = check_cache(c, &pool);
  if (rc == CG_OK) rc = check_seqs(s, pool, &S);
  if (rc != CG_OK) return rc;
  if (n_tokens <= 0) return CG_ERR_SHAPE;
  if (!starts || !aligned(starts, 4) || !aligned(counts, 4) || bad_dtype(dtype) || bad_rows(k) ||
      bad_rows(v) || !aligned(status, 4))
    return CG_ERR_ARG;
  return hip_rc(cg_launch_kv8_store(pool, S, c->head_dim, dtype == CG_KV8_BF16, starts, counts,
                                    n_tokens, rows(*k), rows(*v), status, stream));
}

int cg_kv8_load(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* starts,
                const int32_t* counts, int32_t n_tokens, int32_t dtype, const cg_kv8_rows* k,
                const cg_kv8_rows* v, hipStream_t stream) {
  KvPool pool;
  KvSeqs S;
  int rc = check_cache(c, &pool);
  if (rc == CG_OK) rc = check_seqs(s, pool, &S);
  if (rc != CG_OK) return rc;
  if (n_tokens <= 0) return CG_ERR_SHAPE;
  if (!starts || !aligned(starts, 4) || !aligned(counts, 4) || bad_dtype(dtype) || bad_rows(k) ||
      bad_rows(v))
    return CG_ERR_ARG;
  return hip_rc(cg_launch_kv8_load(pool, S, c->head_dim, dtype == CG_KV8_BF16, starts, counts,
                                   n_tokens, rows(*k), rows(*v), stream));
}

uint64_t cg_kv8_attend_workspace_bytes(const cg_kv8_cache* c, const cg_kv8_seqs* s,
                                       const cg_kv8_attn* a) {
  KvPool pool;
  KvSeqs S;
  KvAttn A;
  if (check_attend(c, s, a, &pool, &S, &A) != CG_OK) return 0;
  return cg_kv8_plan(pool, S, A, c->head_dim).total;
}

int cg_kv8_attend(const cg_kv8_cache* c, const cg_kv8_seqs* s, const cg_kv8_attn* a,
                  void* workspace, uint64_t workspace_bytes, hipStream_t stream) {
  KvPool pool;
  KvSeqs S;
  KvAttn A;
  const int rc = check_attend(c, s, a, &pool, &S, &A);
  if (rc != CG_OK) return rc;
  const uint64_t need = cg_kv8_plan(pool, S, A, c->head_dim).total;
  if (need && (!workspace || !aligned(workspace, 256))) return CG_ERR_ARG;
  if (workspace_bytes < need) return CG_ERR_CAPACITY;
  return hip_rc(cg_launch_kv8_attend(pool, S, c->head_dim, a->dtype == CG_KV8_BF16, A, workspace,
                                     stream));
}

uint64_t cg_kv8_select_workspace_bytes(const cg_kv8_cache* c, const cg_kv8_seqs* s,
                                       const cg_kv8_attn* a) {
  KvPool pool;
  KvSeqs S;
  KvAttn A;
  if (check_cache(c, &pool) != CG_OK || check_seqs(s, pool, &S) != CG_OK ||
      check_queries(a, pool, S, &A) != CG_OK || !score_fits(A.group, c->head_dim))
    return 0;
  return cg_kv8_select_ws(S, pool.H, A.nq, A.max_len);
}

int cg_kv8_select(const cg_kv8_cache* c, const cg_kv8_seqs* s, const cg_kv8_attn* a,
                  int32_t recent, int32_t* picks_out, void* workspace, uint64_t workspace_bytes,
                  hipStream_t stream) {
  KvPool pool;
  KvSeqs S;
  KvAttn A;
  int rc = check_cache(c, &pool);
  if (rc == CG_OK) rc = check_seqs(s, pool, &S);
  if (rc == CG_OK) rc = check_queries(a, pool, S, &A);
  if (rc != CG_OK) return rc;
  if (a->n_picks <= 0 || recent < 0 || !score_fits(A.group, c->head_dim)) return CG_ERR_SHAPE;
  if (!pool.bounds || !picks_out || !aligned(picks_out, 4)) return CG_ERR_ARG;
  const uint64_t need = cg_kv8_select_ws(S, pool.H, A.nq, A.max_len);
  if (need && (!workspace || !aligned(workspace, 256))) return CG_ERR_ARG;
  if (workspace_bytes < need) return CG_ERR_CAPACITY;
  return hip_rc(cg_launch_kv8_select(pool, S, c->head_dim, a->dtype == CG_KV8_BF16, A, recent,
                                     picks_out, workspace, stream));
}

int cg_kv8_evict(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* lengths,
                 int32_t max_len, float* mass, int32_t keep, int32_t recent,
                 const cg_kv8_seqs* to, int32_t* kept, int32_t* new_lengths, hipStream_t stream) {
  KvPool pool;
  KvSeqs S, T;
  int rc = check_cache(c, &pool);
  if (rc == CG_OK) rc = check_seqs(s, pool, &S);
  if (rc == CG_OK) rc = check_seqs(to, pool, &T);
  if (rc != CG_OK) return rc;
  if (max_len < 0 || keep <= 0 || recent < 0 || T.n != S.n) return CG_ERR_SHAPE;
  if (!lengths || !aligned(lengths, 4) || !mass || !aligned(mass, 4) || !kept ||
      !aligned(kept, 4) || !new_lengths || !aligned(new_lengths, 4))
    return CG_ERR_ARG;
  max_len = most_tokens(max_len, S);
  const int64_t most = keep < max_len ? keep : max_len;
  if ((most + kPage - 1) / kPage > T.width) return CG_ERR_CAPACITY;
  return hip_rc(cg_launch_kv8_evict(pool, S, c->head_dim, lengths, max_len, mass, keep, recent, T,
                                    kept, new_lengths, stream));
}

}  // extern "C"
