/*
 * cachegen.h — C ABI of the CacheGen KV-cache codec for AMD Instinct MI355X (gfx950).
 *
 * The codec (CacheGen, SIGCOMM '24, Sec. 5.2 "KV cache encoding") turns an fp16 KV cache into
 * compact bitstreams in four steps, and decodes them back:
 *   1. token groups of G consecutive tokens; the first token of a group is the anchor and is
 *      quantized on its own at 8 bits, the others are coded as a delta against that anchor
 *      (Sec. 5.2 "Change-based encoding"; 8-bit anchors: Sec. 5.2 "Layer-wise quantization");
 *   2. vectorwise quantization whose delta bin width grows with layer depth
 *      (Sec. 5.2 "Layer-wise quantization"; default bins 0.5 / 1 / 1.5: App. C.2), with an
 *      encoding level chosen per context chunk (Sec. 5.3 "Workflow");
 *   3. one symbol distribution per (layer, K/V, channel) for deltas and one for anchors,
 *      counted over the context (Sec. 5.2 "Arithmetic coding"; Sec. 6 "Speed optimization");
 *   4. arithmetic coding of the symbols into bitstreams, and GPU arithmetic decoding back to
 *      fp16 KV (Sec. 5.2 "Arithmetic coding"; Sec. 6 "Speed optimization").
 *
 * Conventions shared by every call
 * --------------------------------
 *  B = n_ctx contexts, L = n_layers, T = n_tokens, C = n_channels per K and per V.
 *  KV layout (fp16 bit patterns, uint16_t): kv[b][l][kv][t][ch], kv = 0 for K and 1 for V,
 *  channel fastest. Element count n_elem = B*L*2*T*C (64-bit).
 *  Chunks: tokens are split into NC = ceil(T/chunk_len) chunks; the last may be partial.
 *  Token groups restart at every chunk start (chunks decode independently, Sec. 5.3).
 *  One arithmetic-coder stream per (b, c, l, kv, ch) with stream index
 *      s = (((b*NC + c)*L + l)*2 + kv)*C + ch        (S = B*NC*L*2*C streams)
 *  so every chunk's streams are contiguous in the payload. Inside a stream the chunk's anchor
 *  symbols come first, in token order, then its delta symbols, in token order (Sec. 5.2 fixes
 *  what is coded and under which distribution, not the order inside one bitstream; anchors
 *  first lets a decoder take every anchor, then every delta, with one table set at hand).
 *  Symbols: a quantized value q in [-127, 127] is symbol q + 127 in [0, 254] (255 symbols).
 *  Scale (per stream): m = max |x| over the chunk's tokens; s = (m == 0) ? 1 : m / 127 (fp32).
 *  Anchor (token j of a chunk with j % G == 0): q = rint(clamp(x / s, -127, 127)); a = q * s.
 *  Delta (other tokens): w = (layer_bin[l] * level_mult[level]) * s; d = x - a;
 *                        q = rint(clamp(d / w, -127, 127)).
 *  Reconstruction: anchor fp16(a); delta fp16(a + q * w). All fp32 arithmetic is IEEE
 *  binary32, round-to-nearest-even, no fused multiply-add; fp16 conversion rounds to nearest even.
 *
 *  CDF tables: uint16_t cum[256] per distribution with cum[0] = 0, cum[i+1] = cum[i] + freq[i]
 *  for i in [0, 253], every freq >= 1, total 65536. Entry 255 is padding (written 0); the
 *  top of the last interval, 65536, is implicit.
 *    cdf_anchor[l][kv][ch][256]                       (level independent)
 *    cdf_delta [level][l][kv][ch][256]                (one table set per encoding level)
 *
 *  Bitstreams: integer arithmetic coder with 32-bit code registers (Witten, Neal and Cleary,
 *  CACM 30(6), 1987), bitwise renormalisation, 2-bit termination. Bits are written MSB-first
 *  into uint32_t words; each stream is zero-padded to a whole word. offsets[0] = 0 and
 *  offsets[s+1] = offsets[s] + (words of stream s), uint64_t, so stream s occupies
 *  words[offsets[s] .. offsets[s+1]).
 *
 *  Memory: every array argument is a DEVICE pointer owned by the caller, except cg_params and
 *  the arrays it points to, which are HOST memory read during the call only. The library
 *  keeps no state between calls and never allocates device memory; scratch comes from the
 *  caller's workspace argument. Calls are asynchronous on the given HIP stream unless a
 *  description says otherwise; a non-zero return means nothing was launched, except
 *  CG_ERR_HIP, which reports a failed launch.
 */
#ifndef CACHEGEN_H
#define CACHEGEN_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Return codes. */
enum {
  CG_OK = 0,
  CG_ERR_ARG = -1,        /* null or misaligned pointer (tables need 16-byte alignment,
                             offsets 8, words and scales 4, the workspace 256), level or
                             chunk range out of range                                       */
  CG_ERR_SHAPE = -2,      /* a dimension <= 0, group_size < 1, chunk_len < 1, n_levels not
                             in [1, 8], or a size whose index space overflows 64 bits       */
  CG_ERR_CAPACITY = -3,   /* words_cap or workspace_bytes below what the call needs        */
  CG_ERR_NONFINITE = -4,  /* the KV input holds NaN or +-Inf (reported by cg_get_status after
                             cg_encode or cg_fit_cdf_levels, and by cg_check_finite)        */
  CG_ERR_HIP = -5,        /* a HIP runtime call or kernel launch failed                     */
  CG_ERR_PARAM = -6,      /* a layer_bin or level_mult entry is not finite and > 0          */
  CG_ERR_SCRATCH = -7     /* cg_encode_noalloc: the cache needs more scratch than
                             CG_NOALLOC_SCRATCH_BYTES                                       */
};

/* cg_decode may read (but never uses) up to this many words past offsets[S]: a words buffer
 * handed to cg_decode must be readable that far. A buffer sized by cg_encode_bound_words is. */
#define CG_TAIL_WORDS 8

typedef struct cg_params {
  int32_t n_ctx;          /* B */
  int32_t n_layers;       /* L */
  int32_t n_tokens;       /* T */
  int32_t n_channels;     /* C = kv_heads * head_dim, the same for K and V */
  int32_t group_size;     /* G, tokens per group, 10 in the paper (Sec. 5.2) */
  int32_t chunk_len;      /* tokens per chunk, 1.5K in the paper (Sec. 5.3); 1536 here */
  int32_t n_levels;       /* number of encoding levels, 1..8 */
  const float* layer_bin; /* [L] base delta bin width per layer in units of the scale s
                             (three layer groups 0.5 / 1 / 1.5 by default, App. C.2)    */
  const float* level_mult;/* [n_levels] multiplier of the bin width per encoding level */
} cg_params;

/* Number of chunks NC and of streams S for these parameters; 0 if the shape is invalid. */
int64_t cg_num_chunks(const cg_params* p);
int64_t cg_num_streams(const cg_params* p);

/* Capacity (in words) that cg_encode requires for its payload buffer: the sum over streams of
 * ceil((18 * n_s + 2) / 32), n_s being the stream's token count (each symbol costs at most 18
 * renormalisation shifts and the termination 2 bits), plus CG_TAIL_WORDS. 0 if the shape is
 * invalid. */
uint64_t cg_encode_bound_words(const cg_params* p);

/* Device scratch that cg_encode needs (bytes): the status word, per-workgroup non-finite
 * flags, a worst-case slot per stream, per-stream lengths and the scan's partial sums. 0 if the
 * shape is invalid. */
uint64_t cg_encode_workspace_bytes(const cg_params* p);

/* Fit the symbol distributions at encoding level `level` (Sec. 5.2 "Arithmetic coding":
 * one distribution per layer-channel for deltas and one for anchors; Sec. 6: counted over the
 * symbols of the context being coded).
 *   kv_f16          [B][L][2][T][C] fp16, device.
 *   level           0 <= level < n_levels: deltas of EVERY chunk are quantized with
 *                   level_mult[level] for this fit.
 *   cdf_anchor      out [L][2][C][256], device; may be NULL to skip the anchor tables.
 *   cdf_delta_level out [L][2][C][256], device: the delta tables of this level, i.e. the
 *                   slice cdf_delta[level] of the layout above.
 * Counts c_i (i in [0, 254]) are taken over all B*NC chunks; with N = sum c_i,
 * freq_i = 1 + floor(c_i * 65281 / N), and the remainder 65536 - sum freq_i is added to the
 * symbol with the largest count (lowest index on ties); N = 0 gives the uniform table.
 * Returns CG_OK, or an error before anything is launched. Does not scan for non-finite input
 * (cg_check_finite does). */
int cg_fit_cdf(const cg_params* p, const uint16_t* kv_f16, int32_t level,
               uint16_t* cdf_anchor, uint16_t* cdf_delta_level, hipStream_t stream);

/* Fit the tables of every encoding level at once (Sec. 5.2 "Arithmetic coding": one
 * distribution per channel-layer for deltas and one for anchors; Sec. 6: counted over the
 * symbols of the context being coded; Sec. 5.3: one table set per encoding level). The result
 * equals cg_fit_cdf at every level (anchor tables from any of them), but the scale and the
 * anchors of each chunk are found once for up to four levels, so the cache is read once per
 * four levels instead of once per level.
 *   kv_f16       [B][L][2][T][C] fp16, device.
 *   cdf_anchor   out [L][2][C][256], device.
 *   cdf_delta    out [n_levels][L][2][C][256], device.
 *   status       NULL, or a device uint32_t (4-byte aligned) that receives 0, or a non-zero
 *                value when the KV holds NaN or +-Inf (the tables are then meaningless);
 *                cg_get_status(status, stream) reads it.
 *   scales       NULL, or out [S] fp32, device (4-byte aligned): every stream's scale s
 *                (Sec. 5.2 "Layer-wise quantization": absmax / 127, 1 for an all-zero stream),
 *                taken from the same maxima the fit quantizes with; these are the scales
 *                cg_encode computes for the same KV, for cg_encode_with_scales.
 * Asynchronous. */
int cg_fit_cdf_levels(const cg_params* p, const uint16_t* kv_f16, uint16_t* cdf_anchor,
                      uint16_t* cdf_delta, uint32_t* status, float* scales,
                      hipStream_t stream);

/* Device scratch that cg_fit_cdf_global needs (bytes). */
#define CG_FIT_GLOBAL_WORKSPACE_BYTES 8192

/* The ablation baseline "one global symbol distribution" (Sec. 5.2 "Arithmetic coding" measures
 * the per channel-layer distributions against it; the ablation of Sec. 7.5 starts from it):
 * like cg_fit_cdf, but the counts of every layer, K/V and channel are pooled into one anchor
 * histogram and one delta histogram, normalised the same way, and that one table is written to
 * every [l][kv][ch] slot of cdf_anchor (may be NULL) and cdf_delta_level, so cg_encode and
 * cg_decode use it unchanged.
 *   workspace    device scratch of workspace_bytes >= CG_FIT_GLOBAL_WORKSPACE_BYTES, 256-byte
 *                aligned; its contents on entry do not matter.
 * Asynchronous. */
int cg_fit_cdf_global(const cg_params* p, const uint16_t* kv_f16, int32_t level,
                      uint16_t* cdf_anchor, uint16_t* cdf_delta_level, void* workspace,
                      uint64_t workspace_bytes, hipStream_t stream);

/* Encode the whole KV cache (Sec. 5.2: delta, layer-wise quantization, arithmetic coding;
 * Sec. 5.3: each chunk at its own level).
 *   kv_f16       [B][L][2][T][C] fp16, device.
 *   chunk_level  [B][NC] uint8, device: level of every (context, chunk); all equal for a
 *                single-level encode.
 *   cdf_anchor   [L][2][C][256], cdf_delta [n_levels][L][2][C][256], device (from cg_fit_cdf).
 *   words        out, device, capacity words_cap >= cg_encode_bound_words(p).
 *   offsets      out [S + 1] uint64, device; offsets[S] is the payload length in words.
 *   scales       out [S] fp32, device: the per-stream scale s.
 *   workspace    device scratch of workspace_bytes >= cg_encode_workspace_bytes(p), 256-byte
 *                aligned; its contents on entry do not matter. After the call its first word
 *                is the call's status: cg_get_status(workspace, stream) reads it.
 * chunk_level values must be < n_levels (an out-of-range level is clamped to n_levels - 1 on
 * the device). Non-finite input (NaN or +-Inf) is outside the quantizer's domain: the encoder
 * detects it on the device while it takes the streams' absolute maxima (no extra pass) and
 * records it in the status word; the payload is then meaningless but every write stays within
 * the buffers above. Asynchronous. */
int cg_encode(const cg_params* p, const uint16_t* kv_f16, const uint8_t* chunk_level,
              const uint16_t* cdf_anchor, const uint16_t* cdf_delta,
              uint32_t* words, uint64_t words_cap, uint64_t* offsets, float* scales,
              void* workspace, uint64_t workspace_bytes, hipStream_t stream);

/* cg_encode with the streams' scales as an input instead of an output (the vectorwise scale of
 * Sec. 5.2 is found once for fit and encode): `scales` [S] fp32, device (4-byte aligned), as
 * cg_fit_cdf_levels wrote them for the same KV. The encoder then takes no absolute maxima, and
 * words and offsets equal those of cg_encode. Other scales code the cache under those scales
 * (a valid payload; its values are whatever they give). Non-finite input is not looked for:
 * the fit's status reports it, and the status word in the workspace is 0. Other arguments,
 * errors and asynchrony as for cg_encode. */
int cg_encode_with_scales(const cg_params* p, const uint16_t* kv_f16, const uint8_t* chunk_level,
                          const uint16_t* cdf_anchor, const uint16_t* cdf_delta,
                          const float* scales, uint32_t* words, uint64_t words_cap,
                          uint64_t* offsets, void* workspace, uint64_t workspace_bytes,
                          hipStream_t stream);

/* Bytes of the static device scratch of cg_encode_noalloc (held by every GPU the library runs
 * on until the process ends). */
#define CG_NOALLOC_SCRATCH_BYTES (64u << 20)

/* cg_encode without any device allocation by the library or the caller beyond the inputs and
 * outputs, for callers that cannot allocate: code being captured into a HIP graph, tight
 * serving loops, harnesses that forbid hipMalloc. Same arguments, results and errors as
 * cg_encode, except:
 *   - no workspace: the encoder's scratch (status word, per-workgroup flags, worst-case slots,
 *     word counts, scan partials) is one static device buffer of CG_NOALLOC_SCRATCH_BYTES per
 *     GPU; a cache whose scratch (cg_encode_workspace_bytes(p)) exceeds it is rejected with
 *     CG_ERR_SCRATCH before anything is launched (e.g. a whole 1536-token chunk of 32 layers
 *     x 1024 channels needs about 227 MB; one such layer about 7 MB);
 *   - status: NULL, or a caller-owned device uint32_t (4-byte aligned) that receives the call's
 *     status word (0, or non-zero if the KV held NaN or +-Inf), written unconditionally.
 * Every call on a GPU shares that GPU's scratch, and nothing in it needs to start at any value;
 * calls that overlap on one GPU (on different streams, or from different host threads without
 * ordering) race and must not be issued. The first call on a device looks up the address of
 * that device's buffer (hipGetSymbolAddress, no allocation). Asynchronous. */
int cg_encode_noalloc(const cg_params* p, const uint16_t* kv_f16, const uint8_t* chunk_level,
                      const uint16_t* cdf_anchor, const uint16_t* cdf_delta, uint32_t* words,
                      uint64_t words_cap, uint64_t* offsets, float* scales, uint32_t* status,
                      hipStream_t stream);

/* Decode chunks [chunk_begin, chunk_end) of every context back to fp16 KV (Sec. 5.2; the
 * GPU decoder of Sec. 6; chunk ranges allow decoding a chunk as soon as it arrives, Sec. 6).
 *   words, offsets [S + 1], scales [S], chunk_level [B][NC], cdf_anchor, cdf_delta: device,
 *                as produced by cg_encode / cg_fit_cdf.
 *   kv_out_f16   out [B][L][2][T][C] fp16, device; only the token rows of the requested
 *                chunks are written.
 * The words buffer must be readable up to offsets[S] + CG_TAIL_WORDS. Bits after a stream's
 * codeword never change its decoded symbols (whatever follows, the code value stays inside the
 * coder's final interval), so the decoder may read into the next stream or the tail. Every
 * loop is bounded by the stream's token count: a corrupt payload yields wrong values but never
 * an out-of-range access, provided offsets is non-decreasing and offsets[S] + CG_TAIL_WORDS
 * words are readable. Asynchronous. */
int cg_decode(const cg_params* p, const uint32_t* words, const uint64_t* offsets,
              const float* scales, const uint8_t* chunk_level,
              const uint16_t* cdf_anchor, const uint16_t* cdf_delta,
              int32_t chunk_begin, int32_t chunk_end, uint16_t* kv_out_f16,
              hipStream_t stream);

/* Timings of one cg_decode_streamed call (milliseconds from the call's first copy). */
typedef struct cg_stream_stats {
  int32_t n_chunks;        /* chunks decoded (NC) */
  double transfer_ms;      /* until the last chunk's payload is on the device */
  double total_ms;         /* until the last chunk is decoded */
  double decode_sum_ms;    /* sum of the per-chunk decode durations */
  double hidden_fraction;  /* 1 - (total_ms - transfer_ms) / decode_sum_ms, clamped to [0, 1]:
                              the share of decoding done while the payload still arrived */
  /* Optional per-chunk event times, host arrays of n_chunks doubles supplied by the caller
   * (NULL: not reported), in milliseconds from the call's first copy: */
  double* chunk_copy_done_ms;     /* chunk c's payload is on the device          */
  double* chunk_decode_begin_ms;  /* chunk c's decode starts                     */
  double* chunk_decode_end_ms;    /* chunk c's decode ends                       */
} cg_stream_stats;

/* Decode the whole cache chunk by chunk while its payload arrives (Sec. 5.3: the cache is
 * split into chunks that are sent and decoded independently; Sec. 6: decoding is pipelined with
 * the transmission so that it adds little delay).
 *   words_host    [offsets[S]] uint32, HOST memory (page-locked, e.g. from hipHostMalloc, or
 *                 the copies cannot overlap the decode): the payload as cg_encode produced it.
 *   offsets_host  [S + 1] uint64, HOST memory: the same offsets (the side information that
 *                 precedes the payload).
 *   words_dev     device buffer of words_cap words, words_cap >= offsets[S] + CG_TAIL_WORDS,
 *                 that receives the payload; the other device arguments are as for cg_decode.
 * offsets_host is checked on the host before anything is issued: it must start at 0, be
 * non-decreasing at every chunk boundary used for a copy and end within words_cap -
 * CG_TAIL_WORDS (else CG_ERR_ARG / CG_ERR_CAPACITY).
 *   link_gbps     rate of the simulated link the payload arrives over, in gigabits per second:
 *                 chunk c's copy is issued when the bytes of chunks 0..c would have arrived
 *                 (the host waits). 0 or less: every copy is issued at once (the host-to-device
 *                 bus is the link).
 *   decode_stream, copy_stream   two HIP streams (the copies overlap the decodes only if they
 *                 differ); chunk c's decode waits for chunk c's copy through an event.
 *   stats         out, host, may be NULL; its chunk_* pointers are read (NULL or arrays of NC
 *                 doubles that receive the per-chunk times).
 * Chunk c of every context is copied (one copy per context: chunk c's streams of context b are
 * contiguous) and decoded with the cg_decode kernels. Creates and destroys HIP events, and
 * returns after the last decode has finished (synchronous). The result equals cg_decode over
 * all chunks. */
int cg_decode_streamed(const cg_params* p, const uint32_t* words_host,
                       const uint64_t* offsets_host, uint32_t* words_dev, uint64_t words_cap,
                       const uint64_t* offsets_dev, const float* scales_dev,
                       const uint8_t* chunk_level_dev, const uint16_t* cdf_anchor_dev,
                       const uint16_t* cdf_delta_dev, uint16_t* kv_out_dev, double link_gbps,
                       hipStream_t decode_stream, hipStream_t copy_stream,
                       cg_stream_stats* stats);

/* Streaming adaptation (Sec. 5.3 "KV cache streaming adaptation"; App. B, Alg. 1): the
 * configuration of each chunk — text (the receiver recomputes its KV) or one encoding level — is
 * chosen while the chunks are sent, so the transfer stays within a time-to-first-token SLO.
 * Host-only logic; it plans and simulates one context's transfer over a given bandwidth trace.
 * Levels are ordered by compression loss: level 0 loses least (largest payload). */
typedef struct cg_adapt_params {
  int32_t n_chunks;
  int32_t n_levels;
  const double* level_bytes;   /* [n_chunks][n_levels] payload bytes of chunk c at level v */
  const double* text_bytes;    /* [n_chunks] bytes of the chunk's text */
  const double* recompute_ms;  /* [n_chunks] time to recompute the chunk's KV from its text;
                                  NULL: text is never chosen */
  double slo_ms;               /* time-to-first-token objective for the whole context */
  double prior_gbps;           /* throughput known before the first chunk; <= 0: unknown */
  int32_t default_level;       /* level of the first chunk when no throughput is known */
} cg_adapt_params;

/* Plan and simulate: for every chunk in order, with the throughput estimate (the previous
 * chunk's measured throughput, or prior_gbps / none for the first) and remaining = slo_ms -
 * elapsed, choose text if the remaining chunks' recompute time fits in remaining (and
 * recompute_ms is given), else the lowest-loss level whose remaining chunks' bytes at that level
 * would arrive within remaining at the estimated throughput, else the most compressed level;
 * the first chunk without an estimate takes default_level (or text if its rule holds). The
 * chunk is then sent at bandwidth_gbps[c] (its actual rate), which is also the next chunk's
 * estimate; elapsed grows by its transfer time, plus its recompute time when sent as text.
 *   bandwidth_gbps  [n_chunks] host, the link rate each chunk experiences (> 0).
 *   choice_out      [n_chunks] host out: the chosen level, or -1 for text.
 *   ttft_ms_out     host out: elapsed time after the last chunk (the simulated TTFT).
 * Returns CG_OK, or CG_ERR_ARG for a null pointer or a non-positive count or rate. */
int cg_adapt_schedule(const cg_adapt_params* a, const double* bandwidth_gbps,
                      int32_t* choice_out, double* ttft_ms_out);

/* Read a status word on the device: the first word of a cg_encode workspace (the status of
 * the last cg_encode that used it), or the status argument of cg_fit_cdf_levels or
 * cg_encode_noalloc. Waits for `stream` (synchronous), then returns CG_OK, or CG_ERR_NONFINITE
 * if the KV of that call held NaN or +-Inf; CG_ERR_ARG for a null or not 4-byte aligned
 * pointer, CG_ERR_HIP if the copy fails. Every call writes its word, so it never needs
 * clearing; calls that share one on different streams race. */
int cg_get_status(const void* workspace, hipStream_t stream);

/* Scan kv_f16 [n_elem] for NaN / Inf (fp16 exponent field all ones), using flag_dev, one
 * caller-owned device uint32_t, as scratch. Synchronises `stream`. Returns CG_OK,
 * CG_ERR_NONFINITE, or an error code. The quantizer is defined for finite input only;
 * callers that cannot vouch for their input run this first. */
int cg_check_finite(const cg_params* p, const uint16_t* kv_f16, uint32_t* flag_dev,
                    hipStream_t stream);

/* ---- Token-parallel stream layout (Sec. 6: the paper's GPU decoder runs one thread per
 * token), for comparison with the channel streams above. One stream per (context, layer,
 * K/V, token) over the token's C channels in order; the symbol of channel ch is coded under the
 * (layer, K/V, ch) tables: cdf_anchor on the first token of each group, the chunk level's delta
 * table otherwise. The quantized symbols and the scales are exactly those of the channel layout
 * (the same fp16 output comes back); only their grouping into streams changes. Stream order:
 * inside context b, chunk c (first token t0, n tokens) holds streams
 * (b T + t0) 2L + (2 l + k) n + (t - t0), so each chunk's streams are contiguous. */

/* Token streams: B * L * 2 * T. 0 if p is invalid. */
int64_t cg_num_token_streams(const cg_params* p);

/* Capacity of the token-layout payload (words): every token stream at its worst case
 * ceil((18 C + 2) / 32), plus CG_TAIL_WORDS. */
uint64_t cg_encode_tokens_bound_words(const cg_params* p);

/* Device scratch of cg_encode_tokens (bytes): the symbol array (one byte per element), a
 * worst-case slot per token stream, per-stream word counts and scan partials. */
uint64_t cg_encode_tokens_workspace_bytes(const cg_params* p);

/* Device scratch of cg_decode_tokens (bytes): the symbol array, one byte per element. */
uint64_t cg_decode_tokens_workspace_bytes(const cg_params* p);

/* Encode in the token layout. Arguments as for cg_encode, except offsets [St + 1] for the St
 * token streams, words_cap >= cg_encode_tokens_bound_words(p) and workspace_bytes >=
 * cg_encode_tokens_workspace_bytes(p); scales [S] are the channel streams' (as cg_encode).
 * Asynchronous. */
int cg_encode_tokens(const cg_params* p, const uint16_t* kv_f16, const uint8_t* chunk_level,
                     const uint16_t* cdf_anchor, const uint16_t* cdf_delta, uint32_t* words,
                     uint64_t words_cap, uint64_t* offsets, float* scales, void* workspace,
                     uint64_t workspace_bytes, hipStream_t stream);

/* Decode the token layout to fp16 KV [B][L][2][T][C] (every chunk). words, offsets [St + 1],
 * scales [S], chunk_level, tables: device, as cg_encode_tokens / cg_fit_cdf produced them; the
 * words buffer must be readable up to offsets[St] + CG_TAIL_WORDS (as for cg_decode: a corrupt
 * payload gives wrong values, never an out-of-range access). workspace_bytes >=
 * cg_decode_tokens_workspace_bytes(p). Asynchronous. */
int cg_decode_tokens(const cg_params* p, const uint32_t* words, const uint64_t* offsets,
                     const float* scales, const uint8_t* chunk_level,
                     const uint16_t* cdf_anchor, const uint16_t* cdf_delta,
                     uint16_t* kv_out_f16, void* workspace, uint64_t workspace_bytes,
                     hipStream_t stream);

/* ---- 8-bit serving cache -------------------------------------------------------------------
 * Where a decoded context is answered from. The paper's system hands the decoded cache to the
 * model (Sec. 6, generate_with_kv); a server that holds many contexts keeps them in 8 bits, the
 * form the paper measures against (Sec. 7.1), and drops the tokens that attention passes by
 * before it encodes again (Sec. 7.2, CacheGen on top of token dropping).
 *
 * A cache is a pool of pages. A page holds CG_KV8_PAGE = 64 consecutive tokens of one sequence,
 * for every KV head, and K and V of a (page, head) are int8 codes under one fp32 scale each:
 * value = code * scale. Attention's two products contract over K's channels and V's tokens, so K
 * lies token by token and V channel by channel. A sequence is a row of page numbers (the table)
 * and a length; token t of it is token t % 64 of page table[t / 64].
 *
 * The struct arguments are HOST memory read during the call; the pointers in them are DEVICE
 * memory of the caller. Page numbers and lengths are read on the device and never trusted: a page
 * number outside [0, n_pages) is a page without tokens, a length is cut to the table's row and to
 * the caller's bound. Every call is asynchronous on the given stream and none allocates. Rows of
 * K, V, queries and outputs are fp16 or bf16 with any strides (the last dimension contiguous); where
 * they are 16-byte aligned, K, V and queries move 16 bytes at a time. */
#define CG_KV8_PAGE 64

/* The workspaces of cg_kv8_attend and cg_kv8_select start with this many bytes of counters, which
 * the caller clears once, before a workspace's first use; every call leaves them zero. The rest of
 * a workspace may hold anything. Calls that may overlap need workspaces of their own, and so do two
 * host threads that call on one stream: a call is up to three launches. */
#define CG_KV8_WORKSPACE_ZEROED 4096

enum { CG_KV8_F16 = 0, CG_KV8_BF16 = 1 };

typedef struct cg_kv8_cache {
  int32_t n_pages;        /* P */
  int32_t n_heads;        /* H, KV heads */
  int32_t head_dim;       /* D: 64, 128 or 256 */
  int8_t* k_codes;        /* [P][H][64][D], 16-byte aligned */
  int8_t* v_codes;        /* [P][H][D][64], 16-byte aligned */
  float* k_scale;         /* [P][H] */
  float* v_scale;         /* [P][H] */
  int8_t* k_bounds;       /* [P][H][2][D], 16-byte aligned: lowest and highest K code of each
                             channel over the page's tokens; NULL: not kept (cg_kv8_select
                             needs them) */
  float* mass;            /* [P][H][64]: token weights as cg_kv8_attend adds them up, which
                             cg_kv8_store clears for the tokens it writes, and which move with the
                             pages in cg_kv8_reserve, copy and compact; NULL: none are touched */
} cg_kv8_cache;

typedef struct cg_kv8_seqs {
  int32_t n_seq;
  int32_t max_pages;      /* columns of the table */
  const int32_t* table;   /* [n_seq][max_pages] page numbers */
} cg_kv8_seqs;

typedef struct cg_kv8_rows {
  void* data;             /* row (seq, token, head) starts at seq * seq_stride + token *
                             token_stride + head * head_stride elements and has head_dim */
  int64_t seq_stride, token_stride, head_stride;
} cg_kv8_rows;

/* Put rows into the pages: row i of sequence b becomes its token starts[b] + i, for i < counts[b].
 *   starts   [n_seq] tokens that each sequence holds already. The tokens before it in its page
 *            keep their values; what the page held from starts[b] on is gone.
 *   counts   [n_seq], at most n_tokens each; NULL: n_tokens for every sequence. Sequences with
 *            none are left alone.
 *   k, v     [n_seq][n_tokens][H] rows of `dtype`.
 *   status   NULL, or a device uint32_t that receives 0, or non-zero where a row held NaN or
 *            +-Inf (cg_get_status). Those set no scale: an Inf becomes code +-127, a NaN code 0.
 * Per page, head and K/V, with m the largest |x| of the page's new rows: scale s = m / 127, or the
 * page's own if that is larger and earlier tokens stay in it; code = rint(clamp(x / s, +-127))
 * (s = 0: code 0). Where s grows, the earlier tokens are coded again from code * old scale. All
 * quotients and products are IEEE fp32, as in the codec. With c->mass, the weights of a written
 * page become 0 from its first new row on: a token starts without weight, whoever had the page
 * before. (A caller that passes no mass clears the weights of a page itself, when the page goes to
 * another sequence.) Pages are shared with no other sequence of the call, or the result is
 * undefined. Asynchronous. */
int cg_kv8_store(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* starts,
                 const int32_t* counts, int32_t n_tokens, int32_t dtype, const cg_kv8_rows* k,
                 const cg_kv8_rows* v, uint32_t* status, hipStream_t stream);

/* Read rows back: row i of sequence b is its token starts[b] + i for i < counts[b] (NULL:
 * n_tokens), the fp32 product code * scale rounded to `dtype`; rows counts[b] .. n_tokens - 1 are zeros, and so
 * are rows of pages that do not exist. Asynchronous. */
int cg_kv8_load(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* starts,
                const int32_t* counts, int32_t n_tokens, int32_t dtype, const cg_kv8_rows* k,
                const cg_kv8_rows* v, hipStream_t stream);

/* Attention of n_q query tokens per sequence over its pages.
 * Token j of a sequence of length n is visible to its query token i of q_lens[b] where
 * j <= n - q_lens[b] + i: the queries are the last tokens, already stored. Query head hq reads KV
 * head hq / (n_q_heads / H). With S = scale * q . k over the visible tokens:
 *   out = softmax(S) v,   lse = log sum exp(S);
 * a query that sees no token, and one with i >= q_lens[b], gets out = 0 and lse = -inf. */
typedef struct cg_kv8_attn {
  int32_t n_q;              /* query tokens per sequence */
  int32_t n_q_heads;        /* a multiple of H */
  int32_t dtype;            /* of q and out */
  float scale;
  const int32_t* lengths;   /* [n_seq] tokens of each sequence, the queries' own among them */
  int32_t max_len;          /* no length is above it (longer ones are cut to it) */
  const int32_t* q_lens;    /* [n_seq] query tokens of each sequence, or NULL: n_q */
  cg_kv8_rows q, out;       /* [n_seq][n_q][n_q_heads] */
  float* lse;               /* NULL, or out [n_seq][n_q][n_q_heads] */
  /* Attention over chosen pages only: picks [n_seq][n_q][H][n_picks], as cg_kv8_select writes
   * them: for each query token and KV head the table columns it reads, each at most once; entries
   * outside the sequence are skipped. NULL: all pages. */
  const int32_t* picks;
  int32_t n_picks;
  /* The weight each token got: mass_out [P][H][64] receives, for every token of the sequences,
   * decay * mass_in + the sum over the query tokens and the heads of its group of their softmax
   * weight on it. mass_in NULL: the sum alone; it may be mass_out. mass_out NULL: no weights. Not
   * together with picks, nor for sequences that share pages. What mass_in holds for a token counts,
   * also for one that has got no weight yet: see cg_kv8_store. */
  const float* mass_in;
  float* mass_out;
  float decay;
} cg_kv8_attn;

/* Device scratch that cg_kv8_attend needs (bytes); 0 if an argument is invalid or none is needed. It
 * follows max_len (or the table's row, if that is shorter), not the lengths, which only the device
 * knows. */
uint64_t cg_kv8_attend_workspace_bytes(const cg_kv8_cache* c, const cg_kv8_seqs* s,
                                       const cg_kv8_attn* a);

/* The attention above. Products take fp16 operands and sum in 32 bits; maxima, sums, lse and mass
 * are 32-bit. The codes and fp16 queries are exact. bf16 queries go in under a power of two per row:
 * exactly down to 2^-17 of the row's largest, off by 2^-25 of it at most below. Softmax weights are
 * rounded to fp16, 2^-11 of a weight, down to 2^-29 of the heaviest in its page where there are few
 * rows, and to 2^-25 of the row's heaviest (lighter ones are off by 2^-36 of it at most) where there
 * are many; there, pages whose V scale is below 2^-60 of the sequence's largest, or subnormal, may
 * add nothing to `out`. Where there are few rows, values are summed with weights of up to 1 before they
 * are divided: the largest |V| times the tokens has to stay below 2^127. Which of the two a call takes
 * follows its sizes and max_len. Results do not depend on the order in which parts of the work end.
 *   workspace   device scratch of workspace_bytes >= cg_kv8_attend_workspace_bytes, 256-byte
 *               aligned (may be NULL where that is 0), its first CG_KV8_WORKSPACE_ZEROED bytes
 *               zero.
 * Asynchronous. */
int cg_kv8_attend(const cg_kv8_cache* c, const cg_kv8_seqs* s, const cg_kv8_attn* a,
                  void* workspace, uint64_t workspace_bytes, hipStream_t stream);

/* Device scratch that cg_kv8_select needs (bytes); 0 if an argument is invalid. */
uint64_t cg_kv8_select_workspace_bytes(const cg_kv8_cache* c, const cg_kv8_seqs* s,
                                       const cg_kv8_attn* a);

/* The pages each query token should read: picks_out [n_seq][n_q][H][a->n_picks], table columns in
 * ascending order, -1 behind the last. Of a query token that sees n tokens, the last `recent` of
 * its ceil(n / 64) pages are taken, and of the others the best by
 *   score(page) = fp32(sum over the group's heads and the channels of max(q8 lo, q8 hi)) * k_scale
 * with q8 = rint(clamp(q * 2^(6 - e), +-127)), 2^e the power of two at or below the largest |q| of
 * the group, and lo, hi the page's bounds: an upper bound of the page's summed q8 . k, in whole
 * numbers (of at most 31 bits: groups past 520 heads of 256 channels, 1040 of 128, 2080 of 64 are
 * CG_ERR_SHAPE). Equal scores go to the lower column. Uses q, lengths, max_len, q_lens, n_picks and
 * dtype of `a`; the workspace as for cg_kv8_attend. Asynchronous. */
int cg_kv8_select(const cg_kv8_cache* c, const cg_kv8_seqs* s, const cg_kv8_attn* a,
                  int32_t recent, int32_t* picks_out, void* workspace, uint64_t workspace_bytes,
                  hipStream_t stream);

/* Cut every sequence longer than `keep` to `keep` tokens, in new pages. Per sequence and KV head
 * the last min(recent, keep) tokens stay, and of the others the heaviest by mass [P][H][64]
 * (equal weights: the earlier token; a NaN weighs least). The tokens that stay are coded again
 * page by page (scale: their largest |code * scale| over 127) into the pages of `to`, in their
 * order, bounds and weights moving along; shorter sequences move whole.
 *   lengths      [n_seq], none above max_len.
 *   to           the same n_seq, at least ceil(min(keep, max_len) / 64) columns; its pages must
 *                be no page of `s`, nor shared within the call.
 *   kept         out [n_seq][H][keep]: the tokens that stay, ascending, -1 behind the last.
 *   new_lengths  out [n_seq] = min(length, keep).
 * Asynchronous. */
int cg_kv8_evict(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* lengths,
                 int32_t max_len, float* mass, int32_t keep, int32_t recent,
                 const cg_kv8_seqs* to, int32_t* kept, int32_t* new_lengths, hipStream_t stream);

/* ---- Requests that share a context ---------------------------------------------------------
 * Sequences may hold the same pages: refs [P] (int32, the caller's, on the device) counts the table
 * rows that hold each page, and 0 marks it free. A context is forked into requests, which share its
 * pages; before a request writes, cg_kv8_reserve gives it pages, and of a page that it shares a copy
 * of its own; cg_kv8_release gives back what a request no longer needs, all of it or what lies
 * behind a length (drafted tokens that were not accepted). Table entries outside [0, n_pages) are
 * "no page" (-1 is written). Every call is asynchronous, allocates nothing, and gives the same
 * result in whatever order its parts run. A page's weights (c->mass, if given) go where the page
 * goes. */

/* Children of sequences: row c of `to` receives the pages of sequence parents[c] of `s` that hold
 * its first min(lengths[parent], ends[c]) tokens, -1 behind them, and each page's count goes up by
 * one for each child.
 *   parents      [to->n_seq]; one outside [0, s->n_seq) makes an empty sequence.
 *   ends         [to->n_seq] tokens to share, or NULL: all.
 *   to           its table is written: at least s->max_pages columns, no memory of a row of `s`
 *                that is a parent's (else the result is undefined). What its rows held is not
 *                released.
 *   new_lengths  out [to->n_seq]. */
int cg_kv8_fork(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* lengths,
                const int32_t* parents, const int32_t* ends, const cg_kv8_seqs* to,
                int32_t* new_lengths, int32_t* refs, hipStream_t stream);

/* Device scratch of cg_kv8_reserve (bytes): 16 a sequence, two bits a column (in words of 64) and up
 * to 4 a page, behind the zeroed front. 0 if an argument is invalid. */
uint64_t cg_kv8_reserve_workspace_bytes(const cg_kv8_cache* c, const cg_kv8_seqs* s);

/* Pages for tokens lengths[b] .. lengths[b] + counts[b] - 1 of every sequence (as far as its row of
 * the table goes), which a cg_kv8_store will write. Of the columns they touch, one that holds earlier
 * tokens keeps its page if its count is 1, and gets a copy of it if that is more (a lost page, -1,
 * stays lost); any other keeps a page whose count is 1 and gets a free one otherwise. The i-th page
 * wanted, by sequence and column, is the i-th free one; its count becomes 1, and that of the page it
 * replaces goes down by one. Sequences of one call that share a page get a copy each, and pages that
 * they all leave are free behind the call, not in it.
 *   s        its table is written.
 *   missing  out [1]: 0, or how many pages more it would have taken; then nothing is changed, and
 *            nothing may be stored: the pages may be others' too (see cg_kv8_reserve_granted).
 *   workspace as for cg_kv8_attend. */
int cg_kv8_reserve(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* lengths,
                   const int32_t* counts, int32_t* refs, int32_t* missing, void* workspace,
                   uint64_t workspace_bytes, hipStream_t stream);

/* The same, and how many tokens each sequence may store behind lengths[b]:
 *   granted  out [n_seq], or NULL: of counts[b] those that its row has room for, 0 of all sequences
 *            where pages were missing. As the counts of the cg_kv8_store that follows, and added to
 *            the lengths, they keep a call that found too few pages from writing to shared ones,
 *            without the host. May be counts. */
int cg_kv8_reserve_granted(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* lengths,
                           const int32_t* counts, int32_t* refs, int32_t* missing,
                           int32_t* granted, void* workspace, uint64_t workspace_bytes,
                           hipStream_t stream);

/* Gives back the pages of every sequence from column ceil(keep[b] / 64) on (keep NULL: all): their
 * counts go down by one (never below 0), the entries become -1. What the pages hold stays until
 * someone else gets them. */
int cg_kv8_release(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* keep, int32_t* refs,
                   hipStream_t stream);

/* Page src[i] to page dst[i] for i < n, codes, scales, bounds and weights. Pairs outside the pool
 * are skipped. No page is the target of two pairs, or of one and the source of another, or the
 * result is undefined. */
int cg_kv8_copy(const cg_kv8_cache* c, const int32_t* src, const int32_t* dst, int32_t n,
                hipStream_t stream);

/* Device scratch of cg_kv8_compact (bytes): 8 a page behind the zeroed front. 0 if c is invalid. */
uint64_t cg_kv8_compact_workspace_bytes(const cg_kv8_cache* c);

/* The pages in use (count above 0) move to the front of the pool: with L of them, the i-th that lies
 * at L or behind goes to the i-th free page before L. The others stay.
 *   s            the sequences' table as it was.
 *   new_table    out [n_seq][max_pages]: the same with the pages' new numbers (may be s->table).
 *   new_refs     out [P]: the counts as the pages lie now (not refs itself).
 *   moved        out [P]: the new number of each page, -1 of one that was free: for other tables.
 *   n_live       out [1]: L. */
int cg_kv8_compact(const cg_kv8_cache* c, const cg_kv8_seqs* s, const int32_t* refs,
                   int32_t* new_table, int32_t* new_refs, int32_t* moved, int32_t* n_live,
                   void* workspace, uint64_t workspace_bytes, hipStream_t stream);

/* The contexts of cg_kv8_attend_shared. */
typedef struct cg_kv8_contexts {
  cg_kv8_seqs seqs;             /* the contexts' pages */
  const int32_t* lengths;       /* [seqs.n_seq] tokens of each */
  int32_t max_len;              /* no length is above it (longer ones are cut to it) */
  const int32_t* firsts;        /* [seqs.n_seq + 1], ascending: context p is read by sequences
                                   firsts[p] .. firsts[p + 1] - 1 of the call */
  int32_t max_users;            /* no context is read by more of them (those behind see none); n_seq
                                   where the host does not know, at little cost */
} cg_kv8_contexts;

/* Device scratch that cg_kv8_attend_shared needs (bytes); 0 if an argument is invalid or none is
 * needed. It follows the numbers of sequences and contexts and the two max_len, whatever max_users
 * leaves room for. CG_ERR_SHAPE: with the smaller of contexts * max_users and n_seq + contexts for the
 * sequences, the query tokens times H are above 2^23, or their rows above 2^30. */
uint64_t cg_kv8_attend_shared_workspace_bytes(const cg_kv8_cache* c, const cg_kv8_contexts* x,
                                              const cg_kv8_seqs* s, const cg_kv8_attn* a);

/* Attention of sequences that share contexts, whose pages are read once for all that share them.
 * The query tokens of a sequence see all of its context (none, if it has none) and, as in
 * cg_kv8_attend, their sequence's own tokens up to their place: with S = scale * q . k over both,
 *   out = softmax(S) v,   lse = log sum exp(S).
 *   s    the sequences' own pages, behind the context; lengths and max_len of `a` are theirs. With
 *        table NULL there are none (max_pages and a->lengths are not read): attention of n_seq
 *        sequences over the contexts alone, as over the states of an encoder.
 *   a    as for cg_kv8_attend; without picks and weights (CG_ERR_ARG).
 * Precision, workspace and the rest as for cg_kv8_attend; what is said there of page scales within
 * a sequence holds within a context and within a sequence's own pages. */
int cg_kv8_attend_shared(const cg_kv8_cache* c, const cg_kv8_contexts* x, const cg_kv8_seqs* s,
                         const cg_kv8_attn* a, void* workspace, uint64_t workspace_bytes,
                         hipStream_t stream);

/* Drafted tokens against the target's probabilities. Sequence b has drafts x_0 .. x_(counts[b] - 1);
 * p_j is row j of its target probabilities (n_drafts + 1 rows: the last is behind all drafts), q_j
 * row j of the draft's. x_j is accepted while u_j q_j(x_j) < p_j(x_j) (so with probability
 * min(1, p / q)); the first that is not ends the drafts, and one more token is drawn, from the
 * weights max(p_j - q_j, 0) there, or from p of the row behind the last accepted draft. With exact u
 * the tokens would be distributed as the target's; the last one is drawn with 24 bits of its u (see
 * cg_verify_drafts), so that its probability is off by up to 2^-24. */
#define CG_VERIFY_MAX_VOCAB (1 << 20)
#define CG_VERIFY_MAX_DRAFTS 1024
enum { CG_KV8_F32 = 2 };        /* a type of probabilities, beside CG_KV8_F16 and CG_KV8_BF16 */

typedef struct cg_verify {
  int32_t n_seq, n_drafts, vocab, dtype;
  const void* target;           /* [n_seq][n_drafts + 1][vocab], rows t_row_stride apart */
  int64_t t_seq_stride, t_row_stride;          /* in elements */
  const void* draft;            /* [n_seq][n_drafts][vocab], or NULL: each draft was sure (q = 1 for
                                   it, 0 for the others) */
  int64_t d_seq_stride, d_row_stride;
  const int32_t* drafts;        /* [n_seq][n_drafts]; a token outside [0, vocab) is not accepted */
  const int32_t* counts;        /* [n_seq], at most n_drafts; below 0 the sequence sits out; NULL:
                                   n_drafts */
  const float* u;               /* [n_seq][n_drafts + 1] in [0, 1): u_j for draft j, the last for the
                                   token that is drawn */
  int32_t* tokens;              /* out [n_seq][n_drafts + 1]: the accepted drafts and the token
                                   drawn, -1 behind it */
  int32_t* accepted;            /* out [n_seq] drafts accepted; 0 of one that sits out */
  const int32_t* lengths;       /* [n_seq] tokens held, the drafts' own among them, and out: */
  int32_t* new_lengths;         /* those less the drafts not accepted (may be lengths), or NULL */
} cg_verify;

/* Device scratch of cg_verify_drafts (bytes); 0 if the sizes are invalid. */
uint64_t cg_verify_workspace_bytes(const cg_verify* v);

/* The above. A probability counts as 0 where it is NaN or below 0 and as 1 above 1; the acceptance
 * is decided exactly; a weight is a difference of probabilities rounded to multiples of 2^-42, and of
 * a row whose weights sum to W such multiples the token drawn is the first with
 * (weights up to it) > floor(floor(u 2^24) W / 2^24), all in whole numbers. Where nothing of p is
 * above q the weights are p's own, and -1 is drawn where those are all 0. n_drafts may be 0. The
 * workspace as for cg_kv8_attend. Asynchronous. */
int cg_verify_drafts(const cg_verify* v, void* workspace, uint64_t workspace_bytes,
                     hipStream_t stream);

/* Static description of a return code; never NULL. */
const char* cg_strerror(int code);

#ifdef __cplusplus
}
#endif

#endif /* CACHEGEN_H */
