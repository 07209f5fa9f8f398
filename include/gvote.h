/*
 * gvote.h — C ABI of the GVote per-request KV-cache compression pass for NVIDIA B200 (sm_100a).
 *
 * The pass is Algorithm 1 of "Adaptive KV-Cache Compression without Manually Setting Budget"
 * (GVote), run once per layer at the end of prefill, per request and per KV head
 * (Section 3.2): fit a diagonal Gaussian to the hidden states (Step 2), draw S synthetic
 * hidden states (Step 3), project them through W_q and rotate them with the RoPE cos/sin
 * averaged over n_f future positions (Step 3), score them against all cached keys, let each
 * synthetic query pick its keys (top-k with k = |C0|, where C0 is the top-p set of the
 * current query, Step 1), OR the picks into one keep-mask per KV head (Step 4) and prune K
 * and V to that set (the pruning step of Algorithm 1).
 *
 * Conventions, valid for every entry point unless it says otherwise
 *  - Every pointer named below is a DEVICE pointer unless its comment says "host".
 *  - The caller owns every buffer.  The library allocates nothing, frees nothing and keeps
 *    no pointer after a call returns (gvote_compress_host is the one exception, see there).
 *  - Work is enqueued on the given CUDA stream (passed as void* = cudaStream_t); calls return
 *    without synchronising.
 *  - Return value: GVOTE_OK (0) or a negative GVOTE_ERR_* code.  On an error detected on the
 *    host nothing has been enqueued.  A bounded device-side wait that ran out is reported
 *    through the status word at the start of the workspace: read it with gvote_poll_status.
 *  - Pointers must be 16-byte aligned; d_h must be a multiple of 8, d_k a multiple of 8.
 *  - A ragged batch packs its requests along the token axis; cu_seqlens [batch+1] int32
 *    (device) holds the prefix sums of the request lengths N_r (request r owns tokens
 *    cu_seqlens[r] .. cu_seqlens[r+1]-1).  `total_tokens` = cu_seqlens[batch] and `max_N` =
 *    the longest request are passed from the host so that no call has to read the device.
 *    A request may be empty (N_r = 0): nothing is read or written for it, its budgets and |C0| are 0.
 *    A non-empty request needs N_r - n_s >= 2 rows for the fit.
 *  - bf16 tensors: W_q [n_q_heads*d_k, d_h], one row per output feature (the paper's W_q
 *    stored transposed, as linear layers keep it), row stride wq_ld elements;
 *    K and V [n_kv_heads, total_tokens, d_k] with element strides (head_stride, tok_stride),
 *    inner dimension contiguous; keys are stored as the model stores them (already rotated).
 *  - Positions: request r's keys sit at positions 0..N_r-1, its current query at N_r-1 and the
 *    n_f future positions are N_r .. N_r+n_f-1.
 *  - Keep-mask: uint32 words, bit (n mod 32) of word (n div 32) is key n of the request; each
 *    request's bit row starts on a word boundary at word gvote_mask_word_offset(cu_seqlens[r], r)
 *    of its head's row; a head's row has gvote_mask_row_words(total_tokens, batch) words;
 *    padding bits are zero.
 */
#ifndef GVOTE_H_
#define GVOTE_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define GVOTE_API __attribute__((visibility("default")))
#else
#define GVOTE_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

enum {
  GVOTE_OK = 0,
  GVOTE_ERR_INVALID_ARG = -1,
  GVOTE_ERR_UNALIGNED = -2,
  GVOTE_ERR_WORKSPACE_TOO_SMALL = -3,
  GVOTE_ERR_UNSUPPORTED_SHAPE = -4,
  GVOTE_ERR_CUDA = -5,
  GVOTE_ERR_TIMEOUT = -6
};

enum { GVOTE_SEL_TOPK_C0 = 0, GVOTE_SEL_TOPP = 1 };
enum { GVOTE_DTYPE_F32 = 0, GVOTE_DTYPE_BF16 = 1 };

/* Hyper-parameters and model shape (Algorithm 1, "Require" line, plus what it uses implicitly). */
typedef struct {
  int32_t d_h;          /* hidden size */
  int32_t n_q_heads;    /* query heads */
  int32_t n_kv_heads;   /* KV heads; n_q_heads must be a multiple */
  int32_t d_k;          /* head dimension */
  double  rope_theta;   /* RoPE base; rotate-half pairing (j, j+d_k/2), w_j = theta^(-2j/d_k) */
  int32_t S;            /* synthetic queries per request (Section 3.5: S >= 8 advised) */
  float   p_nuc;        /* nucleus mass threshold in (0,1] (Section 3.5: 0.95 advised) */
  int32_t n_f;          /* future positions whose cos/sin are averaged (Step 3) */
  int32_t n_s;          /* leading sink tokens the fit ignores (Step 2) */
  int32_t sel_mode;     /* GVOTE_SEL_TOPK_C0: the TopK step of Algorithm 1.  GVOTE_SEL_TOPP: the top-p rule
                           of Section 3.1 applied to every synthetic query instead. */
  int32_t include_c0;   /* non-zero: the current query's set C0 joins the union (Algorithm 1 unions
                           the synthetic sets only; default 0) */
  uint64_t seed;        /* Philox key */
  uint32_t layer_id;    /* Philox counter word: gives every layer its own stream */
  int32_t h_dtype;      /* GVOTE_DTYPE_F32 or GVOTE_DTYPE_BF16: element type of h and h_last */
} gvote_params;

/* Words per head in the keep-mask, and the word where request r's bits start. */
static inline int64_t gvote_mask_row_words(int64_t total_tokens, int32_t batch) {
  return (total_tokens >> 5) + batch;
}
static inline int64_t gvote_mask_word_offset(int64_t cu_seqlens_r, int32_t r) {
  return (cu_seqlens_r >> 5) + r;
}

/* Bytes of scratch every entry point below accepts as `ws` for a batch of this size.  The
 * first 256 bytes hold the status word; a workspace must be zero-filled once after
 * allocation (the library keeps it consistent afterwards).  Returns 0 on invalid params.
 * The size depends on p->sel_mode.  GVOTE_SEL_TOPK_C0 (Algorithm 1) keeps no logits matrix: per synthetic
 * query a few thousand sampled 16-bit keys and a short candidate list, per current query one fp32 row
 * (Section 4.4 names the S x N matrix as what runs out of memory beyond 128K context).  GVOTE_SEL_TOPP
 * needs every row's softmax mass and keeps the fp32 logits of all (S+1) x n_q_heads rows:
 * 4 (S+1) n_q_heads total_tokens bytes more.  A call that asks for the softmax rows (dbg_probs) needs the
 * GVOTE_SEL_TOPP size whatever its mode, as do shapes the fused kernels do not take (d_k other than 64
 * or 128, more than 16 query heads per KV head): gvote_workspace_bytes accounts for that. */
GVOTE_API size_t gvote_workspace_bytes(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N);

/* Where gvote_select and the whole-pass entry points (gvote_compress, gvote_compress_moments, gvote_recompress) leave the
 * rotated queries of Algorithm 1 that their vote used - Q0 (exact position) and the S synthetic queries
 * (averaged cos/sin) of every query head: byte offset into `ws` of a bf16 array
 * [batch][n_kv_heads][G (S+1)][d_k], G = n_q_heads / n_kv_heads, the layout gvote_project writes (per KV
 * head the G*S synthetic rows, query head by query head, then the G current-query rows).  They stay valid
 * until the next call that uses the workspace; gvote_overlap and a caller's own checks can read them there.
 * Returns 0 on invalid params (offset 0 is the status block, never the queries). */
GVOTE_API size_t gvote_workspace_queries(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N);

/* Step 2 of Section 3.2 (the Gaussian fit of Algorithm 1).  mu[r][c], var[r][c] = mean and unbiased variance over rows
 * cu_seqlens[r]+n_s .. cu_seqlens[r+1]-1 of h [total_tokens, d_h] (row stride h_row_stride
 * elements).  Every request needs N_r - n_s >= 2 (the result is NaN otherwise; the host cannot
 * check device-resident lengths, it checks max_N only).  mu, var: [batch, d_h] float. */
GVOTE_API int32_t gvote_fit(const gvote_params* p, const void* h, int64_t h_row_stride,
                  const int32_t* cu_seqlens, int32_t batch, int64_t total_tokens, int64_t max_N,
                  float* mu, float* var, void* ws, size_t ws_bytes, void* stream);

/* Step 2 while the prompt streams by (the Gaussian needs only running moments, not the hidden states:
 * an engine can feed each prefill chunk's layer-norm output and drop it, which takes the fit's read of
 * all hidden states out of the compression pass).
 * state: [batch, 3, d_h] double, zero-filled before the first block; per request and channel it
 * holds the number of rows seen, their mean and their sum of squared deviations.
 * gvote_fit_update folds one block of rows into the state: h_block [total_rows, d_h] holds the new rows
 * of every request, request r owning rows cu_block[r] .. cu_block[r+1]-1 (a request may have none).
 * Every row given is counted: leaving out the n_s sink tokens is the caller's doing here (p->n_s is not
 * used).  Blocks are merged with the pairwise update of Chan, Golub and LeVeque in fp64.
 * gvote_fit_finish turns the state into mu and the unbiased variance (NaN below two rows), the inputs
 * of gvote_sample and gvote_compress_moments. */
GVOTE_API int32_t gvote_fit_update(const gvote_params* p, const void* h_block, int64_t h_row_stride,
                         const int32_t* cu_block, int32_t batch, int64_t total_rows, int64_t max_rows,
                         double* state, void* ws, size_t ws_bytes, void* stream);
GVOTE_API int32_t gvote_fit_finish(const gvote_params* p, const double* state, int32_t batch,
                         float* mu, float* var, void* stream);

/* Fit without any allocation (the paper has no counterpart: this entry point exists for the
 * integration, not for the method).  Same result as gvote_fit, but the per-chunk partial moments
 * live in a fixed 1 MiB array inside the library's device image (GVOTE_FIT_STATIC_MAX_ENTRIES
 * pairs of floats, present on every GPU that loads the library until the process exits), so the
 * caller passes inputs and outputs only and the call obtains no memory, from CUDA or from
 * anyone else.  Use it where asking for device memory is not possible: inside an allocator or
 * memory-pool callback, in a serving loop whose pool is frozen after warm-up, on a thread that
 * may not wait on the allocator's lock.
 *  - Limit: batch * d_h <= GVOTE_FIT_STATIC_MAX_ENTRIES, else GVOTE_ERR_UNSUPPORTED_SHAPE and
 *    nothing is enqueued.  Long inputs are fine: fewer, longer row chunks are used instead.
 *  - The first call on each device looks up the array's device address (with that device
 *    current).  Make that first call before starting any stream capture.
 *  - All calls on a device share the one array.  It needs no clearing (every entry a call reads
 *    it has written itself), but two calls whose kernels may overlap on the GPU (different
 *    streams, no dependency) race on it: serialise them.
 *  - There is no status word here: a bounded device-side wait that ran out shows as NaN in mu.
 * Arguments as in gvote_fit, minus the workspace and total_tokens. */
#define GVOTE_FIT_STATIC_MAX_ENTRIES 131072
GVOTE_API int32_t gvote_fit_static(const gvote_params* p, const void* h, int64_t h_row_stride,
                         const int32_t* cu_seqlens, int32_t batch, int64_t max_N,
                         float* mu, float* var, void* stream);

/* Step 3 of Section 3.2 (the sampling step of Algorithm 1).  H_tilde[r][s][c] = mu[r][c] + sqrt(var[r][c]) * z, z a standard
 * normal drawn by Box-Muller from Philox4x32-10 with key = (seed low, seed high) and counter
 * = (c div 4, s, layer_id, r); word pairs (0,1) and (2,3) of a block give channels 4b..4b+3;
 * u = ((x >> 9) + 0.5) * 2^-23.  H_tilde: [batch, S, d_h] float.  raw_u32_or_null, when given,
 * receives the Philox words [batch, S, d_h] (bit-exact by definition). */
GVOTE_API int32_t gvote_sample(const gvote_params* p, const float* mu, const float* var, int32_t batch,
                     float* H_tilde, uint32_t* raw_u32_or_null, void* stream);

/* Algorithm 1: the current query Q0, AverageCosSin and the synthetic queries.  X = [h_last[r]; H_tilde[r]] is rounded to bf16, multiplied
 * by W_q (fp32 accumulation), b_q added when given ([n_q_heads*d_k] float), then rotated: row 0
 * exactly at position N_r-1, rows 1..S with the mean cos/sin of positions N_r..N_r+n_f-1.
 * Q: [batch, n_kv_heads, G*(S+1), d_k] bf16 with G = n_q_heads / n_kv_heads; the rows of a KV head
 * are ordered for the score contraction: first the S synthetic rows of each of its G query heads
 * (row gl*S + s), then the G current-query rows (row G*S + gl).  h_last: [batch, d_h] of p->h_dtype. */
GVOTE_API int32_t gvote_project(const gvote_params* p, const float* H_tilde, const void* h_last,
                      const void* W_q, int64_t wq_ld, const float* b_q_or_null,
                      const int32_t* cu_seqlens, int32_t batch,
                      void* Q, void* ws, size_t ws_bytes, void* stream);

/* Algorithm 1, the current-query steps (A0, C0, B_step) and the vote (logits, TopK, union), given the rotated queries (layout as written by gvote_project).
 * Per query head g: logits of its
 * S+1 rows against the N_r keys of KV head g div G, scaled by 1/sqrt(d_k); row 0 -> softmax ->
 * top-p -> b_step[r][g] = |C0|; rows 1..S -> top-k(b_step) on logits (or top-p on their softmax
 * in GVOTE_SEL_TOPP); mask[h] = OR over the rows of the head's group; budget[r][h] = popcount.
 * Ties at a selection boundary go to the lower key index.  mask: [n_kv_heads, row_words] is
 * overwritten.  dbg_probs_or_null: [sum_r n_q_heads*(S+1)*N_r] float, request-major, receives the
 * softmax rows (small cases only). */
GVOTE_API int32_t gvote_vote(const gvote_params* p, const void* Q,
                   const void* K, int64_t k_tok_stride, int64_t k_head_stride,
                   const int32_t* cu_seqlens, int32_t batch, int64_t total_tokens, int64_t max_N,
                   uint32_t* mask, int32_t* budget, int32_t* b_step,
                   float* dbg_probs_or_null, void* ws, size_t ws_bytes, void* stream);

/* gvote_project followed by gvote_vote (Algorithm 1 without the fit, the sampling and the pruning); Q lives in ws. */
GVOTE_API int32_t gvote_select(const gvote_params* p, const float* H_tilde, const void* h_last,
                     const void* W_q, int64_t wq_ld, const float* b_q_or_null,
                     const void* K, int64_t k_tok_stride, int64_t k_head_stride,
                     const int32_t* cu_seqlens, int32_t batch, int64_t total_tokens, int64_t max_N,
                     uint32_t* mask, int32_t* budget, int32_t* b_step,
                     float* dbg_probs_or_null, void* ws, size_t ws_bytes, void* stream);

/* Algorithm 1, the pruning step.  In place: for every request r and KV head h the kept rows of K and V
 * move, in ascending key order, to rows cu_seqlens[r] .. cu_seqlens[r]+budget[r][h]-1 of the
 * head's slab; rows behind them are left as they are.  budget [batch, n_kv_heads] is written
 * (popcount of the mask).  Rows are d_k bf16 values, moved in 16-byte pieces. */
GVOTE_API int32_t gvote_compact(const gvote_params* p, void* K, void* V, int64_t tok_stride, int64_t head_stride,
                      const uint32_t* mask, const int32_t* cu_seqlens, int32_t batch,
                      int64_t total_tokens, int64_t max_N, int32_t* budget,
                      void* ws, size_t ws_bytes, void* stream);

/* Section 3.3's yardstick applied to a keep-mask: overlap[r][g] = the share of the current query's
 * attention (softmax weights of Eq. 1 over all N_r keys) of query head g that falls on the keys its
 * KV head keeps; 1 means nothing the query looks at was pruned.  Q as written by gvote_project (the
 * current-query rows are used), K the UNPRUNED keys, mask as written by gvote_vote.  overlap:
 * [batch, n_q_heads] float.  A diagnostic: fp32 logits, not on the compression path. */
GVOTE_API int32_t gvote_overlap(const gvote_params* p, const void* Q,
                      const void* K, int64_t k_tok_stride, int64_t k_head_stride,
                      const uint32_t* mask, const int32_t* cu_seqlens, int32_t batch,
                      int64_t total_tokens, int64_t max_N, float* overlap,
                      void* ws, size_t ws_bytes, void* stream);

/* Section 3.4: the pruned cache in the layout a variable-length attention kernel consumes, written
 * out of place from the UNPRUNED K and V and the keep-mask (use it instead of gvote_compact when
 * the engine wants one dense buffer rather than per-head slabs).  "Sequence" s = r * n_kv_heads + h
 * (request r, KV head h) owns rows cu_seqlens_k[s] .. cu_seqlens_k[s+1]-1 of K_packed and V_packed
 * ([capacity_rows, d_k] bf16, dense), kept rows in ascending key order; cu_seqlens_k
 * [batch*n_kv_heads + 1] int32 and budget [batch, n_kv_heads] are written.  The buffers need
 * cu_seqlens_k[last] rows, at most n_kv_heads * total_tokens; if capacity_rows is smaller than what the
 * mask keeps, the rows that do not fit are not written and the workspace status word reads
 * GVOTE_ERR_WORKSPACE_TOO_SMALL (gvote_poll_status).  K and V are not modified. */
GVOTE_API int32_t gvote_pack(const gvote_params* p, const void* K, const void* V, int64_t tok_stride, int64_t head_stride,
                   const uint32_t* mask, const int32_t* cu_seqlens, int32_t batch,
                   int64_t total_tokens, int64_t max_N, void* K_packed, void* V_packed, int64_t capacity_rows,
                   int32_t* cu_seqlens_k, int32_t* budget, void* ws, size_t ws_bytes, void* stream);

/* Algorithm 1, whole: fit, sample, project, vote, compact for one layer.  The current query's
 * hidden state is the last row of each request in h unless h_last_or_null is given.
 * Outputs: mask, budget, b_step as in gvote_vote; K and V compacted in place. */
GVOTE_API int32_t gvote_compress(const gvote_params* p, const void* h, int64_t h_row_stride, const void* h_last_or_null,
                       const void* W_q, int64_t wq_ld, const float* b_q_or_null,
                       void* K, void* V, int64_t tok_stride, int64_t head_stride,
                       const int32_t* cu_seqlens, int32_t batch, int64_t total_tokens, int64_t max_N,
                       uint32_t* mask, int32_t* budget, int32_t* b_step,
                       void* ws, size_t ws_bytes, void* stream);

/* Algorithm 1 from the sampling step on, for a caller that already has the Gaussian (gvote_fit_finish): sample,
 * project, vote, compact.  mu, var [batch, d_h] float; h_last [batch, d_h] of p->h_dtype is the current
 * query's hidden state.  Other arguments and outputs as in gvote_compress. */
GVOTE_API int32_t gvote_compress_moments(const gvote_params* p, const float* mu, const float* var, const void* h_last,
                               const void* W_q, int64_t wq_ld, const float* b_q_or_null,
                               void* K, void* V, int64_t tok_stride, int64_t head_stride,
                               const int32_t* cu_seqlens, int32_t batch, int64_t total_tokens, int64_t max_N,
                               uint32_t* mask, int32_t* budget, int32_t* b_step,
                               void* ws, size_t ws_bytes, void* stream);

/* The pass applied again to a cache it has pruned before and that has grown since (an extension: in
 * Section 3.4 the pass runs once, after prefill).  The heads of such a cache differ in length, and a slot
 * no longer is a position, so the N of Algorithm 1 splits in two:
 *  - kv_len [batch, n_kv_heads] int32 (device): rows KV head h of request r holds (kept earlier plus
 *    appended since), at the front of its slab cu_seqlens[r] .. ; rows beyond are ignored.  Every query
 *    head votes over the rows of its own KV head only (current-query steps and vote); kv_len may be 0 (budget 0).
 *  - seq_len [batch] int32 (device): tokens the request has seen.  The current query is rotated at
 *    position seq_len - 1, the synthetic queries with the mean over positions seq_len .. seq_len+n_f-1
 *    (the current query and AverageCosSin); keys stay rotated where they were written.
 *  - cu_seqlens / total_tokens / max_N describe the slabs (capacity), as in gvote_compress.
 *  - token_pos_or_null [n_kv_heads, total_tokens] int32 (device, in/out): the original position of every
 *    slot; its kept entries move to the front of the slab with the rows (entries beyond the new budget
 *    are left as they were).
 * mu, var: the caller's running fit (gvote_fit_update / gvote_fit_finish over all tokens seen).
 * Outputs as in gvote_compress: mask over slots, budget = new rows per head, b_step, K and V compacted
 * in place. */
GVOTE_API int32_t gvote_recompress(const gvote_params* p, const float* mu, const float* var, const void* h_last,
                         const void* W_q, int64_t wq_ld, const float* b_q_or_null,
                         void* K, void* V, int64_t tok_stride, int64_t head_stride,
                         const int32_t* cu_seqlens, const int32_t* kv_len, const int32_t* seq_len,
                         int32_t* token_pos_or_null, int32_t batch, int64_t total_tokens, int64_t max_N,
                         uint32_t* mask, int32_t* budget, int32_t* b_step,
                         void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------------
 * The pruned cache in use: rows held in 8 bits, attention of a few tokens over them, and eviction by the
 * attention weight a row has collected (the other common rule for what a cache keeps; Section 4.1 compares
 * the method with such systems).  A prompt goes gvote_compress* or gvote_accumulate + gvote_evict ->
 * gvote_store8 (mask); a token goes gvote_append8 -> gvote_attend8; a full cache goes gvote_evict ->
 * gvote_prune8.
 *
 * The 8-bit cache.  K and V [n_kv_heads, total_tokens, d_k] e4m3 codes (1 sign, 4 exponent, 3 fraction bits, no
 * infinities), in slabs per request as everywhere (cu_seqlens), KV head h of request r holding
 * kv_len[r][h] rows at the front of its slab.  Rows 64 b .. 64 b + 63 of a (request, head) are a block and
 * share one scale for K and one for V: scale word gvote_cache8_block_offset(cu_seqlens[r], r) + b of the
 * head's row of gvote_cache8_row_blocks(total_tokens, batch) floats.  A row's value is code * scale.
 * A scale is a power of two, the smallest 2^e, e >= -126, with max |x| <= 448 * 2^e over the block's finite
 * entries: dividing by it is exact, so a code is its value correctly rounded (nearest, ties to the even
 * code), and a row that moves to a block of another scale keeps its value unless that leaves e4m3's normal
 * range.  A NaN or an infinity is stored as the NaN code.
 *
 * Restrictions of all entry points of this part: d_k a multiple of 16, at most 256; byte strides of the codes
 * multiples of 16; at most 1024 KV heads and 128 query heads per KV head; total_tokens <= 2^30.  Slabs are addressed by 64-bit
 * offsets.  A workspace serves one call at a time: calls (or replays of captured graphs) that may overlap on
 * the GPU need one each; between calls it holds nothing but the status word. */
#define GVOTE_CACHE8_BLOCK 64
typedef struct {
  void* K;                   /* e4m3 codes, device */
  void* V;
  float* k_scale;            /* [n_kv_heads][gvote_cache8_row_blocks] */
  float* v_scale;
  const int32_t* cu_seqlens; /* [batch+1] slab boundaries */
  int32_t* kv_len;           /* [batch][n_kv_heads] rows held; values are clamped to 0 .. slab length */
  int64_t tok_stride;        /* elements (= bytes) between rows, and between heads */
  int64_t head_stride;
  int64_t total_tokens;      /* cu_seqlens[batch] */
  int64_t max_N;             /* longest slab */
  int32_t batch;
  int32_t reserved;
} gvote_cache8;
static inline int64_t gvote_cache8_row_blocks(int64_t total_tokens, int32_t batch) {
  return (total_tokens >> 6) + batch;
}
static inline int64_t gvote_cache8_block_offset(int64_t cu_seqlens_r, int32_t r) {
  return (cu_seqlens_r >> 6) + r;
}

/* Bytes of scratch the entry points of this part accept as `ws`, for slabs of this size and queries of this
 * size (total_q query tokens in all, max_q of one request at most; 0, 0 for calls without queries), and for
 * every call of no larger sizes.  gvote_attend8 of these very sizes without acc_out accepts 4 n_q_heads max_q total_tokens
 * bytes less: it keeps no logits.  Where a call has a source and a destination cache, the larger of both.  Zero-fill
 * it once; status word as everywhere (gvote_poll_status).  0 on invalid arguments. */
GVOTE_API size_t gvote_cache_workspace_bytes(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N,
                                   int64_t total_q, int64_t max_q);

/* The pruning step of Algorithm 1 into the 8-bit cache: the kept rows of K and V (bf16 slabs, as in
 * gvote_compact; not modified), in ascending order, become rows 0 .. of the head's slab in `cache`, and
 * cache->kv_len is written.  mask_or_null: keep-mask over slots (null keeps all); kv_len_or_null: rows that
 * count per (request, head), as in gvote_recompress (bits behind them are ignored).  `cache` has slabs of its own
 * (same batch); rows that do not fit are dropped and the status word reads GVOTE_ERR_WORKSPACE_TOO_SMALL.
 * Per-slot side arrays [n_kv_heads, total_tokens] move with the rows: acc -> acc_out, token_pos ->
 * token_pos_out (with the cache's total_tokens); token_pos_out without token_pos receives the source slot.
 * What lies behind the last row (codes, scales, side arrays) is left as it was. */
GVOTE_API int32_t gvote_store8(const gvote_params* p, const void* K, const void* V, int64_t tok_stride, int64_t head_stride,
                     const uint32_t* mask_or_null, const int32_t* cu_seqlens, const int32_t* kv_len_or_null,
                     int32_t batch, int64_t total_tokens, int64_t max_N, const gvote_cache8* cache,
                     const float* acc_or_null, float* acc_out_or_null, const int32_t* token_pos_or_null,
                     int32_t* token_pos_out_or_null, void* ws, size_t ws_bytes, void* stream);

/* The same from one 8-bit cache into another: the kept rows of `src`, scaled anew block by block.  Here and in
 * gvote_store8 what is read must not share a byte with what is written (GVOTE_ERR_INVALID_ARG).  Rows of the same strides may
 * lie between each other, as windows of one wider buffer; with strides that differ the extents must be apart. */
GVOTE_API int32_t gvote_prune8(const gvote_params* p, const gvote_cache8* src, const uint32_t* mask_or_null,
                     const gvote_cache8* dst, const float* acc_or_null, float* acc_out_or_null,
                     const int32_t* token_pos_or_null, int32_t* token_pos_out_or_null,
                     void* ws, size_t ws_bytes, void* stream);

/* New tokens' rows join the cache.  K_new, V_new [n_kv_heads, total_new, d_k] bf16 with element strides, requests
 * packed by cu_new [batch+1] (device; a request may have none), max_new of one request at most.  They become the
 * rows behind kv_len, and kv_len_out [batch, n_kv_heads] = kv_len + new rows (it may be cache->kv_len itself).
 * The scale of a block that holds rows already is max(its scale, the new rows' own); when it grows, the block's codes
 * are rewritten for it.  acc_or_null / token_pos_or_null [n_kv_heads, total_tokens]: the new slots' weight becomes 0,
 * their position pos_new[row of K_new] (given together with token_pos).  Rows that do not fit the slab are
 * dropped and reported as in gvote_store8. */
GVOTE_API int32_t gvote_append8(const gvote_params* p, const void* K_new, const void* V_new, int64_t tok_stride,
                      int64_t head_stride, const int32_t* cu_new, int64_t total_new, int64_t max_new,
                      const gvote_cache8* cache, int32_t* kv_len_out, float* acc_or_null, int32_t* token_pos_or_null,
                      const int32_t* pos_new_or_null, void* ws, size_t ws_bytes, void* stream);

/* Attention of a few tokens per request over the 8-bit cache.  Q, out [total_q, n_q_heads, d_k] bf16 with element
 * strides (tokens, heads), requests packed by cu_q [batch+1] (device); at most GVOTE_ATTEND8_MAX_Q tokens of a
 * request.  A request's query tokens are the last rows of its cache (append first): token i of n sees rows
 * 0 .. kv_len - n + i of a head; a head with fewer rows than that leaves token i nothing, which gives out = 0,
 * lse = -inf.  Per query head g of KV head h: logits q.k_n / sqrt(d_k), softmax, out = sum of weight * value (products of
 * the stored values, 32-bit sums; 32-bit weights, of every row whose weight times value scale is above 2^-126 of the
 * largest such product; an entry of a query is exact down to 2^-17 of the largest of its row and held to 2^-25 of that
 * below), lse_or_null [total_q, n_q_heads] = log of the softmax's denominator.  acc_out_or_null [n_kv_heads,
 * total_tokens]: for the rows held, acc (null: 0) + the weights summed over the request's tokens and the head's group;
 * acc_or_null may be acc_out itself.  Deterministic.  Where cu_q gives a request more than max_q tokens the status word
 * reads GVOTE_ERR_INVALID_ARG and its outputs are not to be used. */
#define GVOTE_ATTEND8_MAX_Q 32
GVOTE_API int32_t gvote_attend8(const gvote_params* p, const void* Q, int64_t q_tok_stride, int64_t q_head_stride,
                      const int32_t* cu_q, int64_t total_q, int64_t max_q, const gvote_cache8* cache,
                      void* out, int64_t out_tok_stride, int64_t out_head_stride, float* lse_or_null,
                      const float* acc_or_null, float* acc_out_or_null, void* ws, size_t ws_bytes, void* stream);

/* Attention weight each cached key collects from a prompt's queries.  Q [total_q, n_q_heads, d_k] bf16 (rotated, element
 * strides), requests packed by cu_q; K as in gvote_vote (UNPRUNED slabs, or the front of them with kv_len).  A
 * request's query tokens are the last of its rows, causal as in gvote_attend8: all of the prompt, or a window of
 * its last tokens.  acc_out [n_kv_heads, total_tokens]: for the rows that count, acc (null: 0) + the softmax weights
 * summed over the tokens and over the head's group; other entries are left as they were.
 * lse_or_null [total_q, n_q_heads]: the logarithm of each query's softmax denominator over the keys it sees, when
 * the prompt's attention has left it (-inf where it sees none); computed here otherwise.  Deterministic.
 * Weights below 2^-126 are zero.  A key that holds an infinity may get NaN also where every logit with it is -inf (query
 * tiles have empty rows, and zero times an infinity is no number); no other key is touched by it. */
GVOTE_API int32_t gvote_accumulate(const gvote_params* p, const void* Q, int64_t q_tok_stride, int64_t q_head_stride,
                         const int32_t* cu_q, int64_t total_q, int64_t max_q, const void* K, int64_t k_tok_stride,
                         int64_t k_head_stride, const int32_t* cu_seqlens, const int32_t* kv_len_or_null,
                         int32_t batch, int64_t total_tokens, int64_t max_N, const float* lse_or_null,
                         const float* acc_or_null, float* acc_out, void* ws, size_t ws_bytes, void* stream);

/* Eviction by collected weight: which rows stay.  Per request and KV head with n rows (kv_len, or the slab), k =
 * clamp(keep[r][h], 0, n) rows are kept: the last min(n_recent, k), then the first min(p->n_s, what is left of k
 * and n), then those of largest acc, ties to the lower slot (a NaN counts as the lowest weight).  keep
 * [batch, n_kv_heads] int32 (device), so that heads may keep different numbers of rows (a budget written by
 * gvote_vote, for instance).  mask and budget (= k) as in gvote_vote: gvote_compact, gvote_pack, gvote_store8 and
 * gvote_prune8 take the mask. */
GVOTE_API int32_t gvote_evict(const gvote_params* p, const float* acc, const int32_t* cu_seqlens,
                    const int32_t* kv_len_or_null, int32_t batch, int64_t total_tokens, int64_t max_N,
                    const int32_t* keep, int32_t n_recent, uint32_t* mask, int32_t* budget,
                    void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------------
 * Attention over bf16 rows, and a paged cache that gives pruned rows' memory back.  A prompt goes gvote_attend (whose lse
 * gvote_accumulate takes) -> gvote_compress* or gvote_evict -> gvote_page_tables (mask) -> gvote_page_write; a token goes
 * gvote_page_tables (cu_new) -> gvote_page_write -> gvote_page_attend; a slab cache compacted in place is attended to by
 * gvote_attend (kv_len).
 *
 * The paged cache.  K and V [n_pages, page_rows, d_k] bf16 with element strides; a page holds rows of ONE KV head of one
 * request, because the heads of a pruned cache differ in length (Section 3.4).  Row j of head h of request r is row
 * j mod page_rows of page tables[r][h][j / page_rows]; kv_len[r][h] rows are held.  Pages of no head lie on a stack,
 * free_pages[0 .. n_free).  What lies in a page behind the last row may be anything, NaN too.  An engine starts with
 * kv_len = 0, free_pages = every page, n_free = n_pages.
 *
 * Restrictions of all entry points of this part: d_k a multiple of 16, at most 256 (at most 128 where max_q >
 * GVOTE_ATTEND_FEW_Q); at most 128 query heads per KV head, 1024 KV heads, 65535 requests; strides multiples of 8 elements;
 * page_rows a power of two, 16 to 1024; n_pages * page_rows < 2^31; max_pages * page_rows <= 2^26.  A workspace
 * (gvote_attend_workspace_bytes, zero-filled once) is for the entry points of this part alone - between calls it holds the
 * status word and counters that are zero - and serves one call at a time: calls, or replays of captured graphs, that may
 * overlap on the GPU need one each.  After GVOTE_ERR_TIMEOUT zero-fill it again. */
#define GVOTE_ATTEND_FEW_Q 32
typedef struct {
  void* K;                   /* [n_pages][page_rows][d_k] bf16, device */
  void* V;                   /* with the same strides */
  int32_t* tables;           /* [batch][n_kv_heads][max_pages] page of every page_rows rows */
  int32_t* kv_len;           /* [batch][n_kv_heads] rows held; values are clamped to 0 .. max_pages * page_rows */
  int32_t* free_pages;       /* [n_pages] stack of unused pages (gvote_page_tables only) */
  int32_t* n_free;           /* [1] its height */
  int64_t row_stride;        /* elements between the rows of a page, and between pages */
  int64_t page_stride;
  int32_t n_pages;
  int32_t page_rows;
  int32_t max_pages;         /* entries of a table */
  int32_t batch;
} gvote_pages;

/* Bytes of scratch the entry points of this part accept as `ws`, for queries of this size (total_q tokens in all, max_q of one
 * request at most; 0, 0 for calls without queries) and for every call of no larger sizes.  0 on invalid arguments. */
GVOTE_API size_t gvote_attend_workspace_bytes(const gvote_params* p, int32_t batch, int64_t total_q, int64_t max_q);

/* Block tables and slot map from lengths, in one call:
 *  1. every head is cut to cut = min(kv_len, keep) rows (keep_or_null [batch, n_kv_heads]; negative: 0): rejected draft tokens,
 *     requests that have ended (0).  Pages without rows go back on the stack.
 *  2. it grows by the request's new tokens, packed by cu_new_or_null [batch+1] (total_new = cu_new[batch], max_new of one
 *     request at most), or by those of them whose bit is set in mask_or_null (a keep-mask over the new tokens, laid out with
 *     cu_new as everywhere).  Pages come off the stack; kv_len becomes cut + new rows.
 *  3. slots_or_null [n_kv_heads, total_new]: page * page_rows + row of each new row, -1 where the mask drops it or the token
 *     belongs to no request.
 * Order: the k-th of K released pages (by request, head, row) goes to free_pages[n_free + K - 1 - k]; the k-th page taken
 * comes from free_pages[n_free + K - 1 - k]; so cutting what was grown last restores the stack.  Table entries behind the
 * last page, and stack entries above the top, keep what they held.
 * All or nothing: where the stack or a table is too short nothing changes, slots are -1 and the status word reads
 * GVOTE_ERR_WORKSPACE_TOO_SMALL; where n_free is not in 0 .. n_pages, the stack would pass n_pages, or a number that is
 * released or taken names no page, it reads GVOTE_ERR_INVALID_ARG.  New rows that go on in a page that does not exist get slots of
 * -1, and the status word reads GVOTE_ERR_INVALID_ARG, too.  Every page belongs to one head of one request or lies on the
 * stack: a page that two tables name (which gvote_page_attend may read) would be released twice, and that is not found out as
 * long as the stack has room.  Without cu_new nothing grows; mask and slots are null then. */
GVOTE_API int32_t gvote_page_tables(const gvote_params* p, const gvote_pages* pages, const int32_t* keep_or_null,
                          const int32_t* cu_new_or_null, int64_t total_new, int64_t max_new, const uint32_t* mask_or_null,
                          int32_t* slots_or_null, void* ws, size_t ws_bytes, void* stream);

/* New rows into their pages: row t of head h of K_new, V_new [n_kv_heads, total_new, d_k] (bf16, element strides) to place
 * slots[h][t]; negative: dropped.  A slot behind the last page is dropped and the status word reads GVOTE_ERR_INVALID_ARG.
 * Slots that are not negative are to differ, as those of gvote_page_tables do: where rows have the same one, its place holds pieces
 * of 16 bytes of any of them afterwards, K and V each for itself, and this is not reported.  K_new, V_new must not share memory with the pages. */
GVOTE_API int32_t gvote_page_write(const gvote_params* p, const void* K_new, const void* V_new, int64_t tok_stride, int64_t head_stride,
                         const int32_t* slots, int64_t total_new, const gvote_pages* pages, void* ws, size_t ws_bytes, void* stream);

/* Attention over the paged cache.  Q, out [total_q, n_q_heads, d_k] bf16 with element strides (tokens, heads), requests packed
 * by cu_q [batch+1] (device), max_q of one request at most: one token, a few drafts, or the next chunk of a prompt.  A
 * request's query tokens are the last rows of its cache (write them first): token i of n sees rows 0 .. kv_len - n + i of a
 * head; a head with fewer rows than that leaves token i nothing, which gives out = 0, lse = -inf (logits that are all -inf
 * count as nothing, too, whatever the values hold).  Beside other logits a value that is not finite reaches the out of every
 * token that sees its row, though the weight be zero.  Per query head of KV head
 * h: logits q.k / sqrt(d_k), softmax, out = sum of weight * value, rounded to bf16 once; lse_or_null [total_q, n_q_heads] = log
 * of the softmax's denominator.  32-bit logits, references and sums; weights enter the product with the values as 16 bits (two bf16
 * terms) in calls of few query rows (max_q x query heads per KV head at most 16, or d_k > 128) and as bf16 in
 * larger ones, before the division by the denominator: a sum of weights (2^8 at most) times values that passes 2^128 is an
 * infinity.  A row that a token does not see has no influence on it, whatever it holds.  Deterministic.  Tokens of no request
 * (before cu_q[0], behind cu_q[batch]) keep their out and lse.  Where cu_q gives a request more than max_q tokens, or a
 * page that rows are read from does not exist, the status word reads GVOTE_ERR_INVALID_ARG and the outputs are not to be used.
 * out and lse must not share memory with Q or with the pages. */
GVOTE_API int32_t gvote_page_attend(const gvote_params* p, const void* Q, int64_t q_tok_stride, int64_t q_head_stride,
                          const int32_t* cu_q, int64_t total_q, int64_t max_q, const gvote_pages* pages, void* out,
                          int64_t out_tok_stride, int64_t out_head_stride, float* lse_or_null, void* ws, size_t ws_bytes,
                          void* stream);

/* The same over slabs: K, V [n_kv_heads, total_tokens, d_k] bf16 as in gvote_vote, request r's rows from cu_seqlens[r] on, all of
 * them or the first kv_len_or_null [batch, n_kv_heads].  With cu_q = cu_seqlens it is a prompt's causal attention. */
GVOTE_API int32_t gvote_attend(const gvote_params* p, const void* Q, int64_t q_tok_stride, int64_t q_head_stride, const int32_t* cu_q,
                     int64_t total_q, int64_t max_q, const void* K, const void* V, int64_t tok_stride, int64_t head_stride,
                     const int32_t* cu_seqlens, const int32_t* kv_len_or_null, int32_t batch, int64_t total_tokens,
                     int64_t max_N, void* out, int64_t out_tok_stride, int64_t out_head_stride, float* lse_or_null, void* ws,
                     size_t ws_bytes, void* stream);

/* The same pass for a caller whose tensors live in HOST memory (pinned memory gives full copy
 * speed): all pointers are host pointers, K and V are dense ([n_kv_heads, total_tokens, d_k]),
 * h is dense [total_tokens, d_h].  The call copies the inputs to device buffers it keeps in a
 * grow-only per-device arena (released by gvote_host_arena_release), runs gvote_compress on an
 * internal stream, copies mask, budget, b_step and the compacted K and V back, and returns after
 * everything has completed.  This is the only entry point that allocates or synchronises. */
GVOTE_API int32_t gvote_compress_host(const gvote_params* p, const void* h, const void* W_q, const float* b_q_or_null,
                            void* K, void* V, const int32_t* cu_seqlens_host, int32_t batch,
                            uint32_t* mask, int32_t* budget, int32_t* b_step);
GVOTE_API void gvote_host_arena_release(void);

/* Reads the status word of a workspace (synchronises the stream): GVOTE_OK, GVOTE_ERR_TIMEOUT (a bounded
 * device-side wait ran out) or GVOTE_ERR_WORKSPACE_TOO_SMALL (gvote_pack: capacity_rows too small).  The word
 * is only ever set by kernels and STAYS set: every later poll of that workspace reports it again until the
 * caller clears it, with gvote_clear_status (enqueued on the stream) or by zero-filling the first 256 bytes.
 * gvote_compress_host clears the status of its own arena at the start of every call. */
GVOTE_API int32_t gvote_poll_status(void* ws, void* stream);
GVOTE_API int32_t gvote_clear_status(void* ws, void* stream);

/* Diagnostic of the default selection mode (Algorithm 1's TopK step): how many (request, KV head) pairs
 * had to be selected again by the exact route because a row's sampled bracket missed its k-th logit or a
 * candidate list overflowed, since the workspace's status block was last cleared (synchronises the
 * stream).  The result is the same either way; the exact route only costs time.  Negative: an error code. */
GVOTE_API int64_t gvote_exact_heads(void* ws, void* stream);

/* Per-kernel timing for benchmarks.  While enabled, every kernel launch of the library is
 * bracketed by two CUDA events on its stream.  Enabling (or disabling) drops earlier records.
 * gvote_profile_report synchronises the device and writes one text line per kernel,
 * "name launches total_ms", into buf (host, NUL-terminated, truncated to cap); it returns the
 * bytes needed.  Not thread safe against concurrent launches from other threads. */
GVOTE_API void gvote_profile_enable(int32_t on);
GVOTE_API size_t gvote_profile_report(char* buf, size_t cap);

/* Number of kernel launches the library has enqueued in this process (all entry points). */
GVOTE_API int64_t gvote_launch_count(void);

GVOTE_API const char* gvote_status_string(int32_t status);
/* Text of the last CUDA error seen by the calling thread's last failing call ("" if none). */
GVOTE_API const char* gvote_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* GVOTE_H_ */
