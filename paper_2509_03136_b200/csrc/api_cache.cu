// C-ABI entry points of the 8-bit cache and of the eviction (declared in include/gvote.h): argument checks and
// the workspace size; the kernels are in store8.cu, append8.cu, attend8.cu, accumulate.cu and evict.cu.
#include "cache8.cuh"

namespace gvote {
namespace {

int32_t validate_shape(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N) {
  PROPAGATE(validate_params(p));
  PROPAGATE(validate_batch(batch, total_tokens, max_N));
  if (p->d_k % 16 != 0 || p->d_k > kMaxHeadDim8 || p->n_q_heads / p->n_kv_heads > kMaxGroup8) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  // grids: requests on y or z, blocks of every head on x
  if (batch > 65535 || p->n_kv_heads > 1024) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  if (((total_tokens >> 6) + batch) * (int64_t)p->n_kv_heads > 0x3fffffffLL) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  return GVOTE_OK;
}

int32_t validate_queries(const gvote_params* p, int64_t total_q, int64_t max_q) {
  if (total_q < 0 || max_q < 0 || max_q > total_q) return GVOTE_ERR_INVALID_ARG;
  if (total_q > (int64_t)1 << 30 || ((total_q * (p->n_q_heads / p->n_kv_heads) >> 6) + 1) * p->n_kv_heads > 0x3fffffffLL) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  return GVOTE_OK;
}

int32_t validate_cache(const gvote_params* p, const gvote_cache8* c) {
  if (!c) return GVOTE_ERR_INVALID_ARG;
  PROPAGATE(validate_shape(p, c->batch, c->total_tokens, c->max_N));
  REQUIRE_PTR(c->K); REQUIRE_PTR(c->V); REQUIRE_PTR(c->k_scale); REQUIRE_PTR(c->v_scale);
  REQUIRE_PTR(c->cu_seqlens); REQUIRE_PTR(c->kv_len);
  if (c->tok_stride < p->d_k || c->tok_stride % 16 != 0 || c->head_stride % 16 != 0) return GVOTE_ERR_UNALIGNED;
  return GVOTE_OK;
}

bool rows_aligned(int64_t tok, int64_t head, int d_k) { return tok >= d_k && tok % 8 == 0 && head % 8 == 0; }

// Where `heads` x `rows` pieces of `width` bytes lie, at these strides in bytes.
struct Extent {
  int64_t at, head, tok, heads, rows, width;
  int64_t lo() const { return at + (head < 0 ? (heads - 1) * head : 0); }
  int64_t hi() const { return at + (head > 0 ? (heads - 1) * head : 0) + (rows - 1) * tok + width; }
};
Extent extent(const void* p, int64_t heads, int64_t head, int64_t rows, int64_t tok, int64_t width) {
  return {(int64_t)reinterpret_cast<uintptr_t>(p), heads > 1 ? head : 0, tok, heads, rows, width};
}
Extent whole(const void* p, int64_t bytes) { return extent(p, 1, 0, 1, 0, bytes); }

// Whether two arrays share a byte.  Rows of the same strides may lie between each other (windows of one wider buffer): for
// every distance between heads, the row of b nearest to the start of a row of a, and the one before it, are looked at.  Where
// the strides differ a common extent counts as shared.
bool overlap(const Extent& a, const Extent& b) {
  if (!a.at || !b.at || a.heads < 1 || b.heads < 1 || a.rows < 1 || b.rows < 1 || a.width < 1 || b.width < 1) return false;
  if (a.hi() <= b.lo() || b.hi() <= a.lo()) return false;
  const int64_t tok = a.rows > 1 ? a.tok : b.rows > 1 ? b.tok : a.width;
  if (a.head != b.head || (b.rows > 1 && tok != b.tok) || a.heads != b.heads || a.width != b.width || tok < 1) return true;
  for (int64_t dh = 1 - a.heads; dh < a.heads; ++dh) {
    const int64_t apart = b.at - a.at + dh * a.head;                   // plus a multiple of tok: between 1 - a.rows and b.rows - 1 rows
    const int64_t down = apart >= 0 ? -(apart / tok) : (-apart + tok - 1) / tok;
    for (int64_t dt = down - 1; dt <= down; ++dt) {
      const int64_t off = apart + dt * tok;
      if (dt > -a.rows && dt < b.rows && off < a.width && -off < a.width) return true;
    }
  }
  return false;
}

Extent codes_of(const gvote_params* p, const gvote_cache8* c, const void* t) {
  return extent(t, p->n_kv_heads, c->head_stride, c->total_tokens, c->tok_stride, p->d_k);
}
Extent scales_of(const gvote_params* p, const gvote_cache8* c, const void* t) {
  return whole(t, 4 * (int64_t)p->n_kv_heads * gvote_cache8_row_blocks(c->total_tokens, c->batch));
}
Extent lens_of(const gvote_params* p, int32_t batch, const void* t) { return whole(t, 4 * (int64_t)batch * p->n_kv_heads); }
Extent slots_of(const gvote_params* p, int64_t total, const void* t) { return whole(t, 4 * (int64_t)p->n_kv_heads * total); }

// What a call reads of K and V (the same strides) must not lie in the codes it writes.
bool codes_overlap(const gvote_params* p, const Extent& K, const Extent& V, const gvote_cache8* dst) {
  const Extent a = codes_of(p, dst, dst->K), b = codes_of(p, dst, dst->V);
  return overlap(K, a) || overlap(K, b) || overlap(V, a) || overlap(V, b);
}

int64_t larger(int64_t a, int64_t b) { return a > b ? a : b; }

size_t cache_workspace(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t total_q, int64_t max_q) {
  size_t n = store8_map(p, batch, total_tokens).total;
  const size_t a = attend8_workspace(p, batch, total_tokens, total_q, max_q);
  const size_t b = max_q > 0 ? accumulate_workspace(p, batch, total_tokens, total_q) : 0;
  if (a > n) n = a;
  return b > n ? b : n;
}

}  // namespace
}  // namespace gvote

using namespace gvote;

extern "C" {

size_t gvote_cache_workspace_bytes(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N,
                                   int64_t total_q, int64_t max_q) {
  if (validate_shape(p, batch, total_tokens, max_N) != GVOTE_OK || validate_queries(p, total_q, max_q) != GVOTE_OK) return 0;
  return cache_workspace(p, batch, total_tokens, total_q, max_q);
}

int32_t gvote_store8(const gvote_params* p, const void* K, const void* V, int64_t tok_stride, int64_t head_stride,
                     const uint32_t* mask_or_null, const int32_t* cu_seqlens, const int32_t* kv_len_or_null,
                     int32_t batch, int64_t total_tokens, int64_t max_N, const gvote_cache8* cache,
                     const float* acc_or_null, float* acc_out_or_null, const int32_t* token_pos_or_null,
                     int32_t* token_pos_out_or_null, void* ws, size_t ws_bytes, void* stream) {
  PROPAGATE(validate_shape(p, batch, total_tokens, max_N));
  PROPAGATE(validate_cache(p, cache));
  if (cache->batch != batch) return GVOTE_ERR_INVALID_ARG;
  REQUIRE_PTR(K); REQUIRE_PTR(V); REQUIRE_PTR(cu_seqlens); REQUIRE_PTR(ws);
  OPTIONAL_PTR(mask_or_null); OPTIONAL_PTR(kv_len_or_null); OPTIONAL_PTR(acc_or_null); OPTIONAL_PTR(acc_out_or_null);
  OPTIONAL_PTR(token_pos_or_null); OPTIONAL_PTR(token_pos_out_or_null);
  if (!acc_or_null != !acc_out_or_null || (token_pos_or_null && !token_pos_out_or_null)) return GVOTE_ERR_INVALID_ARG;
  if (!rows_aligned(tok_stride, head_stride, p->d_k)) return GVOTE_ERR_UNALIGNED;
  if (overlap(slots_of(p, total_tokens, acc_or_null), slots_of(p, cache->total_tokens, acc_out_or_null)) ||
      overlap(slots_of(p, total_tokens, token_pos_or_null), slots_of(p, cache->total_tokens, token_pos_out_or_null)) ||
      overlap(lens_of(p, batch, kv_len_or_null), lens_of(p, batch, cache->kv_len))) return GVOTE_ERR_INVALID_ARG;
  if (codes_overlap(p, extent(K, p->n_kv_heads, 2 * head_stride, total_tokens, 2 * tok_stride, 2 * p->d_k),
                    extent(V, p->n_kv_heads, 2 * head_stride, total_tokens, 2 * tok_stride, 2 * p->d_k), cache)) return GVOTE_ERR_INVALID_ARG;
  if (ws_bytes < store8_map(p, batch, larger(total_tokens, cache->total_tokens)).total) return GVOTE_ERR_WORKSPACE_TOO_SMALL;
  const SideArrays side{acc_or_null, acc_out_or_null, token_pos_or_null, token_pos_out_or_null};
  return launch_store8(p, (const __nv_bfloat16*)K, (const __nv_bfloat16*)V, tok_stride, head_stride, nullptr, mask_or_null,
                       cu_seqlens, kv_len_or_null, batch, total_tokens, max_N, cache, side, (char*)ws, (cudaStream_t)stream);
}

int32_t gvote_prune8(const gvote_params* p, const gvote_cache8* src, const uint32_t* mask_or_null,
                     const gvote_cache8* dst, const float* acc_or_null, float* acc_out_or_null,
                     const int32_t* token_pos_or_null, int32_t* token_pos_out_or_null, void* ws, size_t ws_bytes,
                     void* stream) {
  PROPAGATE(validate_cache(p, src));
  PROPAGATE(validate_cache(p, dst));
  if (src->batch != dst->batch) return GVOTE_ERR_INVALID_ARG;
  if (codes_overlap(p, codes_of(p, src, src->K), codes_of(p, src, src->V), dst)) return GVOTE_ERR_INVALID_ARG;
  for (const void* s : {src->k_scale, src->v_scale})
    for (const void* d : {dst->k_scale, dst->v_scale})
      if (overlap(scales_of(p, src, s), scales_of(p, dst, d))) return GVOTE_ERR_INVALID_ARG;
  if (overlap(lens_of(p, src->batch, src->kv_len), lens_of(p, dst->batch, dst->kv_len))) return GVOTE_ERR_INVALID_ARG;
  REQUIRE_PTR(ws); OPTIONAL_PTR(mask_or_null); OPTIONAL_PTR(acc_or_null); OPTIONAL_PTR(acc_out_or_null);
  OPTIONAL_PTR(token_pos_or_null); OPTIONAL_PTR(token_pos_out_or_null);
  if (!acc_or_null != !acc_out_or_null || (token_pos_or_null && !token_pos_out_or_null)) return GVOTE_ERR_INVALID_ARG;
  if (overlap(slots_of(p, src->total_tokens, acc_or_null), slots_of(p, dst->total_tokens, acc_out_or_null)) ||
      overlap(slots_of(p, src->total_tokens, token_pos_or_null), slots_of(p, dst->total_tokens, token_pos_out_or_null)))
    return GVOTE_ERR_INVALID_ARG;
  if (ws_bytes < store8_map(p, src->batch, larger(src->total_tokens, dst->total_tokens)).total) return GVOTE_ERR_WORKSPACE_TOO_SMALL;
  const SideArrays side{acc_or_null, acc_out_or_null, token_pos_or_null, token_pos_out_or_null};
  return launch_store8(p, nullptr, nullptr, src->tok_stride, src->head_stride, src, mask_or_null, src->cu_seqlens,
                       src->kv_len, src->batch, src->total_tokens, src->max_N, dst, side, (char*)ws, (cudaStream_t)stream);
}

int32_t gvote_append8(const gvote_params* p, const void* K_new, const void* V_new, int64_t tok_stride,
                      int64_t head_stride, const int32_t* cu_new, int64_t total_new, int64_t max_new,
                      const gvote_cache8* cache, int32_t* kv_len_out, float* acc_or_null, int32_t* token_pos_or_null,
                      const int32_t* pos_new_or_null, void* ws, size_t ws_bytes, void* stream) {
  PROPAGATE(validate_params(p));
  PROPAGATE(validate_cache(p, cache));
  if (total_new < 0 || max_new < 0 || max_new > total_new) return GVOTE_ERR_INVALID_ARG;
  if (total_new > (int64_t)1 << 30) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  if (total_new > 0) {
    REQUIRE_PTR(K_new); REQUIRE_PTR(V_new);
    if (!rows_aligned(tok_stride, head_stride, p->d_k)) return GVOTE_ERR_UNALIGNED;
  }
  REQUIRE_PTR(cu_new); REQUIRE_PTR(kv_len_out); REQUIRE_PTR(ws);
  OPTIONAL_PTR(acc_or_null); OPTIONAL_PTR(token_pos_or_null); OPTIONAL_PTR(pos_new_or_null);
  if (total_new > 0 && !token_pos_or_null != !pos_new_or_null) return GVOTE_ERR_INVALID_ARG;
  if (ws_bytes < kStatusBytes) return GVOTE_ERR_WORKSPACE_TOO_SMALL;
  return launch_append8(p, (const __nv_bfloat16*)K_new, (const __nv_bfloat16*)V_new, tok_stride, head_stride, cu_new,
                        max_new, cache, kv_len_out, acc_or_null, token_pos_or_null, pos_new_or_null, (char*)ws,
                        (cudaStream_t)stream);
}

int32_t gvote_attend8(const gvote_params* p, const void* Q, int64_t q_tok_stride, int64_t q_head_stride,
                      const int32_t* cu_q, int64_t total_q, int64_t max_q, const gvote_cache8* cache, void* out,
                      int64_t out_tok_stride, int64_t out_head_stride, float* lse_or_null, const float* acc_or_null,
                      float* acc_out_or_null, void* ws, size_t ws_bytes, void* stream) {
  PROPAGATE(validate_params(p));
  PROPAGATE(validate_cache(p, cache));
  PROPAGATE(validate_queries(p, total_q, max_q));
  if (max_q < 1) return GVOTE_ERR_INVALID_ARG;
  if (max_q > GVOTE_ATTEND8_MAX_Q) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  REQUIRE_PTR(Q); REQUIRE_PTR(cu_q); REQUIRE_PTR(out); REQUIRE_PTR(ws);
  OPTIONAL_PTR(lse_or_null); OPTIONAL_PTR(acc_or_null); OPTIONAL_PTR(acc_out_or_null);
  if (acc_or_null && !acc_out_or_null) return GVOTE_ERR_INVALID_ARG;
  if (q_head_stride < p->d_k || q_head_stride % 8 != 0 || q_tok_stride % 8 != 0) return GVOTE_ERR_UNALIGNED;
  if (out_head_stride < p->d_k || out_head_stride % 8 != 0 || out_tok_stride % 8 != 0) return GVOTE_ERR_UNALIGNED;
  const AttendMap m = attend8_map(p, cache->batch, cache->total_tokens, total_q, max_q);
  if (ws_bytes < (acc_out_or_null ? m.total : m.logits)) return GVOTE_ERR_WORKSPACE_TOO_SMALL;   // (the logits lie last)
  return launch_attend8(p, (const __nv_bfloat16*)Q, q_tok_stride, q_head_stride, cu_q, total_q, max_q, cache,
                        (__nv_bfloat16*)out, out_tok_stride, out_head_stride, lse_or_null, acc_or_null, acc_out_or_null,
                        (char*)ws, (cudaStream_t)stream);
}

int32_t gvote_accumulate(const gvote_params* p, const void* Q, int64_t q_tok_stride, int64_t q_head_stride,
                         const int32_t* cu_q, int64_t total_q, int64_t max_q, const void* K, int64_t k_tok_stride,
                         int64_t k_head_stride, const int32_t* cu_seqlens, const int32_t* kv_len_or_null, int32_t batch,
                         int64_t total_tokens, int64_t max_N, const float* lse_or_null, const float* acc_or_null,
                         float* acc_out, void* ws, size_t ws_bytes, void* stream) {
  PROPAGATE(validate_shape(p, batch, total_tokens, max_N));
  PROPAGATE(validate_queries(p, total_q, max_q));
  if (max_q < 1) return GVOTE_ERR_INVALID_ARG;
  REQUIRE_PTR(Q); REQUIRE_PTR(cu_q); REQUIRE_PTR(K); REQUIRE_PTR(cu_seqlens); REQUIRE_PTR(acc_out); REQUIRE_PTR(ws);
  OPTIONAL_PTR(kv_len_or_null); OPTIONAL_PTR(lse_or_null); OPTIONAL_PTR(acc_or_null);
  if (q_head_stride < p->d_k || q_head_stride % 8 != 0 || q_tok_stride % 8 != 0) return GVOTE_ERR_UNALIGNED;
  if (!rows_aligned(k_tok_stride, k_head_stride, p->d_k)) return GVOTE_ERR_UNALIGNED;
  if (ws_bytes < accumulate_map(p, batch, total_tokens, max_N, total_q, max_q).total) return GVOTE_ERR_WORKSPACE_TOO_SMALL;
  return launch_accumulate(p, (const __nv_bfloat16*)Q, q_tok_stride, q_head_stride, cu_q, total_q, max_q,
                           (const __nv_bfloat16*)K, k_tok_stride, k_head_stride, cu_seqlens, kv_len_or_null, batch,
                           total_tokens, max_N, lse_or_null, acc_or_null, acc_out, (char*)ws, (cudaStream_t)stream);
}

int32_t gvote_evict(const gvote_params* p, const float* acc, const int32_t* cu_seqlens, const int32_t* kv_len_or_null,
                    int32_t batch, int64_t total_tokens, int64_t max_N, const int32_t* keep, int32_t n_recent,
                    uint32_t* mask, int32_t* budget, void* ws, size_t ws_bytes, void* stream) {
  PROPAGATE(validate_shape(p, batch, total_tokens, max_N));
  REQUIRE_PTR(acc); REQUIRE_PTR(cu_seqlens); OPTIONAL_PTR(kv_len_or_null); REQUIRE_PTR(keep); REQUIRE_PTR(mask);
  REQUIRE_PTR(budget); REQUIRE_PTR(ws);
  if (n_recent < 0) return GVOTE_ERR_INVALID_ARG;
  if (ws_bytes < kStatusBytes) return GVOTE_ERR_WORKSPACE_TOO_SMALL;
  return launch_evict(p, acc, cu_seqlens, kv_len_or_null, batch, total_tokens, max_N, keep, n_recent, mask, budget,
                      (cudaStream_t)stream);
}

}  // extern "C"
