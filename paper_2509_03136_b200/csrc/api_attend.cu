// C-ABI entry points of the paged cache and of the attention over bf16 rows (declared in include/gvote.h): argument checks and
// the workspace size; the kernels are in pages.cu, attend_few.cu and attend_many.cu.
#include "kv_rows.cuh"

namespace gvote {
namespace {

int32_t validate_heads(const gvote_params* p) {
  PROPAGATE(validate_params(p));
  if (p->d_k % 16 != 0 || p->d_k > kMaxHeadDim || p->n_q_heads / p->n_kv_heads > kMaxGroup || p->n_kv_heads > kFewEntries)
    return GVOTE_ERR_UNSUPPORTED_SHAPE;
  return GVOTE_OK;
}

int32_t validate_queries(const gvote_params* p, int32_t batch, int64_t total_q, int64_t max_q) {
  if (batch < 1 || total_q < 0 || max_q < 0 || max_q > total_q) return GVOTE_ERR_INVALID_ARG;
  if (batch > 65535 || total_q > (int64_t)1 << 30) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  if (((total_q * (p->n_q_heads / p->n_kv_heads) >> 6) + batch) * p->n_kv_heads > 0x3fffffffLL) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  if (p->d_k > kMaxHeadDimMany && max_q > GVOTE_ATTEND_FEW_Q) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  return GVOTE_OK;
}

// The stride of a dimension of n rows or heads (of one only it may be anything).
int32_t validate_stride(const gvote_params* p, int64_t stride, int64_t n) {
  if (n <= 1) return GVOTE_OK;
  if (stride < p->d_k || stride % 8 != 0) return GVOTE_ERR_UNALIGNED;
  return stride >= (int64_t)1 << 38 ? GVOTE_ERR_UNSUPPORTED_SHAPE : GVOTE_OK;
}

int32_t validate_pages(const gvote_params* p, const gvote_pages* g) {
  PROPAGATE(validate_heads(p));
  if (!g) return GVOTE_ERR_INVALID_ARG;
  REQUIRE_PTR(g->K); REQUIRE_PTR(g->V); REQUIRE_PTR(g->tables); REQUIRE_PTR(g->kv_len);
  if (g->batch < 1 || g->n_pages < 1 || g->max_pages < 1) return GVOTE_ERR_INVALID_ARG;
  if (g->page_rows < 16 || g->page_rows > 1024 || (g->page_rows & (g->page_rows - 1)) != 0) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  if (g->batch > 65535 || (int64_t)g->n_pages * g->page_rows > 0x7fffffffLL ||
      (int64_t)g->max_pages * g->page_rows > (int64_t)1 << 26) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  PROPAGATE(validate_stride(p, g->row_stride, g->page_rows));
  return validate_stride(p, g->page_stride, g->n_pages);
}

int32_t log2_of(int32_t x) { int32_t n = 0; while ((1 << n) < x) ++n; return n; }

// Checks of what both attention calls share, and the call.
int32_t attend(const gvote_params* p, const AttendCall& c, const RowSource& s, void* ws, size_t ws_bytes, void* stream) {
  if (c.total_q == 0) return GVOTE_OK;
  if (c.max_q < 1) return GVOTE_ERR_INVALID_ARG;
  REQUIRE_PTR(c.Q); REQUIRE_PTR(c.cu_q); REQUIRE_PTR(c.out); REQUIRE_PTR(ws); OPTIONAL_PTR(c.lse);
  PROPAGATE(validate_stride(p, c.q_head, p->n_q_heads)); PROPAGATE(validate_stride(p, c.q_tok, c.total_q));
  PROPAGATE(validate_stride(p, c.o_head, p->n_q_heads)); PROPAGATE(validate_stride(p, c.o_tok, c.total_q));
  if (ws_bytes < gvote_attend_workspace_bytes(p, c.batch, c.total_q, c.max_q)) return GVOTE_ERR_WORKSPACE_TOO_SMALL;
  return attend_takes_few(p, c.max_q) ? launch_attend_few(p, c, s, (char*)ws, (cudaStream_t)stream)
                                      : launch_attend_many(p, c, s, (char*)ws, (cudaStream_t)stream);
}

}  // namespace
}  // namespace gvote

using namespace gvote;

extern "C" {

size_t gvote_attend_workspace_bytes(const gvote_params* p, int32_t batch, int64_t total_q, int64_t max_q) {
  if (validate_heads(p) != GVOTE_OK || validate_queries(p, batch, total_q, max_q) != GVOTE_OK) return 0;
  size_t n = page_map(p, batch).total;
  const size_t a = attend_few_workspace(p, batch, max_q), b = attend_many_workspace(p, batch, total_q, max_q);
  if (a > n) n = a;
  return b > n ? b : n;
}

int32_t gvote_page_tables(const gvote_params* p, const gvote_pages* pages, const int32_t* keep_or_null,
                          const int32_t* cu_new_or_null, int64_t total_new, int64_t max_new, const uint32_t* mask_or_null,
                          int32_t* slots_or_null, void* ws, size_t ws_bytes, void* stream) {
  PROPAGATE(validate_pages(p, pages));
  REQUIRE_PTR(pages->free_pages); REQUIRE_PTR(pages->n_free); REQUIRE_PTR(ws);
  OPTIONAL_PTR(keep_or_null); OPTIONAL_PTR(cu_new_or_null); OPTIONAL_PTR(mask_or_null); OPTIONAL_PTR(slots_or_null);
  if (total_new < 0 || max_new < 0 || max_new > total_new) return GVOTE_ERR_INVALID_ARG;
  if (!cu_new_or_null && (total_new > 0 || mask_or_null || slots_or_null)) return GVOTE_ERR_INVALID_ARG;
  if (total_new > (int64_t)1 << 30) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  const PageMap m = page_map(p, pages->batch);
  if (ws_bytes < m.total) return GVOTE_ERR_WORKSPACE_TOO_SMALL;
  const PageArgs a{pages->tables, pages->kv_len, pages->free_pages, pages->n_free, pages->n_pages, log2_of(pages->page_rows),
                   pages->max_pages, pages->batch, p->n_kv_heads};
  return launch_page_tables(a, keep_or_null, cu_new_or_null, total_new, max_new, mask_or_null, slots_or_null, m, (char*)ws,
                            (cudaStream_t)stream);
}

int32_t gvote_page_write(const gvote_params* p, const void* K_new, const void* V_new, int64_t tok_stride, int64_t head_stride,
                         const int32_t* slots, int64_t total_new, const gvote_pages* pages, void* ws, size_t ws_bytes, void* stream) {
  PROPAGATE(validate_pages(p, pages));
  if (total_new < 0) return GVOTE_ERR_INVALID_ARG;
  if (total_new > (int64_t)1 << 30) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  REQUIRE_PTR(ws);
  if (ws_bytes < kStatusBytes) return GVOTE_ERR_WORKSPACE_TOO_SMALL;
  if (total_new == 0) return GVOTE_OK;
  REQUIRE_PTR(K_new); REQUIRE_PTR(V_new); REQUIRE_PTR(slots);
  PROPAGATE(validate_stride(p, tok_stride, total_new)); PROPAGATE(validate_stride(p, head_stride, p->n_kv_heads));
  return launch_page_write(p, (const __nv_bfloat16*)K_new, (const __nv_bfloat16*)V_new, tok_stride, head_stride, slots, total_new,
                           (__nv_bfloat16*)pages->K, (__nv_bfloat16*)pages->V, pages->row_stride, pages->page_stride,
                           log2_of(pages->page_rows), (int64_t)pages->n_pages * pages->page_rows, (int32_t*)ws,
                           (cudaStream_t)stream);
}

int32_t gvote_page_attend(const gvote_params* p, const void* Q, int64_t q_tok_stride, int64_t q_head_stride, const int32_t* cu_q,
                          int64_t total_q, int64_t max_q, const gvote_pages* pages, void* out, int64_t out_tok_stride,
                          int64_t out_head_stride, float* lse_or_null, void* ws, size_t ws_bytes, void* stream) {
  PROPAGATE(validate_pages(p, pages));
  PROPAGATE(validate_queries(p, pages->batch, total_q, max_q));
  RowSource s = {};
  s.K = (const __nv_bfloat16*)pages->K; s.V = (const __nv_bfloat16*)pages->V;
  s.tok = pages->row_stride; s.outer = pages->page_stride;
  s.kv_len = pages->kv_len; s.tables = pages->tables;
  s.n_pages = pages->n_pages; s.page_log2 = log2_of(pages->page_rows); s.max_pages = pages->max_pages;
  const AttendCall c{(const __nv_bfloat16*)Q, q_tok_stride, q_head_stride, cu_q, total_q, max_q, (__nv_bfloat16*)out, out_tok_stride,
                     out_head_stride, lse_or_null, pages->batch, (int64_t)pages->max_pages * pages->page_rows};
  return attend(p, c, s, ws, ws_bytes, stream);
}

int32_t gvote_attend(const gvote_params* p, const void* Q, int64_t q_tok_stride, int64_t q_head_stride, const int32_t* cu_q,
                     int64_t total_q, int64_t max_q, const void* K, const void* V, int64_t tok_stride, int64_t head_stride,
                     const int32_t* cu_seqlens, const int32_t* kv_len_or_null, int32_t batch, int64_t total_tokens, int64_t max_N,
                     void* out, int64_t out_tok_stride, int64_t out_head_stride, float* lse_or_null, void* ws, size_t ws_bytes,
                     void* stream) {
  PROPAGATE(validate_heads(p));
  PROPAGATE(validate_batch(batch, total_tokens, max_N));
  PROPAGATE(validate_queries(p, batch, total_q, max_q));
  if (((total_tokens >> 6) + 2 * (int64_t)batch) * p->n_kv_heads > 0x3fffffffLL) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  REQUIRE_PTR(cu_seqlens); OPTIONAL_PTR(kv_len_or_null);
  if (total_tokens > 0) {
    REQUIRE_PTR(K); REQUIRE_PTR(V);
    PROPAGATE(validate_stride(p, tok_stride, total_tokens)); PROPAGATE(validate_stride(p, head_stride, p->n_kv_heads));
  } else {
    K = V = Q;                                                     // (nothing is read of them)
    tok_stride = head_stride = p->d_k;
  }
  RowSource s = {};
  s.K = (const __nv_bfloat16*)K; s.V = (const __nv_bfloat16*)V;
  s.tok = tok_stride; s.outer = head_stride;
  s.cu = cu_seqlens; s.kv_len = kv_len_or_null; s.total = total_tokens;
  const AttendCall c{(const __nv_bfloat16*)Q, q_tok_stride, q_head_stride, cu_q, total_q, max_q, (__nv_bfloat16*)out, out_tok_stride,
                     out_head_stride, lse_or_null, batch, max_N};
  return attend(p, c, s, ws, ws_bytes, stream);
}

}  // extern "C"
