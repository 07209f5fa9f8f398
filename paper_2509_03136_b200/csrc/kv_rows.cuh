// Shared by the paged cache (pages.cu) and the attention over bf16 rows (attend_few.cu, attend_many.cu, api_attend.cu): where
// the cached rows of a (request, KV head) lie, the workspace maps and a few helpers of both attention kernels.
#pragma once

#include "common.cuh"
#include "ptx.cuh"

namespace gvote {

constexpr int kMaxHeadDim = 256;        // of a token or a few
constexpr int kMaxHeadDimMany = 128;    // of many tokens
constexpr int kMaxGroup = 128;          // query heads per KV head
constexpr int kNumSms = 148;
// The few-row kernel: entries of a launch (their tiles are added up in shared memory) and groups of query rows.
constexpr int kFewEntries = 1024;
constexpr int kFewGroups = 4;
constexpr int kFewCtas = 2 * kNumSms;
// Behind the status block of a workspace: arrival counters, zero between calls; then the scratch of one call.
constexpr size_t kScratchAt = kStatusBytes + (size_t)kFewGroups * (2 * kFewEntries + kFewCtas) * 4;

// Cached rows, in slabs (K, V [n_kv_heads][total][d_k], request r's rows from cu[r] on) or in pages (K, V
// [n_pages][page_rows][d_k], row j of (r, h) in page tables[r][h][j / page_rows]).
struct RowSource {
  const __nv_bfloat16* K;
  const __nv_bfloat16* V;
  int64_t tok, outer;           // elements between rows; between heads (slabs) or pages
  const int32_t* cu;            // slabs
  const int32_t* kv_len;        // [batch][n_kv_heads]; slabs: or null
  const int32_t* tables;        // pages: [batch][n_kv_heads][max_pages]; null: slabs
  int64_t total;                // slabs
  int32_t n_pages, page_log2, max_pages;
};

struct AttendCall {
  const __nv_bfloat16* Q;
  int64_t q_tok, q_head;
  const int32_t* cu_q;
  int64_t total_q, max_q;
  __nv_bfloat16* out;
  int64_t o_tok, o_head;
  float* lse;                   // or null
  int32_t batch;
  int64_t max_rows;             // a head holds at most
};

struct PageArgs {
  int32_t* tables;
  int32_t* kv_len;
  int32_t* free_pages;
  int32_t* n_free;
  int32_t n_pages, page_log2, max_pages, batch, Hkv;
};

// Scratch of the tables: a refusal mark and the kept new rows of every entry.
struct PageMap { size_t refused, counts, total; };
PageMap page_map(const gvote_params* p, int32_t batch);
size_t attend_few_workspace(const gvote_params* p, int32_t batch, int64_t max_q);
size_t attend_many_workspace(const gvote_params* p, int32_t batch, int64_t total_q, int64_t max_q);
// Whether calls of this size go to the kernel for few query rows.
bool attend_takes_few(const gvote_params* p, int64_t max_q);

int32_t launch_page_tables(const PageArgs& a, const int32_t* keep, const int32_t* cu_new, int64_t total_new, int64_t max_new,
                           const uint32_t* mask, int32_t* slots, const PageMap& m, char* ws, cudaStream_t st);
int32_t launch_page_write(const gvote_params* p, const __nv_bfloat16* K, const __nv_bfloat16* V, int64_t tok, int64_t head,
                          const int32_t* slots, int64_t total_new, __nv_bfloat16* K_out, __nv_bfloat16* V_out, int64_t row_stride,
                          int64_t page_stride, int32_t page_log2, int64_t n_slots, int32_t* status, cudaStream_t st);
int32_t launch_attend_few(const gvote_params* p, const AttendCall& c, const RowSource& s, char* ws, cudaStream_t st);
int32_t launch_attend_many(const gvote_params* p, const AttendCall& c, const RowSource& s, char* ws, cudaStream_t st);

// Tensor maps of K and V, boxes of `rows` rows x 64 channels.
bool row_maps(const gvote_params* p, const RowSource& s, int rows, CUtensorMap* K, CUtensorMap* V);

#ifdef __CUDACC__

// Rows held by KV head h of request r.
__device__ __forceinline__ int rows_held(const RowSource& s, int r, int h, int Hkv) {
  if (s.tables) {
    const int64_t cap = (int64_t)s.max_pages << s.page_log2;
    const int v = s.kv_len[r * Hkv + h];
    return v < 0 ? 0 : (v < cap ? v : (int)cap);
  }
  return valid_keys(s.kv_len, r, Hkv, h, s.cu[r + 1] - s.cu[r]);
}
// Element offset of row j of (r, h), or -1 where its page does not exist.
__device__ __forceinline__ int64_t row_offset(const RowSource& s, int r, int h, int Hkv, int64_t j) {
  if (!s.tables) return (int64_t)h * s.outer + (s.cu[r] + j) * s.tok;
  const int page = s.tables[((int64_t)r * Hkv + h) * s.max_pages + (j >> s.page_log2)];
  if ((uint32_t)page >= (uint32_t)s.n_pages) return -1;
  return (int64_t)page * s.outer + (j & ((1 << s.page_log2) - 1)) * s.tok;
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// What the waits of a CTA look at: whether one of them ran out, and a counter of work done.
struct Watch {
  volatile int stop;
  uint32_t work;
};
__device__ __forceinline__ void count_work(Watch* w) { atomicAdd(&w->work, 1u); }
// Gives up after 2^20 tries (2 s: the hardware lets a try last 2 us) during which no work was done.  So a wait may last as long as
// what it is for, two seconds of a unit of 2^28 rows for instance, as long as whoever is at work counts it at least once in that time.
__device__ __forceinline__ bool wait_or_stop(uint64_t* bar, uint32_t parity, Watch* w) {
  uint32_t seen = 0;
  for (uint32_t i = 0; i < (1u << 20); ++i) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if ((i & 255u) == 255u) {
      if (w->stop) return false;
      const uint32_t now = *reinterpret_cast<volatile uint32_t*>(&w->work);
      if (now != seen) { seen = now; i = 0; }
    }
  }
  w->stop = 1;
  return false;
}
// Before a producer leaves early: the loads of a ring that may still write to this CTA's memory.
__device__ __forceinline__ void await_loads(uint64_t* full, int slots, uint32_t issued) {
  for (uint32_t i = issued > (uint32_t)slots ? issued - slots : 0; i < issued; ++i)
    for (int k = 0; k < (1 << 12) && !ptx::mbar_try_wait(&full[i % slots], (i / slots) & 1); ++k) {}
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ bool any_not_finite(uint32_t w) {            // of a pair of bf16 values
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t finite_only(uint32_t w) {           // what is not finite becomes 0
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}
__device__ __forceinline__ float not_finite_only(float x) { return isfinite(x) ? 0.f : x; }
// A partial result times its factor; what is not finite stays, though the factor be zero.
__device__ __forceinline__ float scaled(float x, float f) { return isfinite(x) ? x * f : x; }

#endif  // __CUDACC__

}  // namespace gvote
