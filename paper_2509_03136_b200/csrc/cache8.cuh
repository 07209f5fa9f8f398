// Shared by the kernels of the 8-bit cache and of the eviction (store8.cu, append8.cu, attend8.cu,
// accumulate.cu, evict.cu, api_cache.cu): the workspace maps, lookups on the ragged layout and the
// conversion to and from e4m3 with a power-of-two scale.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace gvote {

constexpr int kBlock8 = GVOTE_CACHE8_BLOCK;   // rows that share a scale
constexpr int kMaxHeadDim8 = 256;
constexpr int kMaxGroup8 = 128;               // query heads per KV head

// Scratch of one call behind the status block; the maps of the entry points overlap, since nothing outlives a call.
struct StoreMap { size_t list, note, total; };
struct AttendMap { size_t o, ml, info, lse, logits, total; };
struct AccumulateMap { size_t lse, part, total; int64_t q_tiles, key_chunks, q_chunks; int tpt; };

StoreMap store8_map(const gvote_params* p, int32_t batch, int64_t total_tokens);
AttendMap attend8_map(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t total_q, int64_t max_q);
AccumulateMap accumulate_map(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N, int64_t total_q,
                             int64_t max_q);
// Sizes that suffice for a call of these sizes and for every smaller one.
size_t attend8_workspace(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t total_q, int64_t max_q);
size_t accumulate_workspace(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t total_q);

struct SideArrays {            // per-slot arrays that move with the rows
  const float* acc;
  float* acc_out;
  const int32_t* pos;
  int32_t* pos_out;
};

int32_t launch_store8(const gvote_params* p, const __nv_bfloat16* K, const __nv_bfloat16* V, int64_t tok, int64_t head,
                      const gvote_cache8* src8, const uint32_t* mask, const int32_t* cu, const int32_t* kv_len,
                      int32_t batch, int64_t total_tokens, int64_t max_N, const gvote_cache8* dst,
                      const SideArrays& side, char* ws, cudaStream_t st);
int32_t launch_append8(const gvote_params* p, const __nv_bfloat16* K, const __nv_bfloat16* V, int64_t tok, int64_t head,
                       const int32_t* cu_new, int64_t max_new, const gvote_cache8* c, int32_t* kv_len_out, float* acc,
                       int32_t* token_pos, const int32_t* pos_new, char* ws, cudaStream_t st);
int32_t launch_attend8(const gvote_params* p, const __nv_bfloat16* Q, int64_t q_tok, int64_t q_head, const int32_t* cu_q,
                       int64_t total_q, int64_t max_q, const gvote_cache8* c, __nv_bfloat16* out, int64_t o_tok,
                       int64_t o_head, float* lse, const float* acc, float* acc_out, char* ws, cudaStream_t st);
int32_t launch_accumulate(const gvote_params* p, const __nv_bfloat16* Q, int64_t q_tok, int64_t q_head,
                          const int32_t* cu_q, int64_t total_q, int64_t max_q, const __nv_bfloat16* K, int64_t k_tok,
                          int64_t k_head, const int32_t* cu, const int32_t* kv_len, int32_t batch, int64_t total_tokens,
                          int64_t max_N, const float* lse, const float* acc, float* acc_out, char* ws, cudaStream_t st);
int32_t launch_evict(const gvote_params* p, const float* acc, const int32_t* cu, const int32_t* kv_len, int32_t batch,
                     int64_t total_tokens, int64_t max_N, const int32_t* keep, int32_t n_recent, uint32_t* mask,
                     int32_t* budget, cudaStream_t st);

#ifdef __CUDACC__

__device__ __forceinline__ int64_t block8_offset(int cu_r, int r) { return (int64_t)(cu_r >> 6) + r; }

// The request that owns entry `g` of a list with (cu[r] >> shift) + r as the first entry of request r
// (one entry per 2^shift tokens begun, over-allocated by at most one per request).
__device__ __forceinline__ int find_request_by(const int32_t* __restrict__ cu, int batch, int64_t g, int shift) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)(cu[mid] >> shift) + mid <= g) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// The smallest 2^e, e >= -126, with amax <= 448 * 2^e (448 = 1.75 * 2^8, the largest e4m3 value); amax finite, >= 0.
__device__ __forceinline__ float scale8_of(float amax) {
  if (amax <= 448.f * 1.17549435e-38f) return 1.17549435e-38f;
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);   // biased exponent of the scale
  return __uint_as_float((uint32_t)max(e, 1) << 23);
}
__device__ __forceinline__ float inverse_pow2(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// |x| where it counts for the scale: a NaN or an infinity does not.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.402823466e38f ? a : 0.f;
}
// Two values already divided by their scale -> two codes (low byte: a); not finite -> the NaN code.
__device__ __forceinline__ uint32_t encode8x2(float a, float b) {
  uint32_t c = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  if (!(fabsf(a) <= 3.402823466e38f)) c |= 0x7fu;
  if (!(fabsf(b) <= 3.402823466e38f)) c |= 0x7f00u;
  return c;
}
__device__ __forceinline__ float2 decode8x2(uint32_t c) {       // low 16 bits: two codes
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c, __NV_E4M3);
  return __half22float2(__half2(h));
}
// Four e4m3 codes -> two pairs of halves (exact; the NaN code -> NaN).
__device__ __forceinline__ void widen8x4(uint32_t c, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(c));
}
// Two pairs of halves -> four e4m3 codes (nearest, ties to even; beyond 448: 448; NaN: the NaN code).
__device__ __forceinline__ uint32_t narrow8x4(uint32_t lo, uint32_t hi) {
  uint32_t c;
  asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f16x2 l, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 h, %2;\n\tmov.b32 %0, {l, h};\n\t}"
      : "=r"(c)
      : "r"(lo), "r"(hi));
  return c;
}
// The same of four floats.
__device__ __forceinline__ uint32_t narrow8x4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}

#endif  // __CUDACC__

}  // namespace gvote
