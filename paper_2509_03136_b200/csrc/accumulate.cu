// Attention weight each cached key collects from a prompt's queries (gvote_accumulate):
//   acc[h][n] += sum over query tokens i and query heads g of KV head h of exp(q_ig.k_n / sqrt(d_k) - lse_ig).
//
// Two passes over the causal part of Q K^T, which never reaches memory: the first leaves every query row's
// log-sum-exp, the second lets a thread own a key and sum its weights over the query rows (no atomics, one order).
#include "cache8.cuh"

namespace gvote {
namespace {

constexpr int kAccThreads = 256;
constexpr int kAccRows = 8;

struct AccArgs {
  const __nv_bfloat16* Q;
  int64_t q_tok, q_head;
  const int32_t* cu_q;
  const __nv_bfloat16* K;
  int64_t k_tok, k_head, total;
  const int32_t* cu;
  const int32_t* kv_len;
  float* lse;
  const float* acc;
  float* acc_out;
  int Hkv, G, d_k;
  float scale;
};

__device__ __forceinline__ void load_rows(const AccArgs& a, int h, int q0, int row0, int rows, float (*q_sm)[kMaxHeadDim8]) {
  for (int i = threadIdx.x; i < kAccRows * a.d_k; i += kAccThreads) {
    const int j = i / a.d_k, d = i - j * a.d_k;
    float v = 0.f;
    if (row0 + j < rows) {
      const int token = (row0 + j) / a.G, g = (row0 + j) % a.G;
      v = __bfloat162float(a.Q[(int64_t)(q0 + token) * a.q_tok + (int64_t)(h * a.G + g) * a.q_head + d]);
    }
    q_sm[j][d] = v;
  }
}
__device__ __forceinline__ void dots(const AccArgs& a, const __nv_bfloat16* kp, const float (*q_sm)[kMaxHeadDim8], float* l) {
#pragma unroll
  for (int j = 0; j < kAccRows; ++j) l[j] = 0.f;
  for (int u = 0; u < a.d_k / 8; ++u) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(kp) + u);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t w = (&v.x)[e];
      const float x = __uint_as_float(w << 16), y = __uint_as_float(w & 0xffff0000u);
#pragma unroll
      for (int j = 0; j < kAccRows; ++j)
        l[j] = fmaf(q_sm[j][u * 8 + 2 * e], x, fmaf(q_sm[j][u * 8 + 2 * e + 1], y, l[j]));
    }
  }
}

__global__ void __launch_bounds__(kAccThreads)
accumulate_lse_kernel(const __grid_constant__ AccArgs a) {
  __shared__ float q_sm[kAccRows][kMaxHeadDim8];
  __shared__ float red[2][kAccRows][kAccThreads / 32];
  const int h = blockIdx.y, r = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int q0 = a.cu_q[r], nq = a.cu_q[r + 1] - q0;
  const int rows = nq * a.G, row0 = blockIdx.x * kAccRows;
  if (row0 >= rows) return;
  const int start = a.cu[r], n = valid_keys(a.kv_len, r, a.Hkv, h, a.cu[r + 1] - start);
  load_rows(a, h, q0, row0, rows, q_sm);
  __syncthreads();
  float m[kAccRows], s[kAccRows];
#pragma unroll
  for (int j = 0; j < kAccRows; ++j) { m[j] = -INFINITY; s[j] = 0.f; }
  for (int key = tid; key < n; key += kAccThreads) {
    float l[kAccRows];
    dots(a, a.K + (int64_t)h * a.k_head + (int64_t)(start + key) * a.k_tok, q_sm, l);
#pragma unroll
    for (int j = 0; j < kAccRows; ++j) {
      if (key < n - (nq - 1 - (row0 + j) / a.G)) {
        const float v = l[j] * a.scale, top = fmaxf(m[j], v);
        s[j] = s[j] * expf(m[j] - top) + expf(v - top);
        m[j] = top;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kAccRows; ++j) {
    const float top = warp_max(m[j]);
    float v = m[j] == -INFINITY ? 0.f : s[j] * expf(m[j] - top);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) { red[0][j][warp] = top; red[1][j][warp] = v; }
  }
  __syncthreads();
  if (tid < kAccRows && row0 + tid < rows) {
    float top = -INFINITY, v = 0.f;
    for (int w = 0; w < kAccThreads / 32; ++w) top = fmaxf(top, red[0][tid][w]);
    for (int w = 0; w < kAccThreads / 32; ++w)
      if (red[0][tid][w] != -INFINITY) v += red[1][tid][w] * expf(red[0][tid][w] - top);
    const int row = row0 + tid;
    a.lse[(int64_t)(q0 + row / a.G) * a.Hkv * a.G + h * a.G + row % a.G] = top == -INFINITY ? -INFINITY : top + logf(v);
  }
}

__global__ void __launch_bounds__(kAccThreads)
accumulate_kernel(const __grid_constant__ AccArgs a) {
  __shared__ float q_sm[kAccRows][kMaxHeadDim8];
  const int h = blockIdx.y, r = blockIdx.z;
  const int q0 = a.cu_q[r], nq = a.cu_q[r + 1] - q0, rows = nq * a.G;
  const int start = a.cu[r], n = valid_keys(a.kv_len, r, a.Hkv, h, a.cu[r + 1] - start);
  const int key0 = blockIdx.x * kAccThreads, key = key0 + threadIdx.x;
  if (key0 >= n) return;
  double sum = 0.0;
  // the first token that sees the tile's first key
  const int first = max(nq - 1 - (n - 1 - key0), 0) * a.G / kAccRows * kAccRows;
  for (int row0 = first; row0 < rows; row0 += kAccRows) {
    __syncthreads();
    load_rows(a, h, q0, row0, rows, q_sm);
    __syncthreads();
    if (key < n) {
      float l[kAccRows];
      dots(a, a.K + (int64_t)h * a.k_head + (int64_t)(start + key) * a.k_tok, q_sm, l);
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < kAccRows; ++j) {
        const int row = row0 + j;
        if (row < rows && key < n - (nq - 1 - row / a.G))
          part += expf(l[j] * a.scale - a.lse[(int64_t)(q0 + row / a.G) * a.Hkv * a.G + h * a.G + row % a.G]);
      }
      sum += part;
    }
  }
  if (key < n) {
    const int64_t slot = (int64_t)h * a.total + start + key;
    a.acc_out[slot] = (float)((a.acc ? (double)a.acc[slot] : 0.0) + sum);
  }
}

}  // namespace

AccumulateMap accumulate_map(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N, int64_t total_q,
                             int64_t max_q) {
  AccumulateMap m;
  m.lse = kStatusBytes;
  m.part = align_up(m.lse + (size_t)total_q * p->n_q_heads * 4, 256);
  m.q_tiles = m.key_chunks = 0;
  m.total = m.part;
  return m;
}

int32_t launch_accumulate(const gvote_params* p, const __nv_bfloat16* Q, int64_t q_tok, int64_t q_head,
                          const int32_t* cu_q, int64_t total_q, int64_t max_q, const __nv_bfloat16* K, int64_t k_tok,
                          int64_t k_head, const int32_t* cu, const int32_t* kv_len, int32_t batch, int64_t total_tokens,
                          int64_t max_N, const float* lse, const float* acc, float* acc_out, char* ws, cudaStream_t st) {
  const AccumulateMap m = accumulate_map(p, batch, total_tokens, max_N, total_q, max_q);
  AccArgs a;
  a.Q = Q; a.q_tok = q_tok; a.q_head = q_head; a.cu_q = cu_q; a.K = K; a.k_tok = k_tok; a.k_head = k_head;
  a.total = total_tokens; a.cu = cu; a.kv_len = kv_len;
  a.lse = lse ? const_cast<float*>(lse) : (float*)(ws + m.lse);
  a.acc = acc; a.acc_out = acc_out; a.Hkv = p->n_kv_heads; a.G = p->n_q_heads / p->n_kv_heads; a.d_k = p->d_k;
  a.scale = (float)(1.0 / sqrt((double)p->d_k));
  if (!lse && max_q > 0) {
    LaunchScope scope_("accumulate_lse_kernel", st);
    launch_on(accumulate_lse_kernel, dim3((unsigned)ceil_div(max_q * a.G, kAccRows), a.Hkv, batch), dim3(kAccThreads), 0, st, a);
    GVOTE_LAUNCH_CHECK("accumulate_lse_kernel");
  }
  if (max_N > 0) {
    LaunchScope scope_("accumulate_kernel", st);
    launch_on(accumulate_kernel, dim3((unsigned)ceil_div(max_N, kAccThreads), a.Hkv, batch), dim3(kAccThreads), 0, st, a);
    GVOTE_LAUNCH_CHECK("accumulate_kernel");
  }
  return GVOTE_OK;
}

}  // namespace gvote
