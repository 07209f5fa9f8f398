// New tokens' rows join the 8-bit cache (gvote_append8).  The rows land behind the kv_len rows of each head; a
// block that holds rows already keeps the larger of its scale and the one the new rows need, and when that
// grows by 2^j its codes are rewritten as e4m3(code * 2^-j) (exact while they stay normal numbers).
//
// Latency: a decode step appends one row of d_k values per (request, head).  One launch: a cluster of up to eight
// CTAs per (head, request), each taking every eighth of the blocks the new rows touch (one CTA when one
// token comes), the first half of a CTA's threads the keys, the second half the values.  The cluster meets before
// kv_len_out is written, because that array may be kv_len itself and the CTAs read it at their start.
// Measured: 4.4 us in a graph, for one token of each of 16 requests as for three tokens of one; 13.6 us by an eager call,
// which the host bounds.
#include <cooperative_groups.h>

#include "cache8.cuh"

namespace gvote {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendHalf = kAppendThreads / 2;

struct AppendArgs {
  const __nv_bfloat16* src[2];
  int64_t s_tok, s_head;
  const int32_t* cu_new;
  uint8_t* dst[2];
  float* scale[2];
  int64_t d_tok, d_head, total, row_blocks;
  const int32_t* cu;
  const int32_t* kv_len;
  int32_t* kv_len_out;
  float* acc;
  int32_t* token_pos;
  const int32_t* pos_new;
  int32_t* status;
  int Hkv, d_k;
};

__global__ void __launch_bounds__(kAppendThreads)
append8_kernel(const __grid_constant__ AppendArgs a) {
  __shared__ float s_max[kAppendThreads / 32];
  const int h = blockIdx.x, r = blockIdx.y, tid = threadIdx.x;
  const int t = tid / kAppendHalf, lt = tid % kAppendHalf;          // 0: keys, 1: values
  const int start = a.cu[r], cap = a.cu[r + 1] - start;
  const int n = valid_keys(a.kv_len, r, a.Hkv, h, cap);
  const int first = a.cu_new[r], asked = a.cu_new[r + 1] - first;
  const int fit = max(min(asked, cap - n), 0);
  const int dc = a.d_k >> 4;
  const __nv_bfloat16* src = a.src[t] + (int64_t)h * a.s_head + (int64_t)first * a.s_tok;
  uint8_t* dst = a.dst[t] + (int64_t)h * a.d_head + (int64_t)start * a.d_tok;
  float* scales = a.scale[t] + (int64_t)h * a.row_blocks + block8_offset(start, r);
  for (int b = (n >> 6) + (int)blockIdx.z; b * kBlock8 < n + fit; b += gridDim.z) {
    const int have = max(n - b * kBlock8, 0);                        // rows the block holds already
    const int s0 = max(b * kBlock8 - n, 0);                          // its first new row
    const int units = (min(kBlock8, n + fit - b * kBlock8) - have) * dc;
    const float old = have ? scales[b] : 0.f;
    float mx = 0.f;
    for (int u = lt; u < units; u += kAppendHalf) {
      const int j = u / dc, c = u - j * dc;
      const uint4* q = reinterpret_cast<const uint4*>(src + (int64_t)(s0 + j) * a.s_tok + c * 16);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 v = __ldg(q + k);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = (&v.x)[e];
          mx = fmaxf(mx, fmaxf(finite_abs(__uint_as_float(w << 16)), finite_abs(__uint_as_float(w & 0xffff0000u))));
        }
      }
    }
    mx = warp_max(mx);
    if ((tid & 31) == 0) s_max[tid >> 5] = mx;
    __syncthreads();                                                 // (also: everyone has read the old scale)
    const float* half = s_max + t * (kAppendHalf / 32);
    const float top = fmaxf(fmaxf(half[0], half[1]), fmaxf(half[2], half[3]));
    const float scale = fmaxf(scale8_of(top), old), inv = inverse_pow2(scale);
    uint8_t* rows = dst + (int64_t)b * kBlock8 * a.d_tok;
    if (have && scale > old) {
      const float shrink = old * inv;                                // 2^-j; underflows to 0 only where every code does
      for (int u = lt; u < have * dc; u += kAppendHalf) {
        const int j = u / dc, c = u - j * dc;
        uint4* q = reinterpret_cast<uint4*>(rows + (int64_t)j * a.d_tok + c * 16);
        uint4 v = *q;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t& w = (&v.x)[e];
          const float2 f0 = decode8x2(w & 0xffffu), f1 = decode8x2(w >> 16);
          w = encode8x2(f0.x * shrink, f0.y * shrink) | (encode8x2(f1.x * shrink, f1.y * shrink) << 16);
        }
        *q = v;
      }
    }
    for (int u = lt; u < units; u += kAppendHalf) {
      const int j = u / dc, c = u - j * dc;
      const uint4* q = reinterpret_cast<const uint4*>(src + (int64_t)(s0 + j) * a.s_tok + c * 16);
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 v = __ldg(q + k);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t w0 = (&v.x)[2 * e], w1 = (&v.x)[2 * e + 1];
          w[2 * k + e] = encode8x2(__uint_as_float(w0 << 16) * inv, __uint_as_float(w0 & 0xffff0000u) * inv) |
                         (encode8x2(__uint_as_float(w1 << 16) * inv, __uint_as_float(w1 & 0xffff0000u) * inv) << 16);
        }
      }
      *reinterpret_cast<uint4*>(rows + (int64_t)(have + j) * a.d_tok + c * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (lt == 0) scales[b] = scale;
    if (t == 0 && lt < units / dc) {
      const int64_t slot = (int64_t)h * a.total + start + b * kBlock8 + have + lt;
      if (a.acc) a.acc[slot] = 0.f;
      if (a.token_pos) a.token_pos[slot] = a.pos_new[first + s0 + lt];
    }
    __syncthreads();                                                 // s_max is used again
  }
  if (gridDim.z > 1) cooperative_groups::this_cluster().sync(); else __syncthreads();
  if (blockIdx.z == 0 && tid == 0) {
    a.kv_len_out[r * a.Hkv + h] = n + fit;
    if (fit < asked) { atomicExch(&a.status[0], GVOTE_ERR_WORKSPACE_TOO_SMALL); atomicExch(&a.status[1], 9); }
  }
}

}  // namespace

int32_t launch_append8(const gvote_params* p, const __nv_bfloat16* K, const __nv_bfloat16* V, int64_t tok, int64_t head,
                       const int32_t* cu_new, int64_t max_new, const gvote_cache8* c, int32_t* kv_len_out, float* acc,
                       int32_t* token_pos, const int32_t* pos_new, char* ws, cudaStream_t st) {
  AppendArgs a;
  a.src[0] = K; a.src[1] = V; a.s_tok = tok; a.s_head = head; a.cu_new = cu_new;
  a.dst[0] = (uint8_t*)c->K; a.dst[1] = (uint8_t*)c->V; a.scale[0] = c->k_scale; a.scale[1] = c->v_scale;
  a.d_tok = c->tok_stride; a.d_head = c->head_stride; a.total = c->total_tokens;
  a.row_blocks = gvote_cache8_row_blocks(c->total_tokens, c->batch);
  a.cu = c->cu_seqlens; a.kv_len = c->kv_len; a.kv_len_out = kv_len_out;
  a.acc = acc; a.token_pos = token_pos; a.pos_new = pos_new;
  a.status = reinterpret_cast<int32_t*>(ws);
  a.Hkv = p->n_kv_heads; a.d_k = p->d_k;
  // max_new rows touch at most this many blocks of a head (one row: one block)
  const int64_t blocks = max_new <= 1 ? 1 : ceil_div(max_new - 1, kBlock8) + 1;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr;
  cfg.gridDim = dim3(p->n_kv_heads, c->batch, (unsigned)(blocks < 8 ? blocks : 8));
  cfg.blockDim = dim3(kAppendThreads);
  cfg.stream = st;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 1; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = cfg.gridDim.z;
  cfg.attrs = &attr;
  cfg.numAttrs = cfg.gridDim.z > 1 ? 1 : 0;
  {
    LaunchScope scope_("append8_kernel", st);
    (void)cudaLaunchKernelEx(&cfg, append8_kernel, a);
  }
  GVOTE_LAUNCH_CHECK("append8_kernel");
  return GVOTE_OK;
}

}  // namespace gvote
