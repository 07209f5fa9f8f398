// Attention of a few query tokens over the 8-bit cache (gvote_attend8), split over the rows of the cache.
//
// Rows of a head's slab are cut into chunks; attend8_partial_kernel takes one chunk of one (request, KV head) and up
// to eight of its query rows (token-major: row = token * G + query head of the group) and leaves the chunk's
// maximum logit, its sum of exponentials and its unnormalised output; attend8_merge_kernel rescales the
// chunks to the row's maximum and divides; attend8_weights_kernel turns the logits the first kernel kept into
// weights and adds them up per slot.
#include "cache8.cuh"

namespace gvote {
namespace {

constexpr int kAttThreads = 256;
constexpr int kAttRows = 8;
constexpr int kAttKeys = 256;

struct AttendArgs {
  const __nv_bfloat16* Q;
  int64_t q_tok, q_head;
  const int32_t* cu_q;
  const uint8_t* K;
  const uint8_t* V;
  const float* k_scale;
  const float* v_scale;
  int64_t tok, head, total, row_blocks;
  const int32_t* cu;
  const int32_t* kv_len;
  __nv_bfloat16* out;
  int64_t o_tok, o_head;
  float* lse;
  const float* acc;
  float* acc_out;
  float* part_o;       // [chunk][Hkv][max_q * G][d_k]
  float2* part_ml;     // [chunk][Hkv][max_q * G]  (maximum, sum)
  float* logits;       // [Hkv][max_q * G][total] or null
  int64_t chunks;
  int Hkv, G, batch, d_k, max_q;
  float scale;
};

__global__ void __launch_bounds__(kAttThreads)
attend8_partial_kernel(const __grid_constant__ AttendArgs a) {
  __shared__ float q_sm[kAttRows][kMaxHeadDim8];
  __shared__ float p_sm[kAttRows][kAttKeys];
  __shared__ float s_m[kAttRows], s_l[kAttRows];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = (int)(blockIdx.x % a.Hkv);
  const int64_t gc = blockIdx.x / a.Hkv;
  const int r = a.batch == 1 ? 0 : find_request_by(a.cu, a.batch, gc, 8);
  const int start = a.cu[r], cap = a.cu[r + 1] - start;
  const int c = (int)(gc - ((start >> 8) + r));
  const int n = valid_keys(a.kv_len, r, a.Hkv, h, cap);
  const int key0 = c * kAttKeys;
  if (key0 >= n) return;
  const int q0 = a.cu_q[r], nq = a.cu_q[r + 1] - q0;
  const int rows = nq * a.G, row0 = blockIdx.y * kAttRows;
  if (row0 >= rows) return;
  const int nr = min(kAttRows, rows - row0);
  for (int i = tid; i < kAttRows * a.d_k; i += kAttThreads) {
    const int j = i / a.d_k, d = i - j * a.d_k;
    float v = 0.f;
    if (j < nr) {
      const int token = (row0 + j) / a.G, g = (row0 + j) % a.G;
      v = __bfloat162float(a.Q[(int64_t)(q0 + token) * a.q_tok + (int64_t)(h * a.G + g) * a.q_head + d]);
    }
    q_sm[j][d] = v;
  }
  __syncthreads();
  const int key = key0 + tid;
  const int64_t sb = (int64_t)h * a.row_blocks + block8_offset(start, r);
  float l[kAttRows];
#pragma unroll
  for (int j = 0; j < kAttRows; ++j) l[j] = 0.f;
  if (key < n) {
    const uint8_t* kp = a.K + (int64_t)h * a.head + (int64_t)(start + key) * a.tok;
    for (int u = 0; u < a.d_k / 16; ++u) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(kp) + u);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = (&v.x)[e >> 1];
        const float2 f = decode8x2((e & 1) ? w >> 16 : w & 0xffffu);
#pragma unroll
        for (int j = 0; j < kAttRows; ++j)
          l[j] = fmaf(q_sm[j][u * 16 + 2 * e], f.x, fmaf(q_sm[j][u * 16 + 2 * e + 1], f.y, l[j]));
      }
    }
    const float ks = a.k_scale[sb + (key >> 6)] * a.scale;
#pragma unroll
    for (int j = 0; j < kAttRows; ++j) l[j] *= ks;
  }
#pragma unroll
  for (int j = 0; j < kAttRows; ++j) {
    const int token = (row0 + j) / a.G;
    const bool sees = j < nr && key < n - (nq - 1 - token);
    if (!sees) l[j] = -INFINITY;
    p_sm[j][tid] = l[j];
    if (a.logits && j < nr && key < n)
      a.logits[((int64_t)h * a.max_q * a.G + row0 + j) * a.total + start + key] = l[j];
  }
  __syncthreads();
  if (warp < kAttRows) {
    float m = -INFINITY;
    for (int i = lane; i < kAttKeys; i += 32) m = fmaxf(m, p_sm[warp][i]);
    m = warp_max(m);
    const float ref = m == -INFINITY ? 0.f : m;
    float s = 0.f;
    for (int i = lane; i < kAttKeys; i += 32) {
      const float e = expf(p_sm[warp][i] - ref);
      p_sm[warp][i] = e;
      s += e;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) { s_m[warp] = m; s_l[warp] = s; }
  }
  __syncthreads();
  const int cnt = min(kAttKeys, n - key0);
  const int64_t prow = (gc * a.Hkv + h) * a.max_q * a.G + row0;
  if (tid < a.d_k) {
    float o[kAttRows];
#pragma unroll
    for (int j = 0; j < kAttRows; ++j) o[j] = 0.f;
    const uint8_t* vp = a.V + (int64_t)h * a.head + (int64_t)(start + key0) * a.tok + tid;
    for (int i = 0; i < cnt; ++i) {
      const float v = decode8x2(vp[(int64_t)i * a.tok]).x * a.v_scale[sb + ((key0 + i) >> 6)];
#pragma unroll
      for (int j = 0; j < kAttRows; ++j) o[j] = p_sm[j][i] == 0.f ? o[j] : fmaf(p_sm[j][i], v, o[j]);
    }
    for (int j = 0; j < nr; ++j) a.part_o[(prow + j) * a.d_k + tid] = o[j];
  }
  if (tid < nr) a.part_ml[prow + tid] = make_float2(s_m[tid], s_l[tid]);
}

// One warp group per (query head, token): merge the chunks of its request.
__global__ void __launch_bounds__(kMaxHeadDim8)
attend8_merge_kernel(const __grid_constant__ AttendArgs a) {
  const int g = blockIdx.x, r = blockIdx.z, token = blockIdx.y;
  const int q0 = a.cu_q[r], nq = a.cu_q[r + 1] - q0;
  if (token >= nq) return;
  const int h = g / a.G, row = token * a.G + g % a.G;
  const int start = a.cu[r], n = valid_keys(a.kv_len, r, a.Hkv, h, a.cu[r + 1] - start);
  const int chunks = (n + kAttKeys - 1) / kAttKeys;
  const int64_t first = (start >> 8) + r;
  float m = -INFINITY;
  for (int c = 0; c < chunks; ++c) m = fmaxf(m, a.part_ml[((first + c) * a.Hkv + h) * a.max_q * a.G + row].x);
  float l = 0.f, o = 0.f;
  for (int c = 0; c < chunks; ++c) {
    const int64_t p = ((first + c) * a.Hkv + h) * a.max_q * a.G + row;
    const float2 ml = a.part_ml[p];
    if (ml.x == -INFINITY) continue;
    const float w = expf(ml.x - m);
    l = fmaf(w, ml.y, l);
    if (threadIdx.x < a.d_k) o = fmaf(w, a.part_o[p * a.d_k + threadIdx.x], o);
  }
  if (threadIdx.x < a.d_k)
    a.out[(int64_t)(q0 + token) * a.o_tok + (int64_t)g * a.o_head + threadIdx.x] = __float2bfloat16(m == -INFINITY ? 0.f : o / l);
  if (threadIdx.x == 0) a.lse[(int64_t)(q0 + token) * a.Hkv * a.G + g] = m == -INFINITY ? -INFINITY : m + logf(l);
}

__global__ void __launch_bounds__(256)
attend8_weights_kernel(const __grid_constant__ AttendArgs a) {
  const int r = blockIdx.z, h = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  const int start = a.cu[r], n = valid_keys(a.kv_len, r, a.Hkv, h, a.cu[r + 1] - start);
  if (i >= n) return;
  const int q0 = a.cu_q[r], rows = (a.cu_q[r + 1] - q0) * a.G;
  float s = 0.f;
  for (int row = 0; row < rows; ++row) {
    const float lse = a.lse[(int64_t)(q0 + row / a.G) * a.Hkv * a.G + h * a.G + row % a.G];
    if (lse != -INFINITY) s += expf(a.logits[((int64_t)h * a.max_q * a.G + row) * a.total + start + i] - lse);
  }
  const int64_t slot = (int64_t)h * a.total + start + i;
  a.acc_out[slot] = (a.acc ? a.acc[slot] : 0.f) + s;
}

}  // namespace

AttendMap attend8_map(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N, int64_t total_q,
                      int64_t max_q) {
  AttendMap m;
  const int64_t rows = (max_q < GVOTE_ATTEND8_MAX_Q ? max_q : GVOTE_ATTEND8_MAX_Q) * (p->n_q_heads / p->n_kv_heads);
  m.chunk_keys = kAttKeys;
  m.chunks = (total_tokens >> 8) + batch;
  const size_t parts = (size_t)m.chunks * p->n_kv_heads * rows;
  m.o = kStatusBytes;
  m.ml = align_up(m.o + parts * p->d_k * 4, 256);
  m.logits = align_up(m.ml + parts * 8, 256);
  m.total = align_up(m.logits + (size_t)p->n_kv_heads * rows * total_tokens * 4 + (size_t)total_q * p->n_q_heads * 4, 256);
  return m;
}

int32_t launch_attend8(const gvote_params* p, const __nv_bfloat16* Q, int64_t q_tok, int64_t q_head, const int32_t* cu_q,
                       int64_t total_q, int64_t max_q, const gvote_cache8* c, __nv_bfloat16* out, int64_t o_tok,
                       int64_t o_head, float* lse, const float* acc, float* acc_out, char* ws, cudaStream_t st) {
  const AttendMap m = attend8_map(p, c->batch, c->total_tokens, c->max_N, total_q, max_q);
  AttendArgs a;
  a.Q = Q; a.q_tok = q_tok; a.q_head = q_head; a.cu_q = cu_q;
  a.K = (const uint8_t*)c->K; a.V = (const uint8_t*)c->V; a.k_scale = c->k_scale; a.v_scale = c->v_scale;
  a.tok = c->tok_stride; a.head = c->head_stride; a.total = c->total_tokens;
  a.row_blocks = gvote_cache8_row_blocks(c->total_tokens, c->batch);
  a.cu = c->cu_seqlens; a.kv_len = c->kv_len;
  a.out = out; a.o_tok = o_tok; a.o_head = o_head; a.acc = acc; a.acc_out = acc_out;
  a.part_o = (float*)(ws + m.o); a.part_ml = (float2*)(ws + m.ml);
  a.logits = acc_out ? (float*)(ws + m.logits) : nullptr;
  a.Hkv = p->n_kv_heads; a.G = p->n_q_heads / p->n_kv_heads; a.batch = c->batch; a.d_k = p->d_k; a.max_q = (int)max_q;
  a.chunks = m.chunks;
  a.lse = lse ? lse : (float*)(ws + m.logits + (size_t)a.Hkv * max_q * a.G * a.total * 4);
  a.scale = (float)(1.0 / sqrt((double)p->d_k));
  {
    LaunchScope scope_("attend8_partial_kernel", st);
    launch_on(attend8_partial_kernel, dim3((unsigned)(m.chunks * a.Hkv), (unsigned)ceil_div(max_q * a.G, kAttRows)),
              dim3(kAttThreads), 0, st, a);
  }
  GVOTE_LAUNCH_CHECK("attend8_partial_kernel");
  {
    LaunchScope scope_("attend8_merge_kernel", st);
    launch_on(attend8_merge_kernel, dim3(p->n_q_heads, (unsigned)max_q, c->batch), dim3((unsigned)ceil_div(p->d_k, 32) * 32), 0, st, a);
  }
  GVOTE_LAUNCH_CHECK("attend8_merge_kernel");
  if (acc_out && c->max_N > 0) {
    LaunchScope scope_("attend8_weights_kernel", st);
    launch_on(attend8_weights_kernel, dim3((unsigned)ceil_div(c->max_N, 256), a.Hkv, c->batch), dim3(256), 0, st, a);
    GVOTE_LAUNCH_CHECK("attend8_weights_kernel");
  }
  return GVOTE_OK;
}

}  // namespace gvote
