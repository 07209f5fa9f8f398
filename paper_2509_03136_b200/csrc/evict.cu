// Eviction by collected attention weight (gvote_evict): per (request, KV head) the last n_recent rows, the first
// n_s rows, and of those between the ones with the largest weight, ties to the lower slot.
//
// One CTA per (head, request).  A radix search of eight bits per pass over the order-preserving image of the
// weights finds the smallest kept weight T and how many of the rows equal to T are kept; a last sweep writes
// the mask words, counting the equal ones in slot order (every warp owns a run of consecutive words).
#include "cache8.cuh"

namespace gvote {
namespace {

constexpr int kEvictThreads = 1024;
constexpr int kEvictWarps = kEvictThreads / 32;

// Larger weight, larger key; -0 and +0 alike; a NaN below everything.
__device__ __forceinline__ uint32_t weight_key(float w) { return w == w ? ordered_key(w + 0.f) : 0u; }

__global__ void __launch_bounds__(kEvictThreads)
evict_kernel(const float* __restrict__ acc, const int32_t* __restrict__ cu, const int32_t* __restrict__ kv_len,
             const int32_t* __restrict__ keep, int Hkv, int64_t total, int64_t row_words, int n_recent, int n_sink,
             uint32_t* __restrict__ mask, int32_t* __restrict__ budget) {
  __shared__ int hist[256];
  __shared__ int s_digit, s_left;
  __shared__ int s_eq[kEvictWarps];
  const int h = blockIdx.x, r = blockIdx.y;
  const int start = cu[r], N = cu[r + 1] - start;
  const int n = valid_keys(kv_len, r, Hkv, h, N);
  const int k = min(max(keep[r * Hkv + h], 0), n);
  const int recent = min(n_recent, k), sink = min(n_sink, k - recent);
  const int lo = sink, hi = n - recent;                 // the rows weighed
  const int want = k - recent - sink;
  const float* w = acc + (int64_t)h * total + start;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t prefix = 0;                                  // the digits of T found so far
  int left = want;                                      // rows to take among those that share them
  if (want > 0 && want < hi - lo) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kEvictThreads) hist[i] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += kEvictThreads) {
        const uint32_t key = weight_key(w[i]);
        if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255u], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int c = left, d = 255;
        while (d > 0 && hist[d] < c) { c -= hist[d]; --d; }
        s_digit = d;
        s_left = c;
      }
      __syncthreads();
      prefix |= (uint32_t)s_digit << shift;
      left = s_left;
      __syncthreads();
    }
  }
  const bool all = want >= hi - lo;                     // nothing to weigh
  const int words = (N + 31) >> 5;
  const int per = (words + kEvictWarps - 1) / kEvictWarps;
  const int w0 = warp * per, w1 = min(w0 + per, words);
  uint32_t* m = mask + (int64_t)h * row_words + mask_word_offset(start, r);
  int eq = 0;
  if (!all && want > 0) {
    for (int q = w0; q < w1; ++q) {
      const int i = q * 32 + lane;
      eq += __popc(__ballot_sync(0xffffffffu, i >= lo && i < hi && weight_key(w[i]) == prefix));
    }
  }
  if (lane == 0) s_eq[warp] = eq;
  __syncthreads();
  int before = 0;
  for (int i = 0; i < warp; ++i) before += s_eq[i];
  for (int q = w0; q < w1; ++q) {
    const int i = q * 32 + lane;
    bool take = i < n && (i < lo || i >= hi);
    const bool mid = i >= lo && i < hi;
    if (all) {
      take = take || mid;
    } else if (want > 0) {
      const uint32_t key = mid ? weight_key(w[i]) : 0u;
      const bool same = mid && key == prefix;
      const uint32_t same_bits = __ballot_sync(0xffffffffu, same);
      if (mid && key > prefix) take = true;
      if (same && before + __popc(same_bits & ((1u << lane) - 1u)) < left) take = true;
      before += __popc(same_bits);
    }
    const uint32_t bits = __ballot_sync(0xffffffffu, take);
    if (lane == 0) m[q] = bits;
  }
  if (tid == 0) budget[r * Hkv + h] = k;
}

}  // namespace

int32_t launch_evict(const gvote_params* p, const float* acc, const int32_t* cu, const int32_t* kv_len, int32_t batch,
                     int64_t total_tokens, int64_t max_N, const int32_t* keep, int32_t n_recent, uint32_t* mask,
                     int32_t* budget, cudaStream_t st) {
  {
    LaunchScope scope_("evict_kernel", st);
    launch_on(evict_kernel, dim3(p->n_kv_heads, batch), dim3(kEvictThreads), 0, st, acc, cu, kv_len, keep, p->n_kv_heads,
              total_tokens, gvote_mask_row_words(total_tokens, batch), n_recent, p->n_s, mask, budget);
  }
  GVOTE_LAUNCH_CHECK("evict_kernel");
  return GVOTE_OK;
}

}  // namespace gvote
