// Eviction by collected attention weight (gvote_evict): per (request, KV head) the last n_recent rows, the first
// n_s rows, and of those between the ones with the largest weight, ties to the lower slot.
//
// A cluster of CTAs per (head, request), each with a run of the row's mask words.  The weights are read once, as
// order-preserving 32-bit images in shared memory.  A radix search of 11, 11 and 10 bits finds the smallest kept image T:
// every CTA counts its images per digit, adds its peers' counts through distributed shared memory and finds the
// digit for itself (no broadcast).  Then the mask words are written: images above T, and of those equal to T as many as
// are left, lowest slots first; only when T is shared by more rows than are left does the order matter, and the equal
// ones are then counted run by run.  Latency, not bytes, bounds this: 4 bytes per row are 0.1 us of memory time, the five
// steps cost a microsecond or two each.  Cluster size: the largest of 8, 4, 2, 1 that leaves a CTA 2048 rows of the longest
// slab and the grid no more than two CTAs per SM (one row of 128K weights: 17 us with eight CTAs, 138 with one).
// Shares beyond 36K rows per CTA are read from memory again in every step.
#include <cooperative_groups.h>

#include "cache8.cuh"

namespace gvote {
namespace {

namespace cg = cooperative_groups;

constexpr int kEvictThreads = 1024;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kBins = 2048;
constexpr int kCopies = 2;                         // histograms the warps of a CTA share out, against contention
constexpr int kSharedKeys = 36 * 1024;

// Larger weight, larger key; -0 and +0 alike; a NaN below everything.
__device__ __forceinline__ uint32_t weight_key(float w) { return w == w ? ordered_key(w + 0.f) : 0u; }

__global__ void __launch_bounds__(kEvictThreads)
evict_kernel(const float* __restrict__ acc, const int32_t* __restrict__ cu, const int32_t* __restrict__ kv_len,
             const int32_t* __restrict__ keep, int Hkv, int64_t total, int64_t row_words, int n_recent, int n_sink,
             int shared_keys, uint32_t* __restrict__ mask, int32_t* __restrict__ budget) {
  extern __shared__ uint32_t keys_sm[];            // [shared_keys]
  __shared__ int hist[kCopies][kBins];
  __shared__ int folded[3][kBins];                 // this CTA's counts of each step, read by its peers
  __shared__ int warp_tot[kEvictWarps];
  __shared__ int s_digit, s_left, s_equal;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int h = blockIdx.y, r = blockIdx.z;
  const int start = cu[r], N = cu[r + 1] - start;
  const int n = valid_keys(kv_len, r, Hkv, h, N);
  const int k = min(max(keep[r * Hkv + h], 0), n);
  const int recent = min(n_recent, k), sink = min(n_sink, k - recent);
  const int lo = sink, hi = n - recent;            // the rows weighed
  const int want = k - recent - sink;
  const float* w = acc + (int64_t)h * total + start;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int words = (N + 31) >> 5, share = (words + C - 1) / C;
  const int w0 = min(rank * share, words), w1 = min(w0 + share, words);       // this CTA's mask words
  const int i0 = max(w0 * 32, lo), i1 = min(w1 * 32, hi);                     // and weighed rows
  const bool search = want > 0 && want < hi - lo;
  const bool staged = i1 - i0 <= shared_keys;
  auto key_at = [&](int i) { return staged ? keys_sm[i - i0] : weight_key(w[i]); };

  uint32_t T = 0;                                  // the smallest kept image
  int left = want, equal = 0;                      // rows kept among those equal to T, and how many there are
  if (search) {                                    // (the same for every CTA of the cluster)
    if (staged)
      for (int i = i0 + tid; i < i1; i += kEvictThreads) keys_sm[i - i0] = weight_key(w[i]);
#pragma unroll 1
    for (int step = 0; step < 3; ++step) {
      const int shift = step == 0 ? 21 : step == 1 ? 10 : 0, bits = step == 2 ? 10 : 11;
      const uint32_t digit_mask = (1u << bits) - 1u, above = step == 0 ? 0u : 0xffffffffu << (shift + bits);
      for (int i = tid; i < kCopies * kBins; i += kEvictThreads) (&hist[0][0])[i] = 0;
      __syncthreads();
      for (int base = i0; base < i1; base += kEvictThreads) {
        const int i = base + tid;
        const uint32_t key = i < i1 ? key_at(i) : 0u;
        const bool in = i < i1 && (key & above) == (T & above);
        const uint32_t d = (key >> shift) & digit_mask;
        // a warp whose rows all share the digit (equal weights) adds them in one go
        const uint32_t active = __ballot_sync(0xffffffffu, in);
        if (active) {
          const uint32_t d0 = __shfl_sync(0xffffffffu, d, __ffs(active) - 1);
          if (__all_sync(0xffffffffu, !in || d == d0)) {
            if (lane == 0) atomicAdd(&hist[warp & (kCopies - 1)][d0], __popc(active));
          } else if (in) {
            atomicAdd(&hist[warp & (kCopies - 1)][d], 1);
          }
        }
      }
      __syncthreads();
      for (int i = tid; i < kBins; i += kEvictThreads) {
        int c = 0;
#pragma unroll
        for (int q = 0; q < kCopies; ++q) c += hist[q][i];
        folded[step][i] = c;
      }
      cluster.sync();
      // from the largest digit down: thread t has digits 2047 - 2 t and 2046 - 2 t
      int c2[2] = {0, 0};
      for (int p = 0; p < C; ++p) {
        const int* peer = cluster.map_shared_rank(&folded[step][0], p);
        const int2 v = *reinterpret_cast<const int2*>(peer + kBins - 2 - 2 * tid);
        c2[0] += v.y;
        c2[1] += v.x;
      }
      int inc = c2[0] + c2[1];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += u;
      }
      if (lane == 31) warp_tot[warp] = inc;
      __syncthreads();
      int before = inc - c2[0] - c2[1];
      for (int q = 0; q < warp; ++q) before += warp_tot[q];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (before < left && before + c2[j] >= left) {
          s_digit = kBins - 1 - 2 * tid - j;
          s_left = left - before;
          s_equal = c2[j];
        }
        before += c2[j];
      }
      __syncthreads();
      T |= (uint32_t)s_digit << shift;
      left = s_left;
      equal = s_equal;
      __syncthreads();
    }
  }

  // ---- the mask words: each warp has a run of consecutive ones
  const int per = (w1 - w0 + kEvictWarps - 1) / kEvictWarps;
  const int q0 = min(w0 + warp * per, w1), q1 = min(q0 + per, w1);
  const bool ordered = search && left < equal;     // not all of the rows equal to T are kept
  int before = 0;                                  // rows equal to T in lower slots
  if (ordered) {
    const int my_digit = (int)(T & 1023u);
    for (int p = 0; p < rank; ++p) before += *cluster.map_shared_rank(&folded[2][my_digit], p);
    int mine = 0;
    for (int q = q0; q < q1; ++q) {
      const int i = q * 32 + lane;
      mine += __popc(__ballot_sync(0xffffffffu, i >= i0 && i < i1 && key_at(i) == T));
    }
    if (lane == 0) warp_tot[warp] = mine;
    __syncthreads();
    for (int q = 0; q < warp; ++q) before += warp_tot[q];
  }
  uint32_t* m = mask + (int64_t)h * row_words + mask_word_offset(start, r);
  for (int q = q0; q < q1; ++q) {
    const int i = q * 32 + lane;
    const bool mid = i >= i0 && i < i1;
    bool take = i < n && (i < lo || i >= hi);
    if (search) {
      const uint32_t key = mid ? key_at(i) : 0u;
      if (mid && (ordered ? key > T : key >= T)) take = true;
      if (ordered) {
        const uint32_t same = __ballot_sync(0xffffffffu, mid && key == T);
        if (((same >> lane) & 1u) && before + __popc(same & ((1u << lane) - 1u)) < left) take = true;
        before += __popc(same);
      }
    } else if (want > 0) {
      take = take || mid;
    }
    const uint32_t bits = __ballot_sync(0xffffffffu, take);
    if (lane == 0) m[q] = bits;
  }
  if (rank == 0 && tid == 0) budget[r * Hkv + h] = k;
  cluster.sync();                                  // the counts are read until here
}

}  // namespace

int32_t launch_evict(const gvote_params* p, const float* acc, const int32_t* cu, const int32_t* kv_len, int32_t batch,
                     int64_t total_tokens, int64_t max_N, const int32_t* keep, int32_t n_recent, uint32_t* mask,
                     int32_t* budget, cudaStream_t st) {
  int C = 8;
  while (C > 1 && (max_N / C < 2048 || (int64_t)batch * p->n_kv_heads * C > 2 * 148)) C >>= 1;
  const int64_t share = (ceil_div(max_N, 32) + C - 1) / C * 32;
  const int shared_keys = (int)(share < kSharedKeys ? share : kSharedKeys);
  GVOTE_CUDA_CHECK(cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedKeys * 4));
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr;
  cfg.gridDim = dim3(C, p->n_kv_heads, batch);
  cfg.blockDim = dim3(kEvictThreads);
  cfg.dynamicSmemBytes = (size_t)shared_keys * 4;
  cfg.stream = st;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = C; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  {
    LaunchScope scope_("evict_kernel", st);
    (void)cudaLaunchKernelEx(&cfg, evict_kernel, acc, cu, kv_len, keep, (int)p->n_kv_heads, total_tokens,
                             gvote_mask_row_words(total_tokens, batch), (int)n_recent, (int)p->n_s, shared_keys, mask, budget);
  }
  GVOTE_LAUNCH_CHECK("evict_kernel");
  return GVOTE_OK;
}

}  // namespace gvote
