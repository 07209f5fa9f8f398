// Eviction by collected attention weight (gvote_evict): per (request, KV head) the last n_recent rows, the first
// n_s rows, and of those between the ones with the largest weight, ties to the lower slot.
//
// A cluster of CTAs per (head, request), each with a run of the row's mask words.  The weights are read once, as
// order-preserving 32-bit images in shared memory.  A radix search of 11, 11 and 10 bits finds the smallest kept image T:
// every CTA counts its images per digit and per 32 digits, adds its peers' counts of the latter, then of the 32 digits in
// question, through distributed shared memory, and so finds the digit for itself (no broadcast).  Then the mask words are
// written: images above T, and of those equal to T as many as are left, lowest slots first; only when T is shared by more
// rows than are left does the order matter, and the equal ones are then counted run by run.  Latency, not bytes,
// bounds this: 4 bytes per row are 0.1 us of memory time, the five steps cost one to four microseconds each.  Cluster size:
// the largest of 8, 4, 2, 1 that leaves a CTA 2048 rows of the longest slab and the grid no more CTAs than SMs
// (four rows of 128K weights: 19 us with eight CTAs each, 138 with one; 128 rows of 300 to 12K: 15 us with one, 21 with two).
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
  __shared__ int coarse[3][kBins / 32];
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
    if (staged) {
      for (int base = i0 + tid; base < i1; base += 8 * kEvictThreads) {      // eight loads on their way
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = base + j * kEvictThreads < i1 ? w[base + j * kEvictThreads] : 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (base + j * kEvictThreads < i1) keys_sm[base + j * kEvictThreads - i0] = weight_key(v[j]);
      }
    }
#pragma unroll 1
    for (int step = 0; step < 3; ++step) {
      const int shift = step == 0 ? 21 : step == 1 ? 10 : 0, bits = step == 2 ? 10 : 11;
      const uint32_t digit_mask = (1u << bits) - 1u, above = step == 0 ? 0u : 0xffffffffu << (shift + bits);
      for (int i = tid; i < kCopies * kBins; i += kEvictThreads) (&hist[0][0])[i] = 0;
      __syncthreads();
      if (step == 0) {
#pragma unroll 4
        for (int base = i0; base < i1; base += kEvictThreads) {
          const int i = base + tid;
          const uint32_t key = i < i1 ? key_at(i) : 0u, d = key >> shift;
          // a warp whose rows all share the digit (equal weights) adds them in one go
          const uint32_t active = __ballot_sync(0xffffffffu, i < i1);
          const uint32_t d0 = __shfl_sync(0xffffffffu, d, 0);      // (the active lanes are the first ones)
          if (__all_sync(0xffffffffu, i >= i1 || d == d0)) {
            if (lane == 0 && active) atomicAdd(&hist[warp & (kCopies - 1)][d0], __popc(active));
          } else if (i < i1) {
            atomicAdd(&hist[warp & (kCopies - 1)][d], 1);
          }
        }
      } else {
        const uint32_t match = T & above;
#pragma unroll 8
        for (int i = i0 + tid; i < i1; i += kEvictThreads) {
          const uint32_t key = key_at(i);
          if ((key & above) == match) atomicAdd(&hist[warp & (kCopies - 1)][(key >> shift) & digit_mask], 1);
        }
      }
      __syncthreads();
      // this CTA's counts per digit, and per 32 digits; thread t has digits 2 t, 2 t + 1
      {
        int2 c = make_int2(0, 0);
#pragma unroll
        for (int q = 0; q < kCopies; ++q) {
          const int2 v = *reinterpret_cast<const int2*>(&hist[q][2 * tid]);
          c.x += v.x;
          c.y += v.y;
        }
        *reinterpret_cast<int2*>(&folded[step][2 * tid]) = c;
        int both = c.x + c.y;
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) both += __shfl_xor_sync(0xffffffffu, both, o);
        if ((lane & 15) == 0) coarse[step][tid >> 4] = both;
      }
      cluster.sync();
      // From the largest digits down: the first warp finds the run of 32 digits that T lies in, then the digit.  (Adding
      // up all 2048 counts of eight peers took 5700 clocks a step.)
      if (warp == 0) {
        int c2[2] = {0, 0};                                        // runs 63 - 2 lane and 62 - 2 lane
        for (int p = 0; p < C; ++p) {
          const int2 v = *reinterpret_cast<const int2*>(cluster.map_shared_rank(&coarse[step][0], p) + 62 - 2 * lane);
          c2[0] += v.y;
          c2[1] += v.x;
        }
        int inc = c2[0] + c2[1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += u;
        }
        int before = inc - c2[0] - c2[1], run = -1, over = 0;      // `over`: rows in the runs above
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (before < left && before + c2[j] >= left) { run = 63 - 2 * lane - j; over = before; }
          before += c2[j];
        }
        const int src = __ffs(__ballot_sync(0xffffffffu, run >= 0)) - 1;
        run = __shfl_sync(0xffffffffu, run, src);
        over = __shfl_sync(0xffffffffu, over, src);
        int c = 0;                                                 // digit run * 32 + 31 - lane
        for (int p = 0; p < C; ++p) c += cluster.map_shared_rank(&folded[step][0], p)[run * 32 + 31 - lane];
        inc = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += u;
        }
        before = over + inc - c;
        if (before < left && before + c >= left) {
          s_digit = run * 32 + 31 - lane;
          s_left = left - before;
          s_equal = c;
        }
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
    before += __reduce_add_sync(0xffffffffu, lane < warp ? warp_tot[lane] : 0);
  }
  uint32_t* m = mask + (int64_t)h * row_words + mask_word_offset(start, r);
  auto words_at = [&](int q) {
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
  };
  int q = q0;
  if (search && staged && !ordered) {
    for (; q < q1 && q * 32 < i0; ++q) words_at(q);
    for (; q + 4 <= q1 && q * 32 + 128 <= i1; q += 4) {            // words of weighed rows only
      uint32_t bits[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) bits[j] = __ballot_sync(0xffffffffu, keys_sm[(q + j) * 32 + lane - i0] >= T);
      if (lane < 4) m[q + lane] = lane == 0 ? bits[0] : lane == 1 ? bits[1] : lane == 2 ? bits[2] : bits[3];
    }
  }
  for (; q < q1; ++q) words_at(q);
  if (rank == 0) {                                 // padding: words behind the request's last, or before the first request
    const int64_t at = mask_word_offset(start, r), end = r + 1 < (int)gridDim.z ? mask_word_offset(cu[r + 1], r + 1) : row_words;
    for (int64_t i = words + tid; i < end - at; i += kEvictThreads) m[i] = 0u;
    for (int64_t i = tid; r == 0 && i < at; i += kEvictThreads) m[i - at] = 0u;
    if (tid == 0) budget[r * Hkv + h] = k;
  }
  cluster.sync();                                  // the counts are read until here
}

}  // namespace

int32_t launch_evict(const gvote_params* p, const float* acc, const int32_t* cu, const int32_t* kv_len, int32_t batch,
                     int64_t total_tokens, int64_t max_N, const int32_t* keep, int32_t n_recent, uint32_t* mask,
                     int32_t* budget, cudaStream_t st) {
  int C = 8;
  while (C > 1 && (max_N / C < 2048 || (int64_t)batch * p->n_kv_heads * C > 148)) C >>= 1;
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
