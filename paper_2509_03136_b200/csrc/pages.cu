// Block tables and slot maps of the paged cache (gvote_page_tables), and rows into pages (gvote_page_write).
//
// Tables.  An entry is a (request, KV head); pages(x) = ceil(x / page_rows).
//   cut = min(kv_len, keep),  grown = cut + (new rows kept),  released = pages(kv_len) - pages(cut),  taken = pages(grown) - pages(cut)
// Released page k of K, in the order of entries and of rows, goes to free[n_free + K - 1 - k]; taken page k comes from
// free[n_free + K - 1 - k].  So what is cut next is what was grown last, and the stack is as it was.  Everything is one prefix
// sum over entries per direction, and what a thread does next is found by bisecting it: entries that need hundreds of pages
// and entries that need none cost the same per page.  The numbers of all pages that change hands are looked at before anything
// is written: one that names no page refuses the call.
//
// A few thousand integers: bound by latency.  So one CTA does all of a decode step between barriers (lengths and prefix sums;
// releases; takes; slots), and one cluster of eight where more pages or slots may change hands; each CTA of a cluster makes
// the prefix sums for itself and takes its share of the pages.  The slots of long prompts, one per token and head, are a kernel of
// their own, and with a keep-mask the kept rows are counted by one before.  Measured (one B200, in a graph): a step of 2048 heads 10.6
// us, of 4096 23.5, of 16384, whose lengths are read four times, 104; 15,000 pages released and as many taken, 490,000 slots under a mask,
// 15.8 us in three kernels.
#include <cooperative_groups.h>

#include "kv_rows.cuh"

namespace gvote {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanEach = 4;           // entries of a thread
constexpr int kPlanEntries = kPlanThreads * kPlanEach;   // held in shared memory; of more the lengths are read for every phase
constexpr int kHold = 4;               // pages that a thread keeps between looking at their numbers and passing them on
constexpr int kStepTokens = 8;         // new tokens of a request up to which a thread does an entry's slots
constexpr int kSlotLog2 = 10, kSlotTokens = 1 << kSlotLog2;      // tokens of a CTA of the slot kernel (4096: 8 us instead of 4)
constexpr int kSlotThreads = 256;

struct TableArgs {
  PageArgs p;
  const int32_t* keep;
  const int32_t* cu_new;
  const uint32_t* mask;
  int32_t* slots;                      // [Hkv][total_new], or null
  int32_t* counts;                     // [batch][Hkv] kept new rows, when there is a mask
  int32_t* refused;
  int32_t* status;
  int64_t total_new, mask_words;
  int slots_here;                      // the plan kernel writes the slots itself
  int max_new;
};

struct Change { int held, cut, grown; };
// What becomes of entry e; kv_len may be anything.
__device__ __forceinline__ Change change_of(const TableArgs& a, int64_t e) {
  const int64_t cap = (int64_t)a.p.max_pages << a.p.page_log2;
  Change c;
  const int v = a.p.kv_len[e];
  c.held = v < 0 ? 0 : (v < cap ? v : (int)cap);
  c.cut = a.keep ? min(c.held, max(a.keep[e], 0)) : c.held;
  const int r = (int)((uint32_t)e / (uint32_t)a.p.Hkv);
  int more = 0;
  if (a.cu_new) more = a.mask ? a.counts[e] : max(a.cu_new[r + 1] - a.cu_new[r], 0);
  const int64_t grown = (int64_t)c.cut + more;
  c.grown = grown > cap ? -1 : (int)grown;                       // -1: the table is too short
  return c;
}
__device__ __forceinline__ int pages_of(int rows, int log2) { return (rows + (1 << log2) - 1) >> log2; }
// The slot of a head's row; -1 where the table names no page (it has not come by this call: pages that change hands are looked at).
__device__ __forceinline__ int slot_of(const TableArgs& a, int64_t e, int row) {
  const int page = a.p.tables[e * a.p.max_pages + (row >> a.p.page_log2)];
  if ((uint32_t)page < (uint32_t)a.p.n_pages) return (page << a.p.page_log2) + (row & ((1 << a.p.page_log2) - 1));
  atomicExch(&a.status[0], GVOTE_ERR_INVALID_ARG);
  atomicExch(&a.status[1], 28);
  return -1;
}

// Inclusive sum over the CTA's threads.
__device__ __forceinline__ int scan_block(int x, int* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int s = lane < (int)(blockDim.x >> 5) ? warp_sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  return x + (warp ? warp_sums[warp - 1] : 0);
}
// The last i with first[i] <= k, 0 <= i < n (first ascending, first[0] <= k).
__device__ __forceinline__ int find_owner(const int* first, int n, int k) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= k) lo = mid; else hi = mid - 1;
  }
  return lo;
}
__device__ __forceinline__ int request_of(const int32_t* cu, int batch, int64_t t) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

struct PlanShared {
  int cut[kPlanEntries], grown[kPlanEntries];
  int gone[kPlanEntries], want[kPlanEntries];      // pages released, taken by the entries before
  int warp_sums[2][32];
  long long totals[2];
  int sums[2], too_long, no_page;
};

// Lengths and prefix sums of the entries e0 .. e0 + n - 1.
__device__ void plan_entries(const TableArgs& a, PlanShared& s, int64_t e0, int n, bool count) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, log2 = a.p.page_log2;
  int gone[kPlanEach], want[kPlanEach], all_gone = 0, all_want = 0;
  bool too_long = false;
#pragma unroll
  for (int q = 0; q < kPlanEach; ++q) {
    const int k = tid * kPlanEach + q;
    gone[q] = want[q] = 0;
    if (k < n) {
      const Change c = change_of(a, e0 + k);
      too_long |= c.grown < 0;
      s.cut[k] = c.cut;
      s.grown[k] = c.grown;
      gone[q] = pages_of(c.held, log2) - pages_of(c.cut, log2);
      want[q] = max(pages_of(c.grown, log2) - pages_of(c.cut, log2), 0);
    }
    all_gone += gone[q];
    all_want += want[q];
  }
  if (count) {
    const unsigned long long g = warp_sum_u64(all_gone), w = warp_sum_u64(all_want);
    if (lane == 0) {
      atomicAdd((unsigned long long*)&s.totals[0], g);
      atomicAdd((unsigned long long*)&s.totals[1], w);
    }
    if (too_long) s.too_long = 1;
  }
  int up_g = all_gone, up_w = all_want;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, up_g, o), z = __shfl_up_sync(0xffffffffu, up_w, o);
    if (lane >= o) { up_g += y; up_w += z; }
  }
  if (lane == 31) { s.warp_sums[0][warp] = up_g; s.warp_sums[1][warp] = up_w; }
  __syncthreads();
  if (warp < 2) {
    int x = s.warp_sums[warp][lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    s.warp_sums[warp][lane] = x;
    if (lane == 31) s.sums[warp] = x;
  }
  __syncthreads();
  int at_g = up_g - all_gone + (warp ? s.warp_sums[0][warp - 1] : 0), at_w = up_w - all_want + (warp ? s.warp_sums[1][warp - 1] : 0);
#pragma unroll
  for (int q = 0; q < kPlanEach; ++q) {
    const int k = tid * kPlanEach + q;
    if (k < n) { s.gone[k] = at_g; s.want[k] = at_w; }
    at_g += gone[q];
    at_w += want[q];
  }
  __syncthreads();
}

// kCluster: one cluster, else one CTA.
template <bool kCluster>
__global__ void __launch_bounds__(kPlanThreads, 1)
page_plan_kernel(const __grid_constant__ TableArgs a) {
  extern __shared__ __align__(16) uint8_t plan_smem[];
  PlanShared& s = *reinterpret_cast<PlanShared*>(plan_smem);
  const int tid = threadIdx.x, log2 = a.p.page_log2;
  const int64_t entries = (int64_t)a.p.batch * a.p.Hkv;
  const bool once = entries <= kPlanEntries;                     // what is read once stays in shared memory
  const int ctas = kCluster ? gridDim.x : 1, me = kCluster ? blockIdx.x : 0;
  if (tid == 0) { s.totals[0] = s.totals[1] = 0; s.too_long = s.no_page = 0; }
  __syncthreads();
  if (kCluster) cooperative_groups::this_cluster().barrier_arrive();       // (no_page is there for the others)
  ptx::let_next_begin();
  ptx::wait_for_previous();
  auto sync_all = [&] { if (kCluster) cooperative_groups::this_cluster().sync(); else __syncthreads(); };
  auto count_of = [&](int64_t e0) { return (int)min((int64_t)kPlanEntries, entries - e0); };
  // Where page k of those that the entries e0 .. e0 + n - 1 release or take stands in their tables (of entries that start at the same
  // place the last one has the pages).
  auto place_of = [&](const int* first, int64_t e0, int n, int k) {
    const int i = find_owner(first, n, k);
    return a.p.tables + (e0 + i) * a.p.max_pages + pages_of(s.cut[i], log2) + (k - first[i]);
  };
  const int k0 = me * kPlanThreads + tid, stride = ctas * kPlanThreads;

  // sums and checks
  const int n_free = *a.p.n_free;
  bool none = false;                                             // a number that names no page
  auto look = [&](int page) { none |= (uint32_t)page >= (uint32_t)a.p.n_pages; };
  for (int64_t e0 = 0; e0 < entries; e0 += kPlanEntries) {
    plan_entries(a, s, e0, count_of(e0), true);
    if (once) break;
    if (s.totals[0] <= a.p.n_pages)                              // (else the call is refused, and the prefix sums may have wrapped)
      for (int k = k0; k < s.sums[0]; k += stride) look(*place_of(s.gone, e0, count_of(e0), k));
    __syncthreads();
  }
  const long long K = s.totals[0], T = s.totals[1];
  const bool bad = n_free < 0 || n_free > a.p.n_pages || n_free + K > a.p.n_pages;
  bool refuse = bad || s.too_long || T > n_free + K;
  const int top = (int)(n_free + K), most = (int)max(K, T);     // (of a call that is not refused)
  // The k-th page taken lies where the k-th released one went.  So of the first kHold * stride a thread reads page k where it is, and
  // after the barrier it goes to the stack and to the table that takes it (a step 11.3 -> 10.5 us against by way of the stack).
  int page[kHold];
  int32_t* place[kHold];
  if (once && !refuse) {
#pragma unroll
    for (int u = 0; u < kHold; ++u) {
      const int k = k0 + u * stride;
      if (k >= most) break;
      page[u] = k < K ? *place_of(s.gone, 0, (int)entries, k) : a.p.free_pages[top - 1 - k];
      if (k < T) place[u] = place_of(s.want, 0, (int)entries, k);
      look(page[u]);
    }
    for (int k = k0 + kHold * stride; k < most; k += stride)
      look(k < K ? *place_of(s.gone, 0, (int)entries, k) : a.p.free_pages[top - 1 - k]);
  } else if (!refuse) {
    for (int k = (int)K + k0; k < T; k += stride) look(a.p.free_pages[top - 1 - k]);
  }
  if (kCluster) cooperative_groups::this_cluster().barrier_wait();
  if (none)
    for (int c = 0; c < ctas; ++c) *(kCluster ? cooperative_groups::this_cluster().map_shared_rank(&s.no_page, c) : &s.no_page) = 1;
  sync_all();                                                    // every CTA has read n_free, the lengths and the pages
  refuse |= s.no_page != 0;
  const int64_t n_slots = a.total_new * a.p.Hkv;
  if (refuse) {
    if (me == 0 && tid == 0) {
      *a.refused = 1;
      atomicExch(&a.status[0], bad || s.no_page ? GVOTE_ERR_INVALID_ARG : GVOTE_ERR_WORKSPACE_TOO_SMALL);
      atomicExch(&a.status[1], 20);
    }
    if (a.slots_here)
      for (int64_t i = k0; i < n_slots; i += stride) a.slots[i] = -1;
    return;
  }
  if (me == 0 && tid == 0) *a.refused = 0;

  // releases, then takes
  if (once) {
    const int from = k0 + kHold * stride;
    if (most > kHold * stride) {                                 // the others by way of the stack
      for (int k = from; k < K; k += stride) a.p.free_pages[top - 1 - k] = *place_of(s.gone, 0, (int)entries, k);
      sync_all();
    }
#pragma unroll
    for (int u = 0; u < kHold; ++u) {
      const int k = k0 + u * stride;
      if (k < K) a.p.free_pages[top - 1 - k] = page[u];
      if (k < T) *place[u] = page[u];
    }
    for (int k = from; k < T; k += stride) *place_of(s.want, 0, (int)entries, k) = a.p.free_pages[top - 1 - k];
    sync_all();
  }
#pragma unroll 1
  for (int take = 0; take < 2 && !once; ++take) {
    int before = 0;
    for (int64_t e0 = 0; e0 < entries && (take ? T : K) > 0; e0 += kPlanEntries) {
      const int n = count_of(e0);
      plan_entries(a, s, e0, n, false);
      const int all = s.sums[take];
      for (int k = k0; k < all; k += stride) {
        int32_t* at = place_of(take ? s.want : s.gone, e0, n, k);
        int32_t* stack = a.p.free_pages + (top - 1 - before - k);
        if (take) *at = *stack; else *stack = *at;
      }
      before += all;
      __syncthreads();
    }
    sync_all();
  }

  // the slots where they are few, then the lengths
  if (a.slots_here) {
    if (a.max_new <= kStepTokens) {
      for (int64_t e = k0; e < entries; e += stride) {
        const int r = (int)((uint32_t)e / (uint32_t)a.p.Hkv), h = (int)(e - (int64_t)r * a.p.Hkv);
        const int from = a.cu_new[r], to = a.cu_new[r + 1], cut = once ? s.cut[e] : change_of(a, e).cut;
        for (int t = from; t < to; ++t) a.slots[h * a.total_new + t] = slot_of(a, e, cut + t - from);
      }
      const int64_t lead = a.cu_new[0], tail = a.cu_new[a.p.batch];            // tokens of no request
      for (int64_t i = k0; i < (lead + a.total_new - tail) * a.p.Hkv; i += stride) {
        const int64_t t = i / a.p.Hkv;
        a.slots[(i - t * a.p.Hkv) * a.total_new + (t < lead ? t : tail + t - lead)] = -1;
      }
    } else {
      for (int64_t i = k0; i < n_slots; i += stride) {
        const int h = (int)(i / a.total_new);
        const int64_t t = i - h * a.total_new;
        const int r = request_of(a.cu_new, a.p.batch, t);
        const int64_t e = (int64_t)r * a.p.Hkv + h;
        int slot = -1;
        if (t >= a.cu_new[r] && t < a.cu_new[r + 1])
          slot = slot_of(a, e, (once ? s.cut[e] : change_of(a, e).cut) + (int)(t - a.cu_new[r]));
        a.slots[i] = slot;
      }
    }
    if (!once) sync_all();                                       // (the lengths have been read again)
  }
  if (me == 0) {
    for (int64_t e = tid; e < entries; e += kPlanThreads) a.p.kv_len[e] = once ? s.grown[e] : change_of(a, e).grown;
    if (tid == 0) *a.p.n_free = (int)(top - T);
  }
}

// Kept new rows of every entry.
__global__ void __launch_bounds__(kSlotThreads)
page_count_kernel(const __grid_constant__ TableArgs a) {
  __shared__ int part[kSlotThreads / 32];
  const int h = blockIdx.x, r = blockIdx.y;
  ptx::let_next_begin();
  ptx::wait_for_previous();
  const int start = a.cu_new[r], n = a.cu_new[r + 1] - start;
  const uint32_t* words = a.mask + (int64_t)h * a.mask_words + mask_word_offset(start, r);
  int sum = 0;
  for (int w = threadIdx.x; w * 32 < n; w += kSlotThreads) {
    const uint32_t in = n - w * 32 >= 32 ? 0xffffffffu : (1u << (n - w * 32)) - 1;
    sum += __popc(words[w] & in);
  }
  sum = warp_sum_i(sum);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kSlotThreads / 32; ++i) sum += part[i];
    a.counts[(int64_t)r * a.p.Hkv + h] = sum;
  }
}

// The slots of kSlotTokens tokens of one request and head (kv_len is the new length by now).
__global__ void __launch_bounds__(kSlotThreads)
page_slots_kernel(const __grid_constant__ TableArgs a) {
  __shared__ int warp_sums[32];
  __shared__ int rank_of[kSlotTokens / 32];
  const int h = blockIdx.y, tid = threadIdx.x;
  const int64_t g = blockIdx.x;
  ptx::let_next_begin();
  ptx::wait_for_previous();
  // tile g of a list with (cu[r] >> kSlotLog2) + r as the first of request r
  int lo = 0, hi = a.p.batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)(a.cu_new[mid] >> kSlotLog2) + mid <= g) lo = mid; else hi = mid - 1;
  }
  const int r = lo, start = a.cu_new[r], n = a.cu_new[r + 1] - start;
  const int64_t t0 = (g - ((start >> kSlotLog2) + r)) * kSlotTokens;
  // tokens of no request
  if (g == 0)
    for (int64_t i = tid; i < a.cu_new[0]; i += kSlotThreads) a.slots[(int64_t)h * a.total_new + i] = -1;
  if (g == (int64_t)gridDim.x - 1)
    for (int64_t i = a.cu_new[a.p.batch] + tid; i < a.total_new; i += kSlotThreads) a.slots[(int64_t)h * a.total_new + i] = -1;
  if (t0 < 0 || t0 >= n) return;
  const int64_t e = (int64_t)r * a.p.Hkv + h;
  const int here = (int)min((int64_t)kSlotTokens, n - t0);
  int32_t* out = a.slots + (int64_t)h * a.total_new + start + t0;
  if (*a.refused) {
    for (int i = tid; i < here; i += kSlotThreads) out[i] = -1;
    return;
  }
  const uint32_t* words = nullptr;
  int cut;
  if (a.mask) {
    words = a.mask + (int64_t)h * a.mask_words + mask_word_offset(start, r);
    int before = 0;
    for (int w = tid; w < (int)(t0 >> 5); w += kSlotThreads) before += __popc(words[w]);
    words += t0 >> 5;
    const int mine = tid * 32 < here ? __popc(words[tid]) : 0;
    scan_block(before, warp_sums);
    before = warp_sums[kSlotThreads / 32 - 1];
    __syncthreads();
    const int sum = scan_block(mine, warp_sums);
    if (tid < kSlotTokens / 32) rank_of[tid] = before + sum - mine;
    cut = a.p.kv_len[e] - a.counts[e];
    __syncthreads();
  } else {
    cut = a.p.kv_len[e] - n;
  }
  for (int i = tid; i < here; i += kSlotThreads) {
    int row = cut;
    if (a.mask) {
      const uint32_t w = words[i >> 5];
      if (!((w >> (i & 31)) & 1u)) { out[i] = -1; continue; }
      row += rank_of[i >> 5] + __popc(w & ((1u << (i & 31)) - 1));
    } else {
      row += (int)t0 + i;
    }
    out[i] = slot_of(a, e, row);
  }
}

// ---------------------------------------------------------------------------------- rows into pages
// Copies 4 d_k bytes per kept row: bound by memory.  A warp takes 32 slots, and for those that are kept as many lanes per row as
// it has 16-byte pieces; kWriteUnroll rows of K and V per lane are asked for before the first is stored.  Measured: 164 MB (52 % of
// 32K rows of 8 heads) 28.2 us, 5.8 TB/s; one row of 64 requests 4.8 us in a graph.
constexpr int kWriteThreads = 128;
constexpr int kWriteUnroll = 8;

__global__ void __launch_bounds__(kWriteThreads)
page_write_kernel(const __nv_bfloat16* __restrict__ K, const __nv_bfloat16* __restrict__ V, int64_t tok, int64_t head,
                  const int32_t* __restrict__ slots, int64_t total, __nv_bfloat16* K_out, __nv_bfloat16* V_out, int64_t row_stride,
                  int64_t page_stride, int page_log2, int64_t n_slots, int pieces, int lanes_log2, int32_t* status) {
  const int lane = threadIdx.x & 31, h = blockIdx.y;
  const int64_t t0 = ((int64_t)blockIdx.x * (kWriteThreads / 32) + (threadIdx.x >> 5)) * 32;
  ptx::let_next_begin();
  ptx::wait_for_previous();
  if (t0 >= total) return;
  const int slot = t0 + lane < total ? slots[h * total + t0 + lane] : -1;
  const bool is_bad = (int64_t)slot >= n_slots;
  uint32_t todo = __ballot_sync(0xffffffffu, slot >= 0 && !is_bad);
  if (__any_sync(0xffffffffu, is_bad) && lane == 0) {
    atomicExch(&status[0], GVOTE_ERR_INVALID_ARG);
    atomicExch(&status[1], 21);
  }
  const int per = 32 >> lanes_log2, mine = lane >> lanes_log2, piece = lane & ((1 << lanes_log2) - 1);
  const int64_t from0 = (int64_t)h * head + t0 * tok + piece * 8;
  while (todo) {
    uint4 k[kWriteUnroll], v[kWriteUnroll];
    int64_t to[kWriteUnroll];
#pragma unroll
    for (int u = 0; u < kWriteUnroll; ++u) {
      uint32_t rest = todo;
      for (int i = 0; i < mine; ++i) rest &= rest - 1;
      const int j = __ffs(rest) - 1;                             // the lane that holds this lane's row
      const int s = __shfl_sync(0xffffffffu, slot, j & 31);
      to[u] = -1;
      if (j >= 0 && piece < pieces) {
        k[u] = __ldg(reinterpret_cast<const uint4*>(K + from0 + j * tok));
        v[u] = __ldg(reinterpret_cast<const uint4*>(V + from0 + j * tok));
        to[u] = (int64_t)(s >> page_log2) * page_stride + (s & ((1 << page_log2) - 1)) * row_stride + piece * 8;
      }
      for (int i = 0; i < per && todo; ++i) todo &= todo - 1;
    }
#pragma unroll
    for (int u = 0; u < kWriteUnroll; ++u)
      if (to[u] >= 0) {
        *reinterpret_cast<uint4*>(K_out + to[u]) = k[u];
        *reinterpret_cast<uint4*>(V_out + to[u]) = v[u];
      }
  }
}

}  // namespace

PageMap page_map(const gvote_params* p, int32_t batch) {
  PageMap m;
  m.refused = kScratchAt;
  m.counts = kScratchAt + 256;
  m.total = m.counts + align_up((size_t)batch * p->n_kv_heads * 4, 256);
  return m;
}

int32_t launch_page_tables(const PageArgs& p, const int32_t* keep, const int32_t* cu_new, int64_t total_new, int64_t max_new,
                           const uint32_t* mask, int32_t* slots, const PageMap& m, char* ws, cudaStream_t st) {
  TableArgs a;
  a.p = p; a.keep = keep; a.cu_new = cu_new; a.mask = mask; a.slots = slots; a.total_new = total_new;
  a.mask_words = gvote_mask_row_words(total_new, p.batch);
  a.counts = reinterpret_cast<int32_t*>(ws + m.counts);
  a.refused = reinterpret_cast<int32_t*>(ws + m.refused);
  a.status = reinterpret_cast<int32_t*>(ws);
  const int64_t entries = (int64_t)p.batch * p.Hkv, n_slots = slots ? total_new * p.Hkv : 0;
  a.max_new = (int)max_new;
  a.slots_here = n_slots > 0 && !mask && n_slots <= 8 * 1024 ? 1 : 0;
  if (mask) {
    LaunchScope scope_("page_count_kernel", st);
    (void)launch_behind(page_count_kernel, dim3(p.Hkv, p.batch), dim3(kSlotThreads), 0, st, a);
    GVOTE_LAUNCH_CHECK("page_count_kernel");
  }
  {
    const int ctas = entries <= kPlanEntries && !mask && n_slots <= 8 * 1024 ? 1 : 8;
    auto kernel = ctas > 1 ? page_plan_kernel<true> : page_plan_kernel<false>;
    GVOTE_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PlanShared)));
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kPlanThreads);
    cfg.dynamicSmemBytes = sizeof(PlanShared);
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    LaunchScope scope_("page_plan_kernel", st);
    (void)cudaLaunchKernelEx(&cfg, kernel, a);
  }
  GVOTE_LAUNCH_CHECK("page_plan_kernel");
  if (n_slots > 0 && !a.slots_here) {
    LaunchScope scope_("page_slots_kernel", st);
    (void)launch_behind(page_slots_kernel, dim3((unsigned)((total_new >> kSlotLog2) + p.batch), p.Hkv), dim3(kSlotThreads), 0, st, a);
    GVOTE_LAUNCH_CHECK("page_slots_kernel");
  }
  return GVOTE_OK;
}

int32_t launch_page_write(const gvote_params* p, const __nv_bfloat16* K, const __nv_bfloat16* V, int64_t tok, int64_t head,
                          const int32_t* slots, int64_t total_new, __nv_bfloat16* K_out, __nv_bfloat16* V_out, int64_t row_stride,
                          int64_t page_stride, int32_t page_log2, int64_t n_slots, int32_t* status, cudaStream_t st) {
  if (total_new == 0) return GVOTE_OK;
  const int pieces = p->d_k / 8;
  int lanes_log2 = 1;
  while ((1 << lanes_log2) < pieces) ++lanes_log2;
  LaunchScope scope_("page_write_kernel", st);
  (void)launch_behind(page_write_kernel, dim3((unsigned)ceil_div(total_new, kWriteThreads), p->n_kv_heads), dim3(kWriteThreads), 0, st,
                  K, V, tok, head, slots, total_new, K_out, V_out, row_stride, page_stride, page_log2, n_slots, pieces, lanes_log2,
                  status);
  GVOTE_LAUNCH_CHECK("page_write_kernel");
  return GVOTE_OK;
}

}  // namespace gvote
