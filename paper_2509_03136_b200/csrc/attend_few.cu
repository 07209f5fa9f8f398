// Attention of a token or a few over bf16 rows in pages or slabs (gvote_page_attend, gvote_attend).
//
//   l_j = (q.k_j) / sqrt(d_k),  out = sum_j exp(l_j - lse) v_j,  lse = log sum_j exp(l_j)
// with few query rows (tokens x query heads of a KV head) against many cached rows: bound by reading K and V once, 4 d_k bytes per
// cached row.
//
// Split.  The rows of all (request, KV head) pairs ("entries") are cut into tiles of 64 and laid end to end, each entry behind
// kGap tiles for what beginning and ending one costs (about that many tiles' time; a ragged batch took a tenth longer with
// one); CTA b of B takes the tiles from T b / B to T (b + 1) / B of the T places.  So heads of very different length load every
// SM alike, and the lengths stay on the device.  What a CTA has of an entry is a segment.  An
// entry within one CTA goes straight to the output; of the others every segment leaves its reference, sum and output in slot
// entry + CTA, and of kFan neighbouring segments the CTA that arrives last at their counter adds them up in their order, then
// of up to kFan such sums.  So the result does not depend on which CTA that is, and the 74 segments of a long row are not one
// CTA's work (one after the other they took 36 of 81 us).
//
// A CTA: four warps that compute and one that asks for tiles (TMA, 128-byte swizzle, boxes of a page or of 64 rows) into a ring
// of units, K and V of a tile one unit each.  The products are mma.sync m16n8k16 with the query rows on M, 16 of them
// to a group: the tensor work fits under the memory time, and this shape lets a warp keep its 16 cached rows
// of a tile to itself: its own reference, sum and output in registers, no barrier within a segment.  Weights are held as a sum of
// two bf16 terms (16 bits; the outputs have 8), of up to eight rows both in one product; all else in 32 bits.  A reference moves only when a logit passes it by 2^8.
// (A second group of 16 rows in the same CTA was no gain: mma.sync then takes 6000 clocks a tile.)
//
// Measured (one B200): one token of 28 heads over 128K rows of 4 KV heads, 268 MB, 57.5 us: the first tile is there after 5.3 us, the
// last after 41 (7.2 TB/s between them), then the warps' results meet (1.4) and two rounds of joins.  A ragged batch of 128 pruned heads, 131
// MB, 31 us.  The smallest call 9 us in a graph.
//
// Rows that not every token of a group sees, and rows behind the last one, may hold anything: logits are masked by index, values
// that are not finite are taken out of the tile (0 * inf is no number) and added back to the outputs of the tokens that see them.
//
// Every wait is bounded by the time without any work done (kv_rows.cuh); when one runs out GVOTE_ERR_TIMEOUT is recorded and the outputs are not to be used.
#include "kv_rows.cuh"

namespace gvote {
namespace {

constexpr int kTileKeys = 64;
constexpr int kWarps = 4;                       // that compute
constexpr int kThreads = 32 * (kWarps + 1);
constexpr int kRows = 16;                       // query rows of a group
constexpr int kMaxUnits = 8;
constexpr int kGap = 4;
constexpr int kFan = 18;                        // two rounds join every segment of a launch
static_assert(kFan * kFan >= kFewCtas, "");
constexpr float kSlack = 8.f;

struct FewArgs {
  RowSource src;
  const __nv_bfloat16* Q;
  int64_t q_tok, q_head;
  const int32_t* cu_q;
  __nv_bfloat16* out;
  int64_t o_tok, o_head;
  float* lse;            // or null
  float* part_o;         // [groups][entries + CTAs][rows of a group][d_k]
  float2* part_ml;       // [groups][entries + CTAs][rows of a group]
  int32_t* arrived;      // [groups][kFewEntries + kFewCtas: first rounds, by slot][kFewEntries: second rounds], zero between calls
  int32_t* status;
  int Hq, Hkv, G, r0, batch, d_k, max_q;        // requests r0 .. r0 + batch - 1
  int group0, box_rows;                         // this launch's first group of query rows
  int one_group;
  float scale2;          // log2(e) / sqrt(d_k)
};

struct Entry { int r, h, n, nq, q0; };
// n: cached rows the group's last token sees
__device__ __forceinline__ Entry entry_of(const FewArgs& a, int e, int group_last) {
  Entry x;
  const int lr = e / a.Hkv;
  x.h = e - lr * a.Hkv;
  x.r = a.r0 + lr;
  x.q0 = a.cu_q[x.r];
  x.nq = min(a.cu_q[x.r + 1] - x.q0, a.max_q);
  const int last = min(group_last / a.G, x.nq - 1);
  x.n = max(rows_held(a.src, x.r, x.h, a.Hkv) - (x.nq - 1 - last), 0);
  return x;
}

struct Bars {
  uint64_t full[kMaxUnits], empty[kMaxUnits], q_full[2], q_empty[2];
};
struct Tail {
  Bars bars;
  Watch watch;
  int last_one;
  int odd;                                      // bit 0: values that are not finite were taken out; bit 1: outputs are not finite
  alignas(16) float none[kMaxHeadDim];          // what the values of rows that all see add up to, where they are not finite
  float2 join[kFan][kRows];                        // references and sums of the segments that are joined
  int warp_sums[kThreads / 32];
  float2 ml[kWarps][kRows];
  int pref[kFewEntries + 1];
};

template <int kBoxes>                           // 64-channel boxes of a row
struct Layout {
  static constexpr int kUnit = kBoxes * kTileKeys * 128;
  static constexpr int kQPitch = kBoxes * 128 + 16;                   // bytes
  static constexpr int kQ = kRows * kQPitch;
  static constexpr int kSumPitch = kBoxes * 64 + 8;                   // floats
  static constexpr int kSum = kRows * kSumPitch * 4;
  static constexpr bool kTwo = kBoxes <= 2;                           // two CTAs per SM
  static constexpr size_t fixed() { return (size_t)2 * kQ + 2 * kSum + sizeof(Tail); }
  static constexpr int kFit = (int)(((kTwo ? 112 : 226) * 1024 - fixed()) / kUnit);
  static constexpr int kUnits = kFit < kMaxUnits ? kFit : kMaxUnits;
  static constexpr size_t smem() { return fixed() + (size_t)kUnits * kUnit; }
  static_assert(kUnits >= 4, "the ring is too short");
};

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The tiles of a CTA in order, segment by segment (entry e, its tiles s0 .. s1 - 1).
struct Walk {
  int e, s0, s1;
  const int* pref;
  int t0, t1, entries;
  __device__ __forceinline__ Walk(const int* pref_, int t0_, int t1_, int entries_)
      : pref(pref_), t0(t0_), t1(t1_), entries(entries_) {
    int lo = 0, hi = entries - 1;               // the last entry that begins at or before t0
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (pref[mid] <= t0) lo = mid; else hi = mid - 1;
    }
    e = lo;
    enter();
  }
  __device__ __forceinline__ bool done() const { return e >= entries; }
  __device__ __forceinline__ void enter() {
    for (; e < entries; ++e) {
      const int p = pref[e];
      if (p >= t1) break;
      s0 = max(t0 - p - kGap, 0);
      s1 = min(t1, pref[e + 1]) - p - kGap;
      if (s0 < s1) return;
    }
    e = entries;
  }
  __device__ __forceinline__ void next() { ++e; enter(); }
};

template <int kBoxes>
__global__ void __launch_bounds__(kThreads, Layout<kBoxes>::kTwo ? 2 : 1)
attend_few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ FewArgs a) {
  using L = Layout<kBoxes>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* ring = smem;                                            // [unit][box][64 rows][128], swizzled
  uint8_t* q_sm = ring + (size_t)L::kUnits * L::kUnit;             // [2][rows][pitch]
  float* sum_sm = reinterpret_cast<float*>(q_sm + 2 * L::kQ);      // [2][rows][pitch]
  Tail* tail = reinterpret_cast<Tail*>(sum_sm + 2 * kRows * L::kSumPitch);
  int* pref = tail->pref;
  Watch* watch = &tail->watch;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int entries = a.batch * a.Hkv;
  const int row0 = (a.group0 + blockIdx.y) * kRows, row_last = row0 + kRows - 1;   // query rows of this group
  const int boxes = (a.d_k + 63) >> 6, ksteps = a.d_k >> 4;

  if (tid < (int)(sizeof(Bars) / 8)) {
    const bool by_warps = (tid >= kMaxUnits && tid < 2 * kMaxUnits) || tid >= 2 * kMaxUnits + 2;   // empty, q_empty
    ptx::mbar_init(reinterpret_cast<uint64_t*>(&tail->bars) + tid, by_warps ? kWarps : 1);
    ptx::fence_barrier_init();
  }
  if (tid == 0) {
    tail->watch.stop = (ptx::smem_u32(smem) & 1023u) ? 1 : 0;
    tail->watch.work = 0;
    tail->odd = 0;
    ptx::prefetch_tensormap(&tmK);
    ptx::prefetch_tensormap(&tmV);
  }
  // channels of Q behind d_k, and query rows of no token, are zero
  for (uint4* q = reinterpret_cast<uint4*>(q_sm) + tid; q < reinterpret_cast<uint4*>(sum_sm); q += kThreads) *q = make_uint4(0, 0, 0, 0);
  ptx::fence_proxy_async();
  ptx::let_next_begin();
  ptx::wait_for_previous();
  // places before each entry
  {
    const int per = (entries + kThreads - 1) / kThreads, e0 = min(tid * per, entries), e1 = min(e0 + per, entries);
    int sum = 0;
    for (int e = e0; e < e1; ++e) {
      const Entry x = entry_of(a, e, row_last);
      const int places = x.nq * a.G > row0 && x.n > 0 ? (x.n + kTileKeys - 1) / kTileKeys + kGap : 0;
      pref[e + 1] = places;
      sum += places;
      if (blockIdx.x == 0 && row0 == 0 && a.cu_q[x.r + 1] - x.q0 > a.max_q) {
        atomicExch(&a.status[0], GVOTE_ERR_INVALID_ARG);
        atomicExch(&a.status[1], 22);
      }
    }
    int up = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, up, o);
      if (lane >= o) up += y;
    }
    if (lane == 31) tail->warp_sums[warp] = up;
    __syncthreads();
    int at = up - sum;
    for (int w = 0; w < warp; ++w) at += tail->warp_sums[w];
    if (tid == 0) pref[0] = 0;
    for (int e = e0; e < e1; ++e) { at += pref[e + 1]; pref[e + 1] = at; }
    __syncthreads();
  }
  const int T = pref[entries];
  const int B = min((int)gridDim.x, T);                            // (every CTA below B has a place)
  const int b = blockIdx.x;
  const int t0 = b < B ? (int)((int64_t)T * b / B) : 0, t1 = b < B ? (int)((int64_t)T * (b + 1) / B) : 0;

  if (warp == kWarps) {
    // ------------------------------------------------------------------ asks for tiles
    // Rows that no other group reads (a ragged batch 32.7 -> 31.2 us).  Those of pages that requests share are read by several
    // all the same, and may come out of memory once more.
    const uint64_t policy = ptx::l2_policy_evict_first();
    uint32_t unit = 0;
    int seg = 0;
    bool ok = true, bad_page = false;
    for (Walk w(pref, t0, t1, entries); ok && !w.done(); w.next(), ++seg) {
      const Entry x = entry_of(a, w.e, row_last);
      const int rows = min(x.nq * a.G - row0, kRows);
      ok = __all_sync(0xffffffffu, wait_or_stop(&tail->bars.q_empty[seg & 1], ((seg >> 1) & 1) ^ 1, watch));
      if (!ok) break;
      if (lane == 0) ptx::mbar_arrive_expect_tx(&tail->bars.q_full[seg & 1], (uint32_t)(rows * a.d_k * 2));
      __syncwarp();
      if (lane < rows) {
        const int row = row0 + lane, token = row / a.G, g = row - token * a.G;
        ptx::bulk_load(q_sm + (seg & 1) * L::kQ + lane * L::kQPitch,
                       a.Q + (int64_t)(x.q0 + token) * a.q_tok + (int64_t)(x.h * a.G + g) * a.q_head, (uint32_t)(a.d_k * 2),
                       &tail->bars.q_full[seg & 1]);
      }
      const int32_t* table = a.src.tables ? a.src.tables + ((int64_t)x.r * a.Hkv + x.h) * a.src.max_pages : nullptr;
      const int in_page = (1 << a.src.page_log2) - 1;
      const int start = table ? 0 : a.src.cu[x.r];
      const int box = lane % boxes, part = lane / boxes;           // this lane's box of a tile: channels, rows
      int j = w.s0 * kTileKeys + part * a.box_rows;                // its first row
      int page = 0;
      if (table && j < x.n && part * a.box_rows < kTileKeys) page = table[j >> a.src.page_log2];
      for (int t = w.s0; t < w.s1; ++t, j += kTileKeys) {
        const int here = min(x.n - t * kTileKeys, kTileKeys), parts = (here + a.box_rows - 1) / a.box_rows;
        const bool mine = part < parts;
        int next = 0;
        if (table && t + 1 < w.s1 && part * a.box_rows < kTileKeys && j + kTileKeys < x.n) next = table[(j + kTileKeys) >> a.src.page_log2];
        const int cy = table ? (j & in_page) : start + j, cz = table ? page : x.h;
        if (table && mine && (uint32_t)page >= (uint32_t)a.src.n_pages) bad_page = true;   // (the copy reads zeros)
#pragma unroll
        for (int v = 0; v < 2; ++v, ++unit) {
          const uint32_t s = unit % L::kUnits;
          ok = ok && __all_sync(0xffffffffu, wait_or_stop(&tail->bars.empty[s], ((unit / L::kUnits) & 1) ^ 1, watch));
          if (!ok) break;
          if (lane == 0) ptx::mbar_arrive_expect_tx(&tail->bars.full[s], (uint32_t)(parts * boxes * a.box_rows * 128));
          __syncwarp();
          uint8_t* to = ring + (size_t)s * L::kUnit + box * (kTileKeys * 128) + part * a.box_rows * 128;
          if (mine && a.one_group) ptx::tma_load_3d_hint(to, v ? &tmV : &tmK, &tail->bars.full[s], box * 64, cy, cz, policy);
          else if (mine) ptx::tma_load_3d(to, v ? &tmV : &tmK, &tail->bars.full[s], box * 64, cy, cz);
        }
        if (!ok) break;
        page = next;
      }
    }
    if (__any_sync(0xffffffffu, bad_page) && lane == 0) {
      atomicExch(&a.status[0], GVOTE_ERR_INVALID_ARG);
      atomicExch(&a.status[1], 23);
    }
    if (!ok) {
      await_loads(tail->bars.full, L::kUnits, unit);
      await_loads(tail->bars.q_full, 2, (uint32_t)seg);
    }
  } else {
    // ------------------------------------------------------------------ computes
    const int64_t slot0 = (int64_t)blockIdx.y * (entries + gridDim.x);
    uint32_t unit = 0;
    int seg = 0;
    bool ok = true;
    // tokens that see nothing of an entry without places
    for (int e = b; e < entries; e += gridDim.x) {
      if (pref[e + 1] > pref[e]) continue;
      const Entry x = entry_of(a, e, row_last);
      const int rows = min(x.nq * a.G - row0, kRows);
      for (int i = tid; i < rows * (a.d_k >> 3); i += 32 * kWarps) {
        const int lr = i / (a.d_k >> 3), c = i - lr * (a.d_k >> 3), row = row0 + lr, token = row / a.G, head = x.h * a.G + row - token * a.G;
        *reinterpret_cast<uint4*>(a.out + (int64_t)(x.q0 + token) * a.o_tok + (int64_t)head * a.o_head + c * 8) = make_uint4(0, 0, 0, 0);
        if (a.lse && c == 0) a.lse[(int64_t)(x.q0 + token) * a.Hq + head] = -INFINITY;
      }
    }
    for (Walk w(pref, t0, t1, entries); !w.done(); w.next(), ++seg) {
      const Entry x = entry_of(a, w.e, row_last);
      const int rows = min(x.nq * a.G - row0, kRows);
      const int all_see = x.n - (min(row_last / a.G, x.nq - 1) - row0 / a.G);   // rows that every token of the group sees
      const bool packed = rows <= 8;                               // rows 8 to 15 of the product with V are the weights' second terms
      int limit[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int lr = i * 8 + (lane >> 2);
        limit[i] = lr < rows ? all_see + (row0 + lr) / a.G - row0 / a.G : 0;
      }
      float o[kBoxes * 8][4], ref[2], sum[2];
      ref[0] = ref[1] = -INFINITY;
      sum[0] = sum[1] = 0.f;
#pragma unroll
      for (int i = 0; i < kBoxes * 8; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[i][k] = 0.f;
      ok = ok && __all_sync(0xffffffffu, wait_or_stop(&tail->bars.q_full[seg & 1], (seg >> 1) & 1, watch));
      const uint32_t q_addr = ptx::smem_u32(q_sm) + (seg & 1) * L::kQ + ((lane & 15)) * L::kQPitch + (lane >> 4) * 16;
      const int key = 16 * warp;                                   // this warp's rows of a tile
      const uint32_t k_row = key + ((lane >> 4) << 3) + (lane & 7), k_half = (lane >> 3) & 1;
      const uint32_t v_row = key + (((lane >> 3) & 1) << 3) + (lane & 7), v_half = lane >> 4;
      for (int t = w.s0; ok && t < w.s1; ++t) {
        uint32_t s = unit % L::kUnits;
        ok = __all_sync(0xffffffffu, wait_or_stop(&tail->bars.full[s], (unit / L::kUnits) & 1, watch));
        if (!ok) break;
        float l[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) l[i][k] = 0.f;
        const uint32_t k_addr = ptx::smem_u32(ring) + s * L::kUnit + k_row * 128;
#pragma unroll
        for (int c = 0; c < kBoxes * 4; ++c) {
          if (c < ksteps) {
            uint32_t kf[4];
            ldmatrix4(kf, k_addr + (c >> 2) * (kTileKeys * 128) + (((((uint32_t)c & 3) * 2 + k_half) ^ (k_row & 7)) << 4));
            uint32_t qf[4];
            ldmatrix4(qf, q_addr + c * 32);
            mma(l[0], qf, kf[0], kf[1]);
            mma(l[1], qf, kf[2], kf[3]);
          }
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&tail->bars.empty[s]);
        ++unit;
        // weights
        uint32_t hi[4], lo[4];
        const int j0 = t * kTileKeys + key + (lane & 3) * 2;       // this lane's columns: j0, j0 + 1, j0 + 8, j0 + 9
        const bool masked = (t + 1) * kTileKeys > all_see;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (i == 1 && packed) {
            hi[1] = lo[0];
            hi[3] = lo[2];
            break;
          }
          float* p[4] = {&l[0][2 * i], &l[0][2 * i + 1], &l[1][2 * i], &l[1][2 * i + 1]};
          if (masked) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (j0 + (k >> 1) * 8 + (k & 1) >= limit[i]) *p[k] = -INFINITY;
          }
          float top = fmaxf(fmaxf(*p[0], *p[1]), fmaxf(*p[2], *p[3]));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)) * a.scale2;
          const bool move = top > ref[i] + kSlack;
          if (__any_sync(0xffffffffu, move)) {
            const float f = move ? exp2_approx(ref[i] - top) : 1.f;
            if (move) ref[i] = top;
            sum[i] *= f;
#pragma unroll
            for (int n = 0; n < kBoxes * 8; ++n) { o[n][2 * i] *= f; o[n][2 * i + 1] *= f; }
            if (packed) {
#pragma unroll
              for (int n = 0; n < kBoxes * 8; ++n) { o[n][2] *= f; o[n][3] *= f; }
            }
          }
          const float off = ref[i] == -INFINITY ? 0.f : ref[i];
#pragma unroll
          for (int k = 0; k < 4; ++k) *p[k] = exp2_approx(fmaf(*p[k], a.scale2, -off));
          sum[i] += (*p[0] + *p[1]) + (*p[2] + *p[3]);
#pragma unroll
          for (int k = 0; k < 2; ++k) {                          // fragment i + 2 k: columns j0 + 8 k, j0 + 8 k + 1
            const uint32_t h = bf16_pair(*p[2 * k], *p[2 * k + 1]);
            hi[i + 2 * k] = h;
            lo[i + 2 * k] = bf16_pair(*p[2 * k] - __uint_as_float(h << 16), *p[2 * k + 1] - __uint_as_float(h & 0xffff0000u));
          }
        }
        s = unit % L::kUnits;
        ok = __all_sync(0xffffffffu, wait_or_stop(&tail->bars.full[s], (unit / L::kUnits) & 1, watch));
        if (!ok) break;
        if (masked) {
          bool found = false;
          for (int i = lane; i < 16 * boxes * 8; i += 32) {
            const int row = key + i / (boxes * 8), c = i % (boxes * 8), j = t * kTileKeys + row;
            if (j < all_see) continue;
            uint4* at = reinterpret_cast<uint4*>(ring + (size_t)s * L::kUnit + (c >> 3) * (kTileKeys * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4));
            if (j >= x.n) {
              *at = make_uint4(0, 0, 0, 0);
            } else {
              uint4 v = *at;
              if (any_not_finite(v.x) || any_not_finite(v.y) || any_not_finite(v.z) || any_not_finite(v.w)) {
                found = true;
                *at = make_uint4(finite_only(v.x), finite_only(v.y), finite_only(v.z), finite_only(v.w));
              }
            }
          }
          if (__any_sync(0xffffffffu, found) && lane == 0) atomicOr(&tail->odd, 1);
          ptx::fence_proxy_async();                                // (before the unit is filled again)
          __syncwarp();
        }
        const uint32_t v_addr = ptx::smem_u32(ring) + s * L::kUnit + v_row * 128;
#pragma unroll
        for (int c = 0; c < kBoxes * 4; ++c) {                     // 16 channels
          if (c < ksteps) {
            uint32_t vf[4];
            ldmatrix4_trans(vf, v_addr + (c >> 2) * (kTileKeys * 128) + (((((uint32_t)c & 3) * 2 + v_half) ^ (v_row & 7)) << 4));
            mma(o[2 * c], hi, vf[0], vf[1]);
            mma(o[2 * c + 1], hi, vf[2], vf[3]);
            if (!packed) {
              mma(o[2 * c], lo, vf[0], vf[1]);
              mma(o[2 * c + 1], lo, vf[2], vf[3]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&tail->bars.empty[s]);
        ++unit;
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&tail->bars.q_empty[seg & 1]);

      float all = 0.f;
#pragma unroll
      for (int n = 0; n < kBoxes * 8; ++n) {
        if (packed) { o[n][0] += o[n][2]; o[n][1] += o[n][3]; o[n][2] = o[n][3] = 0.f; }
        all += (o[n][0] + o[n][1]) + (o[n][2] + o[n][3]);
      }
      if (__any_sync(0xffffffffu, !isfinite(all)) && lane == 0) atomicOr(&tail->odd, 2);
      // the four warps' results meet: a common reference, then sums in shared memory (warps 2 and 3, then 0 and 1 onto them); of
      // 16 rows those that are a token's, eight at least
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
        if ((lane & 3) == 0) tail->ml[warp][i * 8 + (lane >> 2)] = make_float2(ref[i], sum[i]);
      }
      ptx::named_barrier_sync(1, 32 * kWarps);
      const int odd = tail->odd;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i * 8 >= rows) break;
        const int lr = i * 8 + (lane >> 2);
        float top = tail->ml[0][lr].x;
#pragma unroll
        for (int k = 1; k < kWarps; ++k) top = fmaxf(top, tail->ml[k][lr].x);
        const float f = exp2_approx(ref[i] - (top == -INFINITY ? 0.f : top));
#pragma unroll
        for (int n = 0; n < kBoxes * 8; ++n) { o[n][2 * i] *= f; o[n][2 * i + 1] *= f; }
      }
#pragma unroll
      for (int round = 1; round >= 0; --round) {
        if ((warp >> 1) == round) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (i * 8 >= rows) break;
#pragma unroll
            for (int n = 0; n < kBoxes * 8; ++n) {
              float2* at = reinterpret_cast<float2*>(sum_sm + ((warp & 1) * kRows + i * 8 + (lane >> 2)) * L::kSumPitch + n * 8 + (lane & 3) * 2);
              float2 v = make_float2(o[n][2 * i], o[n][2 * i + 1]);
              if (round == 0) { const float2 u = *at; v.x += u.x; v.y += u.y; }
              *at = v;
            }
          }
        }
        ptx::named_barrier_sync(1, 32 * kWarps);
      }
      const int quads = a.d_k >> 2;
      // Not finite: a value of a row that some token sees was not, and a weight's terms times an infinity may have cancelled or
      // been zero; what such values add up to is the result.  Those of rows that all tokens see are looked for together.
      const int common = min(max(all_see, w.s0 * kTileKeys), w.s1 * kTileKeys);
      if (odd & 2) {
        for (int i = tid; i < a.d_k; i += 32 * kWarps) tail->none[i] = 0.f;
        ptx::named_barrier_sync(1, 32 * kWarps);
        const int per = 32 * kWarps / quads, c = tid % quads * 4;
        uint32_t rows_done = 0;
#pragma unroll 2
        for (int j = w.s0 * kTileKeys + tid / quads; tid < per * quads && j < common; j += per) {
          if ((++rows_done & 1023u) == 0 && tid == 0) count_work(watch);
          const int64_t at = row_offset(a.src, x.r, x.h, a.Hkv, j);
          if (at < 0) continue;
          const uint2 g = *reinterpret_cast<const uint2*>(a.src.V + at + c);
          if (!any_not_finite(g.x) && !any_not_finite(g.y)) continue;
          const uint32_t z[4] = {g.x << 16, g.x & 0xffff0000u, g.y << 16, g.y & 0xffff0000u};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!isfinite(__uint_as_float(z[e]))) atomicAdd(&tail->none[c + e], __uint_as_float(z[e]));   // (sums of infinities and NaN: any order)
        }
        ptx::named_barrier_sync(1, 32 * kWarps);
      }
      const int p0 = pref[w.e] + kGap, p1 = pref[w.e + 1];
      const int first = (int)(((int64_t)(p0 + 1) * B - 1) / T), last = (int)(((int64_t)p1 * B - 1) / T);   // CTAs of this entry
      const int64_t slot = slot0 + w.e + b;
      for (int i = tid; i < rows * quads; i += 32 * kWarps) {
        const int lr = i / quads, c = (i - lr * quads) * 4, row = row0 + lr, token = row / a.G, head = x.h * a.G + row - token * a.G;
        float top = tail->ml[0][lr].x;
#pragma unroll
        for (int k = 1; k < kWarps; ++k) top = fmaxf(top, tail->ml[k][lr].x);
        const float off = top == -INFINITY ? 0.f : top;
        float total = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) total = fmaf(tail->ml[k][lr].y, exp2_approx(tail->ml[k][lr].x - off), total);
        const float4 u = *reinterpret_cast<const float4*>(sum_sm + lr * L::kSumPitch + c);
        const float4 v = *reinterpret_cast<const float4*>(sum_sm + (kRows + lr) * L::kSumPitch + c);
        float4 r = make_float4(u.x + v.x, u.y + v.y, u.z + v.z, u.w + v.w);
        if (odd) {                                                 // and those that were taken out, or that only this token sees
          const int end = min(all_see + row / a.G - row0 / a.G, w.s1 * kTileKeys);
          float4 f = make_float4(0, 0, 0, 0);
          if ((odd & 2) && end > w.s0 * kTileKeys) f = *reinterpret_cast<const float4*>(tail->none + c);
          for (int j = common; j < end; ++j) {
            const int64_t at = row_offset(a.src, x.r, x.h, a.Hkv, j);
            if (at < 0) continue;
            const uint2 g = *reinterpret_cast<const uint2*>(a.src.V + at + c);
            if (!any_not_finite(g.x) && !any_not_finite(g.y)) continue;
            f.x += not_finite_only(__uint_as_float(g.x << 16)); f.y += not_finite_only(__uint_as_float(g.x & 0xffff0000u));
            f.z += not_finite_only(__uint_as_float(g.y << 16)); f.w += not_finite_only(__uint_as_float(g.y & 0xffff0000u));
          }
          if (f.x != 0.f) r.x = f.x;
          if (f.y != 0.f) r.y = f.y;
          if (f.z != 0.f) r.z = f.z;
          if (f.w != 0.f) r.w = f.w;
        }
        if (first == last) {
          if (total == 0.f) r = make_float4(0, 0, 0, 0);           // sees nothing
          const float inv = total == 0.f ? 0.f : 1.f / total;
          *reinterpret_cast<uint2*>(a.out + (int64_t)(x.q0 + token) * a.o_tok + (int64_t)head * a.o_head + c) =
              make_uint2(bf16_pair(r.x * inv, r.y * inv), bf16_pair(r.z * inv, r.w * inv));
          if (a.lse && c == 0)
            a.lse[(int64_t)(x.q0 + token) * a.Hq + head] = total == 0.f ? -INFINITY : off * 0.6931471805599453f + logf(total);
        } else {
          *reinterpret_cast<float4*>(a.part_o + (slot * kRows + lr) * a.d_k + c) = r;
          if (c == 0) a.part_ml[slot * kRows + lr] = make_float2(top, total);
        }
      }
      // the joins: of kFan segments, then of as many joined ones as there are
      const int segs = last - first + 1;
      int32_t* counts = a.arrived + (int64_t)blockIdx.y * (2 * kFewEntries + kFewCtas);
      int k0 = (b - first) / kFan * kFan, n = min(segs - k0, kFan), apart = 1;      // the segments k0, k0 + apart, ..: n of them
      int32_t* count = counts + w.e + first + k0;
      while (segs > 1) {
        ptx::named_barrier_sync(1, 32 * kWarps);
        if (tid == 0) {
          __threadfence();                                         // (of what all wrote: the barrier lies before it)
          const int before = atomicAdd(count, 1);
          tail->last_one = before == n - 1;
          if (before == n - 1) *count = 0;
        }
        ptx::named_barrier_sync(1, 32 * kWarps);
        if (!tail->last_one) break;
        __threadfence();
        const bool final = segs <= kFan || apart > 1;
        const int64_t s0 = slot0 + w.e + first + k0;
        for (int i = tid; i < n * kRows; i += 32 * kWarps)
          tail->join[i / kRows][i % kRows] = __ldcg(a.part_ml + (s0 + (int64_t)(i / kRows) * apart) * kRows + i % kRows);
        ptx::named_barrier_sync(1, 32 * kWarps);
        for (int i = tid; i < rows * quads; i += 32 * kWarps) {
          const int lr = i / quads, c = (i - lr * quads) * 4, row = row0 + lr, token = row / a.G, head = x.h * a.G + row - token * a.G;
          float* po = a.part_o + (s0 * kRows + lr) * a.d_k + c;
          float top = -INFINITY, total = 0.f;
          for (int k = 0; k < n; ++k) top = fmaxf(top, tail->join[k][lr].x);
          const float off = top == -INFINITY ? 0.f : top;
          float4 r = make_float4(0, 0, 0, 0);
#pragma unroll 1
          for (int k1 = 0; k1 < n; k1 += 6) {                      // six loads on their way
            float4 v[6];
#pragma unroll
            for (int k = 0; k < 6; ++k)
              if (k1 + k < n) v[k] = __ldcg(reinterpret_cast<const float4*>(po + (int64_t)(k1 + k) * apart * kRows * a.d_k));
#pragma unroll
            for (int k = 0; k < 6; ++k)
              if (k1 + k < n) {
                const float2 q = tail->join[k1 + k][lr];
                const float f = exp2_approx(q.x - off);
                total = fmaf(q.y, f, total);
                r.x += scaled(v[k].x, f); r.y += scaled(v[k].y, f); r.z += scaled(v[k].z, f); r.w += scaled(v[k].w, f);
              }
          }
          if (final) {
            if (total == 0.f) r = make_float4(0, 0, 0, 0);
            const float inv = total == 0.f ? 0.f : 1.f / total;
            *reinterpret_cast<uint2*>(a.out + (int64_t)(x.q0 + token) * a.o_tok + (int64_t)head * a.o_head + c) =
                make_uint2(bf16_pair(r.x * inv, r.y * inv), bf16_pair(r.z * inv, r.w * inv));
            if (a.lse && c == 0) a.lse[(int64_t)(x.q0 + token) * a.Hq + head] = total == 0.f ? -INFINITY : off * 0.6931471805599453f + logf(total);
          } else {
            *reinterpret_cast<float4*>(po) = r;                    // (nobody else reads these slots any more)
            if (c == 0) a.part_ml[s0 * kRows + lr] = make_float2(top, total);
          }
        }
        if (final) break;
        count = counts + kFewEntries + kFewCtas + w.e;
        n = (segs + kFan - 1) / kFan;
        k0 = 0;
        apart = kFan;
      }
      if (tid == 0) tail->odd = 0;                                 // (everyone has read it: a barrier lies behind)
      ptx::named_barrier_sync(1, 32 * kWarps);
    }
  }
  __syncthreads();
  if (tid == 0 && watch->stop) {
    atomicExch(&a.status[0], GVOTE_ERR_TIMEOUT);
    atomicExch(&a.status[1], 24);
  }
}

int boxes_of(const gvote_params* p) { return p->d_k <= 64 ? 1 : p->d_k <= 128 ? 2 : 4; }

struct FewMap { size_t ml, o, total; int groups, ctas; };
FewMap few_map(const gvote_params* p, int32_t batch, int64_t max_q) {
  FewMap m;
  m.groups = (int)ceil_div(max_q * (p->n_q_heads / p->n_kv_heads), kRows);
  const int at_once = m.groups < kFewGroups ? m.groups : kFewGroups;
  m.ctas = (boxes_of(p) <= 2 ? 2 : 1) * kNumSms / at_once;
  const int64_t all = (int64_t)batch * p->n_kv_heads, slots = (all < kFewEntries ? all : kFewEntries) + m.ctas;
  m.ml = kScratchAt;
  m.o = m.ml + align_up((size_t)at_once * slots * kRows * 8, 256);
  m.total = m.o + align_up((size_t)at_once * slots * kRows * p->d_k * 4, 256);
  return m;
}

template <int kBoxes>
int32_t launch(const CUtensorMap& tk, const CUtensorMap& tv, const FewArgs& a, int ctas, int groups, cudaStream_t st) {
  using L = Layout<kBoxes>;
  GVOTE_CUDA_CHECK(cudaFuncSetAttribute(attend_few_kernel<kBoxes>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::smem()));
  LaunchScope scope_("attend_few_kernel", st);
  (void)launch_behind(attend_few_kernel<kBoxes>, dim3(ctas, groups), dim3(kThreads), L::smem(), st, tk, tv, a);
  GVOTE_LAUNCH_CHECK("attend_few_kernel");
  return GVOTE_OK;
}

}  // namespace

// One group of rows is bound by memory; with a second the cached rows are read and multiplied twice, and the kernel for many
// rows, which takes 256 of them at once, is as fast or faster (20 rows over 512 cached ones 12.5 us against 20).
bool attend_takes_few(const gvote_params* p, int64_t max_q) {
  return p->d_k > kMaxHeadDimMany || max_q * (p->n_q_heads / p->n_kv_heads) <= kRows;
}

size_t attend_few_workspace(const gvote_params* p, int32_t batch, int64_t max_q) {
  size_t n = 0;
  for (int64_t q = 1; q <= max_q && q <= GVOTE_ATTEND_FEW_Q && attend_takes_few(p, q); ++q) {   // (fewer groups have more CTAs: not monotonic)
    const size_t t = few_map(p, batch, q).total;
    if (t > n) n = t;
  }
  return n;
}

bool row_maps(const gvote_params* p, const RowSource& s, int rows, CUtensorMap* K, CUtensorMap* V) {
  const uint64_t dims[3] = {(uint64_t)p->d_k, s.tables ? (uint64_t)1 << s.page_log2 : (uint64_t)(s.total > 0 ? s.total : 1),
                            (uint64_t)(s.tables ? s.n_pages : p->n_kv_heads)};
  // (the stride of a dimension of one is not used and may be anything)
  const uint64_t strides[2] = {(uint64_t)(dims[1] > 1 ? s.tok : p->d_k) * 2, (uint64_t)(dims[2] > 1 ? s.outer : p->d_k) * 2};
  const uint32_t box[3] = {64, (uint32_t)rows, 1};
  return encode_tensor_map_bf16(K, s.K, 3, dims, strides, box) && encode_tensor_map_bf16(V, s.V, 3, dims, strides, box);
}

int32_t launch_attend_few(const gvote_params* p, const AttendCall& c, const RowSource& s, char* ws, cudaStream_t st) {
  const FewMap m = few_map(p, c.batch, c.max_q);
  FewArgs a;
  a.src = s;
  a.Q = c.Q; a.q_tok = c.q_tok; a.q_head = c.q_head; a.cu_q = c.cu_q; a.out = c.out; a.o_tok = c.o_tok; a.o_head = c.o_head;
  a.lse = c.lse;
  a.arrived = reinterpret_cast<int32_t*>(ws + kStatusBytes);
  a.part_ml = reinterpret_cast<float2*>(ws + m.ml);
  a.part_o = reinterpret_cast<float*>(ws + m.o);
  a.status = reinterpret_cast<int32_t*>(ws);
  a.Hq = p->n_q_heads; a.Hkv = p->n_kv_heads; a.G = p->n_q_heads / p->n_kv_heads; a.d_k = p->d_k; a.max_q = (int)c.max_q;
  a.scale2 = (float)(1.4426950408889634 / sqrt((double)p->d_k));
  a.box_rows = s.tables && (1 << s.page_log2) < kTileKeys ? 1 << s.page_log2 : kTileKeys;
  CUtensorMap tk, tv;
  if (!row_maps(p, s, a.box_rows, &tk, &tv)) return GVOTE_ERR_CUDA;
  a.one_group = m.groups == 1;
  const int boxes = boxes_of(p), most = kFewEntries / a.Hkv;
  for (int r0 = 0; r0 < c.batch; r0 += most) {
    a.r0 = r0;
    a.batch = c.batch - r0 < most ? c.batch - r0 : most;
    for (a.group0 = 0; a.group0 < m.groups; a.group0 += kFewGroups) {
      const int n = m.groups - a.group0 < kFewGroups ? m.groups - a.group0 : kFewGroups;
      if (boxes == 4) PROPAGATE(launch<4>(tk, tv, a, m.ctas, n, st));
      else if (boxes == 2) PROPAGATE(launch<2>(tk, tv, a, m.ctas, n, st));
      else PROPAGATE(launch<1>(tk, tv, a, m.ctas, n, st));
    }
  }
  return GVOTE_OK;
}

}  // namespace gvote
