// Causal attention of many query tokens over bf16 rows in slabs or pages (gvote_attend, gvote_page_attend): prompts and chunks.
//
//   l_j = (q.k_j) / sqrt(d_k),  out = sum_j exp(l_j - lse) v_j,  lse = log sum_j exp(l_j),  j over the rows a token sees
// One pass over the keys with a running reference and sum (the output is rescaled where the reference moves), 4 d_k operations
// per (query row, key): bound by the tensor cores and, as much, by the exponentials, one per 4 d_k operations.
//
// A query tile is floor(128 / G) tokens with the G query heads of one KV head (token-major), fetched by one TMA box per 64
// channels, so K and V are read once for the group.  A unit is two such tiles of one (request, KV head) against tiles of 128
// keys.  Persistent CTAs of twelve warps, one per SM:
//   warps 0-3, 4-7   softmax of the first, second tile: thread = query row
//   warp 8           asks for Q, K, V (TMA, 128-byte swizzle; of pages a box each)
//   warp 9           issues the MMAs, all of them tcgen05.mma kind::f16 with 32-bit results
//   warp 10          makes values finite that some token must not see (below)
//   warp 11          lists the CTA's units
//     S_i [128 rows x 128 keys] = Q_i K^T     both from shared memory
//     O_i [128 rows x d_k]     += P_i V       P from tensor memory, where it takes S's place; V as it lies (channels contiguous)
// Tensor memory: S_0, S_1, O_0, O_1.  The MMAs go P_0 V, Q_0 K' (next keys), P_1 V, Q_1 K': while one tile's softmax runs
// the tensor cores work for the other.  S_i is overwritten by the next keys' only behind P_i V, in the order of issue; O_i is
// rescaled by the softmax warps when a logit passes the row's reference by 2^8 (P then reaches 2^8 at most), which after the first
// tiles hardly happens; the next unit's first P_i V waits for them in any case, so a unit's outputs are
// stored while the next one's products run.
//
// P is rounded to bf16, by at most 2^-8 of a weight, as the output is; two terms, as the few-row kernel has them, would
// take half as much tensor time again.  The sum is of the 32-bit weights.
//
// What bounds it: a tile's chain.  The softmax of 128 x 128 logits takes its four warps 2000 clocks (S out of tensor memory and
// its maximum 600, the exponentials 1200, P back 200), the products and their messages 1160, and the two tiles' chains overlap to 3600
// clocks for 2 x 2 products of 128 x 128 x 128, of which the tensor cores work half: 52 % busy, the exponentials' unit 46 %.
// Measured (one B200): a 32K prompt of 32 heads on 8 8.1 to 8.4 ms (8.8 TFLOP, 1.05 to 1.1 PFLOP/s), 8192 tokens 0.51 to
// 0.56 ms as the power allows clocks.  Of that the outputs' stores take 3 %: a lane's 32 bytes are a line of their own, and with 16 at a time
// they took 1 % (of short prompts 2 %) more.
// Slower, or no faster: two S of 64 keys to a tile, so that softmax and products of a tile overlap (the MMAs with N = 64 read
// Q twice as often, 8.5 ms); sixteen softmax warps, two threads to a row (9.5 ms); an issuer for each tile; exponentials before the maximum,
// with the reference of the tile before (registers); none, two or three of eight exponentials on the FMA pipe; a loop over halves with S read
// twice; S read in two halves, the maximum of one while the other comes (8.45 ms for 8.34); the units of a ragged batch sorted by length;
// outputs 64 channels at a time.
//
// Where there are few units (kCutUnits at most) the list is cut evenly over the CTAs, units into pieces, and attend_join_kernel adds
// a unit's pieces up: 500 tokens of 32 heads over pruned 13K rows of 8 KV heads 121 us in a graph instead of 272, 7 of them the join.
// With more units the list is not cut, and a request much longer than the others is one SM's work per KV head: five drafts of 36
// requests, one of 128K rows among 2000, take 1.62 ms, of 32 such requests (272 units) 0.21.
//
// Rows that not every token of a unit sees may hold anything: logits are masked by index, values that are not finite are
// set to 0 in the tile (0 * inf is no number) and added back at the end to the tokens that see them.
//
// Every wait is bounded by the time without any work done (kv_rows.cuh); when one runs out GVOTE_ERR_TIMEOUT is recorded and the outputs are not to be used.
#include <float.h>

#include "f32x2.cuh"
#include "kv_rows.cuh"

namespace gvote {
namespace {

constexpr int kTile = 128;
constexpr int kThreads = 384;
constexpr int kMaxStages = 12;
constexpr int kInfos = 4;
constexpr int kMarks = 8;                 // more than the tiles of V a ring holds
static_assert(kMaxStages / 2 < kMarks, "");
constexpr int kPoly = 1;                  // of 8 exponentials, those computed on the FMA pipe
constexpr float kSlack = 8.f;
// Cut lists (where there are few units): units of a list, places that a unit's beginning and end count as, and what a join takes.
constexpr int kCutUnits = 2 * kNumSms;
constexpr size_t kPiecesBytes = 2560;
static_assert(kCutUnits * sizeof(int2) <= kPiecesBytes && kCutUnits <= kThreads, "");
constexpr int kGap = 3;
constexpr int kPiece = 8;                 // places of a CTA at least
constexpr int kJoinQuads = 8;             // channels / 4 of a CTA of the join
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;     // (with 232 and 40 or 224 and 56 the cut lists' kernel spills)
static_assert(kSoftmaxRegs * 256 + kOtherRegs * 128 <= 168 * kThreads, "the registers a CTA is launched with");

struct ManyArgs {
  RowSource src;
  const int32_t* cu_q;
  __nv_bfloat16* out;
  int64_t o_tok, o_head;
  float* lse;             // or null
  int32_t* status;
  int Hq, Hkv, G, batch, d_k, max_q;
  int tpt;                // tokens of a query tile
  uint32_t pairs, units;  // pairs of tiles (upper bound), times KV heads
  int stages, box_rows;
  int wide;               // out's rows start on 32 bytes
  float4* part_o;         // [2 per CTA][2 tiles][d_k / 4][128 rows]
  float2* part_ml;        // [2 per CTA][2 tiles][128 rows]  (reference, sum), base 2
  int2* pieces;           // [units]  first CTA, pieces
  float c;                // log2(e) / sqrt(d_k)
};

struct Unit {
  int r, h, seq;
  int k0;                 // first tile of keys
  int first, segs;        // in a cut list: the first CTA that has a piece of it, the pieces
  int tok0;               // first token of the first tile, in the packed list
  int count[2];           // tokens of the tiles
  int see[2];             // rows a tile's first token sees (may be negative)
  int tiles[2];           // tiles of keys, from k0 on
  int n;                  // rows the last token sees
};

struct Tail {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t q_full, q_empty;
  uint64_t s_full[2], p_half[2], p_full[2], pv_done[2];
  uint64_t v_raw[kMarks];
  uint64_t info_full[kInfos], info_empty[kInfos];
  uint64_t drain;
  uint32_t tmem_slot;
  Watch watch;
  int mark[kMarks];       // seq of a unit whose values were not all finite
  Unit info[kInfos];      // seq < 0: no more
  int warp_sums[kThreads / 32];
  int pref[kCutUnits + 1];   // a cut list: places before each unit
};

// The largest r with cu[r] / per + r <= g: request of pair g of a list that gives every request one more than it may need.
__device__ __forceinline__ int request_of_pair(const int32_t* __restrict__ cu, int batch, int64_t g, int per) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)(cu[mid] / per) + mid <= g) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// The unit this CTA takes in round k: left to right in even rounds, right to left in odd ones.
__device__ __forceinline__ uint32_t unit_of(uint32_t k) {
  return k * gridDim.x + ((k & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
}

// False: there is nothing at this place of the list.
__device__ __forceinline__ bool unit_info(const ManyArgs& a, uint32_t u, Unit& x) {
  x.k0 = 0;
  x.segs = 1;
  const uint32_t w = u / (uint32_t)a.Hkv;
  x.h = (int)(u - w * (uint32_t)a.Hkv);
  const int64_t v = (int64_t)a.pairs - 1 - w;                      // long rows first
  x.r = a.batch == 1 ? 0 : request_of_pair(a.cu_q, a.batch, v, 2 * a.tpt);
  const int q0 = a.cu_q[x.r], nq = min(a.cu_q[x.r + 1] - q0, a.max_q);
  const int pair = (int)(a.batch == 1 ? v : v - (q0 / (2 * a.tpt) + x.r));
  const int first = pair * 2 * a.tpt;
  if (pair < 0 || first >= nq) return false;
  const int held = rows_held(a.src, x.r, x.h, a.Hkv);
  x.tok0 = q0 + first;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = first + i * a.tpt;
    x.count[i] = max(min(nq - t, a.tpt), 0);
    x.see[i] = held - nq + t + 1;
    const int last = x.see[i] + x.count[i] - 1;
    x.tiles[i] = x.count[i] > 0 && last > 0 ? (last + kTile - 1) / kTile : 0;
  }
  x.n = max(x.count[1] > 0 ? x.see[1] + x.count[1] - 1 : x.see[0] + x.count[0] - 1, 0);
  return true;
}

// Operand of N x K stored as K rows of 64 contiguous N values with the 128-byte swizzle: the next eight K rows 1024 bytes on,
// the next 64 values of N `chunk` bytes on.
__device__ __forceinline__ uint64_t smem_desc_mn_sw128(uint32_t addr, uint32_t chunk) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(chunk >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}

template <int kRegs>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs)); }
template <int kRegs>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs)); }

// A place in the ring: slot and parity, without divisions (by a number that is not known here one takes a hundred clocks).
struct Place {
  uint32_t slot, parity;
  int stages;
  __device__ __forceinline__ explicit Place(int n) : slot(0), parity(0), stages(n) {}
  __device__ __forceinline__ void step() {
    if (++slot == (uint32_t)stages) { slot = 0; parity ^= 1; }
  }
};

// A reader of the unit list.
struct Units {
  Tail* tail;
  int at;
  __device__ __forceinline__ explicit Units(Tail* t) : tail(t), at(0) {}
  // The whole warp: the next unit, or false at the end (or when a wait ran out).
  __device__ __forceinline__ bool next(Unit& x, int lane) {
    const int s = at % kInfos;
    if (!__all_sync(0xffffffffu, wait_or_stop(&tail->info_full[s], (at / kInfos) & 1, &tail->watch))) return false;
    x = tail->info[s];
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&tail->info_empty[s]);
    ++at;
    return x.seq >= 0;
  }
};

// Where piece `seg` of a unit that begins in CTA `first` leaves its sums: the unit's first piece is its CTA's last one, every
// other piece its CTA's first one.
__device__ __forceinline__ int64_t piece_slot(int first, int seg) { return (int64_t)2 * (first + seg) + (seg == 0 ? 1 : 0); }

// The pieces of a unit added up, in their order: a CTA per unit, tile and 4 kJoinQuads channels, two threads per row.  (By the last
// CTA to arrive at a counter, as the few-row kernel does it, a tile's 128 rows were too much for one SM: 70 of 107 us for five
// draft tokens over 32K rows.)
__global__ void __launch_bounds__(2 * kTile)
attend_join_kernel(const __grid_constant__ ManyArgs a) {
  const int u = blockIdx.x, i = blockIdx.y, row = threadIdx.x & (kTile - 1);
  ptx::let_next_begin();
  ptx::wait_for_previous();
  const int2 piece = a.pieces[u];
  const int first = piece.x, n = piece.y;
  if (n < 2) return;
  Unit x;
  unit_info(a, (uint32_t)u, x);
  const int tok_in = row / a.G, head = x.h * a.G + row - tok_in * a.G, quads = a.d_k >> 2;
  if (tok_in >= (i ? x.count[1] : x.count[0]) || row >= a.G * a.tpt) return;
  const int64_t token = x.tok0 + i * a.tpt + tok_in;
  float top = -INFINITY, sum = 0.f;
  for (int k = 0; k < n; ++k) top = fmaxf(top, a.part_ml[(piece_slot(first, k) * 2 + i) * kTile + row].x);
  const float off = top == -INFINITY ? 0.f : top;
  float4 r[kJoinQuads / 2];
#pragma unroll
  for (int c = 0; c < kJoinQuads / 2; ++c) r[c] = make_float4(0, 0, 0, 0);
  const int c0 = blockIdx.z * kJoinQuads + (threadIdx.x >> 7) * (kJoinQuads / 2);
#pragma unroll 2
  for (int k = 0; k < n; ++k) {
    const float2 q = a.part_ml[(piece_slot(first, k) * 2 + i) * kTile + row];
    if (q.x == -INFINITY && q.y == 0.f) continue;                  // no tile: its outputs were not written
    const float f = exp2_fast(q.x - off);
    sum = fmaf(q.y, f, sum);
    const float4* from = a.part_o + ((piece_slot(first, k) * 2 + i) * quads + c0) * kTile + row;
#pragma unroll
    for (int c = 0; c < kJoinQuads / 2; ++c)
      if (c0 + c < quads) {
        const float4 v = from[c * kTile];
        r[c].x += scaled(v.x, f); r[c].y += scaled(v.y, f); r[c].z += scaled(v.z, f); r[c].w += scaled(v.w, f);
      }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  __nv_bfloat16* out = a.out + token * a.o_tok + (int64_t)head * a.o_head;
#pragma unroll
  for (int c = 0; c < kJoinQuads / 2; ++c)
    if (c0 + c < quads) {
      if (sum == 0.f) r[c] = make_float4(0, 0, 0, 0);
      *reinterpret_cast<uint2*>(out + (c0 + c) * 4) = make_uint2(bf16_pair(r[c].x * inv, r[c].y * inv), bf16_pair(r[c].z * inv, r[c].w * inv));
    }
  if (a.lse && c0 == 0) a.lse[token * a.Hq + head] = sum == 0.f ? -INFINITY : off * 0.6931471805599453f + logf(sum);
}

// kCut: the list may be cut.
template <int kBoxes, bool kCut>
__global__ void __launch_bounds__(kThreads, 1)
attend_many_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const __grid_constant__ ManyArgs a) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr uint32_t kTileBytes = kBoxes * kTile * 128;
  uint8_t* q_sm = smem;                                            // [2][box][128 rows][128], swizzled
  uint8_t* ring = q_sm + 2 * kTileBytes;                           // [stage][box][128 rows][128], swizzled: K and V in turns
  Tail* tail = reinterpret_cast<Tail*>(ring + (size_t)a.stages * kTileBytes);
  Watch* watch = &tail->watch;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int q_rows = a.G * a.tpt;                                  // rows a box of Q fills

  if (tid == 0) {
    for (int s = 0; s < kMaxStages; ++s) { ptx::mbar_init(&tail->full[s], 1); ptx::mbar_init(&tail->empty[s], 1); }
    ptx::mbar_init(&tail->q_full, 1);
    ptx::mbar_init(&tail->q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&tail->s_full[i], 1);
      ptx::mbar_init(&tail->p_half[i], 4);
      ptx::mbar_init(&tail->p_full[i], 4);
      ptx::mbar_init(&tail->pv_done[i], 1);
    }
    for (int s = 0; s < kMarks; ++s) ptx::mbar_init(&tail->v_raw[s], 1);
    for (int s = 0; s < kInfos; ++s) { ptx::mbar_init(&tail->info_full[s], 1); ptx::mbar_init(&tail->info_empty[s], 11); }
    ptx::mbar_init(&tail->drain, 1);
    tail->watch.stop = (ptx::smem_u32(smem) & 1023u) ? 1 : 0;
    tail->watch.work = 0;
    for (int s = 0; s < kMarks; ++s) tail->mark[s] = -1;
    ptx::fence_barrier_init();
    ptx::prefetch_tensormap(&tmQ);
    ptx::prefetch_tensormap(&tmK);
    ptx::prefetch_tensormap(&tmV);
  }
  if (warp == 9) {
    ptx::tmem_alloc(&tail->tmem_slot, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tail->tmem_slot, 0);
  ptx::let_next_begin();
  ptx::wait_for_previous();

  // A cut list: the tiles of all units end to end, each behind kGap places for what beginning and ending one costs; this CTA
  // takes the places t0 .. t1 - 1.
  int t0 = 0, t1 = 0, B = 0, T = 0;
  bool cut = false;
  if (kCut) {
    Unit x;
    int places = 0;
    if (tid < (int)a.units && unit_info(a, tid, x)) places = max(x.tiles[0], x.tiles[1]) + kGap;
    int up = places;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, up, o);
      if (lane >= o) up += y;
    }
    if (lane == 31) tail->warp_sums[warp] = up;
    __syncthreads();
    for (int w = 0; w < warp; ++w) up += tail->warp_sums[w];
    if (tid == 0) tail->pref[0] = 0;
    if (tid < (int)a.units) tail->pref[tid + 1] = up;
    __syncthreads();
    T = tail->pref[a.units];
    B = min((int)gridDim.x, T / kPiece);
    cut = T / kPiece > (int)a.units;                               // short units stay whole
    if (blockIdx.x == 0 && tid < (int)a.units) {                   // for the join
      const int p = tail->pref[tid] + kGap, p1 = tail->pref[tid + 1];
      const int first = cut && p < p1 ? (int)(((int64_t)(p + 1) * B - 1) / T) : 0;
      a.pieces[tid] = make_int2(first, cut && p < p1 ? (int)(((int64_t)p1 * B - 1) / T) - first + 1 : 0);
    }
    if ((int)blockIdx.x < B) {
      t0 = (int)((int64_t)T * blockIdx.x / B);
      t1 = (int)((int64_t)T * (blockIdx.x + 1) / B);
    }
  }

  if (warp >= 8) {
    fewer_registers<kOtherRegs>();
    if (warp == 11) {
      // ---------------------------------------------------------------- the list of units
      int at = 0;
      bool ok = true;
      for (uint32_t k = 0; ok; ++k) {
        if ((k & 63u) == 63u && lane == 0) count_work(watch);      // (a list may be long and nearly empty)
        bool end;
        Unit x;
        if (kCut && cut) {
          end = k >= a.units || tail->pref[k] >= t1;
          if (!end) {
            const int p = tail->pref[k], p1 = tail->pref[k + 1];
            if (p1 <= t0 || p1 == p || !unit_info(a, k, x)) continue;
            const int s0 = max(t0 - p - kGap, 0), s1 = min(t1, p1) - p - kGap, n = p1 - p - kGap;     // of its n tiles
            if (n > 0 ? s0 >= s1 : p < t0) continue;               // (without tiles: whose it begins in)
            if (n > 0) {
              x.k0 = s0;
              x.first = (int)(((int64_t)(p + kGap + 1) * B - 1) / T);
              x.segs = (int)(((int64_t)p1 * B - 1) / T) - x.first + 1;
#pragma unroll
              for (int i = 0; i < 2; ++i) x.tiles[i] = max(min(x.tiles[i], s1) - s0, 0);
            }
          }
        } else {
          end = (uint64_t)k * gridDim.x >= a.units;
          const uint32_t u = end ? 0 : unit_of(k);
          if (!end && (u >= a.units || !unit_info(a, u, x))) continue;
        }
        x.seq = end ? -1 : at;
        const int s = at % kInfos;
        ok = __all_sync(0xffffffffu, wait_or_stop(&tail->info_empty[s], ((at / kInfos) & 1) ^ 1, watch));
        if (!ok) break;
        if (lane == 0) {
          tail->info[s] = x;
          ptx::mbar_arrive(&tail->info_full[s]);
        }
        __syncwarp();
        ++at;
        if (end) break;
      }
      if (blockIdx.x == 0)                                         // requests with more tokens than announced
        for (int r = lane; r < a.batch; r += 32)
          if (a.cu_q[r + 1] - a.cu_q[r] > a.max_q) {
            atomicExch(&a.status[0], GVOTE_ERR_INVALID_ARG);
            atomicExch(&a.status[1], 25);
          }
    } else if (warp == 8) {
      // ---------------------------------------------------------------- asks for tiles
      Units units(tail);
      Unit x;
      Place at(a.stages);
      uint32_t it = 0, asked_q = 0, raw = 0;
      bool ok = true, bad_page = false;
      const int boxes = (a.d_k + 63) >> 6, box = lane % boxes, part = lane / boxes;
      const bool in_tile = part * a.box_rows < kTile;
      const int in_page = (1 << a.src.page_log2) - 1;
      while (ok && units.next(x, lane)) {
        const int tiles = max(x.tiles[0], x.tiles[1]);
        if (tiles == 0) continue;
        ok = __all_sync(0xffffffffu, wait_or_stop(&tail->q_empty, (asked_q & 1) ^ 1, watch));
        if (!ok) break;
        ++asked_q;
        const int n_q = x.tiles[1] > 0 ? 2 : 1;                    // (the first tile sees less than the second)
        if (lane == 0) {
          ptx::mbar_arrive_expect_tx(&tail->q_full, (uint32_t)(n_q * boxes * q_rows * 128));
          for (int i = 0; i < n_q; ++i)
            for (int b = 0; b < boxes; ++b)
              ptx::tma_load_3d(q_sm + i * kTileBytes + b * (kTile * 128), &tmQ, &tail->q_full, b * 64, x.h * a.G, x.tok0 + i * a.tpt);
        }
        __syncwarp();
        const int32_t* table = a.src.tables ? a.src.tables + ((int64_t)x.r * a.Hkv + x.h) * a.src.max_pages : nullptr;
        const int start = table ? 0 : a.src.cu[x.r];
        const int masked_from = max(x.see[0], 0) / kTile - x.k0;
        int j = x.k0 * kTile + part * a.box_rows, page = 0;        // this lane's first row of a tile
        if (table && in_tile && j < x.n) page = table[j >> a.src.page_log2];
        for (int t = 0; t < tiles; ++t, j += kTile) {
          const int parts = (min(x.n - (x.k0 + t) * kTile, kTile) + a.box_rows - 1) / a.box_rows;
          const bool mine = part < parts;
          int next = 0;
          if (table && in_tile && t + 1 < tiles && j + kTile < x.n) next = table[(j + kTile) >> a.src.page_log2];
          const int cy = table ? (j & in_page) : start + j, cz = table ? page : x.h;
          if (table && mine && (uint32_t)page >= (uint32_t)a.src.n_pages) bad_page = true;   // (the copy reads zeros)
#pragma unroll
          for (int v = 0; v < 2; ++v, ++it) {
            const uint32_t s = at.slot;
            ok = ok && __all_sync(0xffffffffu, wait_or_stop(&tail->empty[s], at.parity ^ 1, watch));
            if (!ok) break;
            at.step();
            // (values that warp 10 has to look at first: it tells when they are there)
            uint64_t* bar = v && t >= masked_from ? &tail->v_raw[raw++ % kMarks] : &tail->full[s];
            if (lane == 0) ptx::mbar_arrive_expect_tx(bar, (uint32_t)(parts * boxes * a.box_rows * 128));
            __syncwarp();
            if (mine)
              ptx::tma_load_3d(ring + (size_t)s * kTileBytes + box * (kTile * 128) + part * a.box_rows * 128, v ? &tmV : &tmK,
                               bar, box * 64, cy, cz);
          }
          if (!ok) break;
          page = next;
        }
      }
      if (__any_sync(0xffffffffu, bad_page) && lane == 0) {
        atomicExch(&a.status[0], GVOTE_ERR_INVALID_ARG);
        atomicExch(&a.status[1], 26);
      }
      if (watch->stop) {
        await_loads(tail->full, a.stages, it);
        await_loads(tail->v_raw, kMarks, raw);
        if (asked_q) await_loads(&tail->q_full, 1, asked_q);
      }
    } else if (warp == 9) {
      // ---------------------------------------------------------------- issues the MMAs
      Units units(tail);
      Unit x;
      Place at(a.stages);
      uint32_t n_q = 0, n_p[2] = {0, 0};
      bool ok = true;
      const uint32_t idesc_s = ptx::instr_desc_bf16_f32(kTile, kTile);
      const uint32_t idesc_o = ptx::instr_desc_bf16_f32(kTile, a.d_k) | (1u << 16);     // V: channels contiguous
      const uint32_t q_addr = ptx::smem_u32(q_sm), ring_addr = ptx::smem_u32(ring);
      auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_or_stop(bar, parity, watch)); };
      const uint64_t qd0 = ptx::smem_desc_k_sw128(q_addr), kd0 = ptx::smem_desc_k_sw128(ring_addr);
      // (channels behind d_k are zero: every step is taken)
      auto product_qk = [&](int i, uint32_t slot) {
        const uint64_t qd = qd0 + (uint64_t)(i * (int)(kTileBytes >> 4)), kd = kd0 + (uint64_t)(slot * (kTileBytes >> 4));
        if (ptx::elect_one()) {
#pragma unroll
          for (int q = 0; q < kBoxes * 4; ++q) {
            const int to = (q >> 2) * (kTile * 128 / 16) + (q & 3) * 2;
            ptx::umma_bf16(tmem + i * kTile, qd + to, kd + to, idesc_s, q > 0 ? 1u : 0u);
          }
          ptx::umma_commit(&tail->s_full[i]);
        }
        __syncwarp();
      };
      while (ok && units.next(x, lane)) {
        const int tiles = max(x.tiles[0], x.tiles[1]);
        if (tiles == 0) continue;
        ok = wait(&tail->q_full, n_q & 1);
        ++n_q;
        uint32_t k_slot = at.slot;
        ok = ok && wait(&tail->full[k_slot], at.parity);
        at.step();
        if (!ok) break;
        ptx::tc_fence_after_sync();
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (x.tiles[i] > 0) product_qk(i, k_slot);
        if (ptx::elect_one()) {
          ptx::umma_commit(&tail->empty[k_slot]);
          if (tiles == 1) ptx::umma_commit(&tail->q_empty);
        }
        __syncwarp();
        for (int t = 0; ok && t < tiles; ++t) {
          const uint32_t v_slot = at.slot;
          ok = wait(&tail->full[v_slot], at.parity);
          at.step();
          const bool more = t + 1 < tiles;
          if (!ok) break;
          const uint64_t vd = smem_desc_mn_sw128(ring_addr + v_slot * kTileBytes, kTile * 128);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (t < x.tiles[i]) {
              const uint32_t o = tmem + 256 + i * kTile, p = tmem + i * kTile;
              ok = ok && wait(&tail->p_half[i], n_p[i] & 1);
              if (!ok) break;
              ptx::tc_fence_after_sync();
              if (ptx::elect_one()) {
#pragma unroll
                for (int q = 0; q < 4; ++q) ptx::umma_bf16_ts(o, p + q * 8, vd + q * 128, idesc_o, t + q > 0 ? 1u : 0u);
              }
              __syncwarp();
              ok = wait(&tail->p_full[i], n_p[i] & 1);
              ++n_p[i];
              if (!ok) break;
              ptx::tc_fence_after_sync();
              if (ptx::elect_one()) {
#pragma unroll
                for (int q = 4; q < 8; ++q) ptx::umma_bf16_ts(o, p + q * 8, vd + q * 128, idesc_o, 1u);
                ptx::umma_commit(&tail->pv_done[i]);
              }
              __syncwarp();
            }
            if (i == 0 && more) {
              k_slot = at.slot;
              ok = wait(&tail->full[k_slot], at.parity);
              at.step();
              if (!ok) break;
            }
            if (t + 1 < x.tiles[i]) product_qk(i, k_slot);
          }
          if (!ok) break;
          if (ptx::elect_one()) {
            ptx::umma_commit(&tail->empty[v_slot]);
            if (more) ptx::umma_commit(&tail->empty[k_slot]);
            if (t + 2 == tiles) ptx::umma_commit(&tail->q_empty);
            count_work(watch);
          }
          __syncwarp();
        }
      }
      if (watch->stop) {
        if (ptx::elect_one()) ptx::umma_commit(&tail->drain);
        __syncwarp();
        for (int k = 0; k < (1 << 12) && !ptx::mbar_try_wait(&tail->drain, 0); ++k) {}
      }
    } else {
      // ---------------------------------------------------------------- values that some token must not see
      Units units(tail);
      Unit x;
      uint32_t it = 0, raw = 0;
      bool ok = true;
      while (ok && units.next(x, lane)) {
        const int tiles = max(x.tiles[0], x.tiles[1]), from = max(x.see[0], 0);
        for (int t = max(from / kTile - x.k0, 0); t < tiles; ++t, ++raw) {
          ok = __all_sync(0xffffffffu, wait_or_stop(&tail->v_raw[raw % kMarks], (raw / kMarks) & 1, watch));
          if (!ok) break;
          const uint32_t s = (it + 2 * t + 1) % a.stages;
          bool found = false;
          uint8_t* v = ring + (size_t)s * kTileBytes;
          const int r0 = max(from - (x.k0 + t) * kTile, 0), r1 = min(x.n - (x.k0 + t) * kTile, kTile);     // rows r1 .. are nobody's
          for (int b = 0; b < kBoxes; ++b) {
            uint8_t* p = v + b * (kTile * 128);
            const int boxes = (a.d_k + 63) >> 6;
            if (b >= boxes) break;
#pragma unroll 4
            for (int i = r0 * 8 + lane; i < r1 * 8; i += 32) {
              const uint4 w = *reinterpret_cast<const uint4*>(p + i * 16);
              if (any_not_finite(w.x) || any_not_finite(w.y) || any_not_finite(w.z) || any_not_finite(w.w)) {
                found = true;
                *reinterpret_cast<uint4*>(p + i * 16) = make_uint4(finite_only(w.x), finite_only(w.y), finite_only(w.z), finite_only(w.w));
              }
            }
            for (int i = r1 * 8 + lane; i < kTile * 8; i += 32) *reinterpret_cast<uint4*>(p + i * 16) = make_uint4(0, 0, 0, 0);
          }
          if (__any_sync(0xffffffffu, found) && lane == 0) tail->mark[x.seq % kMarks] = x.seq;
          ptx::fence_proxy_async();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->full[s]);
        }
        it += 2 * tiles;
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax: thread = row of a query tile
    more_registers<kSoftmaxRegs>();
    const int i = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t s_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(i * kTile);
    const uint32_t o_addr = s_addr + 256;
    const uint64_t c2 = pack2(a.c, a.c);
    const int tok_in = row / a.G, head_in = row - tok_in * a.G;
    Units units(tail);
    Unit x;
    uint32_t used = 0;
    bool ok = true;
    while (ok && units.next(x, lane)) {
      const int count = i ? x.count[1] : x.count[0], see = i ? x.see[1] : x.see[0], tiles = i ? x.tiles[1] : x.tiles[0];
      if (count == 0) continue;
      const bool holds = tok_in < count && row < q_rows;
      const int limit = holds ? see + tok_in : 0;
      float ref = -INFINITY, sum = 0.f;
      const bool idle = (warp & 3) * 32 >= min(count * a.G, q_rows);   // none of this warp's rows is a token's
      for (int t = 0; t < tiles; ++t, ++used) {
        ok = __all_sync(0xffffffffu, wait_or_stop(&tail->s_full[i], used & 1, watch));
        if (!ok) break;
        if (idle) {                                                // (their weights may be anything)
          if (lane == 0) { ptx::mbar_arrive(&tail->p_half[i]); ptx::mbar_arrive(&tail->p_full[i]); }
          __syncwarp();
          continue;
        }
        ptx::tc_fence_after_sync();
        uint32_t v[4][32];
#pragma unroll
        for (int b = 0; b < 4; ++b) ptx::tmem_ld_32x32(s_addr + b * 32, v[b]);
        ptx::tmem_wait_ld();
        if ((x.k0 + t + 1) * kTile > see) {
          const int seen = limit - (x.k0 + t) * kTile;
#pragma unroll
          for (int k = 0; k < kTile; ++k)
            if (k >= seen) v[k >> 5][k & 31] = 0xff800000u;
        }
        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int k = 0; k < kTile; k += 2)
          m4[(k >> 1) & 3] = fmaxf(fmaxf(__uint_as_float(v[k >> 5][k & 31]), __uint_as_float(v[k >> 5][(k & 31) + 1])), m4[(k >> 1) & 3]);
        const float top = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * a.c;
        const bool move = top > ref + kSlack;
        if (__any_sync(0xffffffffu, move)) {
          const float f = move ? exp2_fast(ref - top) : 1.f;       // (ref = -inf: 0)
          if (move) ref = top;
          sum *= f;
          if (t > 0) {
            ok = __all_sync(0xffffffffu, wait_or_stop(&tail->pv_done[i], (used - 1) & 1, watch));
            if (!ok) break;
            ptx::tc_fence_after_sync();
#pragma unroll 1
            for (int b = 0; b < a.d_k; b += 16) {
              uint32_t o[16];
              ptx::tmem_ld_32x16(o_addr + b, o);
              ptx::tmem_wait_ld();
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
              ptx::tmem_st_32x16(o_addr + b, o);
            }
          }
        }
        const float off = ref == -INFINITY ? 0.f : -ref;
        const uint64_t off2 = pack2(off, off);
        uint64_t s2[2] = {0, 0};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t p[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            const uint32_t* q = &v[half * 2 + (k >> 4)][(2 * k) & 31];
            const uint64_t e = exp2_pair<kPoly>(k & 7, fma2(pack2(__uint_as_float(q[0]), __uint_as_float(q[1])), c2, off2));
            s2[k & 1] = add2(s2[k & 1], e);
            const float2 w = unpack2(e);
            p[k] = bf16_pair(w.x, w.y);
          }
          ptx::tmem_st_32x32(s_addr + half * 32, p);
          ptx::tmem_wait_st();
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(half ? &tail->p_full[i] : &tail->p_half[i]);
        }
        const float2 s = unpack2(add2(s2[0], s2[1]));
        sum += s.x + s.y;
      }
      if (!ok) break;
      if (tiles > 0) {
        ok = __all_sync(0xffffffffu, wait_or_stop(&tail->pv_done[i], (used - 1) & 1, watch));
        if (!ok) break;
        ptx::tc_fence_after_sync();
      }
      // the outputs
      const bool odd = tiles > 0 && *(volatile int*)&tail->mark[x.seq % kMarks] == x.seq;
      const int head = x.h * a.G + head_in;
      const int64_t token = x.tok0 + i * a.tpt + tok_in;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      __nv_bfloat16* out = a.out + token * a.o_tok + (int64_t)head * a.o_head;
      const int64_t slot = kCut ? piece_slot(x.first, (int)blockIdx.x - x.first) : 0;
      const bool piece = kCut && x.segs > 1;
      for (int b = 0; b < a.d_k; b += 16) {
        if (piece && tiles == 0) break;
        uint32_t o[16];
        __syncwarp();
        if (tiles > 0) {
          ptx::tmem_ld_32x16(o_addr + b, o);
          ptx::tmem_wait_ld();
        }
        float f[16];
        float all = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          f[k] = tiles > 0 ? __uint_as_float(o[k]) : 0.f;
          all += f[k];
        }
        // Not finite: some value this token sees was not, and a weight of zero times an infinity may have spoilt it; what such
        // values add up to is the result (rows that all tokens of the unit see: the warp looks for them together).  Values taken
        // out of the unit's tiles are added back.  (A sum that is no number makes the outputs none by itself.)
        const bool again = holds && !isfinite(all) && isfinite(sum);
        const bool search = __any_sync(0xffffffffu, again);
        if (search || odd) {
          const int from = x.k0 * kTile, end = (x.k0 + tiles) * kTile, common = min(max(x.see[0], from), end);
          float g[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) g[k] = 0.f;
          auto add_row = [&](int j) {
            const int64_t at = row_offset(a.src, x.r, x.h, a.Hkv, j);
            if (at < 0) return;
            const uint4* q = reinterpret_cast<const uint4*>(a.src.V + at + b);
            const uint4 w[2] = {q[0], q[1]};
            const uint32_t* z = &w[0].x;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              g[2 * k] += not_finite_only(__uint_as_float(z[k] << 16));
              g[2 * k + 1] += not_finite_only(__uint_as_float(z[k] & 0xffff0000u));
            }
          };
          if (search) {
#pragma unroll 2
            for (int j = from + lane; j < common; j += 32) {
              if (((j - from) & 0xffff) == 0) count_work(watch);   // (the first lane)
              add_row(j);
            }
#pragma unroll
            for (int k = 0; k < 16; ++k)
#pragma unroll
              for (int m = 16; m > 0; m >>= 1) g[k] += __shfl_xor_sync(0xffffffffu, g[k], m);
          }
          if (holds)
            for (int j = common; j < min(limit, end); ++j) add_row(j);
#pragma unroll
          for (int k = 0; k < 16; ++k)
            if (holds && limit > from && g[k] != 0.f) f[k] = g[k];
          __syncwarp();
        }
        if (!holds) continue;
        if (piece) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            a.part_o[((slot * 2 + i) * (a.d_k >> 2) + (b >> 2) + k) * kTile + row] = make_float4(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]);
          continue;
        }
        if (sum == 0.f) {                                          // no rows, or logits that are all -inf
#pragma unroll
          for (int k = 0; k < 16; ++k) f[k] = 0.f;
        }
        uint4 w[2];
#pragma unroll
        for (int k = 0; k < 8; ++k) (&w[k >> 2].x)[k & 3] = bf16_pair(f[2 * k] * inv, f[2 * k + 1] * inv);
        if (a.wide) {                                              // (a lane's row is a line of its own: half as many stores)
          ptx::store_32(out + b, w[0], w[1]);
        } else {
          reinterpret_cast<uint4*>(out + b)[0] = w[0];
          reinterpret_cast<uint4*>(out + b)[1] = w[1];
        }
      }
      ptx::tc_fence_before_sync();
      if (piece) {                                                 // (of weights that are all zero the outputs may be infinities all the same)
        a.part_ml[(slot * 2 + i) * kTile + row] = make_float2(sum == 0.f && tiles > 0 ? -FLT_MAX : ref, sum);
      } else if (holds && a.lse)
        a.lse[token * a.Hq + head] = sum == 0.f ? -INFINITY : (ref == -INFINITY ? 0.f : ref) * 0.6931471805599453f + logf(sum);
    }
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && watch->stop) {
    atomicExch(&a.status[0], GVOTE_ERR_TIMEOUT);
    atomicExch(&a.status[1], 27);
  }
  if (warp == 9) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

template <int kBoxes, bool kCut>
int32_t launch(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, ManyArgs& a, cudaStream_t st) {
  const size_t tile = (size_t)kBoxes * kTile * 128;
  const size_t room = 227 * 1024 - sizeof(Tail) - 2 * tile;
  a.stages = (int)(room / tile) < kMaxStages ? (int)(room / tile) : kMaxStages;
  const size_t smem = (2 + a.stages) * tile + sizeof(Tail);
  auto kernel = attend_many_kernel<kBoxes, kCut>;
  GVOTE_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  LaunchScope scope_("attend_many_kernel", st);
  const unsigned grid = !kCut && a.units < (uint32_t)kNumSms ? a.units : (unsigned)kNumSms;
  (void)launch_behind(kernel, dim3(grid), dim3(kThreads), smem, st, tq, tk, tv, a);
  GVOTE_LAUNCH_CHECK("attend_many_kernel");
  if (kCut) {
    LaunchScope join_("attend_join_kernel", st);
    (void)launch_behind(attend_join_kernel, dim3(a.units, 2, (unsigned)ceil_div(a.d_k / 4, kJoinQuads)), dim3(2 * kTile), 0, st, a);
    GVOTE_LAUNCH_CHECK("attend_join_kernel");
  }
  return GVOTE_OK;
}

}  // namespace

size_t attend_many_workspace(const gvote_params* p, int32_t, int64_t, int64_t max_q) {
  if (attend_takes_few(p, max_q)) return 0;
  return kScratchAt + kPiecesBytes + (size_t)2 * kNumSms * 2 * kTile * (p->d_k * 4 + 8);
}

int32_t launch_attend_many(const gvote_params* p, const AttendCall& c, const RowSource& s, char* ws, cudaStream_t st) {
  ManyArgs a;
  a.src = s;
  a.cu_q = c.cu_q; a.out = c.out; a.o_tok = c.o_tok; a.o_head = c.o_head; a.lse = c.lse;
  a.wide = ((reinterpret_cast<uintptr_t>(c.out) | (uintptr_t)(c.o_tok * 2) | (uintptr_t)(c.o_head * 2)) & 31) == 0;
  a.status = reinterpret_cast<int32_t*>(ws);
  a.Hq = p->n_q_heads; a.Hkv = p->n_kv_heads; a.G = p->n_q_heads / p->n_kv_heads; a.batch = c.batch; a.d_k = p->d_k;
  a.max_q = (int)c.max_q;
  a.tpt = kTile / a.G;
  a.pairs = (uint32_t)(c.batch == 1 ? ceil_div(c.max_q, 2 * a.tpt) : c.total_q / (2 * a.tpt) + c.batch);
  a.units = a.pairs * (uint32_t)a.Hkv;
  // (no unit can be longer than the longest request; where that leaves no more than a piece nothing is cut)
  const int64_t most = ceil_div(c.max_rows, kTile) + kGap;         // places of a unit
  const bool cut = a.units <= (uint32_t)kCutUnits && most > kPiece && most * a.units < (int64_t)1 << 31;
  a.pieces = reinterpret_cast<int2*>(ws + kScratchAt);
  a.part_o = reinterpret_cast<float4*>(ws + kScratchAt + kPiecesBytes);
  a.part_ml = reinterpret_cast<float2*>(ws + kScratchAt + kPiecesBytes + (size_t)2 * kNumSms * 2 * kTile * p->d_k * 4);
  a.c = (float)(1.4426950408889634 / sqrt((double)p->d_k));
  a.box_rows = s.tables && (1 << s.page_log2) < kTile ? 1 << s.page_log2 : kTile;
  // (the stride of a dimension of one is not used and may be anything)
  const uint64_t dims[3] = {(uint64_t)p->d_k, (uint64_t)p->n_q_heads, (uint64_t)c.total_q};
  const uint64_t strides[2] = {(uint64_t)(dims[1] > 1 ? c.q_head : p->d_k) * 2, (uint64_t)(dims[2] > 1 ? c.q_tok : p->d_k) * 2};
  const uint32_t box[3] = {64, (uint32_t)a.G, (uint32_t)a.tpt};
  CUtensorMap tq, tk, tv;
  if (!encode_tensor_map_bf16(&tq, c.Q, 3, dims, strides, box) || !row_maps(p, s, a.box_rows, &tk, &tv)) return GVOTE_ERR_CUDA;
  if (p->d_k <= 64) return cut ? launch<1, true>(tq, tk, tv, a, st) : launch<1, false>(tq, tk, tv, a, st);
  return cut ? launch<2, true>(tq, tk, tv, a, st) : launch<2, false>(tq, tk, tv, a, st);
}

}  // namespace gvote
