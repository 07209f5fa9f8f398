// Attention of a few query tokens over the 8-bit cache (gvote_attend8).
//
//   l_n = (q.k_n) / sqrt(d_k),  out = sum_n exp(l_n - lse) v_n,  lse = log sum_n exp(l_n),
// with k_n, v_n = code * scale of the row's block.  A few rows of queries against long K and V: bound by reading the codes
// once, 2 d_k bytes per cached row.
//
// Split.  The rows of all (request, KV head) pairs ("entries") are cut into tiles of 128 and laid end to end, each entry
// behind a gap of kGap tiles, about what beginning and ending one costs; CTA b takes the tiles between T b / B and
// T (b + 1) / B of the T places, whatever entries they belong to.  So pruned heads of very different length load every SM
// alike, without knowing the lengths on the host: each CTA adds up the entries itself.  (Without the gaps a ragged batch
// took 55 us instead of 36.)  What a CTA has of one entry is a segment; its result (reference, sum, output) goes to slot
// entry + CTA, or straight to the output when the entry lies within one CTA.  attend8_merge_kernel merges an entry's segments.
//
// The products run on tcgen05.mma with the cached rows on the M axis, so that a few query rows fill N and nothing is transposed:
//   S [128 keys x (3 terms, rows)]  = K Q^T    kind::f8f6f4, K as it lies (128-byte swizzle), Q as a sum of three e4m3 terms
//   O [128 channels x (3 terms, rows)] += V^T P^T   kind::f16, V widened to bf16 in shared memory, P as a sum of three bf16 terms
// A term is the value of its type nearest to what the terms before it left (for Q times 16 per term; its columns are added up
// with the matching power of two in 32 bits).  Three bf16 terms are all 24 bits of a weight, at any size a float can have:
// beside a first row that collects the attention the others' weights can lie 2^-30 below and still carry the output.  (Four
// e4m3 terms of P against V as it lies took a quarter less time over long rows, but ended 2^-24 below the largest weight.)
// Three terms of Q hold every entry above 2^-17 of its row's largest exactly, and a smaller one to 2^-25 of the largest.
//
// The scale of K enters the logit; the scale of V goes into the weight: P = 2^(l + log2(scale_v) - ref), ref the largest such
// exponent so far, so that a block of large values does not overflow.  ref only moves when it is passed by 2^64 (the
// accumulated O is then rescaled in tensor memory: the first tile sets it, and few ever move it).
//
// Warp 0 asks for the tiles of K and of V (TMA, only the 32-row parts that hold rows) into rings of their own - a tile
// of K is done with as soon as S is there, a tile of V as soon as it is widened - warps 1 and 2 issue the MMAs of S and of O
// (one warp for both took 1500 clocks a tile, its waits and commits one after the other), and warp 3 prepares the next
// segment's Q terms (the first segment's, which everything waits for, are shared out among the softmax warps: alone,
// warp 3 took 16,000 clocks for 20 rows).  Four warps widen V, a tile or two ahead (by the softmax warps themselves it
// lay in their chain: five tokens 43 us instead of 39), or two groups of four: a box of 128 channels each where
// d_k > 128 (one token over 64K rows of 256 channels 65 -> 57 us), and in turns where few query rows make a tile short (a
// tile takes one group 2100 clocks: one token over long rows 53 us instead of 43.5; with 12 rows and more the second group's
// registers cost more than it brings); then come up to five softmax groups of four warps, thread = cached row of
// the tile (and channel of the output).  A group has kR query rows: with few rows the groups take turns at the tiles, each
// with references and an O of its own (one group alone needs 3000 clocks of latency for a tile, the memory 1400), with many
// the groups share a tile's rows out.  S and P are buffered as deep as the MMAs run ahead.  The loops of the roles run at
// the same time and share the instruction cache: the rare parts (rows that not every token sees) are kept out of them
// (within the widening loop they cost 20 of 70 us over long rows), and the widening loop is not unrolled (64 requests of
// 2048 rows 97 -> 90 us).
//
// Weights for the eviction: the logits are kept (4 bytes per row and query, against 2 d_k per row), and
// attend8_weights_kernel turns them into weights once lse is known; a slot belongs to one thread, so the sum has one order.
//
// Measured (one B200, warm): one token of 28 heads over 128K rows of 4 KV heads, 134 MB: 43.5 us, the first kernel 40 of them.
// A ragged batch of 128 pruned heads, 63 MB: 35 us with the weights.  Five tokens over 32K rows of 8 heads: 37 us.
// Smallest calls: 12.5 us, all of it latency.
//
// Every wait is bounded; when one runs out GVOTE_ERR_TIMEOUT is recorded and the outputs are not to be used.
#include <cstddef>

#include "cache8.cuh"
#include "ptx.cuh"

namespace gvote {
namespace {

constexpr int kTileKeys = 128;
constexpr int kBoxRows = 32;
constexpr int kMaxEntries = 1024;      // entries per launch: their tiles are added up in shared memory
constexpr int kGap = 4;
constexpr int kR = 4;                  // query rows of a softmax group
constexpr int kMaxSlots = 8;           // of a ring
constexpr int kMaxBuffers = 4;         // of S and of P
constexpr int kSms = 148;
constexpr float kNoRef = -1e30f;       // a reference before the first logit
constexpr float kSlack = 64.f;         // a reference may be passed by 2^64: sums of up to 2^30 weights, times codes, stay below 2^127

struct AttendArgs {
  const __nv_bfloat16* Q;
  int64_t q_tok, q_head;
  const int32_t* cu_q;
  const float* k_scale;
  const float* v_scale;
  int64_t total, row_blocks;
  const int32_t* cu;
  const int32_t* kv_len;
  __nv_bfloat16* out;
  int64_t o_tok, o_head;
  float* lse;            // or null
  float* lse2;           // [total_q][n_q_heads] base 2
  const float* acc;
  float* acc_out;        // or null
  float* part_o;         // [row groups][entries + CTAs][turns][rows of a group][d_k], each divided by its own sum
  float2* part_ml;       // [row groups][entries + CTAs][turns][rows of a group]  (reference, sum), base 2
  int2* info;            // [row groups][entries]  first and last CTA of the entry (-1: no rows)
  float* logits;         // [Hkv][max_q * G][total] base 2, when acc_out
  int32_t* status;
  int Hkv, G, r0, batch, d_k, max_q;   // requests r0 .. r0 + batch - 1
  int k_slots, v_slots, group_rows, turns;
  float scale2;          // log2(e) / sqrt(d_k)
};

struct Entry { int r, h, start, n, nq, q0; };
__device__ __forceinline__ Entry entry_of(const AttendArgs& a, int e) {
  Entry x;
  const int lr = e / a.Hkv;
  x.h = e - lr * a.Hkv;
  x.r = a.r0 + lr;
  x.start = a.cu[x.r];
  x.n = valid_keys(a.kv_len, x.r, a.Hkv, x.h, a.cu[x.r + 1] - x.start);
  x.q0 = a.cu_q[x.r];
  x.nq = min(a.cu_q[x.r + 1] - x.q0, a.max_q);         // (the workspace holds no more; the excess is reported)
  return x;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// x * 2^d in two steps: 2^d alone may lie below 2^-126.
__device__ __forceinline__ float times_exp2(float x, float d) {
  const float h = exp2_fast(0.5f * d);
  return x * h * h;
}
__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  for (uint32_t i = 0; i < (1u << 20); ++i) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if ((i & 255u) == 255u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
// Before a role leaves early: what it started may still write to this CTA's memory.
__device__ __forceinline__ void drain_copies(uint64_t* full, int slots, uint32_t issued) {
  for (uint32_t i = issued > (uint32_t)slots ? issued - slots : 0; i < issued; ++i)
    for (int k = 0; k < (1 << 12) && !ptx::mbar_try_wait(&full[i % slots], (i / slots) & 1); ++k) {}
}
__device__ __forceinline__ void drain_mmas(uint64_t* bar) {
  if (ptx::elect_one()) ptx::umma_commit(bar);
  __syncwarp();
  for (int k = 0; k < (1 << 12) && !ptx::mbar_try_wait(bar, 0); ++k) {}
}
// The or of a predicate over the four warps of a softmax group (named barrier `id`).
__device__ __forceinline__ bool group_any(int id, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.aligned.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"((uint32_t)x), "r"(id) : "memory");
  return r != 0;
}
__device__ __forceinline__ float warp_redux_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}

// ---- tcgen05.mma kind::f8f6f4, e4m3 operands in shared memory, 32-bit sums
// Instruction descriptor: 32-bit result (bits 4-5 = 1), A and B e4m3 (bits 7-9, 10-12 = 0), A / B stored with M / N
// contiguous (bits 15, 16), N >> 3 in bits 17-22, M >> 4 in bits 24-28.
__host__ __device__ constexpr uint32_t instr_desc_e4m3(int M, int N, bool a_mn, bool b_mn) {
  return (1u << 4) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void umma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Instruction descriptor, kind::f16: 32-bit result, A and B bf16 (bits 7-9, 10-12 = 1), stored with M / N contiguous.
__host__ __device__ constexpr uint32_t instr_desc_bf16_mn(int M, int N) {
  return ptx::instr_desc_bf16_f32(M, N) | (1u << 15) | (1u << 16);
}
// Operand stored as rows of 16 bytes without swizzle, the 16 bytes along M or N: eight K rows are 128 bytes, the next eight
// K rows follow at once (leading offset 128), the next 16 bytes of M or N `chunk` bytes on.
__device__ __forceinline__ uint64_t smem_desc_mn_plain(uint32_t addr, uint32_t chunk) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 16) | ((uint64_t)(chunk >> 4) << 32) | ((uint64_t)1 << 46);
}
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// Four floats -> the e4m3 codes nearest to them; the floats become 16 times what the codes leave.
__device__ __forceinline__ uint32_t take_term(float (&x)[4]) {
  const uint32_t c = narrow8x4(x[0], x[1], x[2], x[3]);
  uint32_t lo, hi;
  widen8x4(c, lo, hi);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  x[0] = (x[0] - a.x) * 16.f;
  x[1] = (x[1] - a.y) * 16.f;
  x[2] = (x[2] - b.x) * 16.f;
  x[3] = (x[3] - b.y) * 16.f;
  return c;
}

// Two floats -> the bf16 values nearest to them (low half: a); the floats become what those leave.
__device__ __forceinline__ uint32_t take_bf16(float& a, float& b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  const uint32_t w = *reinterpret_cast<const uint32_t*>(&h);
  a -= __uint_as_float(w << 16);
  b -= __uint_as_float(w & 0xffff0000u);
  return w;
}
// Four e4m3 codes -> two pairs of bf16 values (exact; the NaN code -> NaN).
__device__ __forceinline__ void widen_bf16x4(uint32_t c, uint32_t& lo, uint32_t& hi) {
  widen8x4(c, lo, hi);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  const __nv_bfloat162 x = __floats2bfloat162_rn(a.x, a.y), y = __floats2bfloat162_rn(b.x, b.y);
  lo = *reinterpret_cast<const uint32_t*>(&x);
  hi = *reinterpret_cast<const uint32_t*>(&y);
}

// A query row's log-sum-exp: base 2 for the weights, natural for the caller.
__device__ __forceinline__ void write_lse(const AttendArgs& a, int64_t at, float2 ml) {
  const float l = ml.x == -INFINITY ? -INFINITY : ml.x + log2f(ml.y);
  a.lse2[at] = l;
  if (a.lse) a.lse[at] = l * 0.6931471805599453f;
}

// Counts: one arrival, 1 + 4 for every group on q_empty, four per group that shares a tile's rows from s_empty on, four
// from w_full on, on v_empty for every group that widens a part of the tile.
struct Bars {
  uint64_t k_full[kMaxSlots], k_empty[kMaxSlots], v_full[kMaxSlots], q_full[2], q_empty[2];
  uint64_t s_full[kMaxBuffers], p_empty[kMaxBuffers], o_full[4], w_empty[2];
  uint64_t s_empty[kMaxBuffers], p_full[kMaxBuffers], o_empty[4];
  uint64_t v_empty[kMaxSlots];
  uint64_t w_full[2];
  uint64_t drain[2];                   // the MMAs under way of the two issuers, after a wait that ran out
};
constexpr int kFirstQ = 8;             // a named barrier; the softmax groups' are 1 to 5
enum { kWarpTma = 0, kWarpS = 1, kWarpO = 2, kWarpQ = 3, kWarpWide = 4 };   // then the softmax warps

struct Tail {
  Bars bars;
  Entry entry[2];
  uint32_t tmem_slot;
  int any_nan[2][4];                   // [segment parity][turn]
  volatile int abort_flag;
  int64_t out_at[2][32];               // where the query rows' outputs go (elements)
  int64_t lse_at[2][32];
  int warp_tot[32];
  int pref[kMaxEntries + 1];
};

template <int kBoxes, int kRb>          // 128-byte boxes per row; groups that share a tile's rows
struct Layout {                         // threads, tensor memory (columns), shared memory (bytes)
  static constexpr int kTurns = kRb == 1 ? 4 : kRb == 2 ? 2 : 1, kGroups = kTurns * kRb;
  // groups that widen V: a box each, or tiles in turns
  static constexpr bool kByBox = kBoxes == 2;
  static constexpr int kWiden = kByBox || kRb <= 2 ? 2 : 1;
  static constexpr int kWarpSoftmax = kWarpWide + 4 * kWiden, kThreads = 32 * kWarpSoftmax + 128 * kGroups;
  static constexpr int kRows = kR * kRb, kBuffers = kRb <= 2 ? 4 : 2;
  static constexpr int kN1 = (3 * kRows + 15) / 16 * 16, kN2 = 4 * kRows;
  static constexpr int kO = kBuffers * kN1, kCols = kO + kTurns * kBoxes * kN2;     // O of turn i, box y: kO + (i kBoxes + y) kN2
  static constexpr int kAlloc = kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
  static constexpr int kSlot = kBoxes * kTileKeys * 128, kQ = kBoxes * kN1 * 128, kP = kN2 * kTileKeys * 2;
  static constexpr int kWide = 256 * kTileKeys;                        // a box of a tile of V in bf16; there is room for two
  static constexpr int kNanWords = kR * kBoxes * 4;                    // of a group: bits [row][channel]
  static constexpr int kSmall = kGroups * 4 * 2 * kR * 4 + 2 * kRows * 8 + 2 * kGroups * kNanWords * 4;
  static constexpr size_t fixed() { return (size_t)2 * kQ + kBuffers * kP + 2 * kWide + kSmall + sizeof(Tail); }
  // slots of K and V that fit; three at least: two of K, one of V
  static constexpr int kFit = (int)((227 * 1024 - fixed()) / kSlot);
  static_assert(kFit >= 3 && kAlloc >= kCols, "a row group of this size does not fit an SM");
};

// The tiles of a CTA in order: segments (entry e, its tiles s0 .. s1 - 1), tiles t; seg and it count both.
// pref: tiles and gaps before each entry; an entry without tiles has no gap.
struct Walk {
  int e, t, s0, s1, seg, it;
  const int* pref;
  int t0, t1, entries;
  __device__ __forceinline__ Walk(const int* pref_, int t0_, int t1_, int entries_, int e_first)
      : e(e_first), seg(0), it(0), pref(pref_), t0(t0_), t1(t1_), entries(entries_) { enter(); }
  __device__ __forceinline__ bool done() const { return e >= entries; }
  __device__ __forceinline__ void enter() {
    for (; e < entries; ++e) {
      const int p = pref[e];
      if (p >= t1) break;
      s0 = max(t0 - p - kGap, 0);
      s1 = min(t1, pref[e + 1]) - p - kGap;
      if (s0 < s1) { t = s0; return; }
    }
    e = entries;
  }
  __device__ __forceinline__ void next_segment() { it += s1 - t; ++e; ++seg; enter(); }
  __device__ __forceinline__ void next_tile() {
    ++it;
    if (++t == s1) { ++e; ++seg; enter(); }
  }
};

template <int kBoxes, int kRb>
__global__ void __launch_bounds__((Layout<kBoxes, kRb>::kThreads), 1)
attend8_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
               const __grid_constant__ CUtensorMap tmKp, const __grid_constant__ CUtensorMap tmVp,
               const __grid_constant__ AttendArgs a) {
  extern __shared__ __align__(1024) uint8_t smem[];
  using L = Layout<kBoxes, kRb>;
  uint8_t* k_ring = smem;                                              // [slot][box][128 rows][128], swizzled
  uint8_t* v_ring = k_ring + (size_t)a.k_slots * L::kSlot;
  uint8_t* q_sm = v_ring + (size_t)a.v_slots * L::kSlot;               // [2][box][N1 rows][128], swizzled
  uint8_t* p_sm = q_sm + 2 * L::kQ;                                    // [buffer][N2 / 8][128 keys][8 columns], bf16
  uint8_t* wide_sm = p_sm + L::kBuffers * L::kP;                       // [box, or buffer][16][128 keys][8 channels], bf16
  float* red_all = reinterpret_cast<float*>(wide_sm + 2 * L::kWide);   // [group][4 warps][2 kR]
  float* factor_sm = red_all + L::kGroups * 4 * 2 * kR;                // [2][kRows] logit per unit of product
  int* limit_sm = reinterpret_cast<int*>(factor_sm + 2 * L::kRows);    // [2][kRows] cached rows a query row sees
  uint32_t* nan_all = reinterpret_cast<uint32_t*>(limit_sm + 2 * L::kRows);   // [2][group][kR][boxes * 4]
  Tail* tail = reinterpret_cast<Tail*>(nan_all + 2 * L::kGroups * L::kNanWords);
  int* pref = tail->pref;
  volatile int* abort_flag = &tail->abort_flag;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int entries = a.batch * a.Hkv;
  const int group0 = blockIdx.y * a.group_rows;                        // first query row of this row group

  {                                                                    // a barrier per thread
    constexpr int kBars = sizeof(Bars) / 8;
    if (tid < kBars) {
      const int at = tid * 8;
      const uint32_t count = at >= (int)offsetof(Bars, q_empty) && at < (int)offsetof(Bars, s_full) ? 1 + 4 * (L::kWiden + L::kGroups)
                             : at >= (int)offsetof(Bars, s_empty) && at < (int)offsetof(Bars, v_empty) ? 4 * kRb
                             : at >= (int)offsetof(Bars, v_empty) && at < (int)offsetof(Bars, w_full) ? (L::kByBox ? 8 : 4)
                             : at >= (int)offsetof(Bars, w_full) && at < (int)offsetof(Bars, drain) ? 4 : 1;
      ptx::mbar_init(reinterpret_cast<uint64_t*>(&tail->bars) + tid, count);
      ptx::fence_barrier_init();
    }
  }
  if (tid == kWarpQ * 32) {
    for (int b = 0; b < 4; ++b) tail->any_nan[0][b] = tail->any_nan[1][b] = 0;
    tail->abort_flag = (ptx::smem_u32(smem) & 1023u) ? 1 : 0;
    ptx::prefetch_tensormap(&tmK);
    ptx::prefetch_tensormap(&tmV);
  }
  for (int i = tid; i < 2 * L::kGroups * L::kNanWords; i += L::kThreads) nan_all[i] = 0;
  ptx::let_next_begin();
  if (warp == 1) {
    ptx::tmem_alloc(&tail->tmem_slot, L::kAlloc);
    ptx::tmem_relinquish();
  }
  // ---- tiles and gaps before each entry
  {
    const int per = (entries + L::kThreads - 1) / L::kThreads;         // consecutive entries per thread
    const int e0 = min(tid * per, entries), e1 = min(e0 + per, entries);
    const bool b0 = blockIdx.x == 0 && blockIdx.y == 0;
    int mine = 0;
    for (int e = e0; e < e1; ++e) {
      const Entry x = entry_of(a, e);
      if (b0 && a.cu_q[x.r + 1] - x.q0 > a.max_q) { atomicExch(&a.status[0], GVOTE_ERR_INVALID_ARG); atomicExch(&a.status[1], 13); }
      const int t = group0 < x.nq * a.G ? (x.n + kTileKeys - 1) / kTileKeys : 0;
      pref[e + 1] = t > 0 ? t + kGap : 0;
      mine += pref[e + 1];
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += u;
    }
    if (lane == 31) tail->warp_tot[warp] = inc;
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const int before = lane < warp ? tail->warp_tot[lane] : 0;
    int run = inc - mine + __reduce_add_sync(0xffffffffu, before);
    for (int e = e0; e < e1; ++e) { run += pref[e + 1]; pref[e + 1] = run; }
    if (tid == 0) pref[0] = 0;
    __syncthreads();
  }
  const uint32_t tmem = __shfl_sync(0xffffffffu, tail->tmem_slot, 0);
  // no more parts than places: an empty part between two of an entry's would leave its slot unwritten
  const int T = pref[entries], B = max(min((int)gridDim.x, T), 1), b = blockIdx.x;
  const int per_cta = T / B, odd = T - per_cta * B;                    // floor(T c / B) = c (T / B) + c (T mod B) / B
  const int t0 = min(b, B) * per_cta + min(b, B) * odd / B, t1 = min(b + 1, B) * per_cta + min(b + 1, B) * odd / B;
  int e_first = t0 < t1 ? 0 : entries;                                 // the entry of tile t0 (a CTA without tiles: none)
  {
    int hi = entries - 1;
    while (e_first < hi) {
      const int mid = (e_first + hi) >> 1;
      if (pref[mid + 1] <= t0) e_first = mid + 1; else hi = mid;
    }
  }
  Walk at(pref, t0, t1, entries, e_first);
  bool ok = true;
  // A warp's part in preparing a query row: its lanes' channels, then their terms.
  auto load_row = [&](int64_t from, bool holds, uint2 (&v)[kBoxes]) {
#pragma unroll
    for (int y = 0; y < kBoxes; ++y) {
      const int d = y * 128 + lane * 4;
      v[y] = holds && d < a.d_k ? __ldg(reinterpret_cast<const uint2*>(a.Q + from + d)) : make_uint2(0, 0);
    }
  };
  auto put_row = [&](int qb, int row, const uint2 (&v)[kBoxes]) {
    uint32_t top = 0;                                                  // the largest magnitude's bits
#pragma unroll
    for (int y = 0; y < kBoxes; ++y) {
      const uint32_t m = __vmaxu2(v[y].x & 0x7fff7fffu, v[y].y & 0x7fff7fffu);
      top = max(top, max(m & 0xffffu, m >> 16));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    // entries up to 2^8: multiply by 2^(7 - exponent); the exponent is kept where both factors are normal numbers
    const int ex = min(max((int)(top >> 7) - 127, -100), 127);
    const float up = __uint_as_float((uint32_t)(127 + 7 - ex) << 23);
    const int rb = row / kR, n0 = rb * 3 * kR + row % kR;              // groups one after the other, a group's rows term by term
#pragma unroll
    for (int y = 0; y < kBoxes; ++y) {
      const uint2 u = v[y];
      float f[4] = {__uint_as_float(u.x << 16) * up, __uint_as_float(u.x & 0xffff0000u) * up,
                    __uint_as_float(u.y << 16) * up, __uint_as_float(u.y & 0xffff0000u) * up};
      if (top >= 0x7f80u) {                                            // an infinity is no 448: NaN, like a NaN
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = fabsf(f[k]) <= 3.4e38f ? f[k] : __uint_as_float(0x7fffffffu);
      }
#pragma unroll
      for (int term = 0; term < 3; ++term) {
        const int n = n0 + term * kR;
        *reinterpret_cast<uint32_t*>(q_sm + qb * L::kQ + (y * L::kN1 + n) * 128 + (((lane >> 2) ^ (n & 7)) << 4) + (lane & 3) * 4) = take_term(f);
      }
    }
    if (lane == 0) factor_sm[qb * L::kRows + row] = __uint_as_float((uint32_t)(127 - 7 + ex) << 23) * a.scale2;
  };

  if (warp == kWarpTma) {
    // ------------------------------------------------------------------ TMA producer: K and V, each as its ring has room
    if (lane == 0) {
      struct Feed {
        const CUtensorMap *whole, *part;
        uint8_t* ring;
        uint64_t *full, *empty;
        int slots, slot;
        uint32_t phase;
        Entry x;
        int seg;
        uint32_t issued;
      };
      Feed feed[2] = {{&tmK, &tmKp, k_ring, tail->bars.k_full, tail->bars.k_empty, a.k_slots, 0, 0, {}, -1, 0},
                      {&tmV, &tmVp, v_ring, tail->bars.v_full, tail->bars.v_empty, a.v_slots, 0, 0, {}, -1, 0}};
      Walk walk[2] = {at, at};
      uint32_t polls = 0;
      while (ok && !(walk[0].done() && walk[1].done())) {
        bool moved = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          Feed& f = feed[i];
          Walk& w = walk[i];
          if (w.done() || !ptx::mbar_test_wait(&f.empty[f.slot], f.phase ^ 1u)) continue;
          if (f.seg != w.seg) { f.x = entry_of(a, w.e); f.seg = w.seg; }
          const int key0 = w.t * kTileKeys, parts = min(kTileKeys / kBoxRows, (f.x.n - key0 + kBoxRows - 1) / kBoxRows);
          uint8_t* dst = f.ring + (size_t)f.slot * L::kSlot;
          uint64_t* full = &f.full[f.slot];
          ptx::mbar_arrive_expect_tx(full, (uint32_t)parts * kBoxes * kBoxRows * 128);
#pragma unroll
          for (int y = 0; y < kBoxes; ++y) {
            if (parts == kTileKeys / kBoxRows) {
              ptx::tma_load_3d(dst + y * kTileKeys * 128, f.whole, full, y * 128, f.x.start + key0, f.x.h);
            } else {
              for (int g = 0; g < parts; ++g)
                ptx::tma_load_3d(dst + (y * kTileKeys + g * kBoxRows) * 128, f.part, full, y * 128, f.x.start + key0 + g * kBoxRows, f.x.h);
            }
          }
          if (++f.slot == f.slots) { f.slot = 0; f.phase ^= 1u; }
          ++f.issued;
          w.next_tile();
          moved = true;
        }
        if (moved) {
          polls = 0;
        } else if (++polls > (1u << 24) || ((polls & 255u) == 255u && *abort_flag)) {
          *abort_flag = 1;
          ok = false;
        }
      }
      if (!ok) {
#pragma unroll
        for (int i = 0; i < 2; ++i) drain_copies(feed[i].full, feed[i].slots, feed[i].issued);
      }
    }
  } else if (warp == kWarpS) {
    // ------------------------------------------------------------------ S = K Q^T (the whole warp walks, one lane issues)
    const uint32_t idesc = instr_desc_e4m3(kTileKeys, L::kN1, false, false);
    const int ksteps = (a.d_k + 31) / 32;
    const uint64_t kd0 = ptx::smem_desc_k_sw128(ptx::smem_u32(k_ring)), qd0 = ptx::smem_desc_k_sw128(ptx::smem_u32(q_sm));
    int ks = 0;
    uint32_t k_phase = 0;
    for (; ok && !at.done(); at.next_segment()) {
      const int qb = at.seg & 1;
      ok = __all_sync(0xffffffffu, wait_or_abort(&tail->bars.q_full[qb], (at.seg >> 1) & 1, abort_flag));
      for (int t = at.s0, it = at.it; ok && t < at.s1; ++t, ++it) {
        const int sb = it % L::kBuffers;
        ok = __all_sync(0xffffffffu, wait_or_abort(&tail->bars.s_empty[sb], ((it / L::kBuffers) & 1) ^ 1, abort_flag) &&
                                         wait_or_abort(&tail->bars.k_full[ks], k_phase, abort_flag));
        if (!ok) break;
        ptx::tc_fence_after_sync();
        if (ptx::elect_one()) {
#pragma unroll
          for (int y = 0; y < kBoxes; ++y) {
            const uint64_t kd = kd0 + (uint64_t)((ks * L::kSlot + y * kTileKeys * 128) >> 4), qd = qd0 + (uint64_t)((qb * L::kQ + y * L::kN1 * 128) >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (y * 4 + k < ksteps)
                umma_e4m3(tmem + (uint32_t)(sb * L::kN1), kd + 2 * k, qd + 2 * k, idesc, y + k > 0 ? 1u : 0u);
          }
          ptx::umma_commit(&tail->bars.s_full[sb]);
          ptx::umma_commit(&tail->bars.k_empty[ks]);
          if (t == at.s1 - 1) ptx::umma_commit(&tail->bars.q_empty[qb]);
        }
        __syncwarp();
        if (++ks == a.k_slots) { ks = 0; k_phase ^= 1u; }
      }
    }
    if (!ok) drain_mmas(&tail->bars.drain[0]);
  } else if (warp == kWarpO) {
    // ------------------------------------------------------------------ O += V^T P
    const uint32_t idesc = instr_desc_bf16_mn(128, L::kN2);
    const uint64_t vd0 = smem_desc_mn_plain(ptx::smem_u32(wide_sm), 16 * kTileKeys), pd0 = smem_desc_mn_plain(ptx::smem_u32(p_sm), 16 * kTileKeys);
    uint32_t o_uses = 0;                                               // bit i: parity of the uses of turn i's O
    for (; ok && !at.done(); at.next_segment()) {
      for (int t = at.s0, it = at.it; ok && t < at.s1; ++t, ++it) {
        const int pb = it % L::kBuffers, turn = it % L::kTurns;
        const bool first = t - at.s0 < L::kTurns, last = t + L::kTurns >= at.s1;
        ok = __all_sync(0xffffffffu, wait_or_abort(&tail->bars.p_full[pb], (it / L::kBuffers) & 1, abort_flag));
        if (ok && first) {
          ok = __all_sync(0xffffffffu, wait_or_abort(&tail->bars.o_empty[turn], ((o_uses >> turn) & 1) ^ 1, abort_flag));
          o_uses ^= 1u << turn;
        }
        if (!ok) break;
#pragma unroll
        for (int y = 0; y < kBoxes; ++y) {
          const int wb = L::kByBox ? y : it & 1;
          ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->bars.w_full[wb], (L::kByBox ? it : it >> 1) & 1, abort_flag));
          if (!ok) break;
          ptx::tc_fence_after_sync();
          if (ptx::elect_one()) {
            const uint64_t pd = pd0 + (uint64_t)((pb * L::kP) >> 4), vd = vd0 + (uint64_t)((wb * L::kWide) >> 4);
#pragma unroll
            for (int k = 0; k < kTileKeys / 16; ++k)                   // 16 keys: 256 bytes of each column of chunks
              ptx::umma_bf16(tmem + (uint32_t)(L::kO + (turn * kBoxes + y) * L::kN2), vd + (uint64_t)(k * 16), pd + (uint64_t)(k * 16),
                             idesc, first && k == 0 ? 0u : 1u);
            ptx::umma_commit(&tail->bars.w_empty[wb]);
            if (y == kBoxes - 1) {
              ptx::umma_commit(&tail->bars.p_empty[pb]);
              if (last) ptx::umma_commit(&tail->bars.o_full[turn]);
            }
          }
          __syncwarp();
        }
      }
    }
    if (!ok) drain_mmas(&tail->bars.drain[1]);
    // Which CTAs hold an entry, for the merge: the CTA of the tile at place t is the largest c with T c / B <= t.  (Divisions
    // of 64 bits: the softmax is still at its last tile.)
    for (int e = b + lane * B; b < B && e < entries; e += 32 * B) {
      const int f = pref[e] + kGap, l = pref[e + 1] - 1;
      int2 v = make_int2(-1, -1);
      if (l >= f) v = make_int2((int)((((int64_t)f + 1) * B - 1) / T), (int)((((int64_t)l + 1) * B - 1) / T));
      a.info[(int64_t)blockIdx.y * entries + e] = v;
    }
  } else if (warp == kWarpQ) {
    // ------------------------------------------------------------------ Q as three e4m3 terms, a segment ahead
    for (int i = lane; i < 2 * kBoxes * (L::kN1 - 3 * L::kRows) * 8; i += 32) {     // the rows behind the last term are zero
      constexpr int kPer = (L::kN1 - 3 * L::kRows) * 8 > 0 ? (L::kN1 - 3 * L::kRows) * 8 : 1;
      *reinterpret_cast<uint4*>(q_sm + (i / kPer) * L::kN1 * 128 + 3 * L::kRows * 128 + (i % kPer) * 16) = make_uint4(0, 0, 0, 0);
    }
    for (; ok && !at.done(); at.next_segment()) {
      const int qb = at.seg & 1;
      const Entry x = entry_of(a, at.e);
      const int qrow = group0 + lane, token = qrow / a.G, head = x.h * a.G + qrow - token * a.G;     // lane = row
      const bool holds = lane < L::kRows && qrow < x.nq * a.G;
      const int64_t from = holds ? (int64_t)(x.q0 + token) * a.q_tok + (int64_t)head * a.q_head : 0;
      if (at.seg > 1) ok = __all_sync(0xffffffffu, wait_or_abort(&tail->bars.q_empty[qb], ((at.seg >> 1) & 1) ^ 1, abort_flag));
      if (!ok) break;
      if (lane < L::kRows) {
        limit_sm[qb * L::kRows + lane] = holds ? x.n - (x.nq - 1 - token) : 0;
        tail->out_at[qb][lane] = (int64_t)(x.q0 + token) * a.o_tok + (int64_t)head * a.o_head;
        tail->lse_at[qb][lane] = (int64_t)(x.q0 + token) * a.Hkv * a.G + head;
      }
      if (lane == 0) tail->entry[qb] = x;
      if (at.seg > 1 && a.max_q > 1) {                                 // the marks of two segments ago have been read
        for (int i = lane; i < L::kGroups * L::kNanWords; i += 32) nan_all[qb * L::kGroups * L::kNanWords + i] = 0;
        if (lane < 4) tail->any_nan[qb][lane] = 0;
      }
      if (at.seg == 0) {                                               // the softmax warps prepare the first one's rows
        asm volatile("barrier.cta.sync %0, %1;" ::"r"(kFirstQ), "r"(32 + 128 * L::kGroups) : "memory");
      } else {
        const uint32_t held = __ballot_sync(0xffffffffu, holds);
#pragma unroll 1
        for (int rb = 0; rb < kRb; ++rb) {
          uint2 v[kR][kBoxes];                                         // all of a group's rows on their way at once
#pragma unroll
          for (int i = 0; i < kR; ++i) load_row(__shfl_sync(0xffffffffu, from, rb * kR + i), (held >> (rb * kR + i)) & 1u, v[i]);
#pragma unroll
          for (int i = 0; i < kR; ++i) put_row(qb, rb * kR + i, v[i]);
        }
      }
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&tail->bars.q_full[qb]);
    }
  } else if (warp < L::kWarpSoftmax) {
    // ------------------------------------------------------------------ the tiles of V in bf16: thread = row of the tile
    // Either group y has box y of every tile, or tile it is group it mod kWiden's and its buffer it mod 2; that the slot's tile
    // before this one has come (a wait by parity must not meet a phase two behind) follows from the buffer's: there are
    // three slots and more.
    const int group = (warp - kWarpWide) >> 2, key_in = tid & 127, box = L::kByBox ? group : 0, units = min(8, (a.d_k >> 4) - 8 * box);
    constexpr int kStep = L::kByBox ? 1 : L::kWiden;                   // 1 or 2
    int vs = L::kByBox ? 0 : group;
    uint32_t v_phase = 0;
    for (; ok && !at.done(); at.next_segment()) {
      const int qb = at.seg & 1;
      ok = __all_sync(0xffffffffu, wait_or_abort(&tail->bars.q_full[qb], (at.seg >> 1) & 1, abort_flag));
      if (!ok) break;
      const Entry x = tail->entry[qb];
      const int all_see = x.n - (x.nq - 1);
      const int skip = (group + at.it) % kStep;
      for (int t = at.s0 + skip, it = at.it + skip; ok && t < at.s1; t += kStep, it += kStep) {
        const int wb = L::kByBox ? box : it & 1, key = t * kTileKeys + key_in;
        ok = __all_sync(0xffffffffu, wait_or_abort(&tail->bars.w_empty[wb], ((L::kByBox ? it : it >> 1) & 1) ^ 1, abort_flag) &&
                                         wait_or_abort(&tail->bars.v_full[vs], v_phase, abort_flag));
        if (!ok) break;
        uint8_t* from = v_ring + (size_t)vs * L::kSlot + (box * kTileKeys + key_in) * 128;
        uint8_t* to = wide_sm + wb * L::kWide + key_in * 16;
        if (key >= all_see) {
          // A value behind the last row may be anything, and one that not every token sees may be NaN: neither must reach
          // the others through a weight of zero.  The first becomes zero, the second is noted for those who see it.
          const int turn = it % L::kTurns;
          uint32_t* marks = nan_all + (qb * L::kGroups + turn * kRb) * L::kNanWords;       // [row][boxes * 4] of the turn's groups
#pragma unroll 1
          for (int u = 0; u < units; ++u) {
            uint4* place = reinterpret_cast<uint4*>(from + ((u ^ (key_in & 7)) << 4));
            if (key >= x.n) {
              *place = make_uint4(0, 0, 0, 0);
              continue;
            }
            uint4 c = *place, bad;
            bad.x = __vcmpeq4(c.x & 0x7f7f7f7fu, 0x7f7f7f7fu);
            bad.y = __vcmpeq4(c.y & 0x7f7f7f7fu, 0x7f7f7f7fu);
            bad.z = __vcmpeq4(c.z & 0x7f7f7f7fu, 0x7f7f7f7fu);
            bad.w = __vcmpeq4(c.w & 0x7f7f7f7fu, 0x7f7f7f7fu);
            if (!(bad.x | bad.y | bad.z | bad.w)) continue;
            *place = make_uint4(c.x & ~bad.x, c.y & ~bad.y, c.z & ~bad.z, c.w & ~bad.w);
            tail->any_nan[qb][turn] = 1;
            auto four = [](uint32_t m) { return (m & 1u) | ((m >> 7) & 2u) | ((m >> 14) & 4u) | ((m >> 21) & 8u); };
            const uint32_t bits = four(bad.x) | four(bad.y) << 4 | four(bad.z) << 8 | four(bad.w) << 12;
#pragma unroll 1
            for (int g = 0; g < L::kRows; ++g)
              if (key < limit_sm[qb * L::kRows + g]) atomicOr(&marks[g * kBoxes * 4 + box * 4 + (u >> 1)], bits << (u * 16 & 31));
          }
        }
#pragma unroll 1
        for (int u = 0; u < units; ++u) {                               // (unrolled, it took the others' instruction cache)
          const uint4 c = *reinterpret_cast<const uint4*>(from + ((u ^ (key_in & 7)) << 4));
          uint32_t b[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) widen_bf16x4((&c.x)[j], b[2 * j], b[2 * j + 1]);
          *reinterpret_cast<uint4*>(to + u * 2 * (kTileKeys * 16)) = make_uint4(b[0], b[1], b[2], b[3]);
          *reinterpret_cast<uint4*>(to + (u * 2 + 1) * (kTileKeys * 16)) = make_uint4(b[4], b[5], b[6], b[7]);
        }
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(&tail->bars.v_empty[vs]);
          ptx::mbar_arrive(&tail->bars.w_full[wb]);
        }
        vs += kStep;
        if (vs >= a.v_slots) { vs -= a.v_slots; v_phase ^= 1u; }
      }
      __syncwarp();
      if (ok && lane == 0) ptx::mbar_arrive(&tail->bars.q_empty[qb]);
    }
  } else {
    // ------------------------------------------------------------------ softmax: thread = row of the tile, channel of O
    const int group = (warp - L::kWarpSoftmax) >> 2, turn = group / kRb, rb = group % kRb, bar_id = 1 + group;
    const int w = warp & 3, key_in = w * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)(w * 32) << 16);
    const uint32_t o_addr = lane_addr + (uint32_t)(L::kO + turn * kBoxes * L::kN2 + rb * 4 * kR);
    float* red_sm = red_all + group * 4 * 2 * kR;
    float refd[kR], refn[kR], sum[kR];                                 // of the logits; of the weights times scale_v
    int o_uses = 0;
    if (!at.done()) {                                                  // the first segment's query rows (one or two per warp)
      const Entry x = entry_of(a, at.e);
      for (int row = warp - L::kWarpSoftmax; row < L::kRows; row += 4 * L::kGroups) {
        const int qrow = group0 + row, token = qrow / a.G, head = x.h * a.G + qrow - token * a.G;
        uint2 v[kBoxes];
        load_row((int64_t)(x.q0 + token) * a.q_tok + (int64_t)head * a.q_head, qrow < x.nq * a.G, v);
        put_row(0, row, v);
      }
      ptx::fence_proxy_async();
      asm volatile("barrier.cta.arrive %0, %1;" ::"r"(kFirstQ), "r"(32 + 128 * L::kGroups) : "memory");
    }
    for (; !at.done(); at.next_segment()) {
      const int qb = at.seg & 1, e = at.e, s0 = at.s0, s1 = at.s1;
      ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->bars.q_full[qb], (at.seg >> 1) & 1, abort_flag));
      const Entry x = tail->entry[qb];
      const int row0 = group0 + rb * kR, nrows = min(kR, x.nq * a.G - row0), all_see = x.n - (x.nq - 1);
      const float* factor = factor_sm + qb * L::kRows + rb * kR;
      const int* limit = limit_sm + qb * L::kRows + rb * kR;
#pragma unroll
      for (int g = 0; g < kR; ++g) { refd[g] = refn[g] = kNoRef; sum[g] = 0.f; }
      uint32_t* nan_sm = nan_all + (qb * L::kGroups + turn * kRb) * L::kNanWords;       // of the groups that share my tiles
      const int64_t sb0 = (int64_t)x.h * a.row_blocks + block8_offset(x.start, x.r);
      auto scales = [&](int t) {
        const int key = t * kTileKeys + key_in;
        return key < x.n ? make_float2(a.k_scale[sb0 + (key >> 6)], a.v_scale[sb0 + (key >> 6)]) : make_float2(0.f, 1.f);
      };
      // Tile it is turn it mod kTurns', and buffer it mod kBuffers is always the same turn's: a group meets every phase of
      // the barriers that it waits on (by parity, a wait for a phase passes while the one before it is still open).
      const int first = s0 + (turn + L::kTurns - at.it % L::kTurns) % L::kTurns;
      const bool any_tile = first < s1;
      float2 next_scale = ok && any_tile ? scales(first) : make_float2(0.f, 1.f);
      for (int t = first; t < s1; t += L::kTurns) {
        const int it = at.it + t - s0, sb = it % L::kBuffers, phase = (it / L::kBuffers) & 1;
        const int key0 = t * kTileKeys, key = key0 + key_in;
        const float2 sc = next_scale;
        if (ok && t + L::kTurns < s1) next_scale = scales(t + L::kTurns);
        ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->bars.s_full[sb], phase, abort_flag));
        float l[kR];
        const float lv = (float)((int)(__float_as_uint(sc.y) >> 23) - 127);     // log2 of a power of two
        bool over = false;
        if (ok) {
          ptx::tc_fence_after_sync();
          uint32_t c[16];
          const uint32_t s_addr = lane_addr + (uint32_t)(sb * L::kN1 + rb * 3 * kR);
          ptx::tmem_ld_32x16(s_addr, c);                               // (three terms; the last four are not used)
          ptx::tmem_wait_ld();
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->bars.s_empty[sb]);
          const bool edge = key0 + kTileKeys > all_see;
#pragma unroll
          for (int g = 0; g < kR; ++g) {
            auto term = [&](int k) { return __uint_as_float(c[k * kR + g]); };
            l[g] = fmaf(term(2), 0.00390625f, fmaf(term(1), 0.0625f, term(0))) * (sc.x * factor[g]);
            if (edge && key >= limit[g]) l[g] = -INFINITY;
            over = over || l[g] + lv > refn[g] + kSlack || l[g] > refd[g] + kSlack;
          }
          if (a.logits && key < x.n) {
            float* dst = a.logits + ((int64_t)x.h * a.max_q * a.G + row0) * a.total + x.start + key;
#pragma unroll
            for (int g = 0; g < kR; ++g)
              if (g < nrows) dst[(int64_t)g * a.total] = l[g];
          }
        }
        if (group_any(bar_id, over)) {
          // ---- some reference moves: the tile's largest exponents become the references, sums and O are rescaled
#pragma unroll
          for (int g = 0; g < kR; ++g) {
            const float d = warp_redux_max(ok ? l[g] : -INFINITY), n = warp_redux_max(ok ? l[g] + lv : -INFINITY);
            if (lane == 0) *reinterpret_cast<float2*>(&red_sm[w * 2 * kR + 2 * g]) = make_float2(d, n);
          }
          group_any(bar_id, false);
          float shrink[kR];
#pragma unroll
          for (int g = 0; g < kR; ++g) {
            float d = refd[g], n = refn[g];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float2 v = *reinterpret_cast<const float2*>(&red_sm[k * 2 * kR + 2 * g]);
              d = fmaxf(d, v.x);
              n = fmaxf(n, v.y);
            }
            sum[g] = times_exp2(sum[g], refd[g] - d);
            shrink[g] = exp2_fast(0.5f * (refn[g] - n));             // (applied twice)
            refd[g] = d;
            refn[g] = n;
          }
          if (ok && t > first) {                                       // O holds this turn's tiles before this one
            const int before = it - L::kTurns;
            ok = __all_sync(0xffffffffu, wait_or_abort(&tail->bars.p_empty[before % L::kBuffers], (before / L::kBuffers) & 1, abort_flag));
            if (ok) {
              ptx::tc_fence_after_sync();
#pragma unroll
              for (int y = 0; y < kBoxes; ++y) {
                const uint32_t at_o = o_addr + (uint32_t)(y * L::kN2);
                uint32_t v[16];
                ptx::tmem_ld_32x16(at_o, v);
                ptx::tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * shrink[j % kR] * shrink[j % kR]);
                tmem_st_32x16(at_o, v);
              }
              ptx::tmem_wait_st();
              ptx::tc_fence_before_sync();
            }
          }
          group_any(bar_id, false);                                    // red_sm has been read
        }
        // ---- weights and their terms
        ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->bars.p_empty[sb], phase ^ 1, abort_flag));
        if (ok) {
          float f[kR];
#pragma unroll
          for (int g = 0; g < kR; ++g) {
            sum[g] += exp2_fast(l[g] - refd[g]);
            f[g] = exp2_fast(l[g] + lv - refn[g]);
          }
          uint2 p[3];                                                  // a term of the four rows
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            p[k].x = take_bf16(f[0], f[1]);
            p[k].y = take_bf16(f[2], f[3]);
          }
          uint8_t* dst = p_sm + sb * L::kP + rb * 2 * kTileKeys * 16 + key_in * 16;
          *reinterpret_cast<uint4*>(dst) = make_uint4(p[0].x, p[0].y, p[1].x, p[1].y);
          *reinterpret_cast<uint4*>(dst + 16 * kTileKeys) = make_uint4(p[2].x, p[2].y, 0, 0);   // (columns up to a multiple of 16)
          ptx::fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&tail->bars.p_full[sb]);
      }

      // ---- the segment's result
#pragma unroll
      for (int g = 0; g < kR; ++g) {
        float s = sum[g];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) red_sm[w * 2 * kR + g] = s;
      }
      group_any(bar_id, false);
      const bool whole = L::kTurns == 1 && s0 == 0 && s1 == pref[e + 1] - pref[e] - kGap;   // all of the entry, in one O
      const int64_t slot = (((int64_t)blockIdx.y * (entries + (int)gridDim.x) + e + b) * L::kTurns + turn) * a.group_rows + rb * kR;
      if (any_tile) {
        ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->bars.o_full[turn], o_uses & 1, abort_flag));
        ++o_uses;
      }
      if (ok) {
        const bool nan_seen = x.nq > 1 && *(volatile int*)&tail->any_nan[qb][turn] != 0;
        if (any_tile) ptx::tc_fence_after_sync();
#pragma unroll
        for (int y = 0; y < kBoxes; ++y) {
          const int d = y * 128 + key_in;
          uint32_t v[16];
          if (any_tile) {
            ptx::tmem_ld_32x16(o_addr + (uint32_t)(y * L::kN2), v);
            ptx::tmem_wait_ld();
          }
          if (d < a.d_k) {
#pragma unroll
            for (int g = 0; g < kR; ++g) {
              if (g < nrows) {
                const float total = (red_sm[g] + red_sm[2 * kR + g]) + (red_sm[4 * kR + g] + red_sm[6 * kR + g]);
                if (any_tile) {
                  auto term = [&](int k) { return __uint_as_float(v[k * kR + g]); };
                  float o = (term(2) + term(1)) + term(0);
                  o = total == 0.f ? 0.f : times_exp2(o * __frcp_rn(total), refn[g] - refd[g]);
                  if (nan_seen && ((nan_sm[(rb * kR + g) * kBoxes * 4 + (d >> 5)] >> (d & 31)) & 1u)) o = __uint_as_float(0x7fffffffu);
                  if (whole) a.out[tail->out_at[qb][rb * kR + g] + d] = __float2bfloat16(o);
                  else a.part_o[(slot + g) * a.d_k + d] = o;
                }
                if (d == 0) {
                  a.part_ml[slot + g] = make_float2(total == 0.f ? -INFINITY : refd[g], total);
                  if (whole) write_lse(a, tail->lse_at[qb][rb * kR + g], make_float2(total == 0.f ? -INFINITY : refd[g], total));
                }
              }
            }
          }
        }
        ptx::tc_fence_before_sync();
      }
      __syncwarp();
      if (lane == 0) {
        if (any_tile) ptx::mbar_arrive(&tail->bars.o_empty[turn]);
        ptx::mbar_arrive(&tail->bars.q_empty[qb]);
      }
      group_any(bar_id, false);                                        // red_sm has been read
    }
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && tail->abort_flag) { atomicExch(&a.status[0], GVOTE_ERR_TIMEOUT); atomicExch(&a.status[1], 13); }
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, L::kAlloc);
  }
}

// Running (maximum, sum relative to it), joined with another pair; and over a warp.
__device__ __forceinline__ void join(float& M, float& L, float2 x) {
  const float top = fmaxf(M, x.x);
  L = top == -INFINITY ? L + x.y : times_exp2(L, M - top) + times_exp2(x.y, x.x - top);     // (a NaN in the sum stays)
  M = top;
}
__device__ __forceinline__ float2 warp_join(float M, float L) {
  const float all = warp_max(M);
  L = all == -INFINITY ? L : L == 0.f ? 0.f : times_exp2(L, M - all);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
  return make_float2(all, L);
}

// The rows of the entries that lie in several segments (or none), merged.  They are a few KB: what counts is how many loads wait
// for one another, so a block takes a row and its outputs are asked for before the maxima are known.  With many entries, most
// of them in one CTA or two (so of a few parts), it is the number of blocks that counts: then (kRows = 8) a warp takes a row
// of up to 32 parts, and the block the others (512 entries of 2048 rows: 15 us with a block per row).
template <int kRows>
__global__ void __launch_bounds__(256)
attend8_merge_kernel(const __grid_constant__ AttendArgs a, int ctas, int max_rows) {
  __shared__ float4 s_o[8][32 * 2];
  __shared__ float s_f[4 * kSms];
  __shared__ int s_left[8];
  const int entries = a.batch * a.Hkv, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quads = a.d_k >> 2;
  struct Job { Entry x; int e, row, parts; int64_t slot0; };
  auto entry_job = [&](int id) {
    Job j = {};
    if (id < entries * max_rows) {
      j.e = id / max_rows;
      j.row = id - j.e * max_rows;
      j.x = entry_of(a, j.e);
    }
    return j;
  };
  auto job_of = [&](Job j) {                            // parts < 0: nothing to do
    const int e = j.e;
    j.parts = -1;
    if (j.row >= j.x.nq * a.G) return j;
    const int group = j.row / a.group_rows, in_group = j.row - group * a.group_rows;
    const int2 v = a.info[(int64_t)group * entries + e];
    if (a.turns == 1 && v.x >= 0 && v.x == v.y) return j;            // the first kernel has written it
    const int p0 = v.x * a.turns;
    j.parts = v.x < 0 ? 0 : (v.y + 1) * a.turns - p0;
    j.slot0 = (((int64_t)group * (entries + ctas) + e) * a.turns + p0) * a.group_rows + in_group;
    return j;
  };
  auto part_o = [&](const Job& j, int k, int q) {
    return *reinterpret_cast<const float4*>(a.part_o + (j.slot0 + (int64_t)k * a.group_rows) * a.d_k + q * 4);
  };
  auto add = [](float4& s, const float4& p, float f) {  // (0: a turn without tiles has left nothing)
    if (f != 0.f) { s.x = fmaf(f, p.x, s.x); s.y = fmaf(f, p.y, s.y); s.z = fmaf(f, p.z, s.z); s.w = fmaf(f, p.w, s.w); }
  };
  auto finish = [&](const Job& j, int q, const float4& s, float2 ml) {
    const int64_t token = j.x.q0 + j.row / a.G;
    const int g = j.x.h * a.G + j.row % a.G;
    const float inv = ml.x == -INFINITY && ml.y == 0.f ? 0.f : 1.f / ml.y;
    __nv_bfloat162 out[2] = {__floats2bfloat162_rn(s.x * inv, s.y * inv), __floats2bfloat162_rn(s.z * inv, s.w * inv)};
    *reinterpret_cast<uint2*>(a.out + token * a.o_tok + (int64_t)g * a.o_head + q * 4) = *reinterpret_cast<uint2*>(out);
    if (q == 0) write_lse(a, token * a.Hkv * a.G + g, ml);
  };
  auto block_row = [&](const Job& j) {
    constexpr int kAhead = 8;
    float4 pre[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (warp + 8 * i < j.parts && lane < quads) pre[i] = part_o(j, warp + 8 * i, lane);
    float M = -INFINITY, L = 0.f;
    for (int k = lane; k < j.parts; k += 32) join(M, L, a.part_ml[j.slot0 + (int64_t)k * a.group_rows]);
    const float2 ml = warp_join(M, L);
    for (int i = tid; i < j.parts; i += 256) {
      const float2 m = a.part_ml[j.slot0 + (int64_t)i * a.group_rows];
      s_f[i] = m.x == -INFINITY ? 0.f : times_exp2(m.y, m.x - ml.x);
    }
    __syncthreads();
    for (int q = lane; q < quads; q += 32) {
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      int k0 = warp;
      if (q == lane) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
          if (warp + 8 * i < j.parts) add(s, pre[i], s_f[warp + 8 * i]);
        k0 += 8 * kAhead;
      }
#pragma unroll 8
      for (int k = k0; k < j.parts; k += 8) add(s, part_o(j, k, q), s_f[k]);
      s_o[warp][q] = s;
    }
    __syncthreads();
    if (tid < quads) {
      float4 s = s_o[0][tid];
#pragma unroll
      for (int k = 1; k < 8; ++k) {
        const float4 p = s_o[k][tid];
        s.x += p.x; s.y += p.y; s.z += p.z; s.w += p.w;
      }
      finish(j, tid, s, ml);
    }
  };
  const Job mine = entry_job(kRows == 1 ? blockIdx.x : blockIdx.x * kRows + warp);
  ptx::wait_for_previous();
  ptx::let_next_begin();
  if (kRows == 1) {
    const Job j = job_of(mine);
    if (j.parts >= 0) block_row(j);
    return;
  }
  {
    const Job j = job_of(mine);
    if (lane == 0) s_left[warp] = j.parts > 32;
    if (j.parts >= 0 && j.parts <= 32) {
      const float2 m = lane < j.parts ? a.part_ml[j.slot0 + (int64_t)lane * a.group_rows] : make_float2(-INFINITY, 0.f);
      const float2 ml = warp_join(m.x, m.y);
      const float f = m.x == -INFINITY ? 0.f : times_exp2(m.y, m.x - ml.x);
      for (int q = lane; q - lane < quads; q += 32) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < j.parts; ++k) {
          const float fk = __shfl_sync(0xffffffffu, f, k);
          if (q < quads) add(s, part_o(j, k, q), fk);
        }
        if (q < quads) finish(j, q, s, ml);
      }
    }
  }
  __syncthreads();
  for (int w = 0; w < kRows; ++w) {
    if (!s_left[w]) continue;
    block_row(job_of(entry_job(blockIdx.x * kRows + w)));
    __syncthreads();
  }
}

// The weights a row of the cache gets from the request's tokens and the group's heads, added to acc: thread = kSpan / 256 slots.
// Blocks of kSpan slots: request r0 + i has those from (cu >> kSpanBits) - base + i on.
// Latency bound: two slots per thread rather than one halve the blocks (64 requests of 2048 rows 21 -> 15 us of events; a call
// with 128 rows of queries loses 4 of its 224 us to the shorter runs of loads).
constexpr int kSpanBits = 9, kSpan = 1 << kSpanBits;
__global__ void __launch_bounds__(256)
attend8_weights_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int kSlots = kSpan / 256, kRows = 128, kAhead = 4;       // rows whose lse is at hand, logits of a slot on their way at once
  __shared__ float s_lse[kRows];
  const int tid = threadIdx.x, h = blockIdx.y;
  const int64_t gb = blockIdx.x;
  const int base = a.cu[a.r0] >> kSpanBits;
  int i_req = -1;                                       // the last request whose first block is not behind gb
  for (int i0 = 0; i0 < a.batch; i0 += 256) {
    const int i = i0 + tid;
    i_req += __syncthreads_count(i < a.batch && (int64_t)((a.cu[a.r0 + min(i, a.batch - 1)] >> kSpanBits) - base) + i <= gb);
  }
  const int e = i_req * a.Hkv + h;
  const Entry x = entry_of(a, e);
  ptx::wait_for_previous();
  const int i0 = (int)(gb - ((x.start >> kSpanBits) - base + i_req)) * kSpan, i = i0 + tid;
  if (i0 >= x.n) return;
  const int rows = x.nq * a.G;
  const float* l = a.logits + (int64_t)h * a.max_q * a.G * a.total + x.start + i;
  const float* lse = a.lse2 + (int64_t)x.q0 * a.Hkv * a.G + h * a.G;
  const int64_t slot = (int64_t)h * a.total + x.start + i;
  float s[kSlots] = {}, was[kSlots];
#pragma unroll
  for (int c = 0; c < kSlots; ++c) was[c] = a.acc && i + c * 256 < x.n ? a.acc[slot + c * 256] : 0.f;
  for (int row0 = 0; row0 < rows; row0 += kRows) {
    const int some = min(kRows, rows - row0);
    if (row0 > 0) __syncthreads();
    if (tid < some) s_lse[tid] = lse[(int64_t)((row0 + tid) / a.G) * a.Hkv * a.G + (row0 + tid) % a.G];
    for (int k0 = 0; k0 < some; k0 += kAhead, l += kAhead * a.total) {
      float v[kSlots][kAhead];
#pragma unroll
      for (int c = 0; c < kSlots; ++c)
#pragma unroll
        for (int k = 0; k < kAhead; ++k) v[c][k] = i + c * 256 < x.n && k0 + k < some ? l[k * a.total + c * 256] : -INFINITY;
      if (k0 == 0) __syncthreads();
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (int c = 0; c < kSlots; ++c)
          if (v[c][k] != -INFINITY) s[c] += exp2_fast(v[c][k] - s_lse[k0 + k]);
    }
  }
#pragma unroll
  for (int c = 0; c < kSlots; ++c)
    if (i + c * 256 < x.n) a.acc_out[slot + c * 256] = was[c] + s[c];
}

// How a launch is cut: groups that share a tile's rows, row groups, CTAs.
struct Cut { int boxes, rb, turns, rows, groups, requests; int64_t ctas; };
Cut cut_of(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_q) {
  Cut c;
  const int64_t rows = max_q * (p->n_q_heads / p->n_kv_heads);
  c.boxes = p->d_k <= 128 ? 1 : 2;
  // Up to five softmax groups of four rows (four where d_k > 128, whose tiles of V leave less shared memory); beyond those as few
  // and as even row groups as hold the rows, each of which reads the codes again, from L2 (24 rows over 32K: 47 us as two row
  // groups of 12, 55 as three softmax groups of eight rows).
  const int64_t most = c.boxes == 1 ? 20 : 16;
  c.rb = rows > 0 ? (int)ceil_div(ceil_div(rows, ceil_div(rows, most)), kR) : 1;
  c.turns = c.rb == 1 ? 4 : c.rb == 2 ? 2 : 1;
  c.rows = kR * c.rb;
  c.groups = (int)ceil_div(rows > 0 ? rows : 1, c.rows);
  c.requests = kMaxEntries / p->n_kv_heads < batch ? kMaxEntries / p->n_kv_heads : batch;
  // a CTA per SM, and no more than one per tile
  const int64_t most_ctas = (total_tokens / kTileKeys + batch) * p->n_kv_heads;
  c.ctas = most_ctas < kSms ? most_ctas : kSms;
  return c;
}

template <int kBoxes, int kRb>
int32_t run_attend(const Cut& c, const CUtensorMap (&tm)[4], AttendArgs a, cudaStream_t st) {
  using L = Layout<kBoxes, kRb>;
  // the slots that fit, five in twelve to K (a tile of V stays about half as long again)
  a.k_slots = L::kFit * 5 / 12 < 2 ? 2 : L::kFit * 5 / 12 > kMaxSlots ? kMaxSlots : L::kFit * 5 / 12;
  a.v_slots = L::kFit - a.k_slots > kMaxSlots ? kMaxSlots : L::kFit - a.k_slots;
  const size_t smem = L::fixed() + (size_t)(a.k_slots + a.v_slots) * L::kSlot;
  auto kernel = attend8_kernel<kBoxes, kRb>;
  GVOTE_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  {
    LaunchScope scope_("attend8_kernel", st);
    launch_on(kernel, dim3((unsigned)c.ctas, (unsigned)c.groups), dim3(L::kThreads), smem, st, tm[0], tm[1], tm[2],
              tm[3], a);
  }
  GVOTE_LAUNCH_CHECK("attend8_kernel");
  return GVOTE_OK;
}
template <int kBoxes>
int32_t run_attend(const Cut& c, const CUtensorMap (&tm)[4], const AttendArgs& a, cudaStream_t st) {
  if constexpr (kBoxes == 1) {
    if (c.rb == 5) return run_attend<kBoxes, 5>(c, tm, a, st);
  }
  switch (c.rb) {
    case 1: return run_attend<kBoxes, 1>(c, tm, a, st);
    case 2: return run_attend<kBoxes, 2>(c, tm, a, st);
    case 3: return run_attend<kBoxes, 3>(c, tm, a, st);
    default: return run_attend<kBoxes, 4>(c, tm, a, st);
  }
}

}  // namespace

AttendMap attend8_map(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t total_q, int64_t max_q) {
  AttendMap m;
  const Cut c = cut_of(p, batch, total_tokens, max_q);
  const size_t entries = (size_t)c.requests * p->n_kv_heads;
  const size_t rows = (size_t)c.groups * (entries + c.ctas) * c.turns * c.rows;
  m.o = kStatusBytes;
  m.ml = align_up(m.o + rows * p->d_k * 4, 256);
  m.info = align_up(m.ml + rows * 8, 256);
  m.lse = align_up(m.info + c.groups * entries * 8, 256);
  m.logits = align_up(m.lse + (size_t)total_q * p->n_q_heads * 4, 256);
  m.total = align_up(m.logits + (size_t)p->n_q_heads * max_q * total_tokens * 4, 256);
  return m;
}

size_t attend8_workspace(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t total_q, int64_t max_q) {
  size_t most = 0;                                      // (fewer rows can need more: the groups then take turns)
  for (int64_t q = 1; q <= max_q && q <= GVOTE_ATTEND8_MAX_Q; ++q) {
    const size_t n = attend8_map(p, batch, total_tokens, total_q, q).total;
    most = n > most ? n : most;
  }
  return most;
}

int32_t launch_attend8(const gvote_params* p, const __nv_bfloat16* Q, int64_t q_tok, int64_t q_head, const int32_t* cu_q,
                       int64_t total_q, int64_t max_q, const gvote_cache8* c, __nv_bfloat16* out, int64_t o_tok,
                       int64_t o_head, float* lse, const float* acc, float* acc_out, char* ws, cudaStream_t st) {
  const AttendMap m = attend8_map(p, c->batch, c->total_tokens, total_q, max_q);
  const Cut cut = cut_of(p, c->batch, c->total_tokens, max_q);
  AttendArgs a;
  a.Q = Q; a.q_tok = q_tok; a.q_head = q_head; a.cu_q = cu_q;
  a.k_scale = c->k_scale; a.v_scale = c->v_scale;
  a.total = c->total_tokens;
  a.row_blocks = gvote_cache8_row_blocks(c->total_tokens, c->batch);
  a.cu = c->cu_seqlens; a.kv_len = c->kv_len;
  a.out = out; a.o_tok = o_tok; a.o_head = o_head; a.lse = lse; a.acc = acc; a.acc_out = acc_out;
  a.part_o = (float*)(ws + m.o); a.part_ml = (float2*)(ws + m.ml); a.info = (int2*)(ws + m.info);
  a.lse2 = (float*)(ws + m.lse);
  a.logits = acc_out ? (float*)(ws + m.logits) : nullptr;
  a.status = (int32_t*)ws;
  a.Hkv = p->n_kv_heads; a.G = p->n_q_heads / p->n_kv_heads; a.d_k = p->d_k; a.max_q = (int)max_q;
  a.k_slots = a.v_slots = 0; a.group_rows = cut.rows; a.turns = cut.turns;
  a.scale2 = (float)(1.4426950408889634 / sqrt((double)p->d_k));

  CUtensorMap tm[4];                                    // K, V in whole tiles, K, V in parts
  const uint64_t dims[3] = {(uint64_t)p->d_k, (uint64_t)c->total_tokens, (uint64_t)a.Hkv};
  const uint64_t strides[2] = {(uint64_t)c->tok_stride, (uint64_t)(a.Hkv > 1 ? c->head_stride : c->tok_stride)};
  for (int i = 0; i < 4; ++i) {
    const uint32_t box[3] = {128, (uint32_t)(i < 2 ? kTileKeys : kBoxRows), 1};
    if (!encode_tensor_map_u8(&tm[i], i & 1 ? c->V : c->K, 3, dims, strides, box)) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  }

  for (int32_t r0 = 0; r0 < c->batch; r0 += cut.requests) {
    a.r0 = r0;
    a.batch = c->batch - r0 < cut.requests ? c->batch - r0 : cut.requests;
    PROPAGATE(cut.boxes == 1 ? run_attend<1>(cut, tm, a, st) : run_attend<2>(cut, tm, a, st));
    const int64_t rows = max_q * a.G;
    {
      LaunchScope scope_("attend8_merge_kernel", st);
      const int64_t all = (int64_t)a.batch * a.Hkv * rows;
      if (a.batch * a.Hkv < kSms)
        launch_behind(attend8_merge_kernel<1>, dim3((unsigned)all), dim3(256), 0, st, a, (int)cut.ctas, (int)rows);
      else
        launch_behind(attend8_merge_kernel<8>, dim3((unsigned)ceil_div(all, 8)), dim3(256), 0, st, a, (int)cut.ctas, (int)rows);
    }
    GVOTE_LAUNCH_CHECK("attend8_merge_kernel");
    if (acc_out) {
      LaunchScope scope_("attend8_weights_kernel", st);
      launch_behind(attend8_weights_kernel, dim3((unsigned)((c->total_tokens >> kSpanBits) + a.batch), a.Hkv), dim3(256), 0, st, a);
      GVOTE_LAUNCH_CHECK("attend8_weights_kernel");
    }
  }
  return GVOTE_OK;
}

}  // namespace gvote
