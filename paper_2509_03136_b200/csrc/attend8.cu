// Attention of a few query tokens over the 8-bit cache (gvote_attend8).
//
//   l_n = (q.k_n) / sqrt(d_k),  out = sum_n exp(l_n - lse) v_n,  lse = log sum_n exp(l_n),
// with k_n, v_n = code * scale of the row's block.  A few rows of queries against long K and V: bound by reading the codes
// once, 2 d_k bytes per cached row.
//
// Split.  The rows of all (request, KV head) pairs ("entries") are cut into tiles of 128 and laid end to end; CTA b of the
// grid takes tiles T b / grid .. T (b + 1) / grid - 1, whatever entries they belong to.  So pruned heads of very
// different length load every SM alike, without knowing the lengths on the host: each CTA adds up the entries' tiles
// itself.  What a CTA has of one entry is a segment; its result (reference, sum, output) goes to slot entry + CTA, or
// straight to the output when the entry lies within one CTA.  attend8_finish_kernel merges an entry's segments.
//
// The products run on the codes themselves (tcgen05.mma kind::f8f6f4, e4m3 x e4m3, 32-bit sums), with the cached rows on
// the M axis, so that nothing has to be widened or transposed on the way from the TMA boxes to the tensor cores:
//   S [128 keys x (3 terms, rows)]  = K Q^T    K as it lies (128-byte swizzle), Q as a sum of three e4m3 terms
//   O [128 channels x (4 terms, rows)] += V^T P^T   V as it lies, its channels on the M axis; P as a sum of four terms
// A term is the e4m3 value nearest to what the terms before it left, times 16 per term, and its columns are added up
// with the matching power of two in 32 bits.  Three terms hold a row of Q to 2^-12 of each entry and 2^-27 of the
// row's largest (bf16 itself: 2^-8); four hold a weight to 2^-16 of itself and 2^-27 of the largest.  An mma.sync version
// that widened the codes in registers issued 690 instructions per 32 rows and was bound by their latency (one token over
// 128K rows x 4 heads: 30 us for the 20 us of bytes; this kernel ~24).
//
// The scale of K enters the logit; the scale of V goes into the weight: P = 2^(l + log2(scale_v) - ref), ref the largest such
// exponent so far, so that a block of large values neither overflows nor drowns what carries the output.  ref only moves
// when it is passed by 2^4 (the accumulated O is then rescaled in tensor memory: mostly the first tile only).
//
// Warp 0 asks for the tiles (TMA boxes of 32 rows, only those that hold rows), warp 1 issues the MMAs, warps 2 and 3
// prepare the next segment's Q terms, warps 4-7 are the softmax: thread = cached row of the tile (and channel of the output).
// S is double buffered, and the MMA of tile i+1's S is issued before that of tile i's O.
//
// Weights for the eviction: the logits are kept (4 bytes per row and query, against 2 d_k per row), and the finishing
// kernel turns them into weights once lse is known; a slot belongs to one thread, so the sum has one order.
//
// Every wait is bounded; when one runs out GVOTE_ERR_TIMEOUT is recorded and the outputs are not to be used.
#include "cache8.cuh"
#include "ptx.cuh"

namespace gvote {
namespace {

constexpr int kTileKeys = 128;
constexpr int kBoxRows = 32;
constexpr int kMaxEntries = 1024;      // entries per launch: their tiles are added up in shared memory
constexpr int kMaxStages = 6;
constexpr int kThreads = 256;
constexpr int kSms = 148;
constexpr float kNoRef = -1e30f;       // a reference before the first logit
constexpr float kUp = 4.f;             // weights are formed times 2^4: with a slack of 2^4 they stay below 448

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
  const float* acc;
  float* acc_out;        // or null
  float* part_o;         // [row groups][entries + CTAs][rows of a group][d_k], each divided by its segment's sum
  float2* part_ml;       // [row groups][entries + CTAs][rows of a group]  (reference, sum), base 2
  int2* info;            // [row groups][entries]  first and last CTA of the entry (-1: no rows)
  float* logits;         // [Hkv][max_q * G][total] base 2, when acc_out
  int32_t* status;
  int Hkv, G, r0, batch, d_k, max_q;   // requests r0 .. r0 + batch - 1
  int stages, group_rows;
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
  x.nq = a.cu_q[x.r + 1] - x.q0;
  return x;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  for (uint32_t i = 0; i < (1u << 22); ++i) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if ((i & 255u) == 255u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
// The or of a predicate over the softmax warps (named barrier 1).
__device__ __forceinline__ bool softmax_any(bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.aligned.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"((uint32_t)x) : "memory");
  return r != 0;
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
// Operand stored as rows of 16 bytes without swizzle, the 16 bytes along M or N: eight K rows are 128 bytes, the next eight
// K rows follow at once (leading offset 128), the next 16 of M or N `chunk` bytes on.
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

struct Tail {
  uint64_t kv_full[kMaxStages], kv_empty[kMaxStages];
  uint64_t q_full[2], q_empty[2], s_full[2], s_empty[2], p_full[2], p_empty[2], o_full, o_empty;
  Entry entry[2];
  uint32_t tmem_slot;
  int any_nan;
  volatile int abort_flag;
  int warp_tot[8];
  int pref[kMaxEntries + 1];
};

template <int kBoxes, int kRows>
struct Layout {                        // of tensor memory (columns) and shared memory (bytes)
  static constexpr int kN1 = (3 * kRows + 15) / 16 * 16, kN2 = 4 * kRows;
  static constexpr int kCols = 2 * kN1 + kBoxes * kN2;
  static constexpr int kAlloc = kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
  static constexpr int kStage = 2 * kBoxes * kTileKeys * 128, kQ = kBoxes * kN1 * 128, kP = kN2 * kTileKeys;
  static constexpr int kNan = kRows * kBoxes * 4 * 4;                   // bits [row][channel]
  static constexpr int kSmall = 4 * 2 * kRows * 4 + 2 * kRows * 8 + kNan;
  static constexpr size_t fixed() { return (size_t)2 * kQ + 2 * kP + kSmall + sizeof(Tail); }
};

template <int kBoxes, int kRows>       // 128-byte boxes per row; query rows of a group, padded
__global__ void __launch_bounds__(kThreads, 1)
attend8_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
               const __grid_constant__ AttendArgs a) {
  extern __shared__ __align__(1024) uint8_t smem[];
  using L = Layout<kBoxes, kRows>;
  uint8_t* ring = smem;                                                // [stage][K boxes, V boxes][128 rows][128]
  uint8_t* q_sm = ring + (size_t)a.stages * L::kStage;                 // [2][box][N1 rows][128], swizzled
  uint8_t* p_sm = q_sm + 2 * L::kQ;                                    // [2][N2 / 16][128 keys][16]
  float* red_sm = reinterpret_cast<float*>(p_sm + 2 * L::kP);          // [4 warps][2 kRows]
  float* factor_sm = red_sm + 4 * 2 * kRows;                           // [2][kRows] logit per unit of product
  int* limit_sm = reinterpret_cast<int*>(factor_sm + 2 * kRows);       // [2][kRows] cached rows a query row sees
  uint32_t* nan_sm = reinterpret_cast<uint32_t*>(limit_sm + 2 * kRows);
  Tail* tail = reinterpret_cast<Tail*>(nan_sm + L::kNan / 4);
  int* pref = tail->pref;
  volatile int* abort_flag = &tail->abort_flag;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int entries = a.batch * a.Hkv;
  const int group0 = blockIdx.y * a.group_rows;                        // first query row of this group

  if (tid == 0) {
    for (int s = 0; s < kMaxStages; ++s) { ptx::mbar_init(&tail->kv_full[s], 1); ptx::mbar_init(&tail->kv_empty[s], 1); }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(&tail->q_full[b], 2); ptx::mbar_init(&tail->q_empty[b], 5);
      ptx::mbar_init(&tail->s_full[b], 1); ptx::mbar_init(&tail->s_empty[b], 4);
      ptx::mbar_init(&tail->p_full[b], 4); ptx::mbar_init(&tail->p_empty[b], 1);
    }
    ptx::mbar_init(&tail->o_full, 1); ptx::mbar_init(&tail->o_empty, 4);
    tail->abort_flag = (ptx::smem_u32(smem) & 1023u) ? 1 : 0;
    tail->any_nan = 0;
    ptx::fence_barrier_init();
    ptx::prefetch_tensormap(&tmK);
    ptx::prefetch_tensormap(&tmV);
  }
  for (int i = tid; i < L::kNan / 4; i += kThreads) nan_sm[i] = 0;
  if (warp == 1) {
    ptx::tmem_alloc(&tail->tmem_slot, L::kAlloc);
    ptx::tmem_relinquish();
  }
  // ---- tiles before each entry
  {
    const int per = (entries + kThreads - 1) / kThreads;               // consecutive entries per thread
    const int e0 = min(tid * per, entries), e1 = min(e0 + per, entries);
    int mine = 0;
    for (int e = e0; e < e1; ++e) {
      const Entry x = entry_of(a, e);
      const int t = group0 < x.nq * a.G ? (x.n + kTileKeys - 1) / kTileKeys : 0;
      pref[e + 1] = t;
      mine += t;
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
    int run = inc - mine;
    for (int w = 0; w < warp; ++w) run += tail->warp_tot[w];
    for (int e = e0; e < e1; ++e) { run += pref[e + 1]; pref[e + 1] = run; }
    if (tid == 0) pref[0] = 0;
    __syncthreads();
  }
  const uint32_t tmem = __shfl_sync(0xffffffffu, tail->tmem_slot, 0);
  const int T = pref[entries], B = gridDim.x, b = blockIdx.x;
  const int t0 = (int)((int64_t)T * b / B), t1 = (int)((int64_t)T * (b + 1) / B);
  // which CTAs hold an entry: the CTA of tile t is the largest c with T c / B <= t
  if (b == 0) {
    int2* info = a.info + (int64_t)blockIdx.y * entries;
    for (int e = tid; e < entries; e += kThreads) {
      const int f = pref[e], l = pref[e + 1] - 1;
      int2 v = make_int2(-1, -1);
      if (l >= f) v = make_int2((int)((((int64_t)f + 1) * B - 1) / T), (int)((((int64_t)l + 1) * B - 1) / T));
      info[e] = v;
    }
  }
  int e_first = t0 < t1 ? 0 : entries;                                 // the entry of tile t0 (a CTA without tiles: none)
  {
    int hi = entries - 1;
    while (e_first < hi) {
      const int mid = (e_first + hi) >> 1;
      if (pref[mid + 1] <= t0) e_first = mid + 1; else hi = mid;
    }
  }
  bool ok = true;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int it = 0;
      for (int e = e_first; ok && e < entries && pref[e] < t1; ++e) {
        if (pref[e + 1] == pref[e]) continue;
        const Entry x = entry_of(a, e);
        const int s1 = min(t1, pref[e + 1]);
        for (int t = max(t0, pref[e]); t < s1; ++t, ++it) {
          const int s = it % a.stages, key0 = (t - pref[e]) * kTileKeys;
          ok = wait_or_abort(&tail->kv_empty[s], ((it / a.stages) & 1) ^ 1, abort_flag);
          if (!ok) break;
          const int parts = min(kTileKeys / kBoxRows, (x.n - key0 + kBoxRows - 1) / kBoxRows);
          ptx::mbar_arrive_expect_tx(&tail->kv_full[s], (uint32_t)parts * 2 * kBoxes * kBoxRows * 128);
          uint8_t* dst = ring + (size_t)s * L::kStage;
          for (int g = 0; g < parts; ++g)
#pragma unroll
            for (int y = 0; y < kBoxes; ++y)
              ptx::tma_load_3d(dst + (y * kTileKeys + g * kBoxRows) * 128, &tmK, &tail->kv_full[s], y * 128, x.start + key0 + g * kBoxRows, x.h);
          for (int g = 0; g < parts; ++g)
#pragma unroll
            for (int y = 0; y < kBoxes; ++y)
              ptx::tma_load_3d(dst + ((kBoxes + y) * kTileKeys + g * kBoxRows) * 128, &tmV, &tail->kv_full[s], y * 128, x.start + key0 + g * kBoxRows, x.h);
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (the whole warp walks, one lane issues)
    const uint32_t idesc1 = instr_desc_e4m3(kTileKeys, L::kN1, false, false), idesc2 = instr_desc_e4m3(128, L::kN2, true, true);
    const int ksteps = (a.d_k + 31) / 32;
    int it = 0, seg = 0;
    struct { int it, seg; bool first, last, valid; } prev = {0, 0, false, false, false};
    auto second = [&]() {                                              // O of the tile before
      const int s = prev.it % a.stages, pb = prev.it & 1;
      ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->p_full[pb], (prev.it >> 1) & 1, abort_flag));
      if (ok && prev.first) ok = __all_sync(0xffffffffu, wait_or_abort(&tail->o_empty, (prev.seg & 1) ^ 1, abort_flag));
      if (!ok) return;
      ptx::tc_fence_after_sync();
      if (ptx::elect_one()) {
        const uint64_t pd = smem_desc_mn_plain(ptx::smem_u32(p_sm) + (uint32_t)pb * L::kP, 16 * kTileKeys);
#pragma unroll
        for (int y = 0; y < kBoxes; ++y) {
          const uint64_t vd = ptx::smem_desc_k_sw128(ptx::smem_u32(ring) + (uint32_t)(s * L::kStage + (kBoxes + y) * kTileKeys * 128));
#pragma unroll
          for (int k = 0; k < kTileKeys / 32; ++k)                     // 32 keys: 4 KB of V, 512 bytes of P
            umma_e4m3(tmem + (uint32_t)(2 * L::kN1 + y * L::kN2), vd + (uint64_t)(k * (32 * 128 / 16)), pd + (uint64_t)(k * (32 * 16 / 16)),
                      idesc2, prev.first && k == 0 ? 0u : 1u);
        }
        ptx::umma_commit(&tail->p_empty[pb]);
        ptx::umma_commit(&tail->kv_empty[s]);
        if (prev.last) ptx::umma_commit(&tail->o_full);
      }
      __syncwarp();
    };
    for (int e = e_first; ok && e < entries && pref[e] < t1; ++e) {
      if (pref[e + 1] == pref[e]) continue;
      const int s0 = max(t0, pref[e]), s1 = min(t1, pref[e + 1]), qb = seg & 1;
      for (int t = s0; ok && t < s1; ++t, ++it) {
        const int s = it % a.stages, sb = it & 1;
        ok = __all_sync(0xffffffffu, wait_or_abort(&tail->kv_full[s], (it / a.stages) & 1, abort_flag));
        if (ok && t == s0) ok = __all_sync(0xffffffffu, wait_or_abort(&tail->q_full[qb], (seg >> 1) & 1, abort_flag));
        ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->s_empty[sb], ((it >> 1) & 1) ^ 1, abort_flag));
        if (!ok) break;
        ptx::tc_fence_after_sync();
        if (ptx::elect_one()) {
#pragma unroll
          for (int y = 0; y < kBoxes; ++y) {
            const uint64_t kd = ptx::smem_desc_k_sw128(ptx::smem_u32(ring) + (uint32_t)(s * L::kStage + y * kTileKeys * 128));
            const uint64_t qd = ptx::smem_desc_k_sw128(ptx::smem_u32(q_sm) + (uint32_t)(qb * L::kQ + y * L::kN1 * 128));
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (y * 4 + k < ksteps)
                umma_e4m3(tmem + (uint32_t)(sb * L::kN1), kd + 2 * k, qd + 2 * k, idesc1, y + k > 0 ? 1u : 0u);
          }
          ptx::umma_commit(&tail->s_full[sb]);
          if (t == s1 - 1) ptx::umma_commit(&tail->q_empty[qb]);
        }
        __syncwarp();
        if (prev.valid) second();
        prev = {it, seg, t == s0, t == s1 - 1, true};
      }
      ++seg;
    }
    if (ok && prev.valid) second();
  } else if (warp < 4) {
    // ------------------------------------------------------------------ Q as three e4m3 terms, a segment ahead
    int seg = 0;
    for (int e = e_first; ok && e < entries && pref[e] < t1; ++e) {
      if (pref[e + 1] == pref[e]) continue;
      const int qb = seg & 1;
      const Entry x = entry_of(a, e);
      const int rows = x.nq * a.G;
      ok = __all_sync(0xffffffffu, wait_or_abort(&tail->q_empty[qb], ((seg >> 1) & 1) ^ 1, abort_flag));
      if (!ok) break;
      uint8_t* dst = q_sm + qb * L::kQ;
      for (int row = warp - 2; row < (L::kN1 - 2 * kRows); row += 2) {  // the rows, then the padding behind the third term
        const int qrow = group0 + row;
        const bool holds = row < kRows && qrow < rows;
        const int token = holds ? qrow / a.G : 0, g = holds ? qrow - token * a.G : 0;
        const __nv_bfloat16* src = a.Q + (int64_t)(x.q0 + token) * a.q_tok + (int64_t)(x.h * a.G + g) * a.q_head;
        uint2 v[kBoxes];
        uint32_t top = 0;                                              // the largest magnitude's bits
#pragma unroll
        for (int y = 0; y < kBoxes; ++y) {
          const int d = y * 128 + lane * 4;
          v[y] = holds && d < a.d_k ? *reinterpret_cast<const uint2*>(src + d) : make_uint2(0, 0);
          const uint32_t m = __vmaxu2(v[y].x & 0x7fff7fffu, v[y].y & 0x7fff7fffu);
          top = max(top, max(m & 0xffffu, m >> 16));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        // entries up to 2^8: multiply by 2^(7 - exponent); the exponent is kept where both factors are normal numbers
        const int ex = min(max((int)(top >> 7) - 127, -100), 127);
        const float up = __uint_as_float((uint32_t)(127 + 7 - ex) << 23);
#pragma unroll
        for (int y = 0; y < kBoxes; ++y) {
          float f[4] = {__uint_as_float(v[y].x << 16) * up, __uint_as_float(v[y].x & 0xffff0000u) * up,
                        __uint_as_float(v[y].y << 16) * up, __uint_as_float(v[y].y & 0xffff0000u) * up};
          if (top >= 0x7f80u) {                                        // an infinity is no 448: NaN, like a NaN
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = fabsf(f[i]) <= 3.4e38f ? f[i] : __uint_as_float(0x7fffffffu);
          }
#pragma unroll
          for (int term = 0; term < 3; ++term) {
            const int n = row < kRows ? term * kRows + row : 2 * kRows + row;
            const uint32_t c = take_term(f);
            if (row < kRows || term == 0)
              *reinterpret_cast<uint32_t*>(dst + (y * L::kN1 + n) * 128 + (((lane >> 2) ^ (n & 7)) << 4) + (lane & 3) * 4) = c;
          }
        }
        if (lane == 0 && row < kRows) {
          factor_sm[qb * kRows + row] = __uint_as_float((uint32_t)(127 - 7 + ex) << 23) * a.scale2;
          limit_sm[qb * kRows + row] = holds ? x.n - (x.nq - 1 - token) : 0;
        }
      }
      if (warp == 2 && lane == 0) tail->entry[qb] = x;
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&tail->q_full[qb]);
      ++seg;
    }
  } else {
    // ------------------------------------------------------------------ softmax: thread = row of the tile, channel of O
    const int w = warp - 4, key_in = w * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)(w * 32) << 16);
    float refd[kRows], refn[kRows], sum[kRows];                        // of the logits; of the weights times scale_v
    int it = 0, seg = 0;
    for (int e = e_first; e < entries && pref[e] < t1; ++e) {
      if (pref[e + 1] == pref[e]) continue;
      const int s0 = max(t0, pref[e]), s1 = min(t1, pref[e + 1]), qb = seg & 1;
      ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->q_full[qb], (seg >> 1) & 1, abort_flag));
      const Entry x = tail->entry[qb];
      const int nrows = min(kRows, x.nq * a.G - group0), all_see = x.n - (x.nq - 1);
#pragma unroll
      for (int g = 0; g < kRows; ++g) { refd[g] = refn[g] = kNoRef; sum[g] = 0.f; }
      const int64_t sb0 = (int64_t)x.h * a.row_blocks + block8_offset(x.start, x.r);
      auto scales = [&](int t) {
        const int key = (t - pref[e]) * kTileKeys + key_in;
        return key < x.n ? make_float2(a.k_scale[sb0 + (key >> 6)], a.v_scale[sb0 + (key >> 6)]) : make_float2(0.f, 1.f);
      };
      float2 next_scale = ok ? scales(s0) : make_float2(0.f, 1.f);
      for (int t = s0; t < s1; ++t, ++it) {
        const int sb = it & 1, key0 = (t - pref[e]) * kTileKeys, key = key0 + key_in;
        const float2 sc = next_scale;
        if (ok && t + 1 < s1) next_scale = scales(t + 1);
        ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->s_full[sb], (it >> 1) & 1, abort_flag));
        float l[kRows];
        const float lv = log2f(sc.y);                                  // (a power of two: exact)
        bool over = false;
        if (ok) {
          ptx::tc_fence_after_sync();
          uint32_t c[L::kN1 / 16][16];
#pragma unroll
          for (int i = 0; i < L::kN1 / 16; ++i) ptx::tmem_ld_32x16(lane_addr + (uint32_t)(sb * L::kN1 + i * 16), c[i]);
          ptx::tmem_wait_ld();
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->s_empty[sb]);
          const bool edge = key0 + kTileKeys > all_see;
#pragma unroll
          for (int g = 0; g < kRows; ++g) {
            auto term = [&](int k) { return __uint_as_float(c[(k * kRows + g) / 16][(k * kRows + g) % 16]); };
            l[g] = fmaf(term(2), 0.00390625f, fmaf(term(1), 0.0625f, term(0))) * (sc.x * factor_sm[qb * kRows + g]);
            if (edge && key >= limit_sm[qb * kRows + g]) l[g] = -INFINITY;
            over = over || l[g] + lv > refn[g] + kUp || l[g] > refd[g] + 64.f;
          }
          if (a.logits && key < x.n) {
            float* dst = a.logits + ((int64_t)x.h * a.max_q * a.G + group0) * a.total + x.start + key;
#pragma unroll
            for (int g = 0; g < kRows; ++g)
              if (g < nrows) dst[(int64_t)g * a.total] = l[g];
          }
        }
        if (softmax_any(over)) {
          // ---- some reference moves: the tile's largest exponents become the references, sums and O are rescaled
#pragma unroll
          for (int g = 0; g < kRows; ++g) {
            const float d = warp_max(ok ? l[g] : -INFINITY), n = warp_max(ok ? l[g] + lv : -INFINITY);
            if (lane == 0) { red_sm[w * 2 * kRows + 2 * g] = d; red_sm[w * 2 * kRows + 2 * g + 1] = n; }
          }
          softmax_any(false);
          float shrink[kRows];
#pragma unroll
          for (int g = 0; g < kRows; ++g) {
            float d = refd[g], n = refn[g];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              d = fmaxf(d, red_sm[k * 2 * kRows + 2 * g]);
              n = fmaxf(n, red_sm[k * 2 * kRows + 2 * g + 1]);
            }
            sum[g] *= exp2_fast(refd[g] - d);
            shrink[g] = exp2_fast(refn[g] - n);
            refd[g] = d;
            refn[g] = n;
          }
          if (ok && t > s0) {
            ok = __all_sync(0xffffffffu, wait_or_abort(&tail->p_empty[(it - 1) & 1], ((it - 1) >> 1) & 1, abort_flag));
            if (ok) {
              ptx::tc_fence_after_sync();
#pragma unroll
              for (int i = 0; i < kBoxes * L::kN2 / 16; ++i) {
                uint32_t v[16];
                ptx::tmem_ld_32x16(lane_addr + (uint32_t)(2 * L::kN1 + i * 16), v);
                ptx::tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * shrink[(i * 16 + j) % kRows]);
                tmem_st_32x16(lane_addr + (uint32_t)(2 * L::kN1 + i * 16), v);
              }
              ptx::tmem_wait_st();
              ptx::tc_fence_before_sync();
            }
          }
          softmax_any(false);                                          // red_sm has been read
        }
        // ---- weights and their terms
        const int pb = it & 1;
        ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->p_empty[pb], ((it >> 1) & 1) ^ 1, abort_flag));
        if (ok) {
          uint32_t p[L::kN2 / 4];                                      // four codes: rows 4 q .. of term k at k kRows / 4 + q
#pragma unroll
          for (int q = 0; q < kRows / 4; ++q) {
            float f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int g = 4 * q + i;
              sum[g] += exp2_fast(l[g] - refd[g]);
              f[i] = exp2_fast(l[g] + lv - refn[g] + kUp);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) p[k * (kRows / 4) + q] = take_term(f);
          }
          uint8_t* dst = p_sm + pb * L::kP + key_in * 16;
#pragma unroll
          for (int i = 0; i < L::kN2 / 16; ++i)
            *reinterpret_cast<uint4*>(dst + i * 16 * kTileKeys) = make_uint4(p[4 * i], p[4 * i + 1], p[4 * i + 2], p[4 * i + 3]);
          if (key0 + kTileKeys > all_see && key >= all_see) {
            // A value behind the last row may be anything, and one that not every token sees may be NaN: neither must
            // reach the others through a weight of zero.  The first becomes zero, the second is noted for those who see it.
            wait_or_abort(&tail->kv_full[it % a.stages], (it / a.stages) & 1, abort_flag);   // (complete: S came of this tile)
            uint8_t* v = ring + (size_t)(it % a.stages) * L::kStage + (kBoxes * kTileKeys + key_in) * 128;
            for (int y = 0; y < kBoxes; ++y)
              for (int i = 0; i < 8; ++i) {
                uint4* at = reinterpret_cast<uint4*>(v + y * kTileKeys * 128 + ((i ^ (key_in & 7)) << 4));
                uint4 u = make_uint4(0, 0, 0, 0);
                if (key < x.n) {
                  u = *at;
#pragma unroll
                  for (int j = 0; j < 4; ++j) {
                    uint32_t& word = (&u.x)[j];
                    const uint32_t bad = __vcmpeq4(word & 0x7f7f7f7fu, 0x7f7f7f7fu);
                    if (!bad) continue;
                    word &= ~bad;
                    tail->any_nan = 1;
                    const uint32_t four = (bad & 1u) | ((bad >> 7) & 2u) | ((bad >> 14) & 4u) | ((bad >> 21) & 8u);
                    const int d = y * 128 + i * 16 + j * 4;
                    for (int g = 0; g < nrows; ++g)
                      if (key < limit_sm[qb * kRows + g]) atomicOr(&nan_sm[g * kBoxes * 4 + (d >> 5)], four << (d & 31));
                  }
                }
                *at = u;
              }
          }
          ptx::fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&tail->p_full[pb]);
      }

      // ---- the segment's result
#pragma unroll
      for (int g = 0; g < kRows; ++g) {
        float s = sum[g];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) red_sm[w * 2 * kRows + g] = s;
      }
      softmax_any(false);
      const bool nan_seen = tail->any_nan != 0;
      const bool whole = pref[e] >= t0 && pref[e + 1] <= t1;           // the entry lies within this CTA
      const int64_t slot = ((int64_t)blockIdx.y * (entries + B) + e + b) * a.group_rows;
      ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->o_full, seg & 1, abort_flag));
      if (ok) {
        ptx::tc_fence_after_sync();
        constexpr int kPart = kRows < 16 ? kRows : 16;                 // rows at a time
#pragma unroll
        for (int y = 0; y < kBoxes; ++y) {
          const int d = y * 128 + key_in;
#pragma unroll
          for (int g0 = 0; g0 < kRows; g0 += kPart) {
            constexpr int kChunks = 4 * kPart / 16;
            uint32_t v[kChunks][16];
#pragma unroll
            for (int i = 0; i < kChunks; ++i)                          // kPart = 16: term i; below: the terms lie side by side
              ptx::tmem_ld_32x16(lane_addr + (uint32_t)(2 * L::kN1 + y * L::kN2 + (kPart == 16 ? i * kRows + g0 : i * 16)), v[i]);
            ptx::tmem_wait_ld();
            if (d < a.d_k) {
#pragma unroll
              for (int i = 0; i < kPart; ++i) {
                const int g = g0 + i;
                if (g < nrows) {
                  auto term = [&](int k) { return __uint_as_float(v[(k * kPart + i) / 16][(k * kPart + i) % 16]); };
                  float o = fmaf(term(3), 0.000244140625f, fmaf(term(2), 0.00390625f, fmaf(term(1), 0.0625f, term(0))));
                  const float total = (red_sm[g] + red_sm[2 * kRows + g]) + (red_sm[4 * kRows + g] + red_sm[6 * kRows + g]);
                  const float f = exp2_fast(0.5f * (refn[g] - refd[g]));     // (in two steps: it may lie below 2^-126)
                  o = total == 0.f ? 0.f : o * 0.0625f / total * f * f;
                  if (nan_seen && ((nan_sm[g * kBoxes * 4 + (d >> 5)] >> (d & 31)) & 1u)) o = __uint_as_float(0x7fffffffu);
                  const int qrow = group0 + g;
                  if (whole) {
                    const int token = qrow / a.G, head = x.h * a.G + qrow - token * a.G;
                    a.out[(int64_t)(x.q0 + token) * a.o_tok + (int64_t)head * a.o_head + d] = __float2bfloat16(o);
                    if (d == 0 && a.lse)
                      a.lse[(int64_t)(x.q0 + token) * a.Hkv * a.G + head] = total == 0.f ? -INFINITY : (refd[g] + log2f(total)) * 0.6931471805599453f;
                  } else {
                    a.part_o[(slot + g) * a.d_k + d] = o;
                  }
                  if (d == 0) a.part_ml[slot + g] = make_float2(total == 0.f ? -INFINITY : refd[g], total);
                }
              }
            }
          }
        }
        ptx::tc_fence_before_sync();
      }
      __syncwarp();
      if (lane == 0) { ptx::mbar_arrive(&tail->o_empty); ptx::mbar_arrive(&tail->q_empty[qb]); }
      softmax_any(false);                                              // red_sm and the NaN marks have been read
      if (nan_seen) {
        for (int i = key_in; i < L::kNan / 4; i += 128) nan_sm[i] = 0;
        tail->any_nan = 0;
        softmax_any(false);
      }
      ++seg;
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

// What an entry's segments say of one row: the maximum, and the sum relative to it.  A whole warp asks; the segments are
// spread over its lanes, so that their loads are in flight together.
__device__ __forceinline__ float2 merged_ml(const AttendArgs& a, int B, int group, int e, int2 v, int in_group, int entries) {
  const float2* ml = a.part_ml + ((int64_t)group * (entries + B) + e) * a.group_rows + in_group;
  float M = -INFINITY, L = 0.f;
  for (int b = v.x + (int)(threadIdx.x & 31); v.x >= 0 && b <= v.y; b += 32) {
    const float2 x = ml[(int64_t)b * a.group_rows];
    const float top = fmaxf(M, x.x);
    if (top != -INFINITY) L = L * exp2_fast(M - top) + x.y * exp2_fast(x.x - top);
    else L += x.y;                                      // (a NaN in the sum stays)
    M = top;
  }
  const float all = warp_max(M);
  L = all == -INFINITY ? L : L == 0.f ? 0.f : L * exp2_fast(M - all);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
  return make_float2(all, L);
}

// Blocks 0 .. entries * max_rows - 1: one row of one entry, merged from its segments when it has several (or none).
// The others: 256 slots of one entry each, their weights added to acc.
__global__ void __launch_bounds__(256)
attend8_finish_kernel(const __grid_constant__ AttendArgs a, int B, int max_rows, int slot_blocks) {
  __shared__ float4 s_o[8][32 * 2];
  __shared__ float s_neg[GVOTE_ATTEND8_MAX_Q * kMaxGroup8];
  const int entries = a.batch * a.Hkv, tid = threadIdx.x;
  const bool merging = (int64_t)blockIdx.x < (int64_t)entries * max_rows;
  if (merging) {
    const int e = blockIdx.x / max_rows, row = blockIdx.x - e * max_rows;
    const Entry x = entry_of(a, e);
    if (row >= x.nq * a.G) return;
    const int group = row / a.group_rows, in_group = row - group * a.group_rows;
    const int2 v = a.info[(int64_t)group * entries + e];
    if (v.x >= 0 && v.x == v.y) return;                 // the first kernel has written it
    const float2 ml = merged_ml(a, B, group, e, v, in_group, entries);
    const int quads = a.d_k >> 2, part = tid >> 5, lane = tid & 31;
    const int64_t slot0 = ((int64_t)group * (entries + B) + e) * a.group_rows + in_group;
    for (int q = lane; q < quads; q += 32) {
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      if (v.x >= 0) {
#pragma unroll 4
        for (int b = v.x + part; b <= v.y; b += 8) {
          const int64_t slot = slot0 + (int64_t)b * a.group_rows;
          const float2 m = a.part_ml[slot];
          const float4 p = *reinterpret_cast<const float4*>(a.part_o + slot * a.d_k + q * 4);
          const float f = m.x == -INFINITY ? 0.f : exp2_fast(m.x - ml.x) * m.y;
          if (f != 0.f) { s.x = fmaf(f, p.x, s.x); s.y = fmaf(f, p.y, s.y); s.z = fmaf(f, p.z, s.z); s.w = fmaf(f, p.w, s.w); }
        }
      }
      s_o[part][q] = s;
    }
    __syncthreads();
    const int token = row / a.G, g = x.h * a.G + row % a.G;
    if (tid < quads) {
      float4 s = s_o[0][tid];
      for (int k = 1; k < 8; ++k) {
        const float4 p = s_o[k][tid];
        s.x += p.x; s.y += p.y; s.z += p.z; s.w += p.w;
      }
      const float inv = ml.x == -INFINITY && ml.y == 0.f ? 0.f : 1.f / ml.y;
      __nv_bfloat162 out[2] = {__floats2bfloat162_rn(s.x * inv, s.y * inv), __floats2bfloat162_rn(s.z * inv, s.w * inv)};
      *reinterpret_cast<uint2*>(a.out + (int64_t)(x.q0 + token) * a.o_tok + (int64_t)g * a.o_head + tid * 4) = *reinterpret_cast<uint2*>(out);
    }
    if (tid == 0 && a.lse)
      a.lse[(int64_t)(x.q0 + token) * a.Hkv * a.G + g] = ml.x == -INFINITY ? -INFINITY : (ml.x + log2f(ml.y)) * 0.6931471805599453f;
    return;
  }
  const int64_t k = (int64_t)blockIdx.x - (int64_t)entries * max_rows;
  const int h = (int)(k % a.Hkv);
  const int64_t gb = k / a.Hkv;                         // 256-slot blocks of the requests, request r from (cu[r] >> 8) + r on
  const int r = a.r0 + (a.batch == 1 ? 0 : find_request_by(a.cu + a.r0, a.batch, gb + (a.cu[a.r0] >> 8), 8));
  const int e = (r - a.r0) * a.Hkv + h;
  const Entry x = entry_of(a, e);
  const int i0 = (int)(gb - ((x.start >> 8) - (a.cu[a.r0] >> 8) + (r - a.r0))) * 256;
  if (i0 >= x.n || i0 < 0) return;
  const int rows = x.nq * a.G;
  for (int row = tid >> 5; row < rows; row += 8) {
    const int group = row / a.group_rows;
    const float2 ml = merged_ml(a, B, group, e, a.info[(int64_t)group * entries + e], row - group * a.group_rows, entries);
    s_neg[row] = ml.x == -INFINITY ? -INFINITY : -(ml.x + log2f(ml.y));
  }
  __syncthreads();
  const int i = i0 + tid;
  if (i >= x.n) return;
  float s = 0.f;
  const float* l = a.logits + (int64_t)h * a.max_q * a.G * a.total + x.start + i;
#pragma unroll 4
  for (int row = 0; row < rows; ++row) {
    const float v = l[(int64_t)row * a.total];
    if (v != -INFINITY) s += exp2_fast(v + s_neg[row]);
  }
  const int64_t slot = (int64_t)h * a.total + x.start + i;
  a.acc_out[slot] = (a.acc ? a.acc[slot] : 0.f) + s;
}

// How a launch is cut: query rows per group, ring, CTAs.
struct Cut { int boxes, rows, groups, requests; int64_t ctas; };
Cut cut_of(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_q) {
  Cut c;
  const int64_t rows = max_q * (p->n_q_heads / p->n_kv_heads);
  c.boxes = p->d_k <= 128 ? 1 : 2;
  // the padded rows cost columns of both products and the softmax's time; beyond 32 the codes are read again (from L2)
  c.rows = rows <= 4 ? 4 : rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
  c.groups = (int)ceil_div(rows > 0 ? rows : 1, c.rows);
  c.requests = kMaxEntries / p->n_kv_heads < batch ? kMaxEntries / p->n_kv_heads : batch;
  // a CTA per SM, and no more than one per tile
  const int64_t most_ctas = (total_tokens / kTileKeys + batch) * p->n_kv_heads;
  c.ctas = most_ctas < kSms ? most_ctas : kSms;
  return c;
}

template <int kBoxes, int kRows>
int32_t run_attend(const Cut& c, const CUtensorMap& tmK, const CUtensorMap& tmV, AttendArgs a, cudaStream_t st) {
  using L = Layout<kBoxes, kRows>;
  const size_t fit = (227 * 1024 - L::fixed()) / L::kStage;
  a.stages = (int)(fit < kMaxStages ? fit : kMaxStages);
  const size_t smem = L::fixed() + (size_t)a.stages * L::kStage;
  auto kernel = attend8_kernel<kBoxes, kRows>;
  GVOTE_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  {
    LaunchScope scope_("attend8_kernel", st);
    launch_on(kernel, dim3((unsigned)c.ctas, (unsigned)c.groups), dim3(kThreads), smem, st, tmK, tmV, a);
  }
  GVOTE_LAUNCH_CHECK("attend8_kernel");
  return GVOTE_OK;
}
template <int kBoxes>
int32_t run_attend(const Cut& c, const CUtensorMap& tmK, const CUtensorMap& tmV, const AttendArgs& a, cudaStream_t st) {
  switch (c.rows) {
    case 4: return run_attend<kBoxes, 4>(c, tmK, tmV, a, st);
    case 8: return run_attend<kBoxes, 8>(c, tmK, tmV, a, st);
    case 16: return run_attend<kBoxes, 16>(c, tmK, tmV, a, st);
    default: return run_attend<kBoxes, 32>(c, tmK, tmV, a, st);
  }
}

}  // namespace

AttendMap attend8_map(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N, int64_t total_q,
                      int64_t max_q) {
  AttendMap m;
  const int64_t nq = max_q < GVOTE_ATTEND8_MAX_Q ? max_q : GVOTE_ATTEND8_MAX_Q;
  const Cut c = cut_of(p, batch, total_tokens, nq);
  const size_t entries = (size_t)c.requests * p->n_kv_heads;
  const size_t rows = (size_t)c.groups * (entries + c.ctas) * c.rows;
  m.o = kStatusBytes;
  m.ml = align_up(m.o + rows * p->d_k * 4, 256);
  m.info = align_up(m.ml + rows * 8, 256);
  m.logits = align_up(m.info + c.groups * entries * 8, 256);
  m.total = align_up(m.logits + (size_t)p->n_q_heads * nq * total_tokens * 4, 256);
  return m;
}

int32_t launch_attend8(const gvote_params* p, const __nv_bfloat16* Q, int64_t q_tok, int64_t q_head, const int32_t* cu_q,
                       int64_t total_q, int64_t max_q, const gvote_cache8* c, __nv_bfloat16* out, int64_t o_tok,
                       int64_t o_head, float* lse, const float* acc, float* acc_out, char* ws, cudaStream_t st) {
  const AttendMap m = attend8_map(p, c->batch, c->total_tokens, c->max_N, total_q, max_q);
  const Cut cut = cut_of(p, c->batch, c->total_tokens, max_q);
  AttendArgs a;
  a.Q = Q; a.q_tok = q_tok; a.q_head = q_head; a.cu_q = cu_q;
  a.k_scale = c->k_scale; a.v_scale = c->v_scale;
  a.total = c->total_tokens;
  a.row_blocks = gvote_cache8_row_blocks(c->total_tokens, c->batch);
  a.cu = c->cu_seqlens; a.kv_len = c->kv_len;
  a.out = out; a.o_tok = o_tok; a.o_head = o_head; a.lse = lse; a.acc = acc; a.acc_out = acc_out;
  a.part_o = (float*)(ws + m.o); a.part_ml = (float2*)(ws + m.ml); a.info = (int2*)(ws + m.info);
  a.logits = acc_out ? (float*)(ws + m.logits) : nullptr;
  a.status = (int32_t*)ws;
  a.Hkv = p->n_kv_heads; a.G = p->n_q_heads / p->n_kv_heads; a.d_k = p->d_k; a.max_q = (int)max_q;
  a.stages = 0; a.group_rows = cut.rows;
  a.scale2 = (float)(1.4426950408889634 / sqrt((double)p->d_k));

  CUtensorMap tmK, tmV;
  const uint64_t dims[3] = {(uint64_t)p->d_k, (uint64_t)c->total_tokens, (uint64_t)a.Hkv};
  const uint64_t strides[2] = {(uint64_t)c->tok_stride, (uint64_t)(a.Hkv > 1 ? c->head_stride : c->tok_stride)};
  const uint32_t box[3] = {128, (uint32_t)kBoxRows, 1};
  if (!encode_tensor_map_u8(&tmK, c->K, 3, dims, strides, box) || !encode_tensor_map_u8(&tmV, c->V, 3, dims, strides, box))
    return GVOTE_ERR_UNSUPPORTED_SHAPE;

  for (int32_t r0 = 0; r0 < c->batch; r0 += cut.requests) {
    a.r0 = r0;
    a.batch = c->batch - r0 < cut.requests ? c->batch - r0 : cut.requests;
    PROPAGATE(cut.boxes == 1 ? run_attend<1>(cut, tmK, tmV, a, st) : run_attend<2>(cut, tmK, tmV, a, st));
    const int64_t entries = (int64_t)a.batch * a.Hkv, rows = max_q * a.G;
    const int64_t slots = acc_out ? ((c->total_tokens >> 8) + a.batch) * a.Hkv : 0;
    LaunchScope scope_("attend8_finish_kernel", st);
    launch_on(attend8_finish_kernel, dim3((unsigned)(entries * rows + slots)), dim3(256), 0, st, a, (int)cut.ctas, (int)rows,
              (int)slots);
    GVOTE_LAUNCH_CHECK("attend8_finish_kernel");
  }
  return GVOTE_OK;
}

}  // namespace gvote
