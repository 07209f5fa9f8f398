// Attention weight each cached key collects from a prompt's queries (gvote_accumulate):
//   acc[h][n] += sum over query tokens i and query heads g of KV head h of exp(q_ig.k_n / sqrt(d_k) - lse_ig).
//
// Two passes over the causal part of Q K^T on the fifth-generation tensor cores; the logits never reach memory.
//   pass 1  A = 128 query rows, B = 128 keys: a read-out thread owns a query row and keeps its reference and its sum of
//           exponentials in registers; it leaves lse2 = log2 of the softmax denominator (skipped when the caller has it).
//   pass 2  A = 128 keys, B = 128 query rows: a read-out thread owns a key and sums exp2(c s - lse2[row]) over the
//           columns, so that the sum over queries needs neither atomics nor a reduction between threads.
//
// A query tile is floor(128 / G) tokens with the G heads of the group (token-major), fetched by one TMA box per 64
// channels.  A persistent CTA per SM walks units; a unit keeps TWO tiles (of query rows in pass 1, of keys in pass 2)
// stationary and streams the other operand past both, which halves the stream's shared-memory fill (32 KB per
// 2 x 128 x 128 logits).  Warp 0 asks for the tiles (TMA, 128-byte swizzle), warp 1 issues the MMAs, sixteen warps
// read out, two per lane quadrant of a stationary tile (64 columns each); two accumulators of 128 columns each per
// stationary tile (all 512 columns of tensor memory).  The next unit's stationary tiles are fetched while this one runs.
//
// Units differ in length (causal), longest first; a CTA takes them boustrophedon, so that the first CTA does not get the
// longer one in every round.  Where that leaves fewer than four units per SM, the streamed tiles of a unit are split
// into chunks: pass 1 leaves (reference, sum) pairs that accumulate_lse_kernel merges, pass 2 partial sums
// that accumulate_sum_kernel adds in order.
//
// Bound by the exponentials: one per logit and pass, 16 per clock and SM, twice the tensor cores' time.  So
// kPoly of every 8 pairs are evaluated on the FMA pipe instead (exp2_poly2); two or three of 8 were slower, the instructions
// then bound it.  Measured (one B200): all tokens of a 32K prompt, 32 heads on 8: 10.6 ms, 4.8 in pass 1 and 5.8 in
// pass 2 (8.8 TFLOP, the exponentials alone 7.6 ms on their unit, which is 82 % busy in pass 1 and 70 % in pass 2; the
// tensor pipe 45 and 39 %); the last 32 tokens of a 128K prompt, 28 heads on 4: 110 us, 48 + 62, for 117 M exponentials
// per pass (26 us each) and 134 MB.  One issuing lane behind a lane-number branch, eight read-out warps, fetching the
// accumulator a tile ahead, and a pass 1 without a maximum were all slower.
//
// Every wait is bounded: when one runs out the CTA records GVOTE_ERR_TIMEOUT in the status word, frees its tensor
// memory and returns.
#include "cache8.cuh"
#include "ptx.cuh"

namespace gvote {
namespace {

constexpr int kTile = 128;            // rows of A and of B
constexpr int kReadWarps = 16;
constexpr int kAccThreads = 64 + 32 * kReadWarps;
constexpr int kMaxStages = 6;
constexpr int kLseStages = 3;
constexpr int kPoly = 1;                // of 8 exponentials, those computed on the FMA pipe
constexpr int kUnitsPerSm = 4;
constexpr int kSideFloats = (kLseStages + 2) * kTile;   // lse slots and the second halves' sums (pass 1: 2 x 128 pairs)
constexpr int kSms = 148;
constexpr float kLog2e = 1.4426950408889634f;

struct AccArgs {
  const int32_t* cu_q;
  const int32_t* cu;
  const int32_t* kv_len;
  float* lse2;                        // [Hkv][q_tiles][128] the NEGATIVE log2 of the denominators; -inf (weight 0) on rows without
                                      // a query and on queries that see no key
  float2* part;                       // [chunks][Hkv][q_tiles][128] (reference, sum), when pass 1 is split
  float* part_sum;                    // [chunks][Hkv][total], when pass 2 is split
  const float* acc;
  float* acc_out;
  int32_t* status;
  int64_t total, q_tiles;
  uint32_t pairs, units;
  int Hkv, G, batch, d_k, tpt;        // tpt: tokens of a query tile
  int boxes, stages, stat_slots, chunks;
  float c;                            // log2(e) / sqrt(d_k)
};

struct Tail {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t stat_full[2], stat_empty[2];
  uint64_t lse_full[kLseStages], lse_empty[kLseStages];
  uint64_t acc_full[2][2], acc_empty[2][2];
  uint64_t half_full[2], half_empty[2];
  uint64_t drain;                       // the MMAs under way, after a wait that ran out
  uint32_t tmem_slot;
  volatile int abort_flag;
};

__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  for (uint32_t i = 0; i < (1u << 20); ++i) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if ((i & 255u) == 255u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
// Before the producer leaves early: the loads of a ring that may still write to this CTA's memory.
__device__ __forceinline__ void drain_copies(uint64_t* full, int slots, int issued) {
  for (int i = issued > slots ? issued - slots : 0; i < issued; ++i)
    for (int k = 0; k < (1 << 12) && !ptx::mbar_try_wait(&full[i % slots], (i / slots) & 1); ++k) {}
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Packed pairs of 32-bit floats.
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ float2 unpack2(uint64_t d) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(d));
  return f;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// 2^x for a pair, x <= 127, without the special-function unit: x = i + f with i the nearest integer (read off the low bits
// of x + 1.5 * 2^23 + 127, which are i + 127), 2^f by the polynomial of degree 5 with the smallest largest relative error
// on [-1/2, 1/2] (Remez exchange; 1.5e-7 with the coefficients as they are rounded here, 2.1e-7 in 32 bits).  x is taken to
// -127 at least, where the power that i gives is zero: what lies below 2^-126.5 is zero, -inf too; a NaN stays one.
__device__ __forceinline__ uint64_t exp2_poly2(uint64_t x2) {
  float2 x = unpack2(x2);
  x2 = pack2(max_nan(x.x, -127.f), max_nan(x.y, -127.f));
  const uint64_t r2 = add2(x2, pack2(12583039.f, 12583039.f));
  const uint64_t i2 = add2(r2, pack2(-12583039.f, -12583039.f));
  const uint64_t f2 = fma2(i2, pack2(-1.f, -1.f), x2);
  uint64_t p = pack2(1.3276472e-3f, 1.3276472e-3f);
  p = fma2(p, f2, pack2(9.6755410e-3f, 9.6755410e-3f));
  p = fma2(p, f2, pack2(5.5507131e-2f, 5.5507131e-2f));
  p = fma2(p, f2, pack2(2.4022120e-1f, 2.4022120e-1f));
  p = fma2(p, f2, pack2(6.9314694e-1f, 6.9314694e-1f));
  p = fma2(p, f2, pack2(1.0000001f, 1.0000001f));
  const float2 r = unpack2(r2);
  return mul2(p, pack2(__uint_as_float(__float_as_uint(r.x) << 23), __uint_as_float(__float_as_uint(r.y) << 23)));
}
// Of every eight consecutive pairs j, kShare spread evenly go to the FMA pipe.
template <int kShare>
__device__ __forceinline__ uint64_t exp2_pair(int j, uint64_t x2) {
  if (((j + 1) * kShare) / 8 != (j * kShare) / 8) return exp2_poly2(x2);
  const float2 x = unpack2(x2);
  return pack2(exp2_fast(x.x), exp2_fast(x.y));
}

struct UnitInfo {
  int r, h, n, nq, q0, start;
  int stat0, n_stat;                  // stationary tiles (of the request), how many: 0 when the unit is not used
  int s0, s1;                         // streamed tiles
  int chunk;
};

// The largest r with cu[r] / per + r <= g.
__device__ __forceinline__ int find_request_div(const int32_t* __restrict__ cu, int batch, int64_t g, int per) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)(cu[mid] / per) + mid <= g) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Of a batch's first request: where its keys and queries are (the only one's, when there is one).
struct Only { int start, n, q0, nq; };

// The unit this CTA takes in round k: left to right in even rounds, right to left in odd ones.
__device__ __forceinline__ uint32_t unit_of(uint32_t k) {
  return k * gridDim.x + ((k & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
}

template <int kPass>
__device__ __forceinline__ UnitInfo unit_info(const AccArgs& a, const Only& only, uint32_t u) {
  UnitInfo x;
  uint32_t v = u / (uint32_t)a.Hkv;
  x.h = (int)(u - v * (uint32_t)a.Hkv);
  x.chunk = 0;
  if (a.chunks > 1) {
    const uint32_t w = v / (uint32_t)a.chunks;
    x.chunk = (int)(v - w * (uint32_t)a.chunks);
    v = w;
  }
  if (kPass == 1) v = a.pairs - 1 - v;                     // long rows first
  if (a.batch == 1) {                                      // (the lookups cost a short unit a sixth of its time)
    x.r = 0;
    x.start = only.start; x.q0 = only.q0; x.nq = only.nq;
    x.n = valid_keys(a.kv_len, 0, a.Hkv, x.h, only.n);
  } else {
    x.r = kPass == 1 ? find_request_div(a.cu_q, a.batch, v, 2 * a.tpt) : find_request_by(a.cu, a.batch, v, 8);
    x.start = a.cu[x.r];
    x.n = valid_keys(a.kv_len, x.r, a.Hkv, x.h, a.cu[x.r + 1] - x.start);
    x.q0 = a.cu_q[x.r];
    x.nq = a.cu_q[x.r + 1] - x.q0;
  }
  const int q_tiles = (x.nq + a.tpt - 1) / a.tpt;
  if (kPass == 1) {
    x.stat0 = 2 * (int)(v - (x.q0 / (2 * a.tpt) + x.r));
    x.n_stat = max(min(2, q_tiles - x.stat0), 0);
    if (x.stat0 < 0) x.n_stat = 0;                         // (a list that starts behind token 0)
    const int last = min(x.nq, (x.stat0 + x.n_stat) * a.tpt) - 1;
    const int tiles = (max(x.n - (x.nq - 1 - last), 0) + kTile - 1) / kTile;
    x.s0 = 0;
    x.s1 = tiles;
  } else {
    x.stat0 = 2 * (int)(v - ((x.start >> 8) + x.r));
    x.n_stat = max(min(2, (x.n + kTile - 1) / kTile - x.stat0), 0);
    if (x.stat0 < 0) x.n_stat = 0;
    x.s0 = min(max(x.stat0 * kTile - (x.n - x.nq), 0) / a.tpt, q_tiles);
    x.s1 = q_tiles;
  }
  const int first = x.s0, tiles = x.s1 - x.s0;
  if (a.chunks > 1) {
    x.s0 = first + (int)((int64_t)tiles * x.chunk / a.chunks);
    x.s1 = first + (int)((int64_t)tiles * (x.chunk + 1) / a.chunks);
  }
  return x;
}

template <int kPass>
__global__ void __launch_bounds__(kAccThreads, 1)
accumulate_umma_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ AccArgs a) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* base = smem_raw;                       // (no static shared memory: the dynamic part starts on a 1024-byte boundary)
  const uint32_t tile_bytes = (uint32_t)a.boxes * kTile * 128;
  uint8_t* stat_sm = base;                                         // [stat_slots][2][tile]
  uint8_t* ring_sm = stat_sm + (size_t)a.stat_slots * 2 * tile_bytes;
  float* lse_sm = reinterpret_cast<float*>(ring_sm + (size_t)a.stages * tile_bytes);
  // the second half's state at the end of a unit: pass 1 [2][128] (reference, sum), pass 2 [2][128] sums behind the lse slots
  float2* half1_sm = reinterpret_cast<float2*>(lse_sm);
  float* half2_sm = lse_sm + kLseStages * kTile;
  Tail* tail = reinterpret_cast<Tail*>(lse_sm + kSideFloats);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  // the rows of a query tile that no box fills (G does not divide 128) must be finite
  for (uint4* p = reinterpret_cast<uint4*>(base) + threadIdx.x; p < reinterpret_cast<uint4*>(lse_sm); p += kAccThreads)
    *p = make_uint4(0, 0, 0, 0);
  ptx::fence_proxy_async();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kMaxStages; ++s) { ptx::mbar_init(&tail->full[s], 1); ptx::mbar_init(&tail->empty[s], 1); }
    for (int s = 0; s < kLseStages; ++s) { ptx::mbar_init(&tail->lse_full[s], 1); ptx::mbar_init(&tail->lse_empty[s], kReadWarps); }
    for (int s = 0; s < 2; ++s) {
      ptx::mbar_init(&tail->stat_full[s], 1);
      ptx::mbar_init(&tail->stat_empty[s], 1);
      for (int b = 0; b < 2; ++b) { ptx::mbar_init(&tail->acc_full[s][b], 1); ptx::mbar_init(&tail->acc_empty[s][b], 8); }
      ptx::mbar_init(&tail->half_full[s], 4);
      ptx::mbar_init(&tail->half_empty[s], 4);
    }
    ptx::mbar_init(&tail->drain, 1);
    tail->abort_flag = (ptx::smem_u32(smem_raw) & 1023u) ? 1 : 0;
    ptx::fence_barrier_init();
    ptx::prefetch_tensormap(&tmQ);
    ptx::prefetch_tensormap(&tmK);
  }
  if (warp == 1) {
    ptx::tmem_alloc(&tail->tmem_slot, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  ptx::let_next_begin();
  ptx::wait_for_previous();                       // (pass 1, and the first kernel of a call: nothing to wait for)
  const uint32_t tmem = __shfl_sync(0xffffffffu, tail->tmem_slot, 0);
  volatile int* abort_flag = &tail->abort_flag;
  const int q_rows = a.G * a.tpt;                                  // rows a query box fills
  const Only only = {a.cu[0], a.cu[1] - a.cu[0], a.cu_q[0], a.cu_q[1] - a.cu_q[0]};
  const uint32_t q_bytes = (uint32_t)a.boxes * q_rows * 128, k_bytes = tile_bytes;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int unit = 0, it = 0, tiles = 0, rows = 0;                   // (tiles and lse rows asked for)
      bool ok = true;
      for (uint32_t k = 0; ok && k * gridDim.x < a.units; ++k) {
        const uint32_t u = unit_of(k);
        if (u >= a.units) continue;
        const UnitInfo x = unit_info<kPass>(a, only, u);
        if (x.n_stat == 0 || x.s1 <= x.s0) continue;
        const int slot = unit % a.stat_slots;
        ok = wait_or_abort(&tail->stat_empty[slot], ((unit / a.stat_slots) & 1) ^ 1, abort_flag);
        if (!ok) break;
        ++unit;
        ptx::mbar_arrive_expect_tx(&tail->stat_full[slot], (uint32_t)x.n_stat * (kPass == 1 ? q_bytes : k_bytes));
        for (int s = 0; s < x.n_stat; ++s)
          for (int c = 0; c < a.boxes; ++c) {
            uint8_t* dst = stat_sm + (size_t)(slot * 2 + s) * tile_bytes + (size_t)c * kTile * 128;
            if (kPass == 1) ptx::tma_load_3d(dst, &tmQ, &tail->stat_full[slot], c * 64, x.h * a.G, x.q0 + (x.stat0 + s) * a.tpt);
            else ptx::tma_load_3d(dst, &tmK, &tail->stat_full[slot], c * 64, x.start + (x.stat0 + s) * kTile, x.h);
          }
        for (int t = x.s0; t < x.s1; ++t, ++it) {
          const int s = it % a.stages;
          ok = wait_or_abort(&tail->empty[s], ((it / a.stages) & 1) ^ 1, abort_flag);
          if (!ok) break;
          ptx::mbar_arrive_expect_tx(&tail->full[s], kPass == 1 ? k_bytes : q_bytes);
          ++tiles;
          for (int c = 0; c < a.boxes; ++c) {
            uint8_t* dst = ring_sm + (size_t)s * tile_bytes + (size_t)c * kTile * 128;
            if (kPass == 1) ptx::tma_load_3d(dst, &tmK, &tail->full[s], c * 64, x.start + t * kTile, x.h);
            else ptx::tma_load_3d(dst, &tmQ, &tail->full[s], c * 64, x.h * a.G, x.q0 + t * a.tpt);
          }
          if (kPass == 2) {
            const int l = it % kLseStages;
            ok = wait_or_abort(&tail->lse_empty[l], ((it / kLseStages) & 1) ^ 1, abort_flag);
            if (!ok) break;
            ptx::mbar_arrive_expect_tx(&tail->lse_full[l], kTile * 4);
            ++rows;
            ptx::bulk_load(lse_sm + l * kTile, a.lse2 + ((int64_t)x.h * a.q_tiles + x.q0 / a.tpt + x.r + t) * kTile, kTile * 4,
                           &tail->lse_full[l]);
          }
        }
      }
      if (!ok) {
        drain_copies(tail->stat_full, a.stat_slots, unit);
        drain_copies(tail->full, a.stages, tiles);
        drain_copies(tail->lse_full, kLseStages, rows);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    // The whole warp walks the units, so that every operand of the MMAs is uniform over it, and one elected lane issues:
    // with a branch on the lane number instead, an MMA took 70 clocks to issue and bounded the kernel.
    const uint32_t idesc = ptx::instr_desc_bf16_f32(kTile, kTile);
    const int ksteps = a.d_k / 16;
    int unit = 0, it = 0, used0 = 0, used1 = 0;
    bool ok = true;
    for (uint32_t k = 0; ok && k * gridDim.x < a.units; ++k) {
      const uint32_t u = unit_of(k);
      if (u >= a.units) continue;
      const UnitInfo x = unit_info<kPass>(a, only, u);
      if (x.n_stat == 0 || x.s1 <= x.s0) continue;
      const int slot = unit % a.stat_slots;
      ok = __all_sync(0xffffffffu, wait_or_abort(&tail->stat_full[slot], (unit / a.stat_slots) & 1, abort_flag));
      ++unit;
      const uint64_t a_desc = ptx::smem_desc_k_sw128(ptx::smem_u32(stat_sm) + (uint32_t)slot * 2u * tile_bytes);
      for (int t = x.s0; ok && t < x.s1; ++t, ++it) {
        const int s = it % a.stages;
        ok = __all_sync(0xffffffffu, wait_or_abort(&tail->full[s], (it / a.stages) & 1, abort_flag));
        if (!ok) break;
        const uint64_t b_desc = ptx::smem_desc_k_sw128(ptx::smem_u32(ring_sm) + (uint32_t)s * tile_bytes);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (i < x.n_stat) {
            int& used = i ? used1 : used0;
            const int b = used & 1;
            ok = ok && __all_sync(0xffffffffu, wait_or_abort(&tail->acc_empty[i][b], ((used >> 1) & 1) ^ 1, abort_flag));
            if (!ok) break;
            ++used;
            ptx::tc_fence_after_sync();
            if (ptx::elect_one()) {
              // (descriptor addresses count 16 bytes: a K step of 16 channels is 2, the next 64 channels are a box away)
              uint64_t ad = a_desc + (uint64_t)((i * tile_bytes) >> 4), bd = b_desc;
              const uint32_t d = tmem + (uint32_t)((i * 2 + b) * kTile);
              for (int q = 0; q < ksteps; q += 4, ad += kTile * 128 / 16, bd += kTile * 128 / 16) {
                ptx::umma_bf16(d, ad, bd, idesc, q > 0 ? 1u : 0u);
                if (q + 1 < ksteps) ptx::umma_bf16(d, ad + 2, bd + 2, idesc, 1u);
                if (q + 2 < ksteps) ptx::umma_bf16(d, ad + 4, bd + 4, idesc, 1u);
                if (q + 3 < ksteps) ptx::umma_bf16(d, ad + 6, bd + 6, idesc, 1u);
              }
              ptx::umma_commit(&tail->acc_full[i][b]);
              if (i == x.n_stat - 1) ptx::umma_commit(&tail->empty[s]);
              if (i == x.n_stat - 1 && t == x.s1 - 1) ptx::umma_commit(&tail->stat_empty[slot]);
            }
            __syncwarp();
          }
        }
      }
    }
    if (!ok) {
      if (ptx::elect_one()) ptx::umma_commit(&tail->drain);
      __syncwarp();
      for (int k = 0; k < (1 << 12) && !ptx::mbar_try_wait(&tail->drain, 0); ++k) {}
    }
  } else {
    // ------------------------------------------------------------------ read-out: thread = row of a stationary tile
    const int i = (warp - 2) >> 3;                                 // which stationary tile
    const int half = ((warp - 2) >> 2) & 1;                        // which 64 columns
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(i * 2 * kTile + half * 64);
    const uint64_t c2 = pack2(a.c, a.c);
    int it = 0, used = 0, units = 0;
    bool ok = true;
    for (uint32_t k = 0; ok && k * gridDim.x < a.units; ++k) {
      const uint32_t u = unit_of(k);
      if (u >= a.units) continue;
      const UnitInfo x = unit_info<kPass>(a, only, u);
      if (x.n_stat == 0) continue;
      const bool mine = i < x.n_stat;
      if (kPass == 1) {
        if (!mine) continue;
        const int tok0 = (x.stat0 + i) * a.tpt, token = tok0 + row / a.G;
        const bool holds = row < q_rows && token < x.nq;
        const int limit = holds ? x.n - (x.nq - 1 - token) : 0;    // keys this row sees
        const int all_see = x.n - (x.nq - 1 - tok0);               // keys every row of the tile sees
        float ref = -INFINITY, sum = 0.f;
        for (int t = x.s0; t < x.s1; ++t, ++used) {
          const int b = used & 1;
          ok = __all_sync(0xffffffffu, wait_or_abort(&tail->acc_full[i][b], (used >> 1) & 1, abort_flag));
          if (!ok) break;
          ptx::tc_fence_after_sync();
          uint32_t v[2][32];
          ptx::tmem_ld_32x32(lane_addr + (uint32_t)(b * kTile), v[0]);
          ptx::tmem_ld_32x32(lane_addr + (uint32_t)(b * kTile + 32), v[1]);
          ptx::tmem_wait_ld();
          ptx::tc_fence_before_sync();                             // accumulator drained
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->acc_empty[i][b]);
          if ((t + 1) * kTile > all_see) {
            const int k0 = t * kTile + half * 64;
#pragma unroll
            for (int j = 0; j < 64; ++j)
              if (k0 + j >= limit) v[j >> 5][j & 31] = 0xff800000u;
          }
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < 64; j += 2)
            m4[(j >> 1) & 3] = fmaxf(fmaxf(__uint_as_float(v[j >> 5][j & 31]), __uint_as_float(v[j >> 5][(j & 31) + 1])), m4[(j >> 1) & 3]);
          const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
          // the reference moves only when a logit passes it by 2^8: the sum stays far from overflow without it
          if (mx * a.c > ref + 8.f) {
            const float next = mx * a.c;
            sum *= exp2_fast(ref - next);                          // (ref = -inf: 0 * 0)
            ref = next;
          }
          const float off = ref == -INFINITY ? 0.f : -ref;
          const uint64_t off2 = pack2(off, off);
          uint64_t s2[2] = {0, 0};
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const uint32_t* q = &v[j >> 4][(2 * j) & 31];
            s2[j & 1] = add2(s2[j & 1], exp2_pair<kPoly>(j & 7, fma2(pack2(__uint_as_float(q[0]), __uint_as_float(q[1])), c2, off2)));
          }
          const float2 s = unpack2(add2(s2[0], s2[1]));
          sum += s.x + s.y;
        }
        if (!ok) break;
        // the row's two halves meet in shared memory
        if (half == 1) {
          ok = __all_sync(0xffffffffu, wait_or_abort(&tail->half_empty[i], (units & 1) ^ 1, abort_flag));
          half1_sm[i * kTile + row] = make_float2(ref, sum);
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->half_full[i]);
        } else {
          ok = __all_sync(0xffffffffu, wait_or_abort(&tail->half_full[i], units & 1, abort_flag));
          const float2 o = half1_sm[i * kTile + row];
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->half_empty[i]);
          const float top = fmaxf(ref, o.x);
          if (top != -INFINITY) sum = sum * exp2_fast(ref - top) + o.y * exp2_fast(o.x - top);
          const int64_t at = ((int64_t)x.h * a.q_tiles + x.q0 / a.tpt + x.r + x.stat0 + i) * kTile + row;
          if (a.chunks > 1) a.part[(int64_t)x.chunk * a.Hkv * a.q_tiles * kTile + at] = make_float2(top, sum);
          else a.lse2[at] = !holds || top == -INFINITY ? -INFINITY : -(top + log2f(sum));
        }
        ++units;
      } else {
        const int key = (x.stat0 + i) * kTile + row;
        const int shift = key - (x.n - x.nq);                      // the first token that sees this key
        const int last_shift = (x.stat0 + i + 1) * kTile - 1 - (x.n - x.nq);
        double sum = 0.0;
        for (int t = x.s0; t < x.s1; ++t, ++it) {
          const int l = it % kLseStages;
          ok = __all_sync(0xffffffffu, wait_or_abort(&tail->lse_full[l], (it / kLseStages) & 1, abort_flag));
          if (!ok) break;
          if (mine) {
            const int b = used & 1;
            ok = __all_sync(0xffffffffu, wait_or_abort(&tail->acc_full[i][b], (used >> 1) & 1, abort_flag));
            ++used;
            if (!ok) break;
            ptx::tc_fence_after_sync();
            uint32_t v[2][32];
            ptx::tmem_ld_32x32(lane_addr + (uint32_t)(b * kTile), v[0]);
            ptx::tmem_ld_32x32(lane_addr + (uint32_t)(b * kTile + 32), v[1]);
            ptx::tmem_wait_ld();
            ptx::tc_fence_before_sync();                           // accumulator drained
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&tail->acc_empty[i][b]);
            const int tok0 = t * a.tpt;
            // columns of tokens behind the request's last, or of tokens that do not see this key, do not count
            if (tok0 < last_shift || tok0 + a.tpt > x.nq) {
              const int j0 = (shift - tok0) * a.G - half * 64, j1 = min(a.tpt, x.nq - tok0) * a.G - half * 64;
#pragma unroll
              for (int j = 0; j < 64; ++j)
                if (j < j0 || j >= j1) v[j >> 5][j & 31] = 0xff800000u;
            }
            const ulonglong2* lse = reinterpret_cast<const ulonglong2*>(lse_sm + l * kTile + half * 64);
            uint64_t s2[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const ulonglong2 e = lse[j >> 1];
              const uint32_t* q = &v[j >> 4][(2 * j) & 31];
              s2[0] = add2(s2[0], exp2_pair<kPoly>(j & 7, fma2(pack2(__uint_as_float(q[0]), __uint_as_float(q[1])), c2, e.x)));
              s2[1] = add2(s2[1], exp2_pair<kPoly>((j & 7) + 1, fma2(pack2(__uint_as_float(q[2]), __uint_as_float(q[3])), c2, e.y)));
            }
            const float2 s = unpack2(add2(s2[0], s2[1]));
            sum += (double)(s.x + s.y);
          }
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->lse_empty[l]);
        }
        if (!ok) break;
        if (!mine) continue;
        if (half == 1) {
          ok = __all_sync(0xffffffffu, wait_or_abort(&tail->half_empty[i], (units & 1) ^ 1, abort_flag));
          half2_sm[i * kTile + row] = (float)sum;
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->half_full[i]);
        } else {
          ok = __all_sync(0xffffffffu, wait_or_abort(&tail->half_full[i], units & 1, abort_flag));
          sum += (double)half2_sm[i * kTile + row];
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->half_empty[i]);
          if (ok && key < x.n) {
            const int64_t slot = (int64_t)x.h * a.total + x.start + key;
            if (a.chunks > 1) a.part_sum[(int64_t)x.chunk * a.Hkv * a.total + slot] = (float)sum;
            else a.acc_out[slot] = (float)((a.acc ? (double)a.acc[slot] : 0.0) + sum);
          }
        }
        ++units;
      }
    }
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  if (threadIdx.x == 0 && tail->abort_flag) {
    atomicExch(&a.status[0], GVOTE_ERR_TIMEOUT);
    atomicExch(&a.status[1], 10 + kPass);
  }
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// lse2 of the query tiles' rows from the key chunks' (reference, sum) pairs, or from the caller's lse; eight lanes
// share a row's chunks, so that their loads are in flight together.
__global__ void __launch_bounds__(256)
accumulate_lse_kernel(const __grid_constant__ AccArgs a, const float* __restrict__ given) {
  const int h = blockIdx.y, lane = threadIdx.x & 7, row = (blockIdx.x & 3) * 32 + (threadIdx.x >> 3);
  const int64_t tile = blockIdx.x >> 2;
  const int r = a.batch == 1 ? 0 : find_request_div(a.cu_q, a.batch, tile, a.tpt);
  const int q0 = a.cu_q[r], nq = a.cu_q[r + 1] - q0;
  const int tok0 = (int)(tile - (q0 / a.tpt + r)) * a.tpt, token = tok0 + row / a.G;
  ptx::let_next_begin();
  ptx::wait_for_previous();
  if (tok0 < 0 || tok0 >= nq) return;
  const bool holds = row < a.G * a.tpt && token < nq;
  const int64_t at = ((int64_t)h * a.q_tiles + tile) * kTile + row;
  float out = -INFINITY;
  if (given) {
    const float l = holds ? given[(int64_t)(q0 + token) * a.Hkv * a.G + h * a.G + row % a.G] : -INFINITY;
    out = l == -INFINITY ? -INFINITY : -l * kLog2e;
  } else {
    const int64_t pitch = (int64_t)a.Hkv * a.q_tiles * kTile;
    float ref = -INFINITY, sum = 0.f;
    for (int x = lane; x < a.chunks; x += 8) {
      const float2 p = a.part[x * pitch + at];
      const float top = fmaxf(ref, p.x);
      if (top != -INFINITY) sum = sum * exp2_fast(ref - top) + p.y * exp2_fast(p.x - top);
      ref = top;
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
      const float r2 = __shfl_xor_sync(0xffffffffu, ref, o), s2 = __shfl_xor_sync(0xffffffffu, sum, o);
      const float top = fmaxf(ref, r2);
      if (top != -INFINITY) sum = sum * exp2_fast(ref - top) + s2 * exp2_fast(r2 - top);
      ref = top;
    }
    if (holds && ref != -INFINITY) out = -(ref + log2f(sum));
  }
  if (lane == 0) a.lse2[at] = out;
}

// The chunks' partial sums of pass 2, in order.
__global__ void __launch_bounds__(256)
accumulate_sum_kernel(const __grid_constant__ AccArgs a) {
  const int h = blockIdx.y, r = a.batch == 1 ? 0 : find_request_by(a.cu, a.batch, blockIdx.x, 8);
  const int start = a.cu[r], n = valid_keys(a.kv_len, r, a.Hkv, h, a.cu[r + 1] - start);
  const int key = (int)(blockIdx.x - ((start >> 8) + r)) * 256 + threadIdx.x;
  ptx::wait_for_previous();
  if (key < 0 || key >= n) return;
  const int64_t slot = (int64_t)h * a.total + start + key;
  double sum = a.acc ? (double)a.acc[slot] : 0.0;
  for (int x = 0; x < a.chunks; ++x) sum += (double)a.part_sum[(int64_t)x * a.Hkv * a.total + slot];
  a.acc_out[slot] = (float)sum;
}

// Tokens of a query tile: as many as 128 rows hold, fewer where the longest request's tokens can then be dealt out evenly
// (32 tokens of 7 heads are two tiles of 16 rather than 18 and 14: the last tile needs no mask).  Not where the list holds more
// tokens than the batch can have (requests behind others, by a view of the boundaries): there is a tile for each of them.
int tile_tokens(const gvote_params* p, int32_t batch, int64_t total_q, int64_t max_q) {
  const int64_t most = kTile / (p->n_q_heads / p->n_kv_heads);
  if (max_q <= 0 || total_q > batch * max_q) return (int)most;
  return (int)ceil_div(max_q, ceil_div(max_q, most));
}

// Entries of a list with one entry per `per` tokens begun of every request (request r from cu[r] / per + r on): an upper bound
// for a batch, which does not know its lengths on the host, exact for one request.
int64_t list_length(int64_t total, int64_t per, int32_t batch) { return batch == 1 ? ceil_div(total, per) : total / per + batch; }

// Chunks a pass splits its units' streams into, no more than the longest stream has tiles.  Streams of uneven length:
// about kUnitsPerSm units per SM, which the rounds even out.  Even ones (a window of few tokens): one unit per SM.
int64_t chunk_count(int64_t units, int64_t tiles, bool even) {
  if (units < 1) units = 1;
  const int64_t want = even ? kSms / units : ceil_div((int64_t)kUnitsPerSm * kSms, units);
  return want < 1 ? 1 : want < tiles ? want : (tiles > 0 ? tiles : 1);
}

}  // namespace

AccumulateMap accumulate_map(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N, int64_t total_q,
                             int64_t max_q) {
  AccumulateMap m;
  m.tpt = tile_tokens(p, batch, total_q, max_q);
  const int64_t tpt = m.tpt;
  m.q_tiles = list_length(total_q, tpt, batch);
  m.key_chunks = chunk_count(list_length(total_q, 2 * tpt, batch) * p->n_kv_heads, ceil_div(max_N, kTile),
                             batch == 1 && max_q <= max_N / 8);
  m.q_chunks = chunk_count(list_length(total_tokens, 2 * kTile, batch) * p->n_kv_heads, ceil_div(max_q, tpt), false);
  m.lse = kStatusBytes;
  const size_t rows = (size_t)p->n_kv_heads * m.q_tiles * kTile;
  m.part = align_up(m.lse + rows * 4, 256);
  const size_t p1 = m.key_chunks > 1 ? rows * m.key_chunks * 8 : 0;
  const size_t p2 = m.q_chunks > 1 ? (size_t)p->n_kv_heads * total_tokens * m.q_chunks * 4 : 0;
  m.total = align_up(m.part + (p1 > p2 ? p1 : p2), 256);
  return m;
}

// What any call of no larger sizes needs.  A smaller one may be cut into more chunks: the units of a pass with chunks are no
// more than those without and kUnitsPerSm per SM besides, of two tiles each (of two at most: as many pairs as units are
// listed, ceil(n / 2) pairs for n tiles).
size_t accumulate_workspace(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t total_q) {
  const int64_t most = kTile / (p->n_q_heads / p->n_kv_heads), Hkv = p->n_kv_heads, units = kUnitsPerSm * kSms;
  // a tile holds half of what it could at least, or a request's every token and there are two tiles a request at most
  const int64_t rows = Hkv * (2 * total_q / most + 2 * (int64_t)batch + 2) * kTile;
  const int64_t p1 = (units * 2 * kTile + 2 * rows) * 8, p2 = (units * 2 * kTile + 2 * Hkv * total_tokens) * 4;
  return kStatusBytes + (size_t)rows * 4 + (size_t)(p1 > p2 ? p1 : p2) + 1024;
}

int32_t launch_accumulate(const gvote_params* p, const __nv_bfloat16* Q, int64_t q_tok, int64_t q_head,
                          const int32_t* cu_q, int64_t total_q, int64_t max_q, const __nv_bfloat16* K, int64_t k_tok,
                          int64_t k_head, const int32_t* cu, const int32_t* kv_len, int32_t batch, int64_t total_tokens,
                          int64_t max_N, const float* lse, const float* acc, float* acc_out, char* ws, cudaStream_t st) {
  if (max_N == 0) return GVOTE_OK;
  const AccumulateMap m = accumulate_map(p, batch, total_tokens, max_N, total_q, max_q);
  AccArgs a;
  a.cu_q = cu_q; a.cu = cu; a.kv_len = kv_len;
  a.lse2 = (float*)(ws + m.lse); a.part = (float2*)(ws + m.part); a.part_sum = (float*)(ws + m.part);
  a.acc = acc; a.acc_out = acc_out; a.status = (int32_t*)ws; a.total = total_tokens;
  a.Hkv = p->n_kv_heads; a.G = p->n_q_heads / p->n_kv_heads; a.batch = batch; a.d_k = p->d_k; a.tpt = m.tpt;
  a.q_tiles = m.q_tiles;
  a.c = (float)(1.4426950408889634 / sqrt((double)p->d_k));
  a.boxes = (p->d_k + 63) / 64;
  // 227 KB: two slots of two stationary tiles and a ring of at least two tiles where they fit (d_k <= 128)
  const size_t tile = (size_t)a.boxes * kTile * 128, rest = kSideFloats * 4 + sizeof(Tail);
  a.stat_slots = a.boxes <= 2 ? 2 : 1;
  const size_t room = 227 * 1024 - rest - a.stat_slots * 2 * tile;
  a.stages = (int)(room / tile < kMaxStages ? room / tile : kMaxStages);
  const size_t smem = rest + (a.stat_slots * 2 + a.stages) * tile;

  CUtensorMap tmK, tmQ;
  {
    const uint64_t dims[3] = {(uint64_t)p->d_k, (uint64_t)total_tokens, (uint64_t)a.Hkv};
    const uint64_t strides[2] = {(uint64_t)k_tok * 2, (uint64_t)(a.Hkv > 1 ? k_head : k_tok) * 2};
    const uint32_t box[3] = {64, (uint32_t)kTile, 1};
    if (!encode_tensor_map_bf16(&tmK, K, 3, dims, strides, box)) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  }
  {
    const uint64_t dims[3] = {(uint64_t)p->d_k, (uint64_t)p->n_q_heads, (uint64_t)total_q};
    const uint64_t strides[2] = {(uint64_t)q_head * 2, (uint64_t)(total_q > 1 ? q_tok : q_head) * 2};
    const uint32_t box[3] = {64, (uint32_t)a.G, (uint32_t)a.tpt};
    if (!encode_tensor_map_bf16(&tmQ, Q, 3, dims, strides, box)) return GVOTE_ERR_UNSUPPORTED_SHAPE;
  }
  a.chunks = 1;
  if (!lse) {
    a.pairs = (uint32_t)list_length(total_q, 2 * a.tpt, batch);
    a.chunks = (int)m.key_chunks;
    a.units = a.pairs * a.Hkv * a.chunks;
    GVOTE_CUDA_CHECK(cudaFuncSetAttribute(accumulate_umma_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    LaunchScope scope_("accumulate_lse_umma_kernel", st);
    launch_on(accumulate_umma_kernel<1>, dim3((unsigned)(a.units < kSms ? a.units : kSms)), dim3(kAccThreads), smem, st,
              tmQ, tmK, a);
    GVOTE_LAUNCH_CHECK("accumulate_lse_umma_kernel");
  }
  if (lse || a.chunks > 1) {
    LaunchScope scope_("accumulate_lse_kernel", st);
    if (lse) launch_on(accumulate_lse_kernel, dim3((unsigned)(4 * a.q_tiles), a.Hkv), dim3(256), 0, st, a, lse);
    else launch_behind(accumulate_lse_kernel, dim3((unsigned)(4 * a.q_tiles), a.Hkv), dim3(256), 0, st, a, lse);
    GVOTE_LAUNCH_CHECK("accumulate_lse_kernel");
  }
  a.pairs = (uint32_t)list_length(total_tokens, 2 * kTile, batch);
  a.chunks = (int)m.q_chunks;
  a.units = a.pairs * a.Hkv * a.chunks;
  GVOTE_CUDA_CHECK(cudaFuncSetAttribute(accumulate_umma_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  {
    LaunchScope scope_("accumulate_weights_umma_kernel", st);
    launch_behind(accumulate_umma_kernel<2>, dim3((unsigned)(a.units < kSms ? a.units : kSms)), dim3(kAccThreads), smem, st, tmQ,
              tmK, a);
  }
  GVOTE_LAUNCH_CHECK("accumulate_weights_umma_kernel");
  if (a.chunks > 1) {
    LaunchScope scope_("accumulate_sum_kernel", st);
    launch_behind(accumulate_sum_kernel, dim3((unsigned)a.pairs, a.Hkv), dim3(256), 0, st, a);
    GVOTE_LAUNCH_CHECK("accumulate_sum_kernel");
  }
  return GVOTE_OK;
}

}  // namespace gvote
