// Attention of a few query tokens over the 8-bit cache (gvote_attend8).
//
//   l_n = (q.k_n) / sqrt(d_k),  out = sum_n exp(l_n - lse) v_n,  lse = log sum_n exp(l_n),
// with k_n, v_n = code * scale of the row's block.  A few rows of queries against long K and V: bound by reading the codes
// once, 2 d_k bytes per cached row.
//
// Split.  The rows of all (request, KV head) pairs ("entries") are cut into tiles of 32 and laid end to end; CTA b of the
// grid takes tiles T b / grid .. T (b + 1) / grid - 1, whatever entries they belong to.  So pruned heads of very
// different length load every SM alike, without knowing the lengths on the host: each CTA adds up the entries' tiles
// itself.  What a CTA has of one entry is a segment; its result (maximum, sum, output) goes to slot entry + CTA, or
// straight to the output when the entry lies within one CTA.  attend8_finish_kernel merges an entry's segments.
//
// Inside a CTA, warps work on their own: warp (kw, rw) takes every KW-th tile for 8 RT query rows.  A tile comes by TMA
// (128-byte swizzle) into the kw-th ring of shared memory, its two scales by 4-byte asynchronous copies; the ring has
// 8 KB per tile and 128 KB or more in all, which keeps well over the 40 KB in flight that an SM's share of
// the bandwidth times the latency asks for.  The products run on mma.sync (m16n8k16, half precision in, 32-bit sums): a
// tile has at most 16 query rows per warp, a sixteenth of what the fifth-generation tensor cores' smallest shape
// would want, and the codes have to be widened in registers anyway.  An e4m3 code is exactly a half; the two
// products are
//   S^T [16 keys x 8 rows] = K Q^T      a thread's share of a key is 32 consecutive bytes (the order of the channels in a
//                                       contraction is free, so Q is permuted alike)
//   O^T [16 channels x 8 rows] = V^T P^T   two keys' bytes of one channel are paired by a byte permute before they are
//                                       widened: no transposition in shared memory; S^T becomes P^T by movmatrix
// The scale of K enters the logit, the scale of V the sum of a tile: every tile is summed against its own maximum and added
// in 32 bits, so that neither a half's range nor another block's scale costs digits of a row with little weight.
// Q is scaled by a power of two per row to use the half's range (exact down to 2^-31 of the row's largest entry).  Weights
// are rounded to half precision (2^-11) before the second product; out is rounded once, to bf16.
//
// Weights for the eviction: the logits are kept (4 bytes per row and query, against 2 d_k per row), and the finishing
// kernel turns them into weights once lse is known; a slot belongs to one thread, so the sum has one order.
//
// Every wait is bounded; when one runs out GVOTE_ERR_TIMEOUT is recorded and the outputs are not to be used.
#include <type_traits>

#include "cache8.cuh"
#include "ptx.cuh"

namespace gvote {
namespace {

constexpr int kTileKeys = 32;
constexpr int kMaxEntries = 1024;      // entries per launch: their tiles are added up in shared memory
constexpr int kMaxRings = 8;
constexpr int kMaxStages = 6;
constexpr int kSms = 148;
constexpr float kLog2e = 1.4426950408889634f;

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
  float* part_o;         // [row groups][entries + CTAs][rows of a group][d_k]
  float2* part_ml;       // [row groups][entries + CTAs][rows of a group]  (maximum, sum), base 2
  int2* info;            // [row groups][entries]  first and last CTA of the entry (-1: no rows)
  float* logits;         // [Hkv][max_q * G][total] base 2, when acc_out
  int32_t* status;
  int Hkv, G, r0, batch, d_k, max_q;   // requests r0 .. r0 + batch - 1
  int rings, row_warps, stages, group_rows;
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
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// The same with a zero accumulator.
__device__ __forceinline__ void mma_16816_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                               uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// d = part * f + d * g on pairs of 32-bit floats.
__device__ __forceinline__ void scale_add2(float& d0, float& d1, float p0, float p1, uint64_t f, uint64_t g) {
  asm("{\n\t.reg .b64 d, p;\n\tmov.b64 d, {%0, %1};\n\tmov.b64 p, {%2, %3};\n\tmul.rn.f32x2 d, d, %5;\n\t"
      "fma.rn.f32x2 d, p, %4, d;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "+f"(d0), "+f"(d1)
      : "f"(p0), "f"(p1), "l"(f), "l"(g));
}
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
// Two halves: 1 where the code is the NaN code, else 0.
__device__ __forceinline__ uint32_t nan_flags(uint32_t c) {
  return ((c & 0x7fu) == 0x7fu ? 0x3c00u : 0u) | ((c & 0x7f00u) == 0x7f00u ? 0x3c000000u : 0u);
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t h;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(hi), "f"(lo));
  return h;
}

template <int kBoxes, int kRt>      // 128-byte boxes per row; tiles of 8 query rows per warp
__global__ void __launch_bounds__(256, 1)
attend8_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
               const __grid_constant__ AttendArgs a) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr int kBoxBytes = kTileKeys * 128, kStageBytes = 2 * kBoxes * kBoxBytes;
  constexpr int kPitch = kBoxes * 128 + 4;                            // floats per row of the merge area
  const int warps = a.rings * a.row_warps;
  uint8_t* ring_sm = smem;                                            // [ring][stage][K boxes, V boxes]
  float* merge_sm = reinterpret_cast<float*>(ring_sm + (size_t)a.rings * a.stages * kStageBytes);   // [warp][8][kPitch]
  float2* ml_sm = reinterpret_cast<float2*>(merge_sm + (size_t)warps * 8 * kPitch);                  // [warp][8 kRt]
  float2* scale_sm = ml_sm + warps * 8 * kRt;                         // [ring][stage] (k, v)
  uint64_t* full = reinterpret_cast<uint64_t*>(scale_sm + kMaxRings * kMaxStages);                   // [ring][stage]
  uint64_t* empty = full + kMaxRings * kMaxStages;
  int* pref = reinterpret_cast<int*>(empty + kMaxRings * kMaxStages);  // [entries + 1] tiles before each entry
  int* warp_tot = pref + kMaxEntries + 1;                              // [8], then one flag
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = warps * 32;
  const int kw = warp % a.rings, rw = warp / a.rings;
  const int entries = a.batch * a.Hkv;
  const int group0 = blockIdx.y * a.group_rows;                        // first query row of this group

  if (tid < a.rings * a.stages) {
    const int slot = (tid / a.stages) * kMaxStages + tid % a.stages;
    ptx::mbar_init(&full[slot], 2);
    ptx::mbar_init(&empty[slot], a.row_warps);
    ptx::fence_barrier_init();
  }
  if (tid == 0) {
    ptx::prefetch_tensormap(&tmK);
    ptx::prefetch_tensormap(&tmV);
  }
  // ---- tiles before each entry
  {
    const int per = (entries + threads - 1) / threads;                 // consecutive entries per thread
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
    if (lane == 31) warp_tot[warp] = inc;
    __syncthreads();
    int run = inc - mine;
    for (int w = 0; w < warp; ++w) run += warp_tot[w];
    for (int e = e0; e < e1; ++e) { run += pref[e + 1]; pref[e + 1] = run; }
    if (tid == 0) pref[0] = 0;
    __syncthreads();
  }
  const int T = pref[entries], B = gridDim.x, b = blockIdx.x;
  const int t0 = (int)((int64_t)T * b / B), t1 = (int)((int64_t)T * (b + 1) / B);
  // which CTAs hold an entry: the CTA of tile t is the largest c with T c / B <= t
  int2* info = a.info + (int64_t)blockIdx.y * entries;
  if (b == 0) {
    for (int e = tid; e < entries; e += threads) {
      const int f = pref[e], l = pref[e + 1] - 1;
      int2 v = make_int2(-1, -1);
      if (l >= f) v = make_int2((int)((((int64_t)f + 1) * B - 1) / T), (int)((((int64_t)l + 1) * B - 1) / T));
      info[e] = v;
    }
  }
  if (t0 >= t1) return;
  int e_first = 0;                                                     // the entry of tile t0
  {
    int hi = entries - 1;
    while (e_first < hi) {
      const int mid = (e_first + hi) >> 1;
      if (pref[mid + 1] <= t0) e_first = mid + 1; else hi = mid;
    }
  }

  // ---- the ring: one lane of row warp 0 asks for the tiles of its ring, in order, across entries
  uint64_t* my_full = full + kw * kMaxStages;
  uint64_t* my_empty = empty + kw * kMaxStages;
  uint8_t* my_ring = ring_sm + (size_t)kw * a.stages * kStageBytes;
  float2* my_scale = scale_sm + kw * kMaxStages;
  int ask_t = t0 + kw, ask_e = e_first, asked = 0;
  bool ok = true;
  auto ask = [&]() {                                                   // (one lane)
    while (ask_t >= pref[ask_e + 1]) ++ask_e;
    const int lr = ask_e / a.Hkv, h = ask_e - lr * a.Hkv, r = a.r0 + lr;
    const int start = a.cu[r], key0 = (ask_t - pref[ask_e]) * kTileKeys;
    const int s = asked % a.stages;
    uint8_t* dst = my_ring + (size_t)s * kStageBytes;
    ptx::mbar_arrive_expect_tx(&my_full[s], kStageBytes);
#pragma unroll
    for (int x = 0; x < kBoxes; ++x) {
      ptx::tma_load_3d(dst + x * kBoxBytes, &tmK, &my_full[s], x * 128, start + key0, h);
      ptx::tma_load_3d(dst + (kBoxes + x) * kBoxBytes, &tmV, &my_full[s], x * 128, start + key0, h);
    }
    const int64_t sb = (int64_t)h * a.row_blocks + block8_offset(start, r) + (key0 >> 6);
    ptx::cp_async_4(&my_scale[s].x, a.k_scale + sb);
    ptx::cp_async_4(&my_scale[s].y, a.v_scale + sb);
    ptx::cp_async_arrive(&my_full[s]);
    ask_t += a.rings;
    ++asked;
  };
  auto agree = [&]() {                                                 // the warp follows the asking lane's counters
    asked = __shfl_sync(0xffffffffu, asked, 0);
    ask_t = __shfl_sync(0xffffffffu, ask_t, 0);
  };
  if (rw == 0 && lane == 0)
    while (asked < a.stages && ask_t < t1) ask();
  agree();

  const int j8 = lane >> 2, c4 = lane & 3;                             // a lane's place in the mma fragments
  int used = 0, t = t0 + kw;
  for (int e = e_first; e < entries && pref[e] < t1; ++e) {
    if (pref[e + 1] <= t0 || pref[e + 1] == pref[e]) continue;
    const Entry x = entry_of(a, e);
    const int rows = x.nq * a.G, row0 = group0 + rw * 8 * kRt;
    // ---- this warp's query rows as halves, scaled by a power of two per row
    uint32_t q[kRt][kBoxes * 8][2];
    float factor[kRt][2];                                              // of the thread's two rows: logit per unit of product
    int limit[kRt][2];                                                 // rows of the cache they see
#pragma unroll
    for (int rt = 0; rt < kRt; ++rt) {
      const int row = row0 + rt * 8 + j8;
      const bool holds = row < rows;
      const __nv_bfloat16* src = a.Q + (int64_t)(x.q0 + (holds ? row / a.G : 0)) * a.q_tok + (int64_t)(x.h * a.G + (holds ? row % a.G : 0)) * a.q_head;
      uint32_t v[kBoxes][16];
      uint32_t top = 0;                                                // the largest magnitude's bits
#pragma unroll
      for (int y = 0; y < kBoxes; ++y)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int d = y * 128 + c4 * 32 + k * 8;
          uint4 w = make_uint4(0, 0, 0, 0);
          if (holds && d < a.d_k) w = *reinterpret_cast<const uint4*>(src + d);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t u = (&w.x)[i];
            v[y][k * 4 + i] = u;
            top = max(top, max(u & 0x7fffu, (u >> 16) & 0x7fffu));
          }
        }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // entries up to 2^15: multiply by 2^(14 - exponent); the exponent is kept where both factors are normal numbers
      const int ex = min(max((int)(top >> 7) - 127, -100), 127);
      const float up = __uint_as_float((uint32_t)(127 + 14 - ex) << 23);
#pragma unroll
      for (int y = 0; y < kBoxes; ++y)
#pragma unroll
        for (int s = 0; s < 16; ++s)
          q[rt][y * 8 + (s >> 1)][s & 1] = pack_half2(__uint_as_float(v[y][s] << 16) * up, __uint_as_float(v[y][s] & 0xffff0000u) * up);
      const float down = __uint_as_float((uint32_t)(127 - 14 + ex) << 23) * a.scale2;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        factor[rt][i] = __shfl_sync(0xffffffffu, down, (2 * c4 + i) * 4);
        limit[rt][i] = x.n - (x.nq - 1 - (row0 + rt * 8 + 2 * c4 + i) / a.G);
      }
    }
    const int all_see = x.n - (x.nq - 1);                              // rows every query token sees

    float o[kRt][kBoxes * 8][4];
    float m[kRt][2], l[kRt][2];
#pragma unroll
    for (int rt = 0; rt < kRt; ++rt) {
#pragma unroll
      for (int i = 0; i < 2; ++i) { m[rt][i] = -INFINITY; l[rt][i] = 0.f; }
#pragma unroll
      for (int k = 0; k < kBoxes * 8; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[rt][k][i] = 0.f;
    }
    const int seg1 = min(t1, pref[e + 1]);
    for (; t < seg1; t += a.rings, ++used) {
      const int s = used % a.stages;
      ok = ok && __all_sync(0xffffffffu, ptx::mbar_wait(&my_full[s], (used / a.stages) & 1, 1u << 22));
      // One tile.  kEdge: some row does not see all of it, or it reaches behind the last row (kept apart: the tests of
      // the edge would cost every tile as many instructions again).
      auto tile = [&](auto edge_tag) {
        constexpr bool kEdge = decltype(edge_tag)::value;
        const uint8_t* kt = my_ring + (size_t)s * kStageBytes;
        const uint8_t* vt = kt + kBoxes * kBoxBytes;
        const float2 sc = my_scale[s];
        const int key0 = (t - pref[e]) * kTileKeys;
        // ---- S^T: thread holds keys mt * 16 + j8 (+ 8), rows 2 c4, 2 c4 + 1
        float sT[kRt][2][4];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
          for (int y = 0; y < kBoxes; ++y) {
            uint4 ka[2], kb[2];                                        // 32 bytes of keys j8 and j8 + 8
            const uint8_t* ra = kt + y * kBoxBytes + (mt * 16 + j8) * 128;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int at = ((2 * c4 + k) ^ j8) << 4;                 // (rows j8 and j8 + 8 swizzle alike)
              ka[k] = *reinterpret_cast<const uint4*>(ra + at);
              kb[k] = *reinterpret_cast<const uint4*>(ra + 8 * 128 + at);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const uint32_t wa = (&ka[k >> 2].x)[k & 3], wb = (&kb[k >> 2].x)[k & 3];
              uint32_t a0, a1, a2, a3;
              widen8x4(wa, a0, a2);
              widen8x4(wb, a1, a3);
#pragma unroll
              for (int rt = 0; rt < kRt; ++rt) {
                if (y == 0 && k == 0) mma_16816_zero(sT[rt][mt], a0, a1, a2, a3, q[rt][0][0], q[rt][0][1]);
                else mma_16816(sT[rt][mt], a0, a1, a2, a3, q[rt][y * 8 + k][0], q[rt][y * 8 + k][1]);
              }
            }
          }
        }
        uint32_t p[kRt][2][2];
        uint64_t f_old[kRt], f_new[kRt];                               // factors of the sum so far and of this tile's
#pragma unroll
        for (int rt = 0; rt < kRt; ++rt) {
          float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float v = sT[rt][mt][i] * (sc.x * factor[rt][i & 1]);
              if (kEdge && key0 + mt * 16 + j8 + (i >> 1) * 8 >= limit[rt][i & 1]) v = -INFINITY;
              sT[rt][mt][i] = v;
              top[i & 1] = fmaxf(top[i & 1], v);
            }
          if (a.logits) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int row = row0 + rt * 8 + 2 * c4 + (i & 1);
              if (row < rows) {
                float* dst = a.logits + ((int64_t)x.h * a.max_q * a.G + row) * a.total + x.start;
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                  const int key = key0 + mt * 16 + j8 + (i >> 1) * 8;
                  if (key < x.n) dst[key] = sT[rt][mt][i];
                }
              }
            }
          }
          float ref[2], a_old[2], a_new[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int k = 4; k < 32; k <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], k));
            const float next = fmaxf(m[rt][i], top[i]);
            ref[i] = top[i] == -INFINITY ? 0.f : top[i];
            a_old[i] = next == -INFINITY ? 0.f : exp2_fast(m[rt][i] - next);
            a_new[i] = next == -INFINITY ? 0.f : exp2_fast(top[i] - next);
            m[rt][i] = next;
          }
          float add[2] = {0.f, 0.f};
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              w[i] = exp2_fast(sT[rt][mt][i] - ref[i & 1]);
              add[i & 1] += w[i];
            }
            p[rt][mt][0] = transpose_8x8(pack_half2(w[0], w[1]));
            p[rt][mt][1] = transpose_8x8(pack_half2(w[2], w[3]));
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) l[rt][i] = l[rt][i] * a_old[i] + add[i] * a_new[i];
          f_old[rt] = pack2(a_old[0], a_old[1]);
          f_new[rt] = pack2(a_new[0] * sc.y, a_new[1] * sc.y);
        }
        // ---- O^T: thread's 16 channels 16 j8 .. of every 128, keys 2 c4, 2 c4 + 1 (+ 8) of each 16
#pragma unroll
        for (int y = 0; y < kBoxes; ++y) {
          uint4 v[2][4];
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int key = mt * 16 + 2 * c4 + (k & 1) + (k >> 1) * 8;
              v[mt][k] = *reinterpret_cast<const uint4*>(vt + y * kBoxBytes + key * 128 + ((j8 ^ (key & 7)) << 4));
              if (kEdge && key0 + key >= x.n) v[mt][k] = make_uint4(0, 0, 0, 0);     // behind the last row: anything
            }
          bool nan_seen = false;
          if (kEdge && x.nq > 1) {
            // A NaN in a row that some of the tokens do not see must not reach them through a weight of zero: it is
            // taken out of the product here and counted for the tokens that see it below.
            bool any = false;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
              for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int w = 0; w < 4; ++w) any |= __vcmpeq4((&v[mt][k].x)[w] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
            nan_seen = __any_sync(0xffffffffu, any);
          }
#pragma unroll
          for (int w = 0; w < 4; ++w) {                                // m-tiles 2 w, 2 w + 1
            float part[kRt][2][4];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
              uint32_t w0 = (&v[mt][0].x)[w], w1 = (&v[mt][1].x)[w], w2 = (&v[mt][2].x)[w], w3 = (&v[mt][3].x)[w];
              if (kEdge && nan_seen) {
                auto clean = [](uint32_t u) { return u & ~__vcmpeq4(u & 0x7f7f7f7fu, 0x7f7f7f7fu); };
                w0 = clean(w0); w1 = clean(w1); w2 = clean(w2); w3 = clean(w3);
              }
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const uint32_t lo = __byte_perm(w0, w1, i ? 0x7362 : 0x5140), hi = __byte_perm(w2, w3, i ? 0x7362 : 0x5140);
                uint32_t a0, a1, a2, a3;
                widen8x4(lo, a0, a1);
                widen8x4(hi, a2, a3);
#pragma unroll
                for (int rt = 0; rt < kRt; ++rt) {
                  if (mt == 0) mma_16816_zero(part[rt][i], a0, a1, a2, a3, p[rt][0][0], p[rt][0][1]);
                  else mma_16816(part[rt][i], a0, a1, a2, a3, p[rt][1][0], p[rt][1][1]);
                }
              }
            }
#pragma unroll
            for (int rt = 0; rt < kRt; ++rt)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                float (&d)[4] = o[rt][y * 8 + 2 * w + i];
                scale_add2(d[0], d[1], part[rt][i][0], part[rt][i][1], f_new[rt], f_old[rt]);
                scale_add2(d[2], d[3], part[rt][i][2], part[rt][i][3], f_new[rt], f_old[rt]);
              }
          }
          if (kEdge && nan_seen) {
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
              for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int rt = 0; rt < kRt; ++rt) {
                  float count[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                  for (int mt = 0; mt < 2; ++mt) {
                    const uint32_t lo = __byte_perm((&v[mt][0].x)[w], (&v[mt][1].x)[w], i ? 0x7362 : 0x5140);
                    const uint32_t hi = __byte_perm((&v[mt][2].x)[w], (&v[mt][3].x)[w], i ? 0x7362 : 0x5140);
                    uint32_t see[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                      const int key = key0 + mt * 16 + u * 8 + j8;
                      see[u] = transpose_8x8((key < limit[rt][0] ? 0x3c00u : 0u) | (key < limit[rt][1] ? 0x3c000000u : 0u));
                    }
                    mma_16816(count, nan_flags(lo), nan_flags(lo >> 16), nan_flags(hi), nan_flags(hi >> 16), see[0], see[1]);
                  }
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    if (count[k] > 0.f) o[rt][y * 8 + 2 * w + i][k] = __uint_as_float(0x7fffffffu);
                }
          }
        }
      };
      if (ok && row0 < rows) {
        if ((t - pref[e]) * kTileKeys + kTileKeys > all_see) tile(std::true_type{}); else tile(std::false_type{});
      }
      // ---- the slot is free; row warp 0 asks for the ring's next tile
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&my_empty[s]);
      if (rw == 0) {
        // with several row warps, of the tile before: the others need not have finished this one yet
        const int done = a.row_warps > 1 ? used - 1 : used;
        if (ok && done >= 0 && ask_t < t1 && asked == done + a.stages) {
          ok = __all_sync(0xffffffffu, ptx::mbar_wait(&my_empty[done % a.stages], (done / a.stages) & 1, 1u << 22));
          if (ok && lane == 0) ask();
        }
        agree();
      }
    }

    // ---- merge the rings' results of this segment
    const bool whole = pref[e] >= t0 && pref[e + 1] <= t1;             // the entry lies within this CTA
    const int64_t slot = ((int64_t)blockIdx.y * (entries + B) + e + b) * a.group_rows;
#pragma unroll
    for (int rt = 0; rt < kRt; ++rt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) l[rt][i] += __shfl_xor_sync(0xffffffffu, l[rt][i], k);
        if (j8 == 0) ml_sm[warp * 8 * kRt + rt * 8 + 2 * c4 + i] = make_float2(m[rt][i], l[rt][i]);
      }
#pragma unroll
    for (int rt = 0; rt < kRt; ++rt) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float* dst = merge_sm + (size_t)(warp * 8 + 2 * c4 + i) * kPitch + j8 * 16;
#pragma unroll
        for (int y = 0; y < kBoxes; ++y)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            *reinterpret_cast<float4*>(dst + y * 128 + k * 4) = make_float4(o[rt][y * 8 + 2 * k][i], o[rt][y * 8 + 2 * k][2 + i],
                                                                            o[rt][y * 8 + 2 * k + 1][i], o[rt][y * 8 + 2 * k + 1][2 + i]);
      }
      __syncthreads();
      // thread = four channels of one row
      const int quads = a.d_k >> 2;
      for (int u = tid; u < a.row_warps * 8 * quads; u += threads) {
        const int row_in = u / quads, d = (u - row_in * quads) * 4, w = row_in >> 3, row8 = row_in & 7;
        const int in_group = w * 8 * kRt + rt * 8 + row8, row = group0 + in_group;
        if (row < rows) {
          float M = -INFINITY, L = 0.f;
          for (int k = 0; k < a.rings; ++k) M = fmaxf(M, ml_sm[(w * a.rings + k) * 8 * kRt + rt * 8 + row8].x);
          float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int k = 0; k < a.rings; ++k) {
            const float2 ml = ml_sm[(w * a.rings + k) * 8 * kRt + rt * 8 + row8];
            if (ml.x == -INFINITY && ml.y == 0.f) continue;
            const float f = exp2_fast(ml.x - M);
            const float4 v = *reinterpret_cast<const float4*>(merge_sm + (size_t)((w * a.rings + k) * 8 + row8) * kPitch + d);
            L = fmaf(f, ml.y, L);
            s.x = fmaf(f, v.x, s.x); s.y = fmaf(f, v.y, s.y); s.z = fmaf(f, v.z, s.z); s.w = fmaf(f, v.w, s.w);
          }
          if (d == 0) a.part_ml[slot + in_group] = make_float2(M, L);
          if (whole) {
            const int token = row / a.G, g = x.h * a.G + row % a.G;
            const float inv = M == -INFINITY && L == 0.f ? 0.f : 1.f / L;
            __nv_bfloat162 out[2] = {__floats2bfloat162_rn(s.x * inv, s.y * inv), __floats2bfloat162_rn(s.z * inv, s.w * inv)};
            *reinterpret_cast<uint2*>(a.out + (int64_t)(x.q0 + token) * a.o_tok + (int64_t)g * a.o_head + d) = *reinterpret_cast<uint2*>(out);
            if (d == 0 && a.lse)
              a.lse[(int64_t)(x.q0 + token) * a.Hkv * a.G + g] = M == -INFINITY ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
          } else {
            *reinterpret_cast<float4*>(a.part_o + (slot + in_group) * a.d_k + d) = s;
          }
        }
      }
      __syncthreads();
    }
  }
  if (!ok && lane == 0) { atomicExch(&a.status[0], GVOTE_ERR_TIMEOUT); atomicExch(&a.status[1], 13); }
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
          const float m = a.part_ml[slot].x;
          const float4 p = *reinterpret_cast<const float4*>(a.part_o + slot * a.d_k + q * 4);
          const float f = m == -INFINITY ? 0.f : exp2_fast(m - ml.x);
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

// How a launch is cut: query rows per warp and per group, rings of tiles, CTAs.
struct Cut { int boxes, rt, row_warps, rings, stages, group_rows, groups, requests; size_t smem; int64_t ctas; };
Cut cut_of(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_q) {
  Cut c;
  const int64_t rows = max_q * (p->n_q_heads / p->n_kv_heads);
  c.boxes = p->d_k <= 128 ? 1 : 2;
  // Up to 16 rows a warp holds them all; beyond, warps share the tiles of a ring.  Rows of two boxes take the registers of
  // two tiles of 8 rows.
  c.rt = c.boxes == 1 && rows > 8 ? 2 : 1;
  const int most = c.boxes == 1 ? 4 : 2;
  c.row_warps = rows <= 8 * c.rt ? 1 : rows <= 16 * c.rt ? 2 : most;
  if (c.row_warps > most) c.row_warps = most;
  c.rings = c.boxes == 1 ? 8 / c.row_warps : 4;
  c.group_rows = 8 * c.rt * c.row_warps;
  const size_t tile = (size_t)2 * c.boxes * kTileKeys * 128;
  const int warps = c.rings * c.row_warps;
  c.smem = (size_t)warps * 8 * (c.boxes * 128 + 4) * 4 + (size_t)warps * 8 * c.rt * 8 + kMaxRings * kMaxStages * 24 +
           (kMaxEntries + 1 + 16) * 4;
  const int64_t fit = (227 * 1024 - c.smem) / (tile * c.rings);
  c.stages = (int)(fit < kMaxStages ? fit : kMaxStages);
  c.smem += tile * c.rings * c.stages;
  c.groups = (int)ceil_div(rows > 0 ? rows : 1, c.group_rows);
  c.requests = kMaxEntries / p->n_kv_heads < batch ? kMaxEntries / p->n_kv_heads : batch;
  if (c.requests < 1) c.requests = 1;
  // a CTA per SM, and no more than one per tile of each of its rings
  const int64_t most_ctas = ceil_div((total_tokens / kTileKeys + batch) * p->n_kv_heads, c.rings);
  c.ctas = most_ctas < kSms ? most_ctas : kSms;
  return c;
}

template <int kBoxes, int kRt>
int32_t run_attend(const Cut& c, const CUtensorMap& tmK, const CUtensorMap& tmV, const AttendArgs& a, cudaStream_t st) {
  auto kernel = attend8_kernel<kBoxes, kRt>;
  GVOTE_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)c.smem));
  {
    LaunchScope scope_("attend8_kernel", st);
    launch_on(kernel, dim3((unsigned)c.ctas, (unsigned)c.groups), dim3(c.rings * c.row_warps * 32), c.smem, st, tmK, tmV, a);
  }
  GVOTE_LAUNCH_CHECK("attend8_kernel");
  return GVOTE_OK;
}

}  // namespace

AttendMap attend8_map(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N, int64_t total_q,
                      int64_t max_q) {
  AttendMap m;
  const int64_t nq = max_q < GVOTE_ATTEND8_MAX_Q ? max_q : GVOTE_ATTEND8_MAX_Q;
  const Cut c = cut_of(p, batch, total_tokens, nq);
  const size_t entries = (size_t)c.requests * p->n_kv_heads;
  const size_t rows = (size_t)c.groups * (entries + c.ctas) * c.group_rows;
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
  a.rings = cut.rings; a.row_warps = cut.row_warps; a.stages = cut.stages; a.group_rows = cut.group_rows;
  a.scale2 = (float)(1.4426950408889634 / sqrt((double)p->d_k));

  CUtensorMap tmK, tmV;
  const uint64_t dims[3] = {(uint64_t)p->d_k, (uint64_t)c->total_tokens, (uint64_t)a.Hkv};
  const uint64_t strides[2] = {(uint64_t)c->tok_stride, (uint64_t)(a.Hkv > 1 ? c->head_stride : c->tok_stride)};
  const uint32_t box[3] = {128, (uint32_t)kTileKeys, 1};
  if (!encode_tensor_map_u8(&tmK, c->K, 3, dims, strides, box) || !encode_tensor_map_u8(&tmV, c->V, 3, dims, strides, box))
    return GVOTE_ERR_UNSUPPORTED_SHAPE;

  for (int32_t r0 = 0; r0 < c->batch; r0 += cut.requests) {
    a.r0 = r0;
    a.batch = c->batch - r0 < cut.requests ? c->batch - r0 : cut.requests;
    if (cut.boxes == 2) PROPAGATE((run_attend<2, 1>(cut, tmK, tmV, a, st)));
    else if (cut.rt == 2) PROPAGATE((run_attend<1, 2>(cut, tmK, tmV, a, st)));
    else PROPAGATE((run_attend<1, 1>(cut, tmK, tmV, a, st)));
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
