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
// 2 x 128 x 128 logits).  Warp 0 asks for the tiles (TMA, 128-byte swizzle), warp 1 issues the MMAs, warps 2-5 read
// out the first stationary tile, warps 6-9 the second; two accumulators of 128 columns each per stationary tile
// (all 512 columns of tensor memory).  The next unit's stationary tiles are fetched while this one runs.
//
// Few query rows (a window of the last tokens) would give pass 1 fewer units than SMs: the keys are then split
// into chunks whose (reference, sum) pairs accumulate_lse_kernel merges.
//
// Every wait is bounded: when one runs out the CTA records GVOTE_ERR_TIMEOUT in the status word, frees its tensor
// memory and returns.
#include "cache8.cuh"
#include "ptx.cuh"

namespace gvote {
namespace {

constexpr int kTile = 128;            // rows of A and of B
constexpr int kAccThreads = 320;
constexpr int kMaxStages = 6;
constexpr int kLseStages = 3;
constexpr int kSms = 148;
constexpr float kLog2e = 1.4426950408889634f;

struct AccArgs {
  const int32_t* cu_q;
  const int32_t* cu;
  const int32_t* kv_len;
  float* lse2;                        // [Hkv][q_tiles][128], +inf on rows that hold no query
  float2* part;                       // [key_chunks][Hkv][q_tiles][128] (reference, sum), when the keys are split
  const float* acc;
  float* acc_out;
  int32_t* status;
  int64_t total, q_tiles, pairs, units;
  int Hkv, G, batch, d_k, tpt;        // tpt: tokens of a query tile
  int boxes, stages, stat_slots, key_chunks;
  float c;                            // log2(e) / sqrt(d_k)
};

struct Tail {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t stat_full[2], stat_empty[2];
  uint64_t lse_full[kLseStages], lse_empty[kLseStages];
  uint64_t acc_full[2][2], acc_empty[2][2];
  uint32_t tmem_slot;
  volatile int abort_flag;
};

__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  for (uint32_t i = 0; i < (1u << 22); ++i) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if ((i & 255u) == 255u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
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

template <int kPass>
__device__ __forceinline__ UnitInfo unit_info(const AccArgs& a, int64_t u) {
  UnitInfo x;
  x.h = (int)(u % a.Hkv);
  int64_t v = u / a.Hkv;
  x.chunk = 0;
  if (kPass == 1) {
    x.chunk = (int)(v % a.key_chunks);
    v = a.pairs - 1 - v / a.key_chunks;                    // long rows first
    x.r = a.batch == 1 ? 0 : find_request_div(a.cu_q, a.batch, v, 2 * a.tpt);
  } else {
    x.r = a.batch == 1 ? 0 : find_request_by(a.cu, a.batch, v, 8);
  }
  x.start = a.cu[x.r];
  x.n = valid_keys(a.kv_len, x.r, a.Hkv, x.h, a.cu[x.r + 1] - x.start);
  x.q0 = a.cu_q[x.r];
  x.nq = a.cu_q[x.r + 1] - x.q0;
  const int q_tiles = (x.nq + a.tpt - 1) / a.tpt;
  if (kPass == 1) {
    x.stat0 = 2 * (int)(v - (x.q0 / (2 * a.tpt) + x.r));
    x.n_stat = max(min(2, q_tiles - x.stat0), 0);
    const int last = min(x.nq, (x.stat0 + x.n_stat) * a.tpt) - 1;
    const int tiles = (max(x.n - (x.nq - 1 - last), 0) + kTile - 1) / kTile;
    x.s0 = (int)((int64_t)tiles * x.chunk / a.key_chunks);
    x.s1 = (int)((int64_t)tiles * (x.chunk + 1) / a.key_chunks);
  } else {
    x.stat0 = 2 * (int)(v - ((x.start >> 8) + x.r));
    x.n_stat = max(min(2, (x.n + kTile - 1) / kTile - x.stat0), 0);
    x.s0 = min(max(x.stat0 * kTile - (x.n - x.nq), 0) / a.tpt, q_tiles);
    x.s1 = q_tiles;
  }
  return x;
}

template <int kPass>
__global__ void __launch_bounds__(kAccThreads, 1)
accumulate_umma_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ AccArgs a) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t tile_bytes = (uint32_t)a.boxes * kTile * 128;
  uint8_t* stat_sm = base;                                         // [stat_slots][2][tile]
  uint8_t* ring_sm = stat_sm + (size_t)a.stat_slots * 2 * tile_bytes;
  float* lse_sm = reinterpret_cast<float*>(ring_sm + (size_t)a.stages * tile_bytes);
  Tail* tail = reinterpret_cast<Tail*>(lse_sm + kLseStages * kTile);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // the rows of a query tile that no box fills (G does not divide 128) must be finite
  for (uint4* p = reinterpret_cast<uint4*>(base) + threadIdx.x; p < reinterpret_cast<uint4*>(lse_sm); p += kAccThreads)
    *p = make_uint4(0, 0, 0, 0);
  ptx::fence_proxy_async();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kMaxStages; ++s) { ptx::mbar_init(&tail->full[s], 1); ptx::mbar_init(&tail->empty[s], 1); }
    for (int s = 0; s < kLseStages; ++s) { ptx::mbar_init(&tail->lse_full[s], 1); ptx::mbar_init(&tail->lse_empty[s], 8); }
    for (int s = 0; s < 2; ++s) {
      ptx::mbar_init(&tail->stat_full[s], 1);
      ptx::mbar_init(&tail->stat_empty[s], 1);
      for (int b = 0; b < 2; ++b) { ptx::mbar_init(&tail->acc_full[s][b], 1); ptx::mbar_init(&tail->acc_empty[s][b], 4); }
    }
    tail->abort_flag = 0;
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
  const uint32_t tmem = tail->tmem_slot;
  volatile int* abort_flag = &tail->abort_flag;
  const int q_rows = a.G * a.tpt;                                  // rows a query box fills
  const uint32_t q_bytes = (uint32_t)a.boxes * q_rows * 128, k_bytes = tile_bytes;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int unit = 0, it = 0;
      bool ok = true;
      for (int64_t u = blockIdx.x; ok && u < a.units; u += gridDim.x) {
        const UnitInfo x = unit_info<kPass>(a, u);
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
            ptx::bulk_load(lse_sm + l * kTile, a.lse2 + ((int64_t)x.h * a.q_tiles + x.q0 / a.tpt + x.r + t) * kTile, kTile * 4,
                           &tail->lse_full[l]);
          }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      const uint32_t idesc = ptx::instr_desc_bf16_f32(kTile, kTile);
      const int ksteps = a.d_k / 16;
      int unit = 0, it = 0, used[2] = {0, 0};
      bool ok = true;
      for (int64_t u = blockIdx.x; ok && u < a.units; u += gridDim.x) {
        const UnitInfo x = unit_info<kPass>(a, u);
        if (x.n_stat == 0 || x.s1 <= x.s0) continue;
        const int slot = unit % a.stat_slots;
        ok = wait_or_abort(&tail->stat_full[slot], (unit / a.stat_slots) & 1, abort_flag);
        ++unit;
        for (int t = x.s0; ok && t < x.s1; ++t, ++it) {
          const int s = it % a.stages;
          ok = wait_or_abort(&tail->full[s], (it / a.stages) & 1, abort_flag);
          const uint32_t b_addr = ptx::smem_u32(ring_sm + (size_t)s * tile_bytes);
          for (int i = 0; ok && i < x.n_stat; ++i) {
            const int b = used[i] & 1;
            ok = wait_or_abort(&tail->acc_empty[i][b], ((used[i] >> 1) & 1) ^ 1, abort_flag);
            if (!ok) break;
            ++used[i];
            ptx::tc_fence_after_sync();
            const uint32_t a_addr = ptx::smem_u32(stat_sm + (size_t)(slot * 2 + i) * tile_bytes);
            for (int k = 0; k < ksteps; ++k) {
              const uint32_t off = (uint32_t)(k >> 2) * (kTile * 128) + (uint32_t)(k & 3) * 32u;
              ptx::umma_bf16(tmem + (uint32_t)((i * 2 + b) * kTile), ptx::smem_desc_k_sw128(a_addr + off),
                             ptx::smem_desc_k_sw128(b_addr + off), idesc, k > 0 ? 1u : 0u);
            }
            ptx::umma_commit(&tail->acc_full[i][b]);
          }
          if (ok) ptx::umma_commit(&tail->empty[s]);
        }
        if (ok) ptx::umma_commit(&tail->stat_empty[slot]);
      }
    }
  } else {
    // ------------------------------------------------------------------ read-out: thread = row of a stationary tile
    const int i = (warp - 2) >> 2;                                 // which stationary tile
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(i * 2 * kTile);
    int it = 0, used = 0;
    bool ok = true;
    for (int64_t u = blockIdx.x; ok && u < a.units; u += gridDim.x) {
      const UnitInfo x = unit_info<kPass>(a, u);
      if (x.n_stat == 0) continue;
      const bool mine = i < x.n_stat;
      if (kPass == 1) {
        const int tok0 = (x.stat0 + i) * a.tpt, token = tok0 + row / a.G;
        const bool holds = mine && row < q_rows && token < x.nq;
        const int limit = holds ? x.n - (x.nq - 1 - token) : 0;    // keys this row sees
        const int all_see = x.n - (x.nq - 1 - tok0);               // keys every row of the tile sees
        float ref = -INFINITY, sum = 0.f;
        for (int t = x.s0; mine && t < x.s1; ++t, ++used) {
          const int b = used & 1;
          ok = __all_sync(0xffffffffu, wait_or_abort(&tail->acc_full[i][b], (used >> 1) & 1, abort_flag));
          if (!ok) break;
          ptx::tc_fence_after_sync();
          const bool masked = (t + 1) * kTile > all_see;
#pragma unroll
          for (int c = 0; c < kTile; c += 32) {
            uint32_t v[32];
            ptx::tmem_ld_32x32(lane_addr + (uint32_t)(b * kTile + c), v);
            ptx::tmem_wait_ld();
            if (c == kTile - 32) {                                 // accumulator drained
              ptx::tc_fence_before_sync();
              __syncwarp();
              if (lane == 0) ptx::mbar_arrive(&tail->acc_empty[i][b]);
            }
            if (masked) {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (t * kTile + c + j >= limit) v[j] = 0xff800000u;
            }
            float mx = __uint_as_float(v[0]);
#pragma unroll
            for (int j = 1; j < 32; ++j) mx = fmaxf(mx, __uint_as_float(v[j]));
            // the reference moves only when a logit passes it by 2^8: the sum stays far from overflow without it
            if (mx * a.c > ref + 8.f) {
              const float next = mx * a.c;
              sum *= exp2_fast(ref - next);                        // (ref = -inf: 0 * 0)
              ref = next;
            }
            const float off = ref == -INFINITY ? 0.f : ref;
            float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 32; ++j) s4[j & 3] += exp2_fast(fmaf(__uint_as_float(v[j]), a.c, -off));
            sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
          }
        }
        if (mine) {
          const int64_t at = ((int64_t)x.h * a.q_tiles + x.q0 / a.tpt + x.r + x.stat0 + i) * kTile + row;
          if (a.key_chunks > 1) a.part[(int64_t)x.chunk * a.Hkv * a.q_tiles * kTile + at] = make_float2(ref, sum);
          else a.lse2[at] = !holds ? INFINITY : ref == -INFINITY ? -INFINITY : ref + log2f(sum);
        }
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
            const int tok0 = t * a.tpt;
            // columns of tokens behind the request's last, or of tokens that do not see this key, do not count
            const bool masked = tok0 < last_shift || tok0 + a.tpt > x.nq;
            const int j0 = (shift - tok0) * a.G, j1 = min(a.tpt, x.nq - tok0) * a.G;
            const float* lse = lse_sm + l * kTile;
            float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < kTile; c += 32) {
              uint32_t v[32];
              ptx::tmem_ld_32x32(lane_addr + (uint32_t)(b * kTile + c), v);
              ptx::tmem_wait_ld();
              if (c == kTile - 32) {
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&tail->acc_empty[i][b]);
              }
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                const float4 e = *reinterpret_cast<const float4*>(lse + c + j);
                float w0 = exp2_fast(fmaf(__uint_as_float(v[j]), a.c, -e.x));
                float w1 = exp2_fast(fmaf(__uint_as_float(v[j + 1]), a.c, -e.y));
                float w2 = exp2_fast(fmaf(__uint_as_float(v[j + 2]), a.c, -e.z));
                float w3 = exp2_fast(fmaf(__uint_as_float(v[j + 3]), a.c, -e.w));
                if (masked) {
                  const int q = c + j;
                  w0 = q >= j0 && q < j1 ? w0 : 0.f;
                  w1 = q + 1 >= j0 && q + 1 < j1 ? w1 : 0.f;
                  w2 = q + 2 >= j0 && q + 2 < j1 ? w2 : 0.f;
                  w3 = q + 3 >= j0 && q + 3 < j1 ? w3 : 0.f;
                }
                s4[0] += w0; s4[1] += w1; s4[2] += w2; s4[3] += w3;
              }
            }
            sum += (double)((s4[0] + s4[1]) + (s4[2] + s4[3]));
          }
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&tail->lse_empty[l]);
        }
        if (ok && mine && key < x.n) {
          const int64_t slot = (int64_t)x.h * a.total + x.start + key;
          a.acc_out[slot] = (float)((a.acc ? (double)a.acc[slot] : 0.0) + sum);
        }
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

// lse2 of the query tiles' rows from the key chunks' (reference, sum) pairs, or from the caller's lse.
__global__ void __launch_bounds__(kTile)
accumulate_lse_kernel(const __grid_constant__ AccArgs a, const float* __restrict__ given) {
  const int h = blockIdx.y, row = threadIdx.x;
  const int64_t tile = blockIdx.x;
  const int r = a.batch == 1 ? 0 : find_request_div(a.cu_q, a.batch, tile, a.tpt);
  const int q0 = a.cu_q[r], nq = a.cu_q[r + 1] - q0;
  const int token = (int)(tile - (q0 / a.tpt + r)) * a.tpt + row / a.G;
  if (token - row / a.G >= nq) return;
  const bool holds = row < a.G * a.tpt && token < nq;
  const int64_t at = ((int64_t)h * a.q_tiles + tile) * kTile + row;
  float out = INFINITY;
  if (holds && given) {
    out = given[(int64_t)(q0 + token) * a.Hkv * a.G + h * a.G + row % a.G] * kLog2e;
  } else if (holds) {
    const int64_t pitch = (int64_t)a.Hkv * a.q_tiles * kTile;
    float ref = -INFINITY, sum = 0.f;
    for (int x = 0; x < a.key_chunks; ++x) ref = fmaxf(ref, a.part[x * pitch + at].x);
    for (int x = 0; x < a.key_chunks; ++x) {
      const float2 p = a.part[x * pitch + at];
      if (p.x != -INFINITY) sum = fmaf(p.y, exp2_fast(p.x - ref), sum);
    }
    out = ref == -INFINITY ? -INFINITY : ref + log2f(sum);
  }
  a.lse2[at] = out;
}

}  // namespace

AccumulateMap accumulate_map(const gvote_params* p, int32_t batch, int64_t total_tokens, int64_t max_N, int64_t total_q,
                             int64_t max_q) {
  AccumulateMap m;
  const int64_t tpt = kTile / (p->n_q_heads / p->n_kv_heads);
  m.q_tiles = total_q / tpt + batch;
  // pass 1 in about two units per SM at least: chunks of keys where the query rows alone are fewer
  const int64_t units = (total_q / (2 * tpt) + batch) * p->n_kv_heads;
  int64_t chunks = units < 2 * kSms ? ceil_div(2 * kSms, units) : 1;
  const int64_t tiles = ceil_div(max_N > 0 ? max_N : 1, kTile);
  m.key_chunks = chunks < tiles ? chunks : tiles;
  m.lse = kStatusBytes;
  const size_t rows = (size_t)p->n_kv_heads * m.q_tiles * kTile;
  m.part = align_up(m.lse + rows * 4, 256);
  m.total = align_up(m.part + (m.key_chunks > 1 ? rows * m.key_chunks * 8 : 0), 256);
  return m;
}

int32_t launch_accumulate(const gvote_params* p, const __nv_bfloat16* Q, int64_t q_tok, int64_t q_head,
                          const int32_t* cu_q, int64_t total_q, int64_t max_q, const __nv_bfloat16* K, int64_t k_tok,
                          int64_t k_head, const int32_t* cu, const int32_t* kv_len, int32_t batch, int64_t total_tokens,
                          int64_t max_N, const float* lse, const float* acc, float* acc_out, char* ws, cudaStream_t st) {
  if (max_N == 0) return GVOTE_OK;
  const AccumulateMap m = accumulate_map(p, batch, total_tokens, max_N, total_q, max_q);
  AccArgs a;
  a.cu_q = cu_q; a.cu = cu; a.kv_len = kv_len;
  a.lse2 = (float*)(ws + m.lse); a.part = (float2*)(ws + m.part);
  a.acc = acc; a.acc_out = acc_out; a.status = (int32_t*)ws; a.total = total_tokens;
  a.Hkv = p->n_kv_heads; a.G = p->n_q_heads / p->n_kv_heads; a.batch = batch; a.d_k = p->d_k; a.tpt = kTile / a.G;
  a.q_tiles = m.q_tiles;
  a.key_chunks = (int)m.key_chunks;
  a.c = (float)(1.4426950408889634 / sqrt((double)p->d_k));
  a.boxes = (p->d_k + 63) / 64;
  // 227 KB: two slots of two stationary tiles and a ring of at least two tiles where they fit (d_k <= 128)
  const size_t tile = (size_t)a.boxes * kTile * 128, rest = 1024 + kLseStages * kTile * 4 + sizeof(Tail);
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
  if (!lse) {
    a.pairs = total_q / (2 * a.tpt) + batch;
    a.units = a.pairs * a.Hkv * a.key_chunks;
    GVOTE_CUDA_CHECK(cudaFuncSetAttribute(accumulate_umma_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    LaunchScope scope_("accumulate_lse_umma_kernel", st);
    launch_on(accumulate_umma_kernel<1>, dim3((unsigned)(a.units < kSms ? a.units : kSms)), dim3(kAccThreads), smem, st,
              tmQ, tmK, a);
    GVOTE_LAUNCH_CHECK("accumulate_lse_umma_kernel");
  }
  if (lse || a.key_chunks > 1) {
    LaunchScope scope_("accumulate_lse_kernel", st);
    launch_on(accumulate_lse_kernel, dim3((unsigned)a.q_tiles, a.Hkv), dim3(kTile), 0, st, a, lse);
    GVOTE_LAUNCH_CHECK("accumulate_lse_kernel");
  }
  a.pairs = (total_tokens >> 8) + batch;
  a.units = a.pairs * a.Hkv;
  GVOTE_CUDA_CHECK(cudaFuncSetAttribute(accumulate_umma_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  LaunchScope scope_("accumulate_weights_umma_kernel", st);
  launch_on(accumulate_umma_kernel<2>, dim3((unsigned)(a.units < kSms ? a.units : kSms)), dim3(kAccThreads), smem, st, tmQ,
            tmK, a);
  GVOTE_LAUNCH_CHECK("accumulate_weights_umma_kernel");
  return GVOTE_OK;
}

}  // namespace gvote
