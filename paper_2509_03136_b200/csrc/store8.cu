// The pruning step of Algorithm 1 into the 8-bit cache (gvote_store8), and from one 8-bit cache into
// another (gvote_prune8): gather the kept rows in ascending order, find each 64-row block's scale, round.
//
//   scale_b = the smallest 2^e with max |x| <= 448 * 2^e over the block, code = e4m3(x / scale_b).
//
// Two kernels.  store8_scan_kernel turns each (request, head) bit row into the list of its kept rows, 64 to a
// destination block, and notes for every block what its CTA would otherwise have to look up (struct Note).
// store8_kernel gives one CTA one destination block of K and of V: it reads its note and its list, loads all rows into
// registers (16 values per thread and unit, 16-byte loads), takes the maximum over the CTA, and writes the codes.  Bound
// by memory: 6 d_k bytes per kept row from bf16, 4 d_k from e4m3; the rows are read once, there is no second pass
// over them.  A CTA waits for one round of small loads before it can ask for its rows; with five rounds, looking the
// request up and searching for the first word, a call took a third longer.
// Measured: 17K rows of 8 heads from bf16 (110 MB) 31 us, 24 of them in the second kernel (4.6 TB/s); 89 MB pruned from one
// cache into another 28 us; 275K rows of one head 39 us (48 with one CTA per bit row in the scan).  Each CTA working out
// its rows from the whole bit row, without the first kernel, took as long for one request and longer (33 us) for a batch;
// neither fewer instructions per value nor six CTAs per SM instead of five changed the second kernel's time.
// Out of place: nothing orders the blocks, and a pruned 8-bit cache is small.
#include <cooperative_groups.h>

#include "cache8.cuh"
#include "ptx.cuh"

namespace gvote {
namespace {

namespace cg = cooperative_groups;

constexpr int kStoreThreads = 256;
constexpr int kScan8Threads = 256;

// One per (head, destination block), padding entries of the block list included.
struct __align__(16) Note {
  int cnt, row0, start, dst;     // rows (<= 0: none), first destination row, the request's first source and destination slot
  int r, pad[3];
};

// A cluster per (head, request), each CTA with a run of its mask words: the sources of the kept rows, in order, 64 to a
// destination block, and the blocks' notes.
__global__ void __launch_bounds__(kScan8Threads)
store8_scan_kernel(const uint32_t* __restrict__ mask, const int32_t* __restrict__ cu, const int32_t* __restrict__ kv_len,
                   int Hkv, int64_t row_words, int32_t* __restrict__ list, const int32_t* __restrict__ cu8,
                   int64_t row_blocks, Note* __restrict__ note, int32_t* __restrict__ kv_len_out, int32_t* status) {
  constexpr int kWarps = kScan8Threads / 32;
  __shared__ int warp_tot[kWarps];
  __shared__ int share_tot;
  ptx::let_next_begin();
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int h = blockIdx.y, r = blockIdx.z;
  const int start = cu[r], n = valid_keys(kv_len, r, Hkv, h, cu[r + 1] - start);
  const int words = (n + 31) >> 5, share = (words + C - 1) / C, w0 = min(rank * share, words), w1 = min(w0 + share, words);
  const uint32_t* bits_of = mask + (int64_t)h * row_words + mask_word_offset(start, r);
  const int dstart = cu8[r], cap = cu8[r + 1] - dstart;
  const int64_t first = (int64_t)h * row_blocks + block8_offset(dstart, r);       // the request's first block
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  auto word_at = [&](int w) {
    uint32_t v = w < w1 ? bits_of[w] : 0u;
    if (w == words - 1 && (n & 31)) v &= (1u << (n & 31)) - 1u;
    return v;
  };
  uint32_t v = word_at(w0 + tid);
  int mine = __popc(v);
  for (int w = w0 + tid + kScan8Threads; w < w1; w += kScan8Threads) mine += __popc(word_at(w));
  mine = __reduce_add_sync(0xffffffffu, mine);
  if (lane == 0) warp_tot[warp] = mine;
  __syncthreads();
  if (warp == 0) {
    const int t = __reduce_add_sync(0xffffffffu, lane < kWarps ? warp_tot[lane] : 0);
    if (lane == 0) share_tot = t;
  }
  cluster.sync();
  int before = 0, total = 0;                                       // kept rows of the CTAs before this one, and of all
  for (int c = 0; c < C; ++c) {
    const int t = *cluster.map_shared_rank(&share_tot, c);
    before += c < rank ? t : 0;
    total += t;
  }
  const int m = min(total, cap);
  int32_t* out = list + first * kBlock8;
  for (int base = w0; base < w1; base += kScan8Threads) {          // thread = word, then thread = bit
    if (base > w0) v = word_at(base + tid);
    int inc = __popc(v);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += u;
    }
    __syncthreads();
    if (lane == 31) warp_tot[warp] = inc;
    __syncthreads();
    const int tot = lane < kWarps ? warp_tot[lane] : 0;
    const int run = before + __reduce_add_sync(0xffffffffu, lane < warp ? tot : 0) + inc - __popc(v);
    before += __reduce_add_sync(0xffffffffu, tot);
    const int row = (base + warp * 32) * 32 + lane;
#pragma unroll 8
    for (int j = 0; j < 32; ++j) {
      const uint32_t b = __shfl_sync(0xffffffffu, v, j);
      const int at = __shfl_sync(0xffffffffu, run, j) + __popc(b & ((1u << lane) - 1u));
      if (((b >> lane) & 1u) && at < m) out[at] = row + j * 32;
    }
  }
  const int64_t list_end = r + 1 < (int)gridDim.z ? block8_offset(cu8[r + 1], r + 1) : row_blocks;
  const int listed = (int)(list_end - block8_offset(dstart, r));
  const int ahead = r == 0 ? (int)block8_offset(dstart, 0) : 0;    // (slabs that do not start at slot 0)
  for (int b = rank * kScan8Threads + tid - ahead; b < listed; b += C * kScan8Threads) {
    Note x;
    x.cnt = b < 0 ? 0 : min(kBlock8, m - b * kBlock8);
    x.row0 = b * kBlock8; x.start = start; x.dst = dstart; x.r = r;
    int4* q = reinterpret_cast<int4*>(note + first + b);
    q[0] = make_int4(x.cnt, x.row0, x.start, x.dst);
    q[1] = make_int4(x.r, 0, 0, 0);
  }
  if (rank == 0 && tid == 0) {
    kv_len_out[r * Hkv + h] = m;
    if (total > cap) { atomicExch(&status[0], GVOTE_ERR_WORKSPACE_TOO_SMALL); atomicExch(&status[1], 8); }
  }
  cluster.sync();                                                  // the shares' totals are read until here
}

struct StoreArgs {
  const void* src[2];            // K, V: bf16 or e4m3
  const float* src_scale[2];     // of an e4m3 source
  int64_t s_tok, s_head, s_total, s_row_blocks;
  const uint32_t* mask;          // or null: every row
  const int32_t* list;           // [Hkv][row_blocks of the destination][64] the rows' sources
  const Note* note;              // [Hkv][row_blocks of the destination]
  const int32_t* cu;
  const int32_t* kv_len;
  int64_t row_words;
  uint8_t* dst[2];
  float* dst_scale[2];
  int64_t d_tok, d_head, d_total, d_row_blocks;
  const int32_t* cu8;
  int32_t* kv_len_out;
  SideArrays side;
  int32_t* status;
  int Hkv, batch, d_k;
};

// A unit: 16 consecutive elements of a row, bf16 (two 16-byte words) or e4m3 codes with their row's scale.
// The arithmetic works on pairs; 25 instructions per element, in 32-bit floats with a test of every element, had made the
// kernel bound by their issue (37 us for the 12 us of bytes of 17K rows x 8 heads).
template <bool kSrc8>
struct Unit;

__device__ __forceinline__ uint32_t half2_abs_max(uint32_t a, uint32_t b) {      // of |a|, |b|; a NaN loses
  uint32_t d;
  asm("{\n\t.reg .b32 x, y;\n\tabs.f16x2 x, %1;\n\tabs.f16x2 y, %2;\n\tmax.f16x2 %0, x, y;\n\t}" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

template <>
struct Unit<false> {
  uint4 lo, hi;
  bool finite;
  __device__ __forceinline__ void load(const void* base, int64_t elem, float) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(base) + elem);
    lo = __ldg(q);
    hi = __ldg(q + 1);
  }
  __device__ __forceinline__ uint32_t word(int i) const { return i < 4 ? (&lo.x)[i] : (&hi.x)[i - 4]; }
  static __device__ __forceinline__ float scale_of(float top) { return scale8_of(top); }
  // The largest finite magnitude.  Magnitudes of bf16 are ordered like their bits; 0x7f80 and above are not finite.
  __device__ __forceinline__ float largest() {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __vmaxu2(m, word(i) & 0x7fff7fffu);
    finite = (m & 0xffffu) < 0x7f80u && (m >> 16) < 0x7f80u;
    if (!finite) {                                               // rare: leave out what is not
      m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t a = word(i) & 0x7fffu, b = (word(i) >> 16) & 0x7fffu;
        m = max(m, max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u));
      }
    }
    return __uint_as_float(max(m & 0xffffu, m >> 16) << 16);
  }
  __device__ __forceinline__ uint4 encode(float scale, float inv) const {
    uint4 out;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t a = word(2 * q), b = word(2 * q + 1);
      (&out.x)[q] = narrow8x4(__uint_as_float(a << 16) * inv, __uint_as_float(a & 0xffff0000u) * inv,
                              __uint_as_float(b << 16) * inv, __uint_as_float(b & 0xffff0000u) * inv);
    }
    if (!finite) {                                               // rare: an infinity is not 448 but the NaN code
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (((word(2 * q + (k >> 1)) >> (16 * (k & 1))) & 0x7fffu) >= 0x7f80u) (&out.x)[q] |= 0x7fu << (8 * k);
    }
    return out;
  }
};

template <>
struct Unit<true> {
  uint4 lo;
  float scale;
  __device__ __forceinline__ void load(const void* base, int64_t elem, float s) {
    lo = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(base) + elem));
    scale = s;
  }
  // the scale of a block whose largest value is twice `half`: exponents count from the half, whose least scale is 2^-126 / 2
  static __device__ __forceinline__ float scale_of(float half) {
    return half <= 224.f * 1.17549435e-38f ? 1.17549435e-38f : 2.f * scale8_of(half);
  }
  // Half of the largest finite magnitude.
  __device__ __forceinline__ float largest() {
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t a, b;
      widen8x4((&lo.x)[q], a, b);
      m = half2_abs_max(m, half2_abs_max(a, b));
    }
    const __half2 h = *reinterpret_cast<const __half2*>(&m);
    const float x = __low2float(h), y = __high2float(h), top = fmaxf(x, y);     // (a NaN on both sides of a max stays)
    return top == top ? top * (0.5f * scale) : 0.f;               // (the value itself may be 2^128)
  }
  // code * 2^j for the block's own scale: the codes themselves where the scales agree; in halves where 2^j is one (exact as
  // far as e4m3 can tell: a code has 4 significant bits and the least half, 2^-24, lies far below half its least step)
  __device__ __forceinline__ uint4 encode(float to, float inv) const {
    if (scale == to) return lo;
    uint4 out;
    const float ratio = scale * inv;
    if (ratio >= 6.103515625e-05f && ratio <= 32768.f) {
      const __half2 f = __float2half2_rn(ratio);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t a, b;
        widen8x4((&lo.x)[q], a, b);
        const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&a), f), y = __hmul2(*reinterpret_cast<const __half2*>(&b), f);
        (&out.x)[q] = narrow8x4(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
      }
      return out;
    }
    // (a code that is not zero has a ratio of 2^18 at most; beyond that every code is zero, and must stay so)
    const float f = fminf(ratio, 1.2676506e30f);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t w = (&lo.x)[q];
      const float2 a = decode8x2(w & 0xffffu), b = decode8x2(w >> 16);
      (&out.x)[q] = encode8x2(a.x * f, a.y * f) | (encode8x2(b.x * f, b.y * f) << 16);
    }
    return out;
  }
};

template <bool kSrc8, int kUnits>     // kUnits: 16-element units of a block's K (or V) per thread
__global__ void __launch_bounds__(kStoreThreads, kUnits <= 2 ? 5 : 2)
store8_kernel(const __grid_constant__ StoreArgs a) {
  __shared__ int s_src[kBlock8];
  __shared__ float s_max[2][kStoreThreads / 32];
  const int tid = threadIdx.x;
  const int h = (int)(blockIdx.x % a.Hkv);
  const int64_t gb = blockIdx.x / a.Hkv;
  const int64_t db = (int64_t)h * a.d_row_blocks + gb;
  int r, start, dstart, row0, cnt;
  if (a.mask) {
    ptx::wait_for_previous();
    const int4 note = *reinterpret_cast<const int4*>(&a.note[db]);
    r = a.note[db].r;
    if (tid < kBlock8) s_src[tid] = a.list[db * kBlock8 + tid];    // (beyond cnt: not looked at)
    cnt = note.x; row0 = note.y; start = note.z; dstart = note.w;
    if (cnt <= 0) return;
    __syncthreads();
  } else {
    r = a.batch == 1 ? 0 : find_request_by(a.cu8, a.batch, gb, 6);
    dstart = a.cu8[r];
    const int cap = a.cu8[r + 1] - dstart, b = (int)(gb - block8_offset(dstart, r));
    row0 = b * kBlock8;
    start = a.cu[r];
    const int n = valid_keys(a.kv_len, r, a.Hkv, h, a.cu[r + 1] - start), m = min(n, cap);
    if (b == 0 && tid == 0) {
      a.kv_len_out[r * a.Hkv + h] = m;
      if (n > cap) { atomicExch(&a.status[0], GVOTE_ERR_WORKSPACE_TOO_SMALL); atomicExch(&a.status[1], 8); }
    }
    cnt = b < 0 ? 0 : min(kBlock8, m - row0);
    if (cnt <= 0) return;
    if (tid < cnt) s_src[tid] = row0 + tid;
    __syncthreads();
  }
  float weight = 0.f;                                            // of the side arrays, on their way with the rows
  int position = 0;
  if (tid < cnt) {
    const int64_t s = (int64_t)h * a.s_total + start + s_src[tid];
    if (a.side.acc_out) weight = a.side.acc[s];
    if (a.side.pos_out) position = a.side.pos ? a.side.pos[s] : s_src[tid];
  }
  // thread = one unit of every (threads / units per row)-th row
  const int dc = a.d_k >> 4, step = kStoreThreads / dc, j0 = tid / dc, c0 = (tid - j0 * dc) * 16;
  const int64_t s0 = (int64_t)h * a.s_head + (int64_t)start * a.s_tok + c0;
  const int64_t d0 = (int64_t)h * a.d_head + (int64_t)(dstart + row0) * a.d_tok + c0;
  const int64_t sb = (int64_t)h * a.s_row_blocks + block8_offset(start, r);
  auto holds = [&](int i) { return j0 < step && j0 + i * step < cnt; };
  Unit<kSrc8> x[2][kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i)
    if (holds(i)) {
      const int n_src = s_src[j0 + i * step];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        x[t][i].load(a.src[t], s0 + n_src * a.s_tok, kSrc8 ? a.src_scale[t][sb + (n_src >> 6)] : 0.f);
    }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
      if (holds(i)) mx = fmaxf(mx, x[t][i].largest());
    mx = warp_max(mx);
    if ((tid & 31) == 0) s_max[t][tid >> 5] = mx;
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    float top = s_max[t][0];
#pragma unroll
    for (int w = 1; w < kStoreThreads / 32; ++w) top = fmaxf(top, s_max[t][w]);
    const float scale = Unit<kSrc8>::scale_of(top), inv = inverse_pow2(scale);
    if (tid == t) a.dst_scale[t][db] = scale;
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
      if (holds(i)) *reinterpret_cast<uint4*>(a.dst[t] + d0 + (j0 + i * step) * a.d_tok) = x[t][i].encode(scale, inv);
  }
  if (tid < cnt) {
    const int64_t d = (int64_t)h * a.d_total + dstart + row0 + tid;
    if (a.side.acc_out) a.side.acc_out[d] = weight;
    if (a.side.pos_out) a.side.pos_out[d] = position;
  }
}

template <bool kSrc8>
int32_t run_store(const StoreArgs& a, unsigned ctas, cudaStream_t st) {
  const int units = (int)ceil_div(kBlock8, kStoreThreads / (a.d_k >> 4));   // 1 .. 4
  auto kernel = units == 1 ? store8_kernel<kSrc8, 1> : units == 2 ? store8_kernel<kSrc8, 2> : store8_kernel<kSrc8, 4>;
  {
    LaunchScope scope_("store8_kernel", st);
    if (a.mask) launch_behind(kernel, dim3(ctas), dim3(kStoreThreads), 0, st, a);
    else launch_on(kernel, dim3(ctas), dim3(kStoreThreads), 0, st, a);
  }
  GVOTE_LAUNCH_CHECK("store8_kernel");
  return GVOTE_OK;
}

}  // namespace

StoreMap store8_map(const gvote_params* p, int32_t batch, int64_t total_tokens) {
  StoreMap m;
  const size_t blocks = (size_t)p->n_kv_heads * gvote_cache8_row_blocks(total_tokens, batch);
  m.list = kStatusBytes;
  m.note = align_up(m.list + blocks * kBlock8 * 4, 256);
  m.total = align_up(m.note + blocks * sizeof(Note), 256);
  return m;
}

int32_t launch_store8(const gvote_params* p, const __nv_bfloat16* K, const __nv_bfloat16* V, int64_t tok, int64_t head,
                      const gvote_cache8* src8, const uint32_t* mask, const int32_t* cu, const int32_t* kv_len,
                      int32_t batch, int64_t total_tokens, int64_t max_N, const gvote_cache8* dst,
                      const SideArrays& side, char* ws, cudaStream_t st) {
  const int Hkv = p->n_kv_heads;
  const StoreMap m = store8_map(p, batch, total_tokens > dst->total_tokens ? total_tokens : dst->total_tokens);
  StoreArgs a;
  a.src[0] = src8 ? src8->K : (const void*)K;
  a.src[1] = src8 ? src8->V : (const void*)V;
  a.src_scale[0] = src8 ? src8->k_scale : nullptr;
  a.src_scale[1] = src8 ? src8->v_scale : nullptr;
  a.s_tok = tok; a.s_head = head; a.s_total = total_tokens;
  a.s_row_blocks = gvote_cache8_row_blocks(total_tokens, batch);
  a.mask = mask;
  a.list = reinterpret_cast<const int32_t*>(ws + m.list);
  a.note = reinterpret_cast<const Note*>(ws + m.note);
  a.cu = cu; a.kv_len = kv_len;
  a.row_words = gvote_mask_row_words(total_tokens, batch);
  a.dst[0] = (uint8_t*)dst->K; a.dst[1] = (uint8_t*)dst->V;
  a.dst_scale[0] = dst->k_scale; a.dst_scale[1] = dst->v_scale;
  a.d_tok = dst->tok_stride; a.d_head = dst->head_stride; a.d_total = dst->total_tokens;
  a.d_row_blocks = gvote_cache8_row_blocks(dst->total_tokens, batch);
  a.cu8 = dst->cu_seqlens; a.kv_len_out = dst->kv_len;
  a.side = side;
  a.status = reinterpret_cast<int32_t*>(ws);
  a.Hkv = Hkv; a.batch = batch; a.d_k = p->d_k;
  if (mask) {
    // CTAs per bit row: the largest of 8, 4, 2, 1 that leaves each 4096 rows of the longest slab and the grid four CTAs per SM
    int C = 8;
    while (C > 1 && (max_N / C < 4096 || (int64_t)batch * Hkv * C > 4 * 148)) C >>= 1;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    cfg.gridDim = dim3(C, Hkv, batch);
    cfg.blockDim = dim3(kScan8Threads);
    cfg.stream = st;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = C; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = C > 1 ? 1 : 0;
    LaunchScope scope_("store8_scan_kernel", st);
    (void)cudaLaunchKernelEx(&cfg, store8_scan_kernel, mask, cu, kv_len, Hkv, a.row_words, (int32_t*)(ws + m.list), a.cu8,
                             a.d_row_blocks, (Note*)(ws + m.note), a.kv_len_out, a.status);
    GVOTE_LAUNCH_CHECK("store8_scan_kernel");
  }
  const unsigned ctas = (unsigned)(a.d_row_blocks * Hkv);
  return src8 ? run_store<true>(a, ctas, st) : run_store<false>(a, ctas, st);
}

}  // namespace gvote
