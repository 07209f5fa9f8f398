// The pruning step of Algorithm 1 into the 8-bit cache (gvote_store8), and from one 8-bit cache into
// another (gvote_prune8): gather the kept rows in ascending order, find each 64-row block's scale, round.
//
//   scale_b = the smallest 2^e with max |x| <= 448 * 2^e over the block, code = e4m3(x / scale_b).
//
// Two kernels.  store8_scan_kernel turns each (request, head) bit row into an exclusive popcount prefix per
// mask word, and notes for every destination block what its CTA would otherwise have to look up (struct Note).
// store8_kernel gives one CTA one destination block of K and of V: its threads take a bit each of the words from
// the noted one on, load all rows into registers (16 values per thread and unit, 16-byte loads), take the maximum
// over the CTA, and write the codes.  Bound by memory: 6 d_k bytes per kept row from bf16, 4 d_k from e4m3; the rows are
// read once, there is no second pass over them.  What a CTA waits for before it can ask for its rows is two rounds of
// small loads (the note; words and prefixes); with five rounds, looking the request up and searching for the first
// word, a call took a third longer.
// Measured: 17K rows of 8 heads from bf16 (110 MB) 31 us, 24 of them in the second kernel (4.6 TB/s); 89 MB pruned from one cache
// into another 28 us.  Each CTA working out its rows from the whole bit row, without the first kernel, took as long (31 us) for
// one request and longer (33 us) for a batch.
// Out of place: nothing orders the blocks, and a pruned 8-bit cache is small.
#include "cache8.cuh"
#include "ptx.cuh"

namespace gvote {
namespace {

constexpr int kStoreThreads = 256;
constexpr int kScan8Threads = 1024;

// One per (head, destination block), padding entries of the block list included.
struct __align__(16) Note {
  int word, cnt, words, row0;    // first mask word (of the request's), rows, mask words that count, first destination row
  int r, start, dst, pad;        // request, its first source slot and first destination slot
};

// One CTA per (head, request): prefix[h][word] = kept keys among the n rows that count, before this word.
__global__ void __launch_bounds__(kScan8Threads)
store8_scan_kernel(const uint32_t* __restrict__ mask, const int32_t* __restrict__ cu, const int32_t* __restrict__ kv_len,
                   int Hkv, int64_t row_words, int32_t* __restrict__ prefix, const int32_t* __restrict__ cu8,
                   int64_t row_blocks, Note* __restrict__ note, int32_t* __restrict__ kv_len_out, int32_t* status) {
  __shared__ int warp_tot[kScan8Threads / 32];
  __shared__ int carry;
  ptx::let_next_begin();
  const int h = blockIdx.x, r = blockIdx.y;
  const int start = cu[r], n = valid_keys(kv_len, r, Hkv, h, cu[r + 1] - start);
  const int words = (n + 31) >> 5;
  const int64_t woff = (int64_t)h * row_words + mask_word_offset(start, r);
  const int dstart = cu8[r], cap = cu8[r + 1] - dstart;
  Note* my_note = note + (int64_t)h * row_blocks + block8_offset(dstart, r);
  const int64_t list_end = r + 1 < (int)gridDim.y ? block8_offset(cu8[r + 1], r + 1) : row_blocks;
  const int listed = (int)(list_end - block8_offset(dstart, r));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) carry = 0;
  __syncthreads();
  for (int base = 0; base < words; base += 4 * kScan8Threads) {
    const int w0 = base + 4 * tid;
    int c[4], mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int w = w0 + j;
      uint32_t v = w < words ? mask[woff + w] : 0u;
      if (w == words - 1 && (n & 31)) v &= (1u << (n & 31)) - 1u;
      c[j] = __popc(v);
      mine += c[j];
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += u;
    }
    if (lane == 31) warp_tot[warp] = inc;
    __syncthreads();
    if (warp == 0) {
      int t = warp_tot[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, t, o);
        if (lane >= o) t += u;
      }
      warp_tot[lane] = t;
    }
    __syncthreads();
    int run = carry + (warp ? warp_tot[warp - 1] : 0) + inc - mine;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (w0 + j < words) prefix[woff + w0 + j] = run;
      // the block whose first row is one of this word's
      const int b = (run + kBlock8 - 1) >> 6;
      if (b * kBlock8 < run + c[j] && b * kBlock8 < cap) my_note[b].word = w0 + j;
      run += c[j];
    }
    __syncthreads();
    if (tid == 0) carry += warp_tot[kScan8Threads / 32 - 1];
    __syncthreads();
  }
  const int m = min(carry, cap);
  const int before = r == 0 ? (int)block8_offset(dstart, 0) : 0;   // (slabs that do not start at slot 0)
  for (int b = tid - before; b < listed; b += kScan8Threads) {
    my_note[b].cnt = b < 0 ? 0 : min(kBlock8, m - b * kBlock8);    // (<= 0: no rows)
    my_note[b].words = words;
    my_note[b].row0 = b * kBlock8;
    *reinterpret_cast<int4*>(&my_note[b].r) = make_int4(r, start, dstart, 0);
  }
  if (tid == 0) {
    kv_len_out[r * Hkv + h] = m;
    if (carry > cap) { atomicExch(&status[0], GVOTE_ERR_WORKSPACE_TOO_SMALL); atomicExch(&status[1], 8); }
  }
}

struct StoreArgs {
  const void* src[2];            // K, V: bf16 or e4m3
  const float* src_scale[2];     // of an e4m3 source
  int64_t s_tok, s_head, s_total, s_row_blocks;
  const uint32_t* mask;          // or null: every row
  const int32_t* prefix;
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
    return top == top ? finite_abs(top * scale) : 0.f;
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
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t w = (&lo.x)[q];
      const float2 a = decode8x2(w & 0xffffu), b = decode8x2(w >> 16);
      (&out.x)[q] = encode8x2(a.x * scale * inv, a.y * scale * inv) | (encode8x2(b.x * scale * inv, b.y * scale * inv) << 16);
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
    const int4 note = *reinterpret_cast<const int4*>(&a.note[db]), where = *reinterpret_cast<const int4*>(&a.note[db].r);
    cnt = note.y; row0 = note.w; r = where.x; start = where.y; dstart = where.z;
    if (cnt <= 0) return;
    const int64_t woff = (int64_t)h * a.row_words + mask_word_offset(start, r);
    // thread = one bit of a word, four words per warp and round
    constexpr int kWarps = kStoreThreads / 32;
    const int lane = tid & 31;
    for (int base = note.x + (tid >> 5);; base += 4 * kWarps) {
      uint32_t bits[4];
      int rank[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int w = base + j * kWarps;
        bits[j] = w < note.z ? a.mask[woff + w] : 0u;
        rank[j] = w < note.z ? a.prefix[woff + w] - row0 : cnt;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // (bits behind the rows that count come after the last of the cnt ranks)
        const int mine = rank[j] + __popc(bits[j] & ((1u << lane) - 1u));
        if (((bits[j] >> lane) & 1u) && mine >= 0 && mine < cnt) s_src[mine] = (base + j * kWarps) * 32 + lane;
      }
      if (__syncthreads_or(rank[3] + __popc(bits[3]) >= cnt)) break;   // (ranks grow with the words)
    }
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
    const float scale = scale8_of(top), inv = inverse_pow2(scale);
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
  m.prefix = kStatusBytes;
  m.note = align_up(m.prefix + (size_t)p->n_kv_heads * gvote_mask_row_words(total_tokens, batch) * 4, 256);
  m.total = align_up(m.note + (size_t)p->n_kv_heads * gvote_cache8_row_blocks(total_tokens, batch) * sizeof(Note), 256);
  return m;
}

int32_t launch_store8(const gvote_params* p, const __nv_bfloat16* K, const __nv_bfloat16* V, int64_t tok, int64_t head,
                      const gvote_cache8* src8, const uint32_t* mask, const int32_t* cu, const int32_t* kv_len,
                      int32_t batch, int64_t total_tokens, const gvote_cache8* dst, const SideArrays& side, char* ws,
                      cudaStream_t st) {
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
  a.prefix = reinterpret_cast<const int32_t*>(ws + m.prefix);
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
    LaunchScope scope_("store8_scan_kernel", st);
    launch_on(store8_scan_kernel, dim3(Hkv, batch), dim3(kScan8Threads), 0, st, mask, cu, kv_len, Hkv, a.row_words,
              (int32_t*)(ws + m.prefix), a.cu8, a.d_row_blocks, (Note*)(ws + m.note), a.kv_len_out, a.status);
    GVOTE_LAUNCH_CHECK("store8_scan_kernel");
  }
  const unsigned ctas = (unsigned)(a.d_row_blocks * Hkv);
  return src8 ? run_store<true>(a, ctas, st) : run_store<false>(a, ctas, st);
}

}  // namespace gvote
