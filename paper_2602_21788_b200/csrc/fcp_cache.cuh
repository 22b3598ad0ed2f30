// Kernels on a paged cache of 8-bit keys and values: append, attention of the newest tokens, the weights it leaves, eviction.
#pragma once
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "fcp_cache_index.hpp"
#include "sm100_ptx.cuh"

namespace fcp {

// ---------------------------------------------------------------------------------------------
// Views and checks
// ---------------------------------------------------------------------------------------------
struct CacheView {
  uint8_t *k, *v;
  float *k_scale, *v_scale, *weight;
  int32_t* status;
  int32_t n_pages, page_tokens, page_shift, hkv;      // page_tokens = 1 << page_shift
};
struct BatchView {
  int32_t B, rows, max_new, table_width, capacity;     // capacity: tokens that a row of the page table can name
  const int32_t *page_table, *length, *row_offset;
  const int32_t* only;                                 // NULL, or one word per sequence: the others count as without new tokens
};

__device__ __forceinline__ int32_t ld_i32(const int32_t* p) {
  int32_t x;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(x) : "l"(p));
  return x;
}
__device__ __forceinline__ void mark_bad(int32_t* status, int32_t code, int32_t b) {
  if (atomicCAS(status, 0, FCP_ERR_INVALID_ARG) == 0) {
    status[1] = code;
    status[2] = b;
  }
}
__device__ __forceinline__ SeqView load_seq(const BatchView& s, int b) {
  SeqView v = seq_view(ld_i32(s.row_offset + b), ld_i32(s.row_offset + b + 1), ld_i32(s.length + b), s.rows, s.max_new, s.capacity);
  if (s.only && ld_i32(s.only + b) == 0) v.n = 0;
  return v;
}
__device__ __forceinline__ bool usable_scale(float x) { return x >= FCP_CACHE_MIN_SCALE && x <= FCP_CACHE_MAX_SCALE; }

// ---------------------------------------------------------------------------------------------
// Codes
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
// Two codes (the low or the high half of a word) -> two halves, exactly: e4m3 has 4 significant bits, int8 8, a half 11.
template <int KIND>
__device__ __forceinline__ uint32_t halves_lo(uint32_t w) {
  uint32_t r;
  if (KIND == FCP_CACHE_E4M3) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
    return r;
  }
  // byte + 128 under the exponent of 1024 is the half 1024 + 128 + value
  r = __byte_perm(w ^ 0x80808080u, 0x64646464u, 0x4140);
  return h2_bits(__hsub2(*reinterpret_cast<const __half2*>(&r), __float2half2_rn(1152.f)));
}
template <int KIND>
__device__ __forceinline__ uint32_t halves_hi(uint32_t w) {
  uint32_t r;
  if (KIND == FCP_CACHE_E4M3) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
    return r;
  }
  r = __byte_perm(w ^ 0x80808080u, 0x64646464u, 0x4342);
  return h2_bits(__hsub2(*reinterpret_cast<const __half2*>(&r), __float2half2_rn(1152.f)));
}
// Four values over their scale -> four codes, nearest, ties to even; too large ones the largest code.
template <int KIND>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  if (KIND == FCP_CACHE_E4M3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
  }
  auto one = [](float x) { return (uint32_t)min(127, max(-127, __float2int_rn(x))) & 0xffu; };       // NaN: 0
  return one(a) | (one(b) << 8) | (one(c) << 16) | (one(d) << 24);
}
// The same for finite values within the range of the codes, times the inverse of a power of two.  int8: added to 1.5 * 2^23 a value
// is rounded to an integer, ties to even, which the low byte holds; limits, shifts and conversions took 19 instructions a value.
template <int KIND>
__device__ __forceinline__ uint32_t small_codes(const float4& f, float inverse) {
  if (KIND == FCP_CACHE_E4M3) return to_codes<KIND>(f.x * inverse, f.y * inverse, f.z * inverse, f.w * inverse);
  const float magic = 12582912.f;
  const uint32_t a = __float_as_uint(fmaf(f.x, inverse, magic)), b = __float_as_uint(fmaf(f.y, inverse, magic));
  const uint32_t c = __float_as_uint(fmaf(f.z, inverse, magic)), d = __float_as_uint(fmaf(f.w, inverse, magic));
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
template <int KIND>
__device__ __forceinline__ uint32_t rescale_codes(uint32_t w, float ratio) {
  const uint32_t lo = halves_lo<KIND>(w), hi = halves_hi<KIND>(w);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  return to_codes<KIND>(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio);
}
// The same for a power of two of at most 1, in halves.  A code times it is exact, or below 2^-14, where e4m3 has nothing but 0; an
// int8 code times it plus 1.5 * 2^10 is rounded to an integer, which the low byte holds.
template <int KIND>
__device__ __forceinline__ uint32_t shrink_codes(uint32_t w, __half2 ratio) {
  const uint32_t lo = halves_lo<KIND>(w), hi = halves_hi<KIND>(w);
  const __half2 a = *reinterpret_cast<const __half2*>(&lo), b = *reinterpret_cast<const __half2*>(&hi);
  if (KIND == FCP_CACHE_E4M3) {
    const __half2 x = __hmul2(a, ratio), y = __hmul2(b, ratio);
    return (uint32_t)__nv_cvt_halfraw2_to_fp8x2(*reinterpret_cast<const __half2_raw*>(&x), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_halfraw2_to_fp8x2(*reinterpret_cast<const __half2_raw*>(&y), __NV_SATFINITE, __NV_E4M3) << 16;
  }
  const __half2 magic = __float2half2_rn(1536.f);
  return __byte_perm(h2_bits(__hfma2(a, ratio, magic)), h2_bits(__hfma2(b, ratio, magic)), 0x6420);
}
template <int KIND>
__device__ __forceinline__ uint4 moved_codes(const uint4& x, float ratio) {
  if (ratio == 1.f) return x;
  if ((__float_as_uint(ratio) & 0x7fffffu) == 0 && ratio < 1.f) {
    const __half2 r = __float2half2_rn(ratio);        // below 2^-24: 0, and so are the codes
    return make_uint4(shrink_codes<KIND>(x.x, r), shrink_codes<KIND>(x.y, r), shrink_codes<KIND>(x.z, r), shrink_codes<KIND>(x.w, r));
  }
  return make_uint4(rescale_codes<KIND>(x.x, ratio), rescale_codes<KIND>(x.y, ratio), rescale_codes<KIND>(x.z, ratio), rescale_codes<KIND>(x.w, ratio));
}
// |x| of a bf16 as ordered bits; infinities count as the largest finite value, NaN as 0
__device__ __forceinline__ uint32_t abs_bits(uint32_t h) {
  h &= 0x7fffu;
  return h > 0x7f80u ? 0u : min(h, 0x7f7fu);
}
// Smallest power of two s >= FCP_CACHE_MIN_SCALE with a / s <= the largest code; a: bits of a finite bf16.  From the exponent
// alone: 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6.
template <int KIND>
__device__ __forceinline__ float fresh_scale(uint32_t a) {
  const int e = (int)(a >> 7) - 127, top = KIND == FCP_CACHE_E4M3 ? 8 : 6;
  const uint32_t m = a & 0x7fu, most = KIND == FCP_CACHE_E4M3 ? 0x60u : 0x7eu;       // bf16 mantissas of 1.75 and 1.984375
  const int s = max(e - top + (m > most ? 1 : 0), -100);       // a subnormal a (e = -127) ends at the lower limit
  return __uint_as_float((uint32_t)(s + 127) << 23);
}
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// ---------------------------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------------------------
struct AppendArgs {
  CacheView c;
  BatchView s;
  const __nv_bfloat16 *k, *v;
  int64_t k_stride, v_stride;
  int32_t slots;
};

// Offsets that fall can keep the search below from a sequence, so one block looks at them all.  Out of line: within the kernel, whose blocks
// live for 2 us, it cost all of them 4 %.
__device__ __noinline__ void report_sequences(const BatchView& s, int32_t* status, int threads) {
  for (int b = threadIdx.x; b < s.B; b += threads) {
    const int32_t bad = load_seq(s, b).bad;
    if (bad) mark_bad(status, bad, b);
  }
}
// One piece of work per (page touched, head, K or V), for as many warps as give a thread N pieces of 16 values, which stay in
// registers between the maximum and the codes.  HBM bound: 64K tokens of 8 heads, pages of 64, int8: 70 us,
// 5.8 TB/s (pages of 16, a warp each: 73 us).
constexpr int append_warps(int page_tokens, int D, int N) { return page_tokens * D / (512 * N) < 1 ? 1 : page_tokens * D / (512 * N); }
__host__ __device__ constexpr int append_threads(int warps) { return 32 * (warps < 4 ? 4 : warps); }
template <int D, int KIND, int N, int WARPS>
__global__ void __launch_bounds__(append_threads(WARPS)) cache_append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int THREADS = append_threads(WARPS), GROUP = 32 * WARPS;        // of the block, of a piece of work
  __shared__ uint32_t warp_max[THREADS / 32];
  grid_begin();
  const int w = blockIdx.x, part = blockIdx.y * (THREADS / GROUP) + threadIdx.x / GROUP, h = part >> 1, tid = threadIdx.x % GROUP;
  const bool is_v = part & 1;
  const int page_tokens = a.c.page_tokens;
  int b = w;                                         // one token, one page: a slot per sequence
  if (a.s.max_new != 1) {
    // the last b whose first slot is at most w, by all threads: THREADS sequences a round
    int lo = 0, hi = a.s.B - 1;
    while (lo < hi) {
      const int step = (hi - lo + THREADS - 1) / THREADS, at = lo + ((int)threadIdx.x + 1) * step;
      const int below = __syncthreads_count(at <= hi && append_slot(ld_i32(a.s.row_offset + min(at, a.s.B - 1)), min(at, a.s.B - 1), page_tokens) <= w);
      lo += below * step;
      hi = min(hi, lo + step - 1);
    }
    b = lo;
    if (blockIdx.x == 0 && blockIdx.y == 0) report_sequences(a.s, a.c.status, THREADS);
  }
  if (h >= a.c.hkv) return;
  const SeqView sv = load_seq(a.s, b);
  const int slot = a.s.max_new == 1 ? 0 : w - append_slot(sv.row0, b, page_tokens);
  if (sv.bad) {
    if (tid == 0) mark_bad(a.c.status, sv.bad, b);
    return;
  }
  if (slot < 0) return;
  const AppendSpan sp = append_span(sv, slot, page_tokens);
  if (sp.lo >= sp.hi || sp.page >= a.s.table_width) return;
  const int32_t page = ld_i32(a.s.page_table + (int64_t)b * a.s.table_width + sp.page);
  const int held = sp.lo - sp.page * page_tokens, filled = sp.hi - sp.page * page_tokens;      // slots [held, filled) are new
  constexpr int C = D / 16;
  const __nv_bfloat16* x = (is_v ? a.v : a.k) + h * D;
  const int64_t stride = is_v ? a.v_stride : a.k_stride;
  const int64_t first = (int64_t)sv.row0 + sv.n - sv.length + (int64_t)sp.page * page_tokens;  // row of the page's slot 0
  uint4 r[N][2];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * GROUP + tid, s = e / C, c = e % C;
    r[i][0] = r[i][1] = make_uint4(0, 0, 0, 0);
    if (s >= held && s < filled) {
      const __nv_bfloat16* p = x + (first + s) * stride + c * 16;
      r[i][0] = ld_v4(p);
      r[i][1] = ld_v4(p + 8);
    }
  }
  const int32_t row = page_row(page, a.c.n_pages, a.c.hkv, h, page_tokens);
  const int32_t cell = page * a.c.hkv + h;
  float* scales = is_v ? a.c.v_scale : a.c.k_scale;
  float old = 0.f;
  if (row < 0) {
    if (tid == 0) mark_bad(a.c.status, FCP_CACHE_BAD_PAGE, b);
    return;
  }
  if (held > 0) old = ld_f32(scales + cell);
  auto group_sync = [&] {                            // also: every thread has read the old scale before one writes it
    // barrier numbers that the compiler sees: with one in a register a block takes all 16, which leaves room for few blocks (64K
    // tokens 98 us instead of 69)
    if (WARPS == 1) __syncwarp();
    else if (WARPS >= 4) __syncthreads();
    else if (threadIdx.x < GROUP) asm volatile("bar.sync 1, %0;" ::"n"(GROUP) : "memory");
    else asm volatile("bar.sync 2, %0;" ::"n"(GROUP) : "memory");
  };
  auto group_max = [&](uint32_t x) {
    x = __reduce_max_sync(0xffffffffu, x);
    if (WARPS == 1) return x;
    if ((tid & 31) == 0) warp_max[threadIdx.x >> 5] = x;
    group_sync();
#pragma unroll
    for (int i = 0; i < WARPS; ++i) x = max(x, warp_max[threadIdx.x / GROUP * WARPS + i]);
    return x;
  };
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(r[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) most = __vmaxu2(most, u[j] & 0x7fff7fffu);
  }
  most = group_max(max(most & 0xffffu, most >> 16));
  const bool odd = most >= 0x7f80u;                  // an infinity or a NaN on this page: again, with care
  if (odd) {
    most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t* u = reinterpret_cast<const uint32_t*>(r[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) most = max(most, max(abs_bits(u[j]), abs_bits(u[j] >> 16)));
    }
    group_sync();
    most = group_max(most);
  }
  uint8_t* codes = (is_v ? a.c.v : a.c.k) + (int64_t)row * D;
  float scale = fresh_scale<KIND>(most);
  if (held > 0) scale = fmaxf(old, scale);
  if (WARPS == 1) __syncwarp();
  if (tid == 0 && !(held > 0 && scale == old)) scales[cell] = scale;
  const float inverse = 1.f / scale;                 // exact for powers of two; x / scale otherwise below
  const bool exact = (__float_as_uint(scale) & 0x7fffffu) == 0;
  if (!is_v && a.c.weight)
    for (int s = held + tid; s < filled; s += GROUP) a.c.weight[(int64_t)row + s] = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * GROUP + tid, s = e / C, c = e % C;
    if (s >= held && s < filled) {
      const uint32_t* u = reinterpret_cast<const uint32_t*>(r[i]);
      uint32_t out[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 f = make_float4(bf_lo(u[2 * j]), bf_hi(u[2 * j]), bf_lo(u[2 * j + 1]), bf_hi(u[2 * j + 1]));
        out[j] = exact && !odd ? small_codes<KIND>(f, inverse)
                 : exact       ? to_codes<KIND>(f.x * inverse, f.y * inverse, f.z * inverse, f.w * inverse)
                               : to_codes<KIND>(__fdiv_rn(f.x, scale), __fdiv_rn(f.y, scale), __fdiv_rn(f.z, scale), __fdiv_rn(f.w, scale));
      }
      *reinterpret_cast<uint4*>(codes + s * D + c * 16) = make_uint4(out[0], out[1], out[2], out[3]);
    } else if (s < held && scale != old) {
      const float ratio = __fdiv_rn(old, scale);
      const uint4 u = ld_v4(codes + s * D + c * 16);
      *reinterpret_cast<uint4*>(codes + s * D + c * 16) = moved_codes<KIND>(u, ratio);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------------------------
// Bound by the cache's bytes as long as a KV head has few rows (new tokens times query heads of the KV head), so: every CTA
// takes the same number of key tiles, whatever the lengths (the tiles of all (sequence, KV head, row tile) groups in a row,
// cut evenly); codes come by TMA through a ring and go from shared memory straight into the fragments of 16 x 8 x 16 products
// of halves, which hold codes and probabilities exactly enough; a group that several CTAs share leaves one partial result
// per CTA, joined by a second kernel in a fixed order.
//
// Products by mma.sync, not tcgen05, up to 32 rows: a decode step has 1 to 16 rows per KV head, tcgen05 wants 64 or 128, and codes
// have to pass through registers to become halves anyway.  Keys and value columns are the 16-row operand, the rows the 8
// columns: S^T = K Q^T, O^T = V^T P^T, so that 8 rows (one token of 8 query heads) fill a product.
constexpr int CT_KEYS = 128;                          // keys of a tile
constexpr int CT_STEP = 32;                           // keys that a warp takes at a time
constexpr int CT_WARPS = 8;                           // consumer warps; two more load keys and values
constexpr int CT_THREADS = (CT_WARPS + 2) * 32;
constexpr int WEIGHT_CTAS = 2;                        // per SM, of the kernel that adds up weights

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A weight is 2^(a - ref), a the score plus y, the log2 of its value scale; the probabilities are the weights over the value scales.  With y
// from -100 (pages of zeros) to 122 (infinite values) neither the plain sum of the probabilities nor the weights of keys whose scale
// is small beside others' stay in fp32's range.  So:
//   - the sum is kept times 2^CT_SHIFT: between 2^(8 - 40 - 60), a row's largest weight alone with y = 60, and 2^(46 - 40 + 100), 2^31
//     weights of 2^15 with y = -100; in rows whose largest weight has a greater y, times 2^CT_SHIFT_HUGE (cache_tile_kernel, whose
//     warps hold parts of a row's sum under one reference: where the part asks for it);
//   - from the first tiles of a group on that hold keys whose y is 60 from another's, tiles are marked ST_APART, and from its first key with
//     y >= 60 on ST_HUGE besides: their probabilities get exponentials of their own, because the weights may vanish where the
//     probabilities do not.
// Against sums taken from the weights alone, us: one token of 64 sequences of 300 to 8K 76.8 -> 79.1, of one of 384K 129.9 -> 130.8; 25 rows
// per KV head 189 -> 178 (the step compiled twice, the marked form apart).  A running top scale in every step took 80.3 for the first and 4 % more for the second.
constexpr int CT_APART = 60, CT_HUGE = 60;
constexpr float CT_SHIFT = -40.f, CT_SHIFT_HUGE = 20.f, CT_UNIT = 0x1p-40f, CT_UNIT_HUGE = 0x1p20f;
// l times 2^e, for -250 < e < 250 where the result is in range; 0 stays 0
__device__ __forceinline__ float times_exp2(float l, float e) {
  const float half = exp2_approx(0.5f * e);
  return l * half * half;
}
// A sum times 2^CT_SHIFT_HUGE is passed on with a minus sign.
__device__ __forceinline__ float sum_shift(float l) { return l < 0.f ? CT_SHIFT_HUGE : CT_SHIFT; }
// The logarithm's error grows with its size, so the exponent goes by itself.
__device__ __forceinline__ float log2_split(float z) {
  const uint32_t u = __float_as_uint(z);
  return z < INFINITY ? (float)((int)(u >> 23) - 127) + __log2f(__uint_as_float((u & 0x7fffffu) | 0x3f800000u)) : z;
}

// A partial output may pass fp32's range where the whole one does not: an infinite value is stored as 448 * 2^120 or 127 * 2^122, and
// its weight may be 1 among one CTA's keys and 0 among all.  Partial outputs are held 2^-12 times: their sum over 148 CTAs then
// stays below 2^127, and the smallest bf16 keeps 11 bits.
constexpr float CT_PART_UNIT = 0x1p-12f;

struct AttnArgs {
  CacheView c;
  BatchView s;
  const __nv_bfloat16* q;
  int64_t q_stride;
  __nv_bfloat16* o;
  float* lse;
  float scale_log2;
  int32_t hq, group;                                  // group: query heads of a KV head
  int32_t box;                                        // keys of a TMA box
  float* part_o;                                      // workspace: [2 * CTAs][rows of a tile][D], [2 * CTAs][rows], [CTAs][SP_W]
  float* part_lse;
  int32_t* split;
};

struct StageMeta {                                    // what a stage holds, for the consumers
  int32_t row0, n, length, head;                      // of the sequence and group
  int32_t row_tile, key0, flags, part;
  // per 16 keys: key scale (0: absent), log2 and 2^CT_SHIFT times the inverse (ST_APART: 0) of the value scale, row of the first code (bits)
  float4 sub[CT_KEYS / 16];
};
enum { ST_FIRST = 1, ST_LAST = 2, ST_WHOLE = 4, ST_END = 8, ST_APART = 16, ST_HUGE = 32 };
enum { SP_COUNT = 0, SP_ROW0, SP_N, SP_HEAD, SP_ROW_TILE, SP_W = 8 };

// NR blocks of 8 rows per warp, WR warps side by side: 8 * NR * WR rows of a group (WR = 0: the weights, NR blocks at a time).
template <int D, int NR, int WR>
struct AttnSmem {
  static constexpr int BLOCKS = NR * (WR ? WR : 1), ROWS = 8 * BLOCKS;
  static constexpr int TILE = CT_KEYS * D;            // bytes of K or of V
  static constexpr int STAGE = WR ? 2 * TILE : TILE;
  static constexpr int STAGES = WR == 0 ? 4 : D == 64 ? 8 : NR == 2 ? 4 : 5;
  static constexpr int RING = STAGES * STAGE;
  // the queries of a group travel with its first tile where they are few; else the warps fetch them
  static constexpr int QUERY_BYTES = WR == 1 ? ROWS * D * 2 : 0;
  static constexpr int FRAGS = ROWS * D * 2;          // the queries as operands
  static constexpr int JOIN = WR == 0 ? 0 : CT_WARPS * 8 * NR * D * 4;           // the warps' partial outputs
  static constexpr int DYN_BYTES = RING + STAGES * QUERY_BYTES + FRAGS + JOIN + 1024;
};

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"(m), "r"(bar), "r"(c0), "r"(c1)
               : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// D (fp32) += A (16 x 16 halves) * B (16 x 8 halves)
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 halves held as (row g, columns 2t, 2t + 1) -> (column g, rows 2t, 2t + 1)
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) { return h2_bits(__floats2half2_rn(lo, hi)); }

// How the tiles of a batch lie in a row: sequence after sequence, its KV heads, their row tiles, their key tiles.
// A group counts for GROUP_COST tiles more than it has, for what its queries and its end take.  64 sequences of 300 to 8K tokens, 8 KV heads,
// us: 0 tiles 114, 1 tile 90, 2 tiles 78, 4 tiles 72 with pages of 128; 114, 90, 79, 82 with pages of 16.
struct TileOrder {
  static constexpr int GROUP_COST = 2;
  int32_t rows_per_tile, group, hkv;
  bool all_rows;                                      // one group per KV head, whatever its rows (the weights)
  __device__ __forceinline__ int32_t row_tiles(const SeqView& s) const {
    return s.n <= 0 ? 0 : all_rows ? 1 : (s.n * group + rows_per_tile - 1) / rows_per_tile;
  }
  __device__ __forceinline__ int32_t key_tiles(const SeqView& s) const { return s.length <= 0 ? 1 : (s.length + CT_KEYS - 1) / CT_KEYS; }
  __device__ __forceinline__ int64_t tiles(const SeqView& s) const { return (int64_t)row_tiles(s) * hkv * (key_tiles(s) + GROUP_COST); }
};

struct CtaRange {
  int64_t begin, end, per;                            // tiles of this CTA, tiles of every CTA
  int64_t seq_begin;                                  // first tile of sequence b
  int32_t b;
};

// All threads: the CTA's share of the tiles and the sequence it begins in.  Sequences that are not usable are reported by CTA 0.
__device__ __forceinline__ CtaRange cta_range(const BatchView& s, const TileOrder& order, int32_t* status, int64_t* scratch /* [16] */) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int64_t total = 0, mine = 0;
  for (int b0 = 0; b0 < s.B; b0 += CT_WARPS * 32) {
    const int b = b0 + tid;
    mine = 0;
    if (tid < CT_WARPS * 32 && b < s.B) {
      const SeqView v = load_seq(s, b);
      if (v.bad && blockIdx.x == 0) mark_bad(status, v.bad, b);
      mine = order.tiles(v);
    }
    int64_t sum = mine;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();
    if (lane == 0 && warp < CT_WARPS) scratch[warp] = sum;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < CT_WARPS; ++i) total += scratch[i];
  }
  CtaRange r;
  r.per = (total + gridDim.x - 1) / gridDim.x;
  r.begin = min(total, (int64_t)blockIdx.x * r.per);
  r.end = min(total, r.begin + r.per);
  int64_t running = 0;
  for (int b0 = 0; b0 < s.B; b0 += CT_WARPS * 32) {
    const int b = b0 + tid;
    if (s.B > CT_WARPS * 32) mine = tid < CT_WARPS * 32 && b < s.B ? order.tiles(load_seq(s, b)) : 0;
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    __syncthreads();
    if (lane == 31 && warp < CT_WARPS) scratch[warp] = upto;
    __syncthreads();
    int64_t before = running;
    for (int i = 0; i < CT_WARPS; ++i) {
      if (i < warp) before += scratch[i];
      running += scratch[i];
    }
    if (warp < CT_WARPS && r.begin < r.end && before + upto - mine <= r.begin && r.begin < before + upto) {
      scratch[8] = b;
      scratch[9] = before + upto - mine;
    }
  }
  __syncthreads();
  r.b = (int32_t)scratch[8];
  r.seq_begin = scratch[9];
  return r;
}

// The rows of a group's tile in shared memory: queries as the 8-column operand of S^T = K Q^T, and what goes with each row.
// Thread (g, t) of the operand holds row g of a block and of it the columns [t * D / 4, (t + 1) * D / 4): the sum over columns
// may be taken in any order, as long as queries and keys agree.  In registers they would take half a warp's budget.
struct RowInfo {
  float factor;                                       // score of the product -> log2 units, without the key scale
  int32_t limit;                                      // keys in front of this position are seen; 0: no such row
  float lse2;                                         // for the weights
  int32_t unused;
};
template <int D>
struct QueryArea {
  static constexpr int KS = D / 16;                   // steps of 16 columns
  uint2* frag;                                        // [block][KS][32 lanes]
  RowInfo* row;

  // Blocks of 8 rows from first_row on, a warp each.  `raw`: where the rows lie in shared memory; NULL: they are fetched.
  template <bool WEIGHTS>
  __device__ __forceinline__ void fill(const AttnArgs& A, const StageMeta& m, int first_row, int blocks, const uint8_t* raw, int warp, int lane) const {
    const int g = lane >> 2, t = lane & 3, n_rows = m.n * A.group;
    for (int i = warp; i < blocks; i += CT_WARPS) {
      const int r = first_row + 8 * i + g, j = r / A.group;
      const int64_t token = m.row0 + j;
      const int head = m.head * A.group + r - j * A.group;
      uint32_t w[D / 8];
      if (r < n_rows) {
        const __nv_bfloat16* p = A.q + token * A.q_stride + head * D + t * (D / 4);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const uint4 x = raw ? *reinterpret_cast<const uint4*>(raw + (8 * i + g) * (2 * D) + t * (D / 2) + c * 16) : ld_v4(p + c * 8);
          w[4 * c] = x.x; w[4 * c + 1] = x.y; w[4 * c + 2] = x.z; w[4 * c + 3] = x.w;
        }
      } else {
#pragma unroll
        for (int c = 0; c < D / 8; ++c) w[c] = 0;
      }
      // the row times a power of two that brings its largest value to [2^8, 2^9): a half then holds every bf16 down to
      // 2^-22 of the largest exactly
      uint32_t top = 0;
#pragma unroll
      for (int c = 0; c < D / 8; ++c) top = max(top, max(w[c] & 0x7fffu, (w[c] >> 16) & 0x7fffu));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = max((int)(top >> 7), 20);         // biased exponent; 20: smaller rows are taken as they are scaled then
      const float up = __uint_as_float((uint32_t)(262 - e) << 23);                     // 2^(8 - (e - 127)), e <= 255
#pragma unroll
      for (int k = 0; k < KS; ++k)
        frag[(i * KS + k) * 32 + lane] = make_uint2(pack_half(bf_lo(w[2 * k]) * up, bf_hi(w[2 * k]) * up),
                                                    pack_half(bf_lo(w[2 * k + 1]) * up, bf_hi(w[2 * k + 1]) * up));
      if (t == 0) {
        RowInfo x;
        x.factor = A.scale_log2 * __uint_as_float((uint32_t)(e - 8) << 23);            // 2^(e - 127 - 8)
        x.limit = r < n_rows ? m.length - m.n + j + 1 : 0;
        x.lse2 = WEIGHTS && r < n_rows ? ld_f32(A.lse + token * A.hq + head) * 1.4426950408889634f : INFINITY;
        x.unused = 0;
        row[8 * i + g] = x;
      }
    }
  }
};
// A barrier of the eight consumer warps that gives up like every other wait: a warp that has left may not hold up the others.
struct ConsumerSync {
  uint32_t bar, phase;
  __device__ __forceinline__ bool operator()(const WaitCtx& ctx, int lane, int where) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
    const bool ok = mbar_wait_warp(bar, phase, ctx, where);
    phase ^= 1;
    return ok;
  }
};

// 16 bytes `chunk` of key `key` of a tile, as TMA has swizzled them.
template <int D>
__device__ __forceinline__ const uint8_t* tile_at(const uint8_t* tile, int key, int chunk) {
  return D == 128 ? tile + key * 128 + ((chunk ^ (key & 7)) << 4) : tile + key * 64 + ((chunk ^ ((key >> 1) & 3)) << 4);
}
__device__ __forceinline__ void words(const uint8_t* p, uint32_t* w) {
  const uint4 x = *reinterpret_cast<const uint4*>(p);
  w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
}

// Scores of HB blocks of 16 keys from `key0` of the tile on, against NR blocks of rows: s[h][i] = (key g | g + 8) x (row 2t | 2t + 1).
template <int D, int KIND, int HB, int NR>
__device__ __forceinline__ void scores(const uint2* frag, const uint8_t* tile, int key0, int lane, float (&s)[HB][NR][4]) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int h = 0; h < HB; ++h)
#pragma unroll
    for (int i = 0; i < NR; ++i) s[h][i][0] = s[h][i][1] = s[h][i][2] = s[h][i][3] = 0.f;
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    uint32_t lo[HB][4], hi[HB][4];                    // of keys g and g + 8
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      words(tile_at<D>(tile, key0 + 16 * h + g, t * (D / 64) + c), lo[h]);
      words(tile_at<D>(tile, key0 + 16 * h + g + 8, t * (D / 64) + c), hi[h]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint2 b[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) b[i] = frag[(i * (D / 16) + 4 * c + k) * 32 + lane];
#pragma unroll
      for (int h = 0; h < HB; ++h) {
        const uint32_t a0 = halves_lo<KIND>(lo[h][k]), a1 = halves_lo<KIND>(hi[h][k]), a2 = halves_hi<KIND>(lo[h][k]), a3 = halves_hi<KIND>(hi[h][k]);
#pragma unroll
        for (int i = 0; i < NR; ++i) mma_f16(s[h][i], a0, a1, a2, a3, b[i].x, b[i].y);
      }
    }
  }
}

// A run of at most four tiles of one group, as the loading warp sees it.  Lane l stands for 16 keys of it: tile l / 8, sub-block l % 8.
struct TileRun {
  SeqView s;
  int32_t b, head, row_tile, tile, tiles, seen;       // seen: keys in front of this position are of use
  bool first, last, begins, ends;                     // of the group's tiles on this CTA; of the group
  int32_t page, row;                                  // this lane's page, and the row of its first code (-1: none)
  float ks, vs;
};

// A loading warp walks the CTA's tiles.  Page numbers are fetched two runs ahead, the scales they lead to one run ahead, so that
// the loop waits for neither; fetched when needed, the two in a row held the ring up for 1 to 2 us in every four tiles.
// S: the layout of shared memory (AttnSmem, TileSmem).
template <int D, class S, bool WEIGHTS>
struct AttnProducer {
  static constexpr int SUBS = CT_KEYS / 16;
  const AttnArgs& A;
  const TileOrder& order;
  const CtaRange& range;
  int64_t at, group_end;                              // next tile to hand out (in the order's units), end of its group
  int64_t seq_begin;
  SeqView s, ahead;                                   // of sequence b and of the next one
  int32_t b, kt, rt_n, head, rt, tile;
  bool fresh;                                         // no run handed out yet
  int32_t split[SP_W];

  __device__ __forceinline__ AttnProducer(const AttnArgs& A, const TileOrder& order, const CtaRange& range) : A(A), order(order), range(range) {
#pragma unroll
    for (int i = 0; i < SP_W; ++i) split[i] = 0;
    fresh = true;
    at = range.begin;
    seq_begin = range.seq_begin;
    b = range.b;
    if (at >= range.end) return;
    s = load_seq(A.s, b);
    look_ahead();
    enter();
  }
  __device__ __forceinline__ void look_ahead() {
    ahead = {0, 0, 0, 0};
    if (b + 1 < A.s.B) ahead = load_seq(A.s, b + 1);
  }
  // The group that `at` lies in.  It occupies GROUP_COST units more than it has tiles, the first ones.
  __device__ __forceinline__ void enter() {
    while (at >= seq_begin + order.tiles(s)) {
      seq_begin += order.tiles(s);
      ++b;
      s = ahead;
      look_ahead();
    }
    kt = order.key_tiles(s);
    rt_n = order.row_tiles(s);
    const int64_t rel = at - seq_begin, grp = rel / (kt + TileOrder::GROUP_COST);
    head = (int)(grp / rt_n);
    rt = (int)(grp - (int64_t)head * rt_n);
    group_end = seq_begin + (grp + 1) * (kt + TileOrder::GROUP_COST);
    at = max(at, group_end - kt);
    tile = kt - (int)(group_end - at);
  }
  // The next run, its pages on their way; false: none left.
  __device__ __forceinline__ bool next(TileRun& r, int lane) {
    if (at >= range.end) return false;
    const int left = (int)(min(group_end, range.end) - at);
    r.s = s;
    r.b = b;
    r.head = head;
    r.row_tile = rt;
    r.tile = tile;
    r.tiles = min(left, 4);
    r.begins = tile == 0;
    r.first = tile == 0 || fresh;
    fresh = false;
    r.last = r.tiles == left;
    r.ends = group_end <= range.end;
    const int last_row = min((rt + 1) * order.rows_per_tile, s.n * A.group) - 1;
    r.seen = WEIGHTS ? s.length : s.length - s.n + last_row / A.group + 1;
    const int key = (tile + lane / SUBS) * CT_KEYS + (lane % SUBS) * 16;
    r.page = -1;
    r.row = -2;                                       // nothing to load
    if (lane / SUBS < r.tiles && key < r.seen) {
      r.page = ld_i32(A.s.page_table + (int64_t)b * A.s.table_width + (key >> A.c.page_shift));
      r.row = key & (A.c.page_tokens - 1);
    }
    if (tile == 0 && !r.ends) {
      split[SP_COUNT] = (int)((group_end - 1) / range.per) - (int)blockIdx.x;
      split[SP_ROW0] = s.row0; split[SP_N] = s.n; split[SP_HEAD] = head; split[SP_ROW_TILE] = rt;
    }
    at += r.tiles;
    tile += r.tiles;
    if (at >= group_end && at < range.end) enter();
    return true;
  }
  __device__ __forceinline__ void fetch_scales(TileRun& r) {
    r.ks = r.vs = 0.f;
    if (r.row < 0) return;
    const int32_t at_page = page_row(r.page, A.c.n_pages, A.c.hkv, r.head, A.c.page_tokens);
    if (at_page < 0) {
      r.row = -1;
      return;
    }
    r.row += at_page;
    r.ks = ld_f32(A.c.k_scale + r.page * A.c.hkv + r.head);
    r.vs = ld_f32(A.c.v_scale + r.page * A.c.hkv + r.head);
  }

  // `map`, `ring`: of the keys, or of the values (is_v); the keys' warp also describes the stages and fetches the queries.
  __device__ __forceinline__ void run(const CUtensorMap* map, int is_v, uint32_t ring, uint32_t queries, StageMeta* meta, uint32_t full,
                                      uint32_t empty, const WaitCtx& ctx) {
    const int lane = threadIdx.x & 31, sub = lane & (SUBS - 1);
    const bool leads = (sub * 16) % A.box == 0;       // this lane's sub-block begins a box
    int stage = 0;
    uint32_t phase = 0;
    TileRun now, soon, later;
    bool have = next(now, lane), have_soon = have && next(soon, lane), have_later = false;
    if (have) fetch_scales(now);
    bool ok = true, whole = false, from_start = false;
    int top = 0, least = 255, apart = 0;              // largest and smallest biased exponent of a value scale of the group so far; marks
    while (have) {
      if (have_soon) fetch_scales(soon);
      have_later = have_soon && next(later, lane);
      const bool bad = now.row == -1 || (now.row >= 0 && (!usable_scale(now.ks) || !usable_scale(now.vs)));
      if (bad) {
        mark_bad(A.c.status, now.row == -1 ? FCP_CACHE_BAD_PAGE : FCP_CACHE_BAD_SCALE, now.b);
        now.row = -1;
      }
      const bool usable = now.row >= 0;
      if (!WEIGHTS && !is_v) {
        const int e = (int)(__float_as_uint(now.vs) >> 23);
        const int high = __reduce_max_sync(0xffffffffu, usable ? e : 0), low = __reduce_min_sync(0xffffffffu, usable ? e : 255);
        top = now.first ? high : max(top, high);
        least = now.first ? low : min(least, low);
        apart = (least + CT_APART < top ? ST_APART : 0) | (top >= 127 + CT_HUGE ? ST_APART | ST_HUGE : 0);
      }
      const float4 about = usable ? make_float4(now.ks, __log2f(now.vs), apart ? 0.f : CT_UNIT / now.vs, __int_as_float(now.row)) : make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = 0; i < now.tiles; ++i) {
        if (!mbar_wait_warp(empty + stage * 8, phase ^ 1, ctx, 911)) {
          ok = false;
          break;
        }
        const bool here = lane / SUBS == i, loads = here && leads && usable;
        const bool first = now.first && i == 0, last = now.last && i == now.tiles - 1;
        const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, loads));
        StageMeta& m = meta[stage];
        if (here && !is_v) m.sub[sub] = about;
        if (first) {
          from_start = now.begins;
          whole = now.begins && now.ends;
        }
        if (lane == 0 && !is_v) {
          m.row0 = now.s.row0; m.n = now.s.n; m.length = now.s.length; m.head = now.head;
          m.row_tile = now.row_tile;
          m.key0 = (now.tile + i) * CT_KEYS;
          m.flags = (first ? ST_FIRST : 0) | (last ? ST_LAST : 0) | (whole ? ST_WHOLE : 0) | apart;
          m.part = 2 * (int)blockIdx.x + (from_start ? 1 : 0);
        }
        __syncwarp();
        const uint32_t bar = full + stage * 8;
        // the queries of a group travel with its first tile, a row per lane
        const int row = now.row_tile * order.rows_per_tile + lane;
        const bool asks = S::QUERY_BYTES > 0 && !is_v && first && lane < order.rows_per_tile && row < now.s.n * A.group;
        const uint32_t rows = __popc(__ballot_sync(0xffffffffu, asks));
        if (lane == 0) {
          const uint32_t bytes = boxes * (uint32_t)(A.box * D) + rows * (uint32_t)(2 * D);
          if (bytes) mbar_expect_tx(bar, bytes);
          else mbar_arrive(bar);
        }
        __syncwarp();
        if (asks) {
          const int j = row / A.group;
          bulk_load(queries + (stage * order.rows_per_tile + lane) * (2 * D),
                    A.q + (int64_t)(now.s.row0 + j) * A.q_stride + (now.head * A.group + row - j * A.group) * D, 2 * D, bar);
        }
        if (loads) tma_load_2d(ring + stage * S::STAGE + sub * 16 * D, map, bar, 0, now.row);
        __syncwarp();
        if (++stage == S::STAGES) {
          stage = 0;
          phase ^= 1;
        }
      }
      if (!ok) break;
      now = soon;
      soon = later;
      have = have_soon;
      have_soon = have_later;
    }
    grid_launch_next();
    if (ok && mbar_wait_warp(empty + stage * 8, phase ^ 1, ctx, 912)) {
      if (lane == 0) {
        if (!is_v) meta[stage].flags = ST_END;
        mbar_arrive(full + stage * 8);
      }
    }
    if (!WEIGHTS && !is_v && lane < SP_W) {
      int32_t x = 0;
#pragma unroll
      for (int i = 0; i < SP_W; ++i) x = lane == i ? split[i] : x;
      A.split[blockIdx.x * SP_W + lane] = x;
    }
  }
};

// WR warps side by side (1 or 2) hold the rows of a tile, 8 * NR each; the 8 / WR warps behind each other take 32 keys each: of
// a tile, or with one warp side by side of every second tile.
template <int D, int KIND, int NR, int WR>
struct AttnConsumer {
  using S = AttnSmem<D, NR, WR>;
  static constexpr int RT = 8 * NR * WR, KG = CT_WARPS / WR, MT = D / 16;
  const uint2* frag;                                  // this warp's rows
  float factor[NR][2];                                // of rows 2t and 2t + 1 of each block
  int32_t limit[NR][2], least, most;                  // least, most: limits of the first and the last row that exist
  float o[NR][MT][4];                                 // O^T: block j of 16 columns: columns g MT*2 + 2j (| + 1) x rows 2t (| + 1)
  float ref[NR][2], l[NR][2];                         // weights are 2^(a - ref); sum of the probabilities, times 2^CT_SHIFT
  uint32_t huge;                                      // bit 2i + r: that row's sum is times 2^CT_SHIFT_HUGE
  __device__ __forceinline__ float shift(int i, int r) const { return huge >> (2 * i + r) & 1u ? CT_SHIFT_HUGE : CT_SHIFT; }

  // 32 keys from `key` (position) on, at `at` in the stage.  APART: of a tile with that mark; `with_huge`: with the other one.
  template <bool APART>
  __device__ __forceinline__ void step(const uint8_t* ktile, const uint8_t* vtile, int at, int key, const float4 (&about)[2], bool with_huge, int lane) {
    const int g = lane >> 2, t = lane & 3;
    float s[2][NR][4];
    scores<D, KIND, 2, NR>(frag, ktile, at, lane, s);
    // a = score in log2 units plus log2 of the value scale, so that 2^(a - ref) are the weights of the value codes, and the sum
    // of the probabilities is that of the weights over the value scale.  ref follows the largest a from 8 below it and is left
    // alone until a weight would pass 2^15: a half holds weights down to 2^-24, 2^-32 of the largest and less.
    const bool edge = key + 32 > least || about[0].x == 0.f || about[1].x == 0.f;
    float top[NR][2];
    bool high = false;
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float f = factor[i][r] * about[h].x;
          float &x = s[h][i][r], &y = s[h][i][r + 2];
          x = fmaf(x, f, about[h].y);
          y = fmaf(y, f, about[h].y);
          if (edge) {
            if (about[h].x == 0.f || key + 16 * h + g >= limit[i][r]) x = -INFINITY;
            if (about[h].x == 0.f || key + 16 * h + g + 8 >= limit[i][r]) y = -INFINITY;
          }
        }
        top[i][r] = fmaxf(fmaxf(s[0][i][r], s[0][i][r + 2]), fmaxf(s[1][i][r], s[1][i][r + 2]));
        high |= top[i][r] > ref[i][r] + 15.f;
      }
    if (__any_sync(0xffffffffu, high)) {
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float m = top[i][r];
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
          float rise = 0.f;
          if (APART && with_huge) {
            float at = -INFINITY;                     // the largest with such a value scale
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (about[h].y >= (float)CT_HUGE) at = fmaxf(at, fmaxf(s[h][i][r], s[h][i][r + 2]));
            at = fmaxf(at, __shfl_xor_sync(0xffffffffu, at, 4));
            at = fmaxf(at, __shfl_xor_sync(0xffffffffu, at, 8));
            at = fmaxf(at, __shfl_xor_sync(0xffffffffu, at, 16));
            if (at >= m && m - 8.f > ref[i][r] && shift(i, r) == CT_SHIFT) {
              rise = CT_SHIFT_HUGE - CT_SHIFT;
              huge |= 1u << (2 * i + r);
            }
          }
          m = fmaxf(ref[i][r], m - 8.f);
          // in two halves: the sum may outlast what o loses
          const float half = exp2_approx(0.5f * (ref[i][r] - m)), shrink = half * half;
          l[i][r] = APART ? times_exp2(l[i][r], ref[i][r] - m + rise) : l[i][r] * half * half;
          ref[i][r] = m;
#pragma unroll
          for (int j = 0; j < MT; ++j) {
            o[i][j][r] *= shrink;
            o[i][j][r + 2] *= shrink;
          }
        }
    }
    if (APART) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) l[i][c & 1] += about[h].x == 0.f ? 0.f : exp2_approx(s[h][i][c] - ref[i][c & 1] + (shift(i, c & 1) - about[h].y));
    }
    uint32_t p[2][NR][2];                             // P^T as the second operand: keys 2t, 2t + 1 (| + 8) x row g
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < NR; ++i) {
#pragma unroll
        for (int c = 0; c < 4; ++c) s[h][i][c] = exp2_approx(s[h][i][c] - ref[i][c & 1]);
        if (!APART) {
          l[i][0] = fmaf(s[h][i][0] + s[h][i][2], about[h].z, l[i][0]);
          l[i][1] = fmaf(s[h][i][1] + s[h][i][3], about[h].z, l[i][1]);
        }
        p[h][i][0] = transpose8(pack_half(s[h][i][0], s[h][i][1]));
        p[h][i][1] = transpose8(pack_half(s[h][i][2], s[h][i][3]));
      }
    // value codes: thread (g, t) reads columns [g D/8, (g + 1) D/8) of keys 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t v[4][D / 32];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int kk = at + 16 * h + 2 * t + (i & 1) + 8 * (i >> 1);
        if (D == 128) {
          words(tile_at<D>(vtile, kk, g), v[i]);
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(tile_at<D>(vtile, kk, g >> 1) + (g & 1) * 8);
          v[i][0] = x.x;
          v[i][1] = x.y;
        }
      }
      if (edge) {
        // What lies behind the last key that any row sees is whatever the page held, and a NaN of a new token must reach the
        // rows that see it and no other: neither may meet a zero weight.
        bool any = false;
        uint32_t nan[4][D / 32];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool past = about[h].x == 0.f || key + 16 * h + 2 * t + (i & 1) + 8 * (i >> 1) >= most;
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            if (past) v[i][c] = 0;
            if (KIND == FCP_CACHE_E4M3) {
              nan[i][c] = __vcmpeq4(v[i][c] & 0x7f7f7f7fu, 0x7f7f7f7fu);
              any |= nan[i][c] != 0;
              v[i][c] &= ~nan[i][c];
            }
          }
        }
        if (KIND == FCP_CACHE_E4M3 && __any_sync(0xffffffffu, any)) {
          // ones where a value is NaN times ones where a row sees the key: NaN where the product is not 0
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            uint32_t sees[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int pos = key + 16 * h + g + 8 * k;
              sees[k] = transpose8(pack_half(pos < limit[i][0] ? 1.f : 0.f, pos < limit[i][1] ? 1.f : 0.f));
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const uint32_t b0 = __byte_perm(nan[0][c], nan[1][c], e ? 0x7362 : 0x5140) & 0x38383838u;
                const uint32_t b1 = __byte_perm(nan[2][c], nan[3][c], e ? 0x7362 : 0x5140) & 0x38383838u;
                float d[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(d, halves_lo<KIND>(b0), halves_hi<KIND>(b0), halves_lo<KIND>(b1), halves_hi<KIND>(b1), sees[0], sees[1]);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  if (d[r] != 0.f) o[i][2 * c + e][r] = __int_as_float(0x7fffffff);
              }
          }
        }
      }
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          // bytes of two keys side by side: columns 4c + 2e (low half) and 4c + 2e + 1 of the thread's run
          const uint32_t b0 = __byte_perm(v[0][c], v[1][c], e ? 0x7362 : 0x5140), b1 = __byte_perm(v[2][c], v[3][c], e ? 0x7362 : 0x5140);
          const uint32_t a0 = halves_lo<KIND>(b0), a1 = halves_hi<KIND>(b0), a2 = halves_lo<KIND>(b1), a3 = halves_hi<KIND>(b1);
#pragma unroll
          for (int i = 0; i < NR; ++i) mma_f16(o[i][2 * c + e], a0, a1, a2, a3, p[h][i][0], p[h][i][1]);
        }
    }
  }

  // Place of 16 bytes `f` of a row of the join area, spread over the banks.
  __device__ static __forceinline__ int join_slot(int row, int f) {
    const int t = (row >> 1) & 3;
    return row * (D / 4) + (D == 128 ? f ^ t : f ^ ((t & 1) | (t >> 1) << 2));
  }

  // The end of a group's tiles on this CTA: joins the warps and writes the rows, or their partial result.
  __device__ __forceinline__ bool finish(const AttnArgs& A, const StageMeta& meta, float4* join, float2* stats, ConsumerSync& sync, const WaitCtx& ctx, int warp,
                                         int lane) {
    const int g = lane >> 2, t = lane & 3, tid = warp * 32 + lane;
    if (!sync(ctx, lane, 923)) return false;          // the join area's last readers are done
    float4* mine = join + warp * 8 * NR * (D / 4);
    const int n_rows = min(RT, meta.n * A.group - meta.row_tile * RT);
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l[i][r] += __shfl_xor_sync(0xffffffffu, l[i][r], 4);
        l[i][r] += __shfl_xor_sync(0xffffffffu, l[i][r], 8);
        l[i][r] += __shfl_xor_sync(0xffffffffu, l[i][r], 16);
        const int row = 8 * i + 2 * t + r;
        if (warp % WR * 8 * NR + row >= n_rows) continue;
        if (g == 0) stats[warp * 8 * NR + row] = make_float2(ref[i][r], shift(i, r) == CT_SHIFT ? l[i][r] : -l[i][r]);
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
          mine[join_slot(row, g * (D / 32) + c)] = make_float4(o[i][2 * c][r], o[i][2 * c][r + 2], o[i][2 * c + 1][r], o[i][2 * c + 1][r + 2]);
      }
    if (!sync(ctx, lane, 924)) return false;
    for (int e = tid; e < n_rows * (D / 4); e += CT_WARPS * 32) {
      const int r = e / (D / 4), f = e % (D / 4), wr = r / (8 * NR), row = r % (8 * NR);
      float top = -3e38f, shift = CT_SHIFT;
#pragma unroll
      for (int k = 0; k < KG; ++k) top = fmaxf(top, stats[(k * WR + wr) * 8 * NR + row].x);
      float z = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < KG; ++k) {
        const float2 ml = stats[(k * WR + wr) * 8 * NR + row];
        const float w = exp2_approx(ml.x - top);
        const float4 y = join[(k * WR + wr) * 8 * NR * (D / 4) + join_slot(row, f)];
        z = fmaf(ml.y, w, z);
        x.x = fmaf(y.x, w, x.x); x.y = fmaf(y.y, w, x.y); x.z = fmaf(y.z, w, x.z); x.w = fmaf(y.w, w, x.w);
      }
      if (meta.flags & ST_APART) {                    // sums in different units, or beside which w vanishes
        z = 0.f;
#pragma unroll 1
        for (int k = 0; k < KG; ++k) shift = fmaxf(shift, sum_shift(stats[(k * WR + wr) * 8 * NR + row].y));
#pragma unroll 1
        for (int k = 0; k < KG; ++k) {
          const float2 ml = stats[(k * WR + wr) * 8 * NR + row];
          z += times_exp2(fabsf(ml.y), ml.x - top + (shift - sum_shift(ml.y)));
        }
      }
      const float inverse = z == 0.f ? 0.f : 1.f / z;
      const float lse2 = z == 0.f ? -INFINITY : top - shift + log2_split(z);
      const float unit = (shift == CT_SHIFT ? CT_UNIT : CT_UNIT_HUGE) * (meta.flags & ST_WHOLE ? 1.f : CT_PART_UNIT);
      x.x = x.x * inverse * unit; x.y = x.y * inverse * unit; x.z = x.z * inverse * unit; x.w = x.w * inverse * unit;
      if (meta.flags & ST_WHOLE) {
        const int gr = meta.row_tile * RT + r, j = gr / A.group;
        const int64_t out = (int64_t)(meta.row0 + j) * A.hq + meta.head * A.group + gr - j * A.group;
        *reinterpret_cast<uint2*>(A.o + out * D + f * 4) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
        if (f == 0) A.lse[out] = lse2 * 0.69314718055994531f;
      } else {
        *reinterpret_cast<float4*>(A.part_o + ((int64_t)meta.part * RT + r) * D + f * 4) = x;
        if (f == 0) A.part_lse[(int64_t)meta.part * RT + r] = lse2;
      }
    }
    return true;
  }

  __device__ __forceinline__ void run(const AttnArgs& A, const uint8_t* ring, const uint8_t* queries, const QueryArea<D>& area, const StageMeta* metas, float4* join, float2* stats,
                                      uint32_t full, uint32_t empty, ConsumerSync sync, const WaitCtx& ctx) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wr = warp % WR, kg = warp / WR;
    const int turn = WR == 1 ? kg >> 2 : 0, i = WR == 1 ? kg & 3 : kg;       // which tiles, which 32 keys of them
    int stage = 0, tile = 0;
    uint32_t phase = 0;
    frag = area.frag + wr * NR * (D / 16) * 32;
    while (mbar_wait_warp(full + stage * 8, phase, ctx, 921)) {
      const StageMeta& meta = metas[stage];
      const int flags = meta.flags;
      if (flags & ST_END) break;
      if (flags & ST_FIRST) {
        area.template fill<false>(A, meta, meta.row_tile * RT, S::BLOCKS, S::QUERY_BYTES ? queries + stage * S::QUERY_BYTES : nullptr, warp, lane);
        if (!sync(ctx, lane, 922)) break;
        const int first_row = meta.row_tile * RT + wr * 8 * NR, n_rows = meta.n * A.group;
        const int last_row = min(first_row + 8 * NR, n_rows) - 1;
        least = meta.length - meta.n + first_row / A.group + 1;
        huge = 0;
        most = first_row < n_rows ? meta.length - meta.n + last_row / A.group + 1 : 0;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const RowInfo x = area.row[(wr * NR + i) * 8 + 2 * (lane & 3) + r];
            factor[i][r] = x.factor;
            limit[i][r] = x.limit;
          }
          ref[i][0] = ref[i][1] = -3e38f;
          l[i][0] = l[i][1] = 0.f;
#pragma unroll
          for (int j = 0; j < MT; ++j) o[i][j][0] = o[i][j][1] = o[i][j][2] = o[i][j][3] = 0.f;
        }
      }
      if (WR > 1 || (tile & 1) == turn) {
        const uint8_t* ktile = ring + stage * S::STAGE;
        const int key = meta.key0 + i * CT_STEP;
        const float4 about[2] = {meta.sub[2 * i], meta.sub[2 * i + 1]};
        if (key < most && (about[0].x != 0.f || about[1].x != 0.f)) {
          if (!(flags & ST_APART)) step<false>(ktile, ktile + S::TILE, i * CT_STEP, key, about, false, lane);
          else step<true>(ktile, ktile + S::TILE, i * CT_STEP, key, about, flags & ST_HUGE, lane);
        }
      }
      if ((flags & ST_LAST) && !finish(A, meta, join, stats, sync, ctx, warp, lane)) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(empty + stage * 8);
      ++tile;
      if (++stage == S::STAGES) {
        stage = 0;
        phase ^= 1;
      }
    }
  }
};

// Weights of the cached keys: the scores once more, against the finished log-sum-exps.  A warp holds 16 keys and goes over the
// rows in blocks of 8, NR blocks in shared memory at a time, so that a key's sum is taken by four threads in a fixed order.
template <int D, int KIND, int NR>
__device__ __forceinline__ void weight_consumer(const AttnArgs& A, const uint8_t* ring, const QueryArea<D>& area, const StageMeta* metas,
                                                uint32_t full, uint32_t empty, ConsumerSync sync, const WaitCtx& ctx) {
  using S = AttnSmem<D, NR, 0>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  int stage = 0;
  uint32_t phase = 0;
  while (mbar_wait_warp(full + stage * 8, phase, ctx, 931)) {
    const StageMeta& meta = metas[stage];
    if (meta.flags & ST_END) break;
    const int key = meta.key0 + warp * 16, n_rows = meta.n * A.group;
    const float4 about = meta.sub[warp];
    float sum[2] = {0.f, 0.f};                        // of keys g and g + 8
#pragma unroll 1
    for (int r0 = 0; r0 < n_rows; r0 += 8 * NR) {
      const int blocks = min(NR, (n_rows - r0 + 7) / 8), least = meta.length - meta.n + r0 / A.group + 1;
      if (n_rows > 8 * NR || (meta.flags & ST_FIRST)) {
        if (!sync(ctx, lane, 932)) return;            // the rows before have been read
        area.template fill<true>(A, meta, r0, (blocks + 3) / 4 * 4, nullptr, warp, lane);
        if (!sync(ctx, lane, 933)) return;
      }
      if (key >= meta.length || about.x == 0.f) continue;
      uint32_t a[D / 16][4];                          // the keys as operands
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        uint32_t lo[4], hi[4];
        words(tile_at<D>(ring + stage * S::STAGE, warp * 16 + g, t * (D / 64) + c), lo);
        words(tile_at<D>(ring + stage * S::STAGE, warp * 16 + g + 8, t * (D / 64) + c), hi);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          a[4 * c + k][0] = halves_lo<KIND>(lo[k]);
          a[4 * c + k][1] = halves_lo<KIND>(hi[k]);
          a[4 * c + k][2] = halves_hi<KIND>(lo[k]);
          a[4 * c + k][3] = halves_hi<KIND>(hi[k]);
        }
      }
      // four blocks side by side, so that a product need not wait for the one before it (blocks behind the last hold no rows)
#pragma unroll 1
      for (int i0 = 0; i0 < blocks; i0 += 4) {
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint2 x = area.frag[((i0 + i) * (D / 16) + k) * 32 + lane];
            mma_f16(s[i], a[k][0], a[k][1], a[k][2], a[k][3], x.x, x.y);
          }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i0 + i >= blocks) break;
          const RowInfo rows[2] = {area.row[8 * (i0 + i) + 2 * t], area.row[8 * (i0 + i) + 2 * t + 1]};
          const float f[2] = {rows[0].factor * about.x, rows[1].factor * about.x};
#pragma unroll
          for (int c = 0; c < 4; ++c) s[i][c] = fmaf(s[i][c], f[c & 1], -rows[c & 1].lse2);
          if (key + 16 > least) {                     // some row may not see some key
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (key + g + 8 * (c >> 1) >= rows[c & 1].limit) s[i][c] = -INFINITY;
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) sum[c >> 1] += exp2_approx(s[i][c]);
        }
      }
    }
    if (key < meta.length && about.x != 0.f) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], 1);
        sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], 2);
      }
      // one addition per place and call, so the result does not depend on any order; as an atomic it is not waited for
      if (t < 2 && key + g + 8 * t < meta.length) atomicAdd(A.c.weight + (int64_t)__float_as_int(about.w) + g + 8 * t, t ? sum[1] : sum[0]);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty + stage * 8);
    if (++stage == S::STAGES) {
      stage = 0;
      phase ^= 1;
    }
  }
}

// WR = 0: the weights, of NR blocks of rows at a time.
template <int D, int KIND, int NR, int WR>
__global__ void __launch_bounds__(CT_THREADS, WR == 0 ? WEIGHT_CTAS : 1)
cache_attn_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv, const __grid_constant__ AttnArgs A) {
  using S = AttnSmem<D, NR, WR>;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[2 * S::STAGES + 1];
  __shared__ __align__(16) StageMeta metas[S::STAGES];
  __shared__ float2 stats[WR ? CT_WARPS * 8 * NR : 1];
  __shared__ __align__(16) RowInfo rows[S::ROWS];
  __shared__ int64_t scratch[16];
  __shared__ int abort_flag;
  const int warp = threadIdx.x >> 5;
  const uint32_t full = smem_u32(bars), empty = full + S::STAGES * 8;
  const ConsumerSync sync = {empty + S::STAGES * 8, 0};
  // the swizzle pattern repeats every 1024 bytes of address
  const uint32_t skip = (1024u - (smem_u32(smem) & 1023u)) & 1023u;
  uint8_t* ring = smem + skip;
  uint8_t* queries = ring + S::RING;
  const QueryArea<D> area = {reinterpret_cast<uint2*>(queries + S::STAGES * S::QUERY_BYTES), rows};
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < S::STAGES; ++i) {
      mbar_init(full + i * 8, WR ? 2 : 1);
      mbar_init(empty + i * 8, CT_WARPS);
    }
    mbar_init(sync.bar, CT_WARPS);
    fence_mbar_init();
    prefetch_tmap(&tk);
    prefetch_tmap(&tv);
  }
  grid_wait();
  __syncthreads();
  const WaitCtx ctx = {&abort_flag, A.c.status, (uint32_t)FCP_WAIT_NS};
  const TileOrder order = {8 * NR * (WR ? WR : 1), A.group, A.c.hkv, WR == 0};
  const CtaRange range = cta_range(A.s, order, A.c.status, scratch);
  if (warp >= CT_WARPS) {
    AttnProducer<D, S, WR == 0> producer(A, order, range);
    if (warp == CT_WARPS || WR > 0) producer.run(warp == CT_WARPS ? &tk : &tv, warp - CT_WARPS, smem_u32(ring) + (warp - CT_WARPS) * S::TILE, smem_u32(queries), metas, full, empty, ctx);
  } else if constexpr (WR == 0) {
    weight_consumer<D, KIND, NR>(A, ring, area, metas, full, empty, sync, ctx);
  } else {
    AttnConsumer<D, KIND, NR, WR> consumer;
    consumer.run(A, ring, queries, area, metas, reinterpret_cast<float4*>(queries + S::STAGES * S::QUERY_BYTES + S::FRAGS), stats, full, empty, sync, ctx);
  }
  __syncthreads();
  wait_teardown(ctx);
}

// ---------------------------------------------------------------------------------------------
// Attention of tiles of up to 128 rows
// ---------------------------------------------------------------------------------------------
// From 33 rows per KV head on the products go to tcgen05: eight warps turn a tile's codes into halves in shared memory, once for
// all rows, S = Q K^T and O += P V run on 128 rows whether they are all there or not (1024 clk per tile of 128 keys, D = 128), and
// sixteen warps keep the softmax, a quarter of a row per thread, with P and O in tensor memory.  A tile takes about 4400 clk, neither
// the products' nor the bytes' time: codes to halves (2000 to 3000 clk), the softmax warps' way from S to P (of it 1000 for the
// exponentials) and the products wait for one another.  16 sequences of 4K to 32K tokens, 40/8 heads, us: 224 for 35 rows, 237 for 100 rows
// per KV head with int8, 218 and 235 with e4m3; cache_attn_kernel takes 325 and 645, 286 and 569.
// Tried, with eight softmax warps: 222, 236 with int8 and 247 for 100 rows with e4m3; V's halves in one buffer 253 for 35 rows; masking rows that do not
// exist 245; the next scores fetched before P is handed over 232; even and odd tiles to four softmax warps each, with an output of
// their own, 264; polling in front of waits 228; halves made before their place is free 221, e4m3 249.  Four converting warps for K
// and four for V took 142 against 111 (4 sequences, 64 new tokens).
//   warps 0..7    codes -> halves: queries at the start of a group, K of tile t, V of tile t - 1
//   warps 8, 9    the loading warps above
//   warp 10       issues the products: S of tile t, then O += P V of tile t - 1
//   warps 12..27  softmax and output: four per quarter of the tensor memory's lanes, each with 32 of a tile's columns
// Tensor memory: S of two tiles in turn | P of two tiles | O.
constexpr int TILE_THREADS = 896;
constexpr int TILE_ROWS = 128;
constexpr int TILE_CONVERT = 8;                       // converting warps
constexpr int TILE_RING = 8;                          // what goes with a tile: nobody is more than four behind; with a group: three
constexpr int TILE_GROUPS = 4;
template <int D>
struct TileSmem {
  // codes of K and of V in rings of their own; halves of a tile of K, of two of V in turn, and the queries
  static constexpr int TILE = CT_KEYS * D, STAGE = TILE, STAGES = D == 64 ? 5 : 2, QUERY_BYTES = 0;
  static constexpr int RING = STAGES * STAGE, HALVES = 128 * D * 2;
  static constexpr int DYN_BYTES = 2 * RING + 4 * HALVES + 1024;
};
struct TileMeta {
  int32_t flags, key0, row0, n, length, head, row_tile, part;
  float4 sub[CT_KEYS / 16];                           // as in StageMeta
};
struct TileGroup {                                    // of a group's rows
  float factor[TILE_ROWS];
  int32_t limit[TILE_ROWS];
  int32_t least, nan_any;
};

// Instruction descriptor like make_idesc, for halves.
__host__ __device__ constexpr uint32_t make_idesc_f16(int M, int N, int b_mn_major) {
  return (1u << 4) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// 16 codes -> 32 bytes of halves at columns [16 c, 16 c + 16) of row r of a tile of [128][64]-element swizzled blocks.
template <int D, int KIND>
__device__ __forceinline__ void put_halves(uint8_t* tile, int r, int c, const uint32_t (&w)[4]) {
  const uint4 lo = make_uint4(halves_lo<KIND>(w[0]), halves_hi<KIND>(w[0]), halves_lo<KIND>(w[1]), halves_hi<KIND>(w[1]));
  const uint4 hi = make_uint4(halves_lo<KIND>(w[2]), halves_hi<KIND>(w[2]), halves_lo<KIND>(w[3]), halves_hi<KIND>(w[3]));
  uint8_t* row = tile + (c >> 2) * 16384 + r * 128;
  const int a = ((c & 3) * 2) ^ (r & 7);
  // lanes of the second block write their upper half first, so that eight lanes cover all banks
  const bool swap = c >> 2;
  *reinterpret_cast<uint4*>(row + ((swap ? a ^ 1 : a) << 4)) = swap ? hi : lo;
  *reinterpret_cast<uint4*>(row + ((swap ? a : a ^ 1) << 4)) = swap ? lo : hi;
}

template <int D, int KIND>
__global__ void __launch_bounds__(TILE_THREADS, 1)
cache_tile_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv, const __grid_constant__ AttnArgs A) {
  using S = TileSmem<D>;
  constexpr uint32_t S_COL = 0, P_COL = 256, O_COL = 384;      // P: 64 columns for every other tile
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[4 * S::STAGES + 19];
  __shared__ __align__(16) StageMeta stages[S::STAGES];
  __shared__ __align__(16) TileMeta tiles[TILE_RING];
  __shared__ TileGroup groups[TILE_GROUPS];
  constexpr bool NANS = KIND == FCP_CACHE_E4M3;
  __shared__ uint16_t nans[NANS ? TILE_GROUPS : 1][NANS ? 128 : 1][D / 16];       // columns that are NaN in the keys from `least` on
  __shared__ int64_t scratch[16];
  __shared__ int abort_flag;
  __shared__ float tops[2][4][TILE_ROWS], sums[4][TILE_ROWS];
  __shared__ uint32_t tmem_slot;
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t full = smem_u32(bars), empty = full + 2 * S::STAGES * 8, bar0 = empty + 2 * S::STAGES * 8;         // K's, then V's
  // two of each but one, for even and odd tiles: a waiter may be two tiles behind, which one phase bit does not tell
  const uint32_t v_full = bar0, k_full = bar0 + 16, k_free = bar0 + 32, s_full = bar0 + 48, s_free = bar0 + 64, p_full = bar0 + 80, pv_done = bar0 + 96;
  ConsumerSync sync = {bar0 + 112, 0};
  const uint32_t quartet = bar0 + 120;                // the four softmax warps of a quarter, four times
  const uint32_t skip = (1024u - (smem_u32(smem) & 1023u)) & 1023u;
  uint8_t* ring = smem + skip;
  uint8_t* k16 = ring + 2 * S::RING;
  uint8_t* v16 = k16 + S::HALVES;
  uint8_t* q16 = v16 + 2 * S::HALVES;
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < 2 * S::STAGES; ++i) {
      mbar_init(full + i * 8, 1);
      mbar_init(empty + i * 8, TILE_CONVERT);
    }
    mbar_init(sync.bar, TILE_CONVERT);
    for (int i = 0; i < 4; ++i) mbar_init(quartet + i * 8, 4);
    for (int i = 0; i < 2; ++i) {
      mbar_init(k_full + i * 8, TILE_CONVERT);
      mbar_init(v_full + i * 8, TILE_CONVERT);
      mbar_init(k_free + i * 8, 1);
      mbar_init(p_full + i * 8, 16);
      mbar_init(pv_done + i * 8, 2);
      mbar_init(s_full + i * 8, 2);
      mbar_init(s_free + i * 8, 16);
    }
    fence_mbar_init();
    prefetch_tmap(&tk);
    prefetch_tmap(&tv);
  }
  if (warp == 10) {
    tmem_alloc(smem_u32(&tmem_slot), 512);
    tmem_relinquish();
  }
  grid_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const WaitCtx ctx = {&abort_flag, A.c.status, (uint32_t)FCP_WAIT_NS};
  const TileOrder order = {TILE_ROWS, A.group, A.c.hkv, false};
  const CtaRange range = cta_range(A.s, order, A.c.status, scratch);
  if (warp < TILE_CONVERT) {
    // ------------------------------------------------------------------ codes -> halves
    // K of tile t comes before V of tile t - 1: its product does not wait for anything that V's does
    int seg = -1, k_stage = 0, v_stage = 0, v_seg = 0, v_least = 0, v_most = 0, v_key0 = 0, next_least = 0, next_most = 0;
    float v_scale = 0.f;                              // key scale of this warp's 16 keys of the tile whose V is next; 0: absent
    uint32_t k_phase = 0, v_phase = 0;
    constexpr int KEYS = CT_KEYS / TILE_CONVERT, C = D / 16, PER = KEYS * C / 32;        // pieces of 16 codes per lane and tile
    for (int t = 0;; ++t) {
      if (!mbar_wait_warp(full + k_stage * 8, k_phase, ctx, 941)) break;
      const StageMeta& meta = stages[k_stage];
      const int flags = meta.flags, key0 = meta.key0;
      const float scale = meta.sub[warp].x;
      if (t > 0 && !mbar_wait_warp(k_free + ((t - 1) & 1) * 8, ((t - 1) >> 1) & 1, ctx, 944)) break;
      TileMeta& tile = tiles[t % TILE_RING];
      if (warp == 0) {
        if (lane < CT_KEYS / 16) tile.sub[lane] = meta.sub[lane];
        if (lane == 0) {
          tile.flags = flags; tile.key0 = meta.key0; tile.row0 = meta.row0; tile.n = meta.n; tile.length = meta.length;
          tile.head = meta.head; tile.row_tile = meta.row_tile; tile.part = meta.part;
        }
      }
      if (!(flags & ST_END)) {
        if (flags & ST_FIRST) {
          ++seg;
          TileGroup& grp = groups[seg % TILE_GROUPS];
          const int n_rows = meta.n * A.group, row0 = meta.row_tile * TILE_ROWS, last = min(row0 + TILE_ROWS, n_rows) - 1;
          next_least = meta.length - meta.n + row0 / A.group + 1;
          next_most = meta.length - meta.n + last / A.group + 1;
          if (NANS) {
            for (int i = threadIdx.x; i < 128 * C; i += TILE_CONVERT * 32) (&nans[seg % TILE_GROUPS][0][0])[i] = 0;
            if (threadIdx.x == 0) {
              grp.least = next_least;
              grp.nan_any = 0;
            }
            if (!sync(ctx, lane, 946)) break;         // in front of any warp's values of this group
          }
          // a row at a time; times a power of two as in QueryArea
#pragma unroll 4
          for (int i = 0; i < TILE_ROWS / TILE_CONVERT; ++i) {
            const int r = warp * (TILE_ROWS / TILE_CONVERT) + i, row = row0 + r, j = row / A.group;
            uint2 x = make_uint2(0, 0);
            if (row < n_rows) {
              const __nv_bfloat16* p = A.q + (int64_t)(meta.row0 + j) * A.q_stride + (meta.head * A.group + row - j * A.group) * D;
              if (D == 128) asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "l"(p + 4 * lane));
              else asm volatile("ld.global.u32 %0, [%1];" : "=r"(x.x) : "l"(p + 2 * lane));
            }
            uint32_t top = max(max(x.x & 0x7fffu, (x.x >> 16) & 0x7fffu), max(x.y & 0x7fffu, (x.y >> 16) & 0x7fffu));
            top = __reduce_max_sync(0xffffffffu, top);
            const int e = max((int)(top >> 7), 20);
            const float up = __uint_as_float((uint32_t)(262 - e) << 23);
            if (lane == 0) {
              grp.factor[r] = A.scale_log2 * __uint_as_float((uint32_t)(e - 8) << 23);
              grp.limit[r] = min(meta.length - meta.n + j + 1, next_most);       // rows that do not exist mask nothing
            }
            const uint32_t h0 = pack_half(bf_lo(x.x) * up, bf_hi(x.x) * up), h1 = pack_half(bf_lo(x.y) * up, bf_hi(x.y) * up);
            if (D == 128)
              *reinterpret_cast<uint2*>(q16 + (lane >> 4) * 16384 + r * 128 + ((((lane & 15) >> 1) ^ (r & 7)) << 4) + (lane & 1) * 8) = make_uint2(h0, h1);
            else
              *reinterpret_cast<uint32_t*>(q16 + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4) = h0;
          }
        }
        const uint8_t* raw = ring + k_stage * S::STAGE;
        uint32_t w[PER][4];
#pragma unroll
        for (int i = 0; i < PER; ++i) words(tile_at<D>(raw, warp * KEYS + (i * 32 + lane) / C, lane % C), w[i]);
#pragma unroll
        for (int i = 0; i < PER; ++i) put_halves<D, KIND>(k16, warp * KEYS + (i * 32 + lane) / C, lane % C, w[i]);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(k_full + (t & 1) * 8);
        if (!(flags & ST_END)) mbar_arrive(empty + k_stage * 8);
      }
      if (t > 0) {
        // V of the tile before
        if (!mbar_wait_warp(full + (S::STAGES + v_stage) * 8, v_phase, ctx, 945)) break;
        if (t > 2 && !mbar_wait_warp(pv_done + ((t - 3) & 1) * 8, ((t - 3) >> 1) & 1, ctx, 943)) break;
        uint8_t* half = v16 + ((t - 1) & 1) * S::HALVES;
        const uint8_t* raw = ring + S::RING + v_stage * S::STAGE;
        uint32_t all[PER][4];
#pragma unroll
        for (int i = 0; i < PER; ++i) words(tile_at<D>(raw, warp * KEYS + (i * 32 + lane) / C, lane % C), all[i]);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int r = warp * KEYS + (i * 32 + lane) / C, c = lane % C, pos = v_key0 + r;
          uint32_t (&w)[4] = all[i];
          if (v_key0 + CT_KEYS <= v_least && v_scale != 0.f) {       // every row sees every key of the tile
            put_halves<D, KIND>(half, r, c, w);
            continue;
          }
          // what no row sees is whatever the page held, and must not meet a zero weight; nor must a NaN that some rows see
          if (pos >= v_most || v_scale == 0.f) w[0] = w[1] = w[2] = w[3] = 0;
          if (NANS && pos >= v_least) {
            uint32_t bits = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t m = __vcmpeq4(w[j] & 0x7f7f7f7fu, 0x7f7f7f7fu);
              w[j] &= ~m;
              bits |= ((m & 1u) | (m >> 7 & 2u) | (m >> 14 & 4u) | (m >> 21 & 8u)) << (4 * j);
            }
            if (bits) {
              nans[v_seg % TILE_GROUPS][pos - v_least][c] = (uint16_t)bits;
              groups[v_seg % TILE_GROUPS].nan_any = 1;
            }
          }
          put_halves<D, KIND>(half, r, c, w);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(v_full + ((t - 1) & 1) * 8);
          mbar_arrive(empty + (S::STAGES + v_stage) * 8);
        }
        if (++v_stage == S::STAGES) {
          v_stage = 0;
          v_phase ^= 1;
        }
      }
      if (flags & ST_END) break;
      v_key0 = key0;
      v_scale = scale;
      v_seg = seg;
      v_least = next_least;
      v_most = next_most;
      if (++k_stage == S::STAGES) {
        k_stage = 0;
        k_phase ^= 1;
      }
    }
  } else if (warp < 10) {
    AttnProducer<D, S, false> producer(A, order, range);
    const uint32_t v = warp - 8;
    producer.run(v ? &tv : &tk, v, smem_u32(ring) + v * S::RING, 0, stages, full + v * S::STAGES * 8, empty + v * S::STAGES * 8, ctx);
  } else if (warp == 10) {
    // ------------------------------------------------------------------ products
    constexpr uint32_t IDESC_QK = make_idesc_f16(128, 128, 0), IDESC_PV = make_idesc_f16(128, D, 1);
    int before = 0;                                   // flags of the tile before
    for (int t = 0;; ++t) {
      if (!mbar_wait_warp(k_full + (t & 1) * 8, (t >> 1) & 1, ctx, 951)) break;
      const int flags = __shfl_sync(0xffffffffu, tiles[t % TILE_RING].flags, 0);
      if (!(flags & ST_END)) {
        if (!mbar_wait_warp(s_free + (t & 1) * 8, ((t >> 1) & 1) ^ 1, ctx, 952)) break;
        tc_fence_after();
        umma_loop_kk<0, D / 16>(tmem + S_COL + (t & 1) * 128, smem_u32(q16), smem_u32(k16), IDESC_QK);
        tc_commit(s_full + (t & 1) * 8);
        tc_commit(k_free + (t & 1) * 8);
        if (lane == 0) mbar_arrive(s_full + (t & 1) * 8);      // passes on what the converting warps wrote about the tile
      }
      if (t > 0) {
        if (!mbar_wait_warp(v_full + ((t - 1) & 1) * 8, ((t - 1) >> 1) & 1, ctx, 954)) break;
        if (!mbar_wait_warp(p_full + ((t - 1) & 1) * 8, ((t - 1) >> 1) & 1, ctx, 955)) break;
        tc_fence_after();
        umma_loop_ts<0, 8>(tmem + O_COL, tmem + P_COL + ((t - 1) & 1) * 64, false, smem_u32(v16) + ((t - 1) & 1) * S::HALVES, IDESC_PV, before & ST_FIRST ? 0u : 1u);
        tc_commit(pv_done + ((t - 1) & 1) * 8);
        if (lane == 0) mbar_arrive(pv_done + ((t - 1) & 1) * 8);
      }
      if (flags & ST_END) {
        tc_commit(s_full + (t & 1) * 8);
        if (lane == 0) mbar_arrive(s_full + (t & 1) * 8);
        break;
      }
      before = flags;
    }
  } else if (warp >= 12) {
    // ------------------------------------------------------------------ softmax
    const int quarter = warp & 3, part = (warp - 12) >> 2, row = quarter * 32 + lane;
    const uint32_t t_o = tmem_addr(tmem, quarter * 32, O_COL + part * (D / 4));
    ConsumerSync all = {quartet + quarter * 8, 0};
    float factor = 0.f, ref = -3e38f, l = 0.f;
    bool huge = false;                                // the row's sum is times 2^CT_SHIFT_HUGE
    int limit = 0, seg = -1;
    bool there = false, begun = false;                // these warps have rows; O holds something of this group
    for (int t = 0;; ++t) {
      if (!mbar_wait_warp(s_full + (t & 1) * 8, (t >> 1) & 1, ctx, 961)) break;
      tc_fence_after();
      const TileMeta& meta = tiles[t % TILE_RING];
      const int flags = meta.flags;
      if (flags & ST_END) break;
      if (flags & ST_FIRST) {
        ++seg;
        factor = groups[seg % TILE_GROUPS].factor[row];
        limit = groups[seg % TILE_GROUPS].limit[row];
        there = meta.row_tile * TILE_ROWS + quarter * 32 < meta.n * A.group;
        ref = -3e38f;
        l = 0.f;
        huge = false;
        begun = false;
      }
      uint32_t x[32];                                 // this warp's part of the row's scores
      float top = -INFINITY;
      const int seen = limit - meta.key0 - 32 * part; // columns of the part that the row sees
      const bool edge = __any_sync(0xffffffffu, seen < 32);
      if (there) {
        const uint32_t t_s = tmem_addr(tmem, quarter * 32, S_COL + (t & 1) * 128 + 32 * part);
        tmem_ld32(t_s, x);
        tc_wait_ld(x);
        // a = score in log2 units plus log2 of the value scale, as in AttnConsumer
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 about = meta.sub[2 * part + h];
          if (edge || about.x == 0.f) {
            const int n = about.x == 0.f ? 0 : seen - 16 * h;
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (i >= n) x[16 * h + i] = 0xff800000u;
          }
          float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            m0 = max3(m0, __uint_as_float(x[16 * h + i]), __uint_as_float(x[16 * h + i + 1]));
            m1 = max3(m1, __uint_as_float(x[16 * h + i + 2]), __uint_as_float(x[16 * h + i + 3]));
          }
          if (about.x != 0.f) top = fmaxf(top, fmaf(fmaxf(m0, m1), fmaxf(factor * about.x, 1.2e-38f), about.y));
        }
        tops[t & 1][part][row] = top;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(s_free + (t & 1) * 8);
      // this tile's place for P is free.  Warps without rows wait too, so that none arrives twice in one phase of p_full.
      if (t > 1 && !mbar_wait_warp(pv_done + (t & 1) * 8, ((t - 2) >> 1) & 1, ctx, 962)) break;
      if (there) {
        if (!all(ctx, lane, 965)) break;
        top = fmaxf(fmaxf(tops[t & 1][0][row], tops[t & 1][1][row]), fmaxf(tops[t & 1][2][row], tops[t & 1][3][row]));
        tc_fence_after();
        if (__any_sync(0xffffffffu, top > ref + 15.f)) {       // the same in all four warps
          const float m = top > ref + 15.f ? top - 8.f : ref, shrink = exp2_approx(ref - m);
          // the sum keeps what it can of its range
          const bool rises = (flags & ST_HUGE) && !huge && (float)((int)(__float_as_uint(l) >> 23) - 127) + (ref - m) < -60.f;
          l = times_exp2(l, ref - m + (rises ? CT_SHIFT_HUGE - CT_SHIFT : 0.f));
          huge |= rises;
          ref = m;
          if (begun) {                                // O is at rest once the tile before is in it
            if (!mbar_wait_warp(pv_done + ((t - 1) & 1) * 8, ((t - 1) >> 1) & 1, ctx, 963)) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 64; ++c) {
              uint32_t o[16];
              tmem_ld16(t_o + 16 * c, o);
              tc_wait_ld(o);
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * shrink);
              tmem_st16(t_o + 16 * c, o);
            }
          }
        }
        if (flags & ST_APART) {
          auto e = [&](int h, int i) {                // score over the reference, without the value scale
            const float4 about = meta.sub[2 * part + h];
            return fmaf(__uint_as_float(x[16 * h + i]), fmaxf(factor * about.x, 1.2e-38f), about.y) - ref - about.y;
          };
          if (flags & ST_HUGE) {
            float most = -INFINITY;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (meta.sub[2 * part + (i >> 4)].x != 0.f) most = fmaxf(most, e(i >> 4, i & 15));
            const bool up = !huge && most < -50.f && l < 0x1p-60f, down = huge && most > 40.f;
            if (up) l /= CT_UNIT / CT_UNIT_HUGE;
            if (down) l *= CT_UNIT / CT_UNIT_HUGE;
            huge = up || (huge && !down);
          }
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (meta.sub[2 * part + (i >> 4)].x != 0.f) l += exp2_approx(e(i >> 4, i & 15) + (huge ? CT_SHIFT_HUGE : CT_SHIFT));
        }
        uint32_t p[16];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 about = meta.sub[2 * part + h];
          const float f = about.x != 0.f ? fmaxf(factor * about.x, 1.2e-38f) : 1.f;       // not 0: times -infinity; absent keys have -infinity
          float z0 = 0.f, z1 = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = 16 * h + 2 * i;
            // rounded as the reference was before it is taken off: in one step a score of 2^26 or more would differ from its own
            // reference by the rounding, and its weight would overflow
            const float2 s2 = add2(fma2(make_float2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), make_float2(f, f), make_float2(about.y, about.y)), make_float2(-ref, -ref));
            const float a = exp2_approx(s2.x), b = exp2_approx(s2.y);
            z0 += a;
            z1 += b;
            p[8 * h + i] = pack_half(a, b);
          }
          l = fmaf(z0 + z1, about.z, l);
        }
        tmem_st16(tmem_addr(tmem, quarter * 32, P_COL + (t & 1) * 64 + 16 * part), p);
        tc_wait_st();
        begun = true;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full + (t & 1) * 8);
      if (flags & ST_LAST) {
        if (there) {
          sums[part][row] = huge ? -l : l;
          if (!all(ctx, lane, 966)) break;
          float z = (sums[0][row] + sums[1][row]) + (sums[2][row] + sums[3][row]);
          if (flags & ST_HUGE) {
            float shift = CT_SHIFT;
            z = 0.f;
#pragma unroll 1
            for (int i = 0; i < 4; ++i) shift = fmaxf(shift, sum_shift(sums[i][row]));
#pragma unroll 1
            for (int i = 0; i < 4; ++i) z += times_exp2(fabsf(sums[i][row]), shift - sum_shift(sums[i][row]));
            huge = shift == CT_SHIFT_HUGE;
          }
          if (!mbar_wait_warp(pv_done + (t & 1) * 8, (t >> 1) & 1, ctx, 964)) break;
          tc_fence_after();
          const int gr = meta.row_tile * TILE_ROWS + row, j = gr / A.group;
          const bool is = gr < meta.n * A.group;
          const float inverse = z == 0.f ? 0.f : 1.f / z, lse2 = z == 0.f ? -INFINITY : ref - (huge ? CT_SHIFT_HUGE : CT_SHIFT) + log2_split(z);
          const float unit = (huge ? CT_UNIT_HUGE : CT_UNIT) * (flags & ST_WHOLE ? 1.f : CT_PART_UNIT);
          const int64_t out = (int64_t)(meta.row0 + j) * A.hq + meta.head * A.group + gr - j * A.group, place = (int64_t)meta.part * TILE_ROWS + row;
          const TileGroup& grp = groups[seg % TILE_GROUPS];
#pragma unroll 1
          for (int c = 0; c < D / 64; ++c) {          // this warp's part of the columns
            uint32_t o[16];
            tmem_ld16(t_o + 16 * c, o);
            tc_wait_ld(o);
            const int col = part * (D / 64) + c;
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(z == 0.f ? 0.f : __uint_as_float(o[i]) * inverse * unit);
            if (NANS && grp.nan_any) {
              uint32_t bits = 0;
              for (int k = 0; k < min(limit - grp.least, 128); ++k) bits |= nans[seg % TILE_GROUPS][k][col];
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (bits >> i & 1) o[i] = 0x7fffffffu;
            }
            if (!is) continue;
            if (flags & ST_WHOLE) {
              uint32_t y[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = pack_bf16(__uint_as_float(o[2 * i]), __uint_as_float(o[2 * i + 1]));
              uint4* dst = reinterpret_cast<uint4*>(A.o + out * D + 16 * col);
              dst[0] = make_uint4(y[0], y[1], y[2], y[3]);
              dst[1] = make_uint4(y[4], y[5], y[6], y[7]);
            } else {
              uint4* dst = reinterpret_cast<uint4*>(A.part_o + place * D + 16 * col);
#pragma unroll
              for (int i = 0; i < 4; ++i) dst[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
          }
          if (is && part == 0) {
            if (flags & ST_WHOLE) A.lse[out] = lse2 * 0.69314718055994531f;
            else A.part_lse[place] = lse2;
          }
          tc_fence_before();                          // O is free for the next group with this warp's next arrival at p_full
        }
      }
    }
  }
  wait_teardown(ctx);
  tc_fence_before();
  __syncthreads();
  if (warp == 10) {
    __syncwarp();
    tmem_dealloc(tmem, 512);
  }
}

// Joins the partial results of groups that several CTAs shared: block c takes the group that began on CTA c, in the CTAs' order.
constexpr int MERGE_THREADS = 256;
template <int D>
__global__ void __launch_bounds__(MERGE_THREADS) cache_merge_kernel(const __grid_constant__ AttnArgs A, int rows_per_tile) {
  grid_begin();
  const int32_t* S = A.split + blockIdx.x * SP_W;
  const int count = ld_i32(S + SP_COUNT);
  if (count <= 0) return;
  const int row0 = ld_i32(S + SP_ROW0), n = ld_i32(S + SP_N), head = ld_i32(S + SP_HEAD), first = ld_i32(S + SP_ROW_TILE) * rows_per_tile;
  const int n_rows = min(rows_per_tile, n * A.group - first);
  auto part = [&](int i) { return i == 0 ? 2 * (int)blockIdx.x + 1 : 2 * ((int)blockIdx.x + i); };
  for (int e = threadIdx.x; e < n_rows * (D / 4); e += MERGE_THREADS) {
    const int r = e / (D / 4), f = e % (D / 4);
    float ref = -3e38f, z = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int U = 4;                              // partial results in flight
    for (int i0 = 0; i0 <= count; i0 += U) {
      float l[U], top = ref;
      float4 y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = (int64_t)part(min(i0 + u, count)) * rows_per_tile + r;
        l[u] = ld_f32(A.part_lse + at);
        y[u] = ld_stream_f4(A.part_o + at * D + f * 4);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + u > count) l[u] = -INFINITY;
        top = fmaxf(top, l[u]);
      }
      const float shrink = exp2_approx(ref - top);
      ref = top;
      z *= shrink;
      x.x *= shrink; x.y *= shrink; x.z *= shrink; x.w *= shrink;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = exp2_approx(l[u] - ref);
        if (i0 + u > count) continue;                 // a repeated one, whose values may be NaN
        z += w;
        x.x = fmaf(y[u].x, w, x.x); x.y = fmaf(y[u].y, w, x.y); x.z = fmaf(y[u].z, w, x.z); x.w = fmaf(y[u].w, w, x.w);
      }
    }
    const float inverse = z == 0.f ? 0.f : 1.f / z;
    const int gr = first + r, j = gr / A.group;
    const int64_t out = (int64_t)(row0 + j) * A.hq + head * A.group + gr - j * A.group;
    x.x = x.x * inverse / CT_PART_UNIT; x.y = x.y * inverse / CT_PART_UNIT; x.z = x.z * inverse / CT_PART_UNIT; x.w = x.w * inverse / CT_PART_UNIT;
    *reinterpret_cast<uint2*>(A.o + out * D + f * 4) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
    if (f == 0) A.lse[out] = z == 0.f ? -INFINITY : (ref + __log2f(z)) * 0.69314718055994531f;
  }
}

// ---------------------------------------------------------------------------------------------
// Attention of long chunks of new tokens
// ---------------------------------------------------------------------------------------------
// With many new tokens the products decide, and those of whole tiles of 128 tokens belong to tcgen05: the cached keys and values
// are written out as bf16 once (exactly, where the scale is a power of two), [sequence][capacity][hkv][D], and the packed
// attention of this library (fcp_fwd_kernel) runs over them, with work units and row limits made on the device.  Its weights are bf16, so
// that keys and values of any size meet them: 2.3e-3 from 64 bits in the mean over 4 chunks of 512 tokens, of which the rounding of o is
// 1.7e-3; the kernels above, with halves, stay at 1.7e-3.
//
// Sequences that this cannot serve exactly are marked and left to cache_attn_kernel or cache_tile_kernel: tokens on pages that do not
// exist, more new rows than tokens, a NaN value among the new tokens (it would meet zero weights of rows that do not see it), key
// scales above CHUNK_MOST_K.
struct ChunkArgs {
  CacheView c;
  BatchView s;
  __nv_bfloat16 *k, *v;                               // [B * stride][hkv][D]
  int32_t stride;                                     // rows per sequence: the capacity in whole tiles
  int32_t* careful;                                   // [B], zero before
  int32_t *units, *groups, *row_limit, *counter;      // [B * units_per_seq][FCP_FWD_UNIT_W], [4], [rows], the grid's work counter
  int32_t units_per_seq;
};

constexpr int UNPACK_THREADS = 256;
// fcp_fwd_kernel's weights overflow at scores of 2^31.  Keys of up to 2^17 stay clear of that.
constexpr float CHUNK_MOST_K = 0x1p8f;
// code * scale as it goes into a bf16.  From scales of 2^119 on it may be beyond one (an infinite value is stored with 2^120 or 2^122),
// and an infinity would meet the zero weights of rows that do not see it: the largest bf16 instead.
__device__ __forceinline__ float held_by_bf16(float x) {
  const float most = __uint_as_float(0x7f7f0000u);
  return fabsf(x) > most ? copysignf(most, x) : x;     // a NaN stays one
}
// 16 codes -> 16 bf16
template <int KIND>
__device__ __forceinline__ void unpack16(const uint4& x, float scale, uint4 (&out)[2]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = halves_lo<KIND>(w[i]), hi = halves_hi<KIND>(w[i]);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    y[2 * i] = pack_bf16(a.x * scale, a.y * scale);
    y[2 * i + 1] = pack_bf16(b.x * scale, b.y * scale);
    if (scale > 0x1p118f) {
      y[2 * i] = pack_bf16(held_by_bf16(a.x * scale), held_by_bf16(a.y * scale));
      y[2 * i + 1] = pack_bf16(held_by_bf16(b.x * scale), held_by_bf16(b.y * scale));
    }
  }
  out[0] = make_uint4(y[0], y[1], y[2], y[3]);
  out[1] = make_uint4(y[4], y[5], y[6], y[7]);
}
// One block per (128 tokens, KV head, sequence).  The rest of a sequence's last tile is zeroed: its probabilities are zero, and a
// product with them must not meet what the memory held.
template <int D, int KIND>
__global__ void __launch_bounds__(UNPACK_THREADS) cache_unpack_kernel(const __grid_constant__ ChunkArgs a) {
  __shared__ int32_t rows[CT_KEYS];
  __shared__ float scales[2][CT_KEYS];
  grid_begin();
  const int b = blockIdx.z, h = blockIdx.y, t0 = blockIdx.x * CT_KEYS, tid = threadIdx.x;
  const SeqView s = load_seq(a.s, b);
  if (s.n == 0 || t0 >= s.length) {
    if (tid == 0 && s.n > s.length) a.careful[b] = 1;
    return;
  }
  bool careful = s.n > s.length;
  if (tid < CT_KEYS) {
    const int pos = t0 + tid;
    int32_t row = -2;
    float ks = 0.f, vs = 0.f;
    if (pos < s.length) {
      const int32_t page = ld_i32(a.s.page_table + (int64_t)b * a.s.table_width + (pos >> a.c.page_shift));
      row = page_row(page, a.c.n_pages, a.c.hkv, h, a.c.page_tokens);
      if (row >= 0) {
        ks = ld_f32(a.c.k_scale + page * a.c.hkv + h);
        vs = ld_f32(a.c.v_scale + page * a.c.hkv + h);
        row += pos & (a.c.page_tokens - 1);
      }
      if (row < 0 || !usable_scale(ks) || !usable_scale(vs)) {
        row = -2;
        careful = true;
      }
      careful |= ks > CHUNK_MOST_K;
    }
    rows[tid] = row;
    scales[0][tid] = ks;
    scales[1][tid] = vs;
  }
  __syncthreads();
  constexpr int C = D / 16, N = 2 * CT_KEYS * C / UNPACK_THREADS;
  uint4 x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * UNPACK_THREADS + tid, which = e / (CT_KEYS * C), t = e / C % CT_KEYS, c = e % C;
    x[i] = make_uint4(0, 0, 0, 0);
    if (rows[t] >= 0) x[i] = ld_v4((which ? a.c.v : a.c.k) + (int64_t)rows[t] * D + c * 16);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * UNPACK_THREADS + tid, which = e / (CT_KEYS * C), t = e / C % CT_KEYS, c = e % C;
    if (KIND == FCP_CACHE_E4M3 && which && t0 + t >= s.length - s.n) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) careful |= __vcmpeq4(w[j] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
    }
    uint4 y[2];
    unpack16<KIND>(x[i], scales[which][t], y);
    __nv_bfloat16* out = (which ? a.v : a.k) + (((int64_t)b * a.stride + t0 + t) * a.c.hkv + h) * D + c * 16;
    *reinterpret_cast<uint4*>(out) = y[0];
    *reinterpret_cast<uint4*>(out + 8) = y[1];
  }
  if (careful) a.careful[b] = 1;
}

// The work units of fcp_fwd_kernel (pairs of tiles of 128 new tokens), the one work group, the row limits.  The units go by their
// number of key tiles, most first, so that the last ones to be handed out are short; up to CHUNK_SORT units, because every unit
// looks at every other.
constexpr int CHUNK_THREADS = 256;
constexpr int CHUNK_SORT = 8192;
__global__ void __launch_bounds__(CHUNK_THREADS) cache_chunk_kernel(const __grid_constant__ ChunkArgs a) {
  __shared__ int32_t place;
  grid_begin();
  const int b = blockIdx.y, u = blockIdx.x, tid = threadIdx.x, n_units = (int)(gridDim.x * gridDim.y), self = b * (int)gridDim.x + u;
  const SeqView s = load_seq(a.s, b);
  const bool serves = ld_i32(a.careful + b) == 0;
  const int first = u * FCP_FWD_UNIT_ROWS, n = serves ? max(0, min(FCP_FWD_UNIT_ROWS, s.n - first)) : 0;
  const int seen = s.length - s.n + first + 1;        // keys that the unit's first row sees
  if (tid < n) a.row_limit[s.row0 + first + tid] = b * a.stride + seen + tid;
  if (tid == 0) place = 0;
  __syncthreads();
  if (n_units <= CHUNK_SORT) {
    const int mine = n > 0 ? (seen + n - 1 + FCP_TILE - 1) / FCP_TILE : 0;
    int before = 0;
    for (int i = tid; i < n_units; i += CHUNK_THREADS) {
      const int bi = i / (int)gridDim.x, fi = (i - bi * (int)gridDim.x) * FCP_FWD_UNIT_ROWS;
      const SeqView x = load_seq(a.s, bi);
      const int ni = ld_i32(a.careful + bi) == 0 ? max(0, min(FCP_FWD_UNIT_ROWS, x.n - fi)) : 0;
      const int other = ni > 0 ? (x.length - x.n + fi + ni + FCP_TILE - 1) / FCP_TILE : 0;
      before += other > mine || (other == mine && i < self);
    }
    before = __reduce_add_sync(0xffffffffu, before);
    if ((tid & 31) == 0) atomicAdd(&place, before);
  } else if (tid == 0) {
    place = self;
  }
  __syncthreads();
  if (tid < FCP_FWD_UNIT_W) {
    auto tiles = [&](int rows) { return (seen + rows - 1 + FCP_TILE - 1) / FCP_TILE; };        // of keys, for the first `rows` rows
    int x = 0;
    switch (tid) {
      case FU_Q_ROW0: x = s.row0 + first; break;
      case FU_Q_ROWS: x = n; break;
      case FU_N_RANGES: x = 1; break;
      case FU_KV0_BEGIN: x = b * a.stride; break;
      case FU_KV0_END: x = b * a.stride + seen + n - 1; break;
      case FU_KV0_DIAG: x = 1; break;
      case FU_NT_STAGE0: x = n > 0 ? tiles(min(n, FCP_TILE)) : 0; break;
      case FU_NT_STAGE1: x = n > FCP_TILE ? tiles(n) : 0; break;
      case FU_NT_RANGE0: x = 0x7fffffff; break;       // no second range
      case FU_SINGLE_SLOT: x = 1; break;
    }
    a.units[(int64_t)place * FCP_FWD_UNIT_W + tid] = x;
  }
  if (b == 0 && u == 0 && tid == 0) {
    *a.counter = 0;
    a.groups[WG_FIRST] = 0;
    a.groups[WG_N_UNITS] = (int32_t)(gridDim.x * gridDim.y);
    a.groups[WG_HEADS] = a.c.hkv;
    a.groups[WG_RSV] = 0;
  }
}

// ---------------------------------------------------------------------------------------------
// Eviction
// ---------------------------------------------------------------------------------------------
struct EvictArgs {
  CacheView c;
  BatchView s;
  int32_t n_sink, n_heavy, n_recent;
  const int32_t* dst_table;
  int32_t dst_width;
  int32_t *new_length, *kept;
};

__device__ __forceinline__ int32_t usable_length(const BatchView& s, int b) {
  const int32_t n = ld_i32(s.length + b);
  return n < 0 || n > s.capacity ? -1 : n;
}

// Weights as unsigned keys of the same order; NaN and what lies on a page that does not exist come last.  0 is no candidate.
__device__ __forceinline__ uint32_t weight_key(float x) {
  if (x != x) return 1u;
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// Which tokens of a head stay: one cluster of blocks per (KV head, sequence), each with its slice of the candidates.  The n_heavy
// largest weights by three counting passes over 11, 11 and 10 bits of the keys, from the top, the counts added up over the cluster;
// then one pass writes the kept positions in order.
// Keys go four at a time: they lie side by side in a page, and one place in the page table, one load and one address serve them
// (key by key the kernel was bound by its instructions, 120 000 warp instructions per block).  2 sequences of 128K tokens, 8 heads: 44 us,
// 8 blocks per head, bound by the chain of counting passes and cluster barriers; reading the weights alone takes 1.4 us.
constexpr int SELECT_THREADS = 1024;
constexpr int SELECT_KEYS = 49152;                    // as many keys of a slice stay in shared memory
constexpr int SELECT_BINS = 2048;
constexpr int SELECT_BLOCKS = 8;                      // most blocks of a cluster
__global__ void __launch_bounds__(SELECT_THREADS, 2) cache_select_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ __align__(16) uint4 keys[];
  __shared__ __align__(8) uint32_t sums[2][SELECT_BINS];       // of this block, read by the others: one per pass in turn
  __shared__ uint32_t warp_count[32][2];
  __shared__ uint32_t share[2];                       // kept and equal keys of this block, read by the others
  __shared__ uint32_t chosen[2];                      // digit, how many are still wanted among the keys that have it
  grid_begin();
  const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int h = blockIdx.x / blocks, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int keep = a.n_sink + a.n_heavy + a.n_recent;
  const int length = usable_length(a.s, b);
  const bool reports = blockIdx.x == 0 && tid == 0;
  if (length < 0 && reports) mark_bad(a.c.status, FCP_CACHE_BAD_LENGTH, b);
  int32_t* kept = a.kept + ((int64_t)b * a.c.hkv + h) * keep;
  if (reports) a.new_length[b] = max(0, min(length, keep));
  const int first = rank * SELECT_THREADS + tid, stride = blocks * SELECT_THREADS;
  if (length <= keep) {
    for (int i = first; i < keep; i += stride) kept[i] = i < length ? i : -1;
    return;
  }
  const int page_tokens = a.c.page_tokens, end = length - a.n_recent;          // candidates: positions [n_sink, end)
  for (int i = first; i < a.n_sink; i += stride) kept[i] = i;
  for (int i = first; i < a.n_recent; i += stride) kept[a.n_sink + a.n_heavy + i] = end + i;
  if (a.n_heavy == 0) return;
  // fours of positions, and this block's share of them
  const int q_begin = a.n_sink >> 2, q_all = ((end + 3) >> 2) - q_begin, per = (q_all + blocks - 1) / blocks;
  const int from = q_begin + min(q_all, rank * per), n = q_begin + min(q_all, rank * per + per) - from;
  auto page_of = [&](int i) { return ld_i32(a.s.page_table + (int64_t)b * a.s.table_width + (((from + i) * 4) >> a.c.page_shift)); };
  auto keys_of = [&](int i, int32_t page) {
    const int pos = (from + i) * 4;
    const int32_t row = page_row(page, a.c.n_pages, a.c.hkv, h, page_tokens);
    float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row >= 0) {
      const uint4 x = ld_v4(a.c.weight + (int64_t)row + (pos & (page_tokens - 1)));
      w = make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
    }
    auto key = [&](float x, int p) { return p < a.n_sink || p >= end ? 0u : row < 0 ? 1u : weight_key(x); };
    return make_uint4(key(w.x, pos), key(w.y, pos + 1), key(w.z, pos + 2), key(w.w, pos + 3));
  };
  const bool in_smem = 4 * n <= SELECT_KEYS;
  if (in_smem) {
    constexpr int U = 4;                              // places in the page table in flight per thread
    for (int i0 = tid; i0 < n; i0 += U * SELECT_THREADS) {
      int32_t page[U];
#pragma unroll
      for (int u = 0; u < U; ++u) page[u] = i0 + u * SELECT_THREADS < n ? page_of(i0 + u * SELECT_THREADS) : -1;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * SELECT_THREADS < n) keys[i0 + u * SELECT_THREADS] = keys_of(i0 + u * SELECT_THREADS, page[u]);
    }
  }
  auto four = [&](int i) { return in_smem ? keys[i] : keys_of(i, page_of(i)); };
  uint32_t prefix = 0, wanted = (uint32_t)a.n_heavy;
  for (int pass = 0; pass < 3; ++pass) {              // 11, 11 and 10 bits
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    const uint32_t mask = (1u << bits) - 1u;
    uint32_t* mine = sums[pass & 1];
    for (int i = tid; i < SELECT_BINS; i += SELECT_THREADS) mine[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += SELECT_THREADS) {
      const uint4 k = four(i);
      auto count = [&](uint32_t x) {
        if (x != 0u && (pass == 0 || x >> (shift + bits) == prefix)) atomicAdd(&mine[(x >> shift) & mask], 1u);
      };
      count(k.x);
      count(k.y);
      count(k.z);
      count(k.w);
    }
    if (blocks > 1) cluster.sync();
    else __syncthreads();
    // from the highest digit down, two digits per thread
    static_assert(SELECT_BINS == 2 * SELECT_THREADS, "");
    uint32_t c[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < SELECT_BLOCKS; ++k) {
      if (k >= blocks) break;
      const uint2 x = reinterpret_cast<const uint2*>(cluster.map_shared_rank(mine, k))[SELECT_THREADS - 1 - tid];
      c[0] += x.y;
      c[1] += x.x;
    }
    uint32_t upto = c[0] + c[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) warp_count[warp][0] = upto;
    __syncthreads();
    uint32_t w = warp_count[lane][0];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += x;
    }
    w = __shfl_sync(0xffffffffu, w, (warp - 1) & 31);
    uint32_t before = upto - c[0] - c[1] + (warp ? w : 0u);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (before < wanted && wanted <= before + c[j]) {
        chosen[0] = (uint32_t)(SELECT_BINS - 1 - (2 * tid + j));
        chosen[1] = wanted - before;
      }
      before += c[j];
    }
    __syncthreads();
    prefix = prefix << bits | chosen[0];
    wanted = chosen[1];
  }
  // prefix is the smallest kept key, `wanted` of its equals are kept: the first ones
  // every warp takes a run of the keys, so that only its first place needs the others
  const int run = (n + SELECT_THREADS - 1) / SELECT_THREADS * 32, w0 = min(n, warp * run), w1 = min(n, w0 + run);
  auto above_in = [&](const uint4& k) { return (uint32_t)(k.x > prefix) + (k.y > prefix) + (k.z > prefix) + (k.w > prefix); };
  auto equal_in = [&](const uint4& k) { return (uint32_t)(k.x == prefix) + (k.y == prefix) + (k.z == prefix) + (k.w == prefix); };
  uint32_t above_n = 0, equal_n = 0;
  for (int i = w0 + lane; i < w1; i += 32) {
    const uint4 k = four(i);
    above_n += above_in(k);
    equal_n += equal_in(k);
  }
  above_n = __reduce_add_sync(0xffffffffu, above_n);
  equal_n = __reduce_add_sync(0xffffffffu, equal_n);
  if (lane == 0) {
    warp_count[warp][0] = above_n;
    warp_count[warp][1] = equal_n;
  }
  __syncthreads();
  if (warp == 0) {
    above_n = __reduce_add_sync(0xffffffffu, warp_count[lane][0]);
    equal_n = __reduce_add_sync(0xffffffffu, warp_count[lane][1]);
    if (lane == 0) {
      share[0] = above_n;
      share[1] = equal_n;
    }
  }
  cluster.sync();
  // kept and equal keys in front of this warp: blocks and warps before it
  uint32_t a_base = lane < warp ? warp_count[lane][0] : 0u, e_base = lane < warp ? warp_count[lane][1] : 0u;
  if (lane < rank) {
    const uint32_t* x = cluster.map_shared_rank(share, lane);
    a_base += x[0];
    e_base += x[1];
  }
  a_base = __reduce_add_sync(0xffffffffu, a_base);
  e_base = __reduce_add_sync(0xffffffffu, e_base);
  for (int i0 = w0; i0 < w1; i0 += 32) {
    const int i = i0 + lane;
    const uint4 k = i < w1 ? four(i) : make_uint4(0u, 0u, 0u, 0u);
    uint32_t upto = above_in(k) | equal_in(k) << 16;  // at most 128 of each in a trip
    const uint32_t own = upto;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    uint32_t a_before = a_base + ((upto - own) & 0xffffu), e_before = e_base + ((upto - own) >> 16);
    auto put = [&](uint32_t x, int pos) {
      const bool above = x > prefix, equal = x == prefix;
      if (above || (equal && e_before < wanted)) kept[a.n_sink + a_before + min(e_before, wanted)] = pos;
      a_before += above;
      e_before += equal;
    };
    const int pos = (from + i) * 4;
    put(k.x, pos);
    put(k.y, pos + 1);
    put(k.z, pos + 2);
    put(k.w, pos + 3);
    const uint32_t total = __shfl_sync(0xffffffffu, upto, 31);
    a_base += total & 0xffffu;
    e_base += total >> 16;
  }
  cluster.sync();                                     // no block leaves while another reads its shares
}

// The kept tokens into their new pages: one block per 128 of a head, i.e. 1 to 8 new pages.  Loads depend on one another three
// deep: length, position and new page; old page; scales, weight and codes.
constexpr int MOVE_THREADS = 256;
constexpr int MOVE_TOKENS = 128;
template <int D, int KIND>
__global__ void __launch_bounds__(MOVE_THREADS) cache_move_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ int32_t src_row[MOVE_TOKENS];            // of every token; -1: none
  __shared__ int32_t dst_row[MOVE_TOKENS];            // of every token; -1: nowhere
  __shared__ float src_scale[2][MOVE_TOKENS], top[2][MOVE_TOKENS / 16];
  grid_begin();
  const int t0 = blockIdx.x * MOVE_TOKENS, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int keep = a.n_sink + a.n_heavy + a.n_recent, page_tokens = a.c.page_tokens;
  float weight = 0.f;
  int32_t dst = -1, dst_page = -1;
  if (tid < MOVE_TOKENS) {
    const int i = t0 + tid;
    const bool in = i < keep;
    const int32_t length = usable_length(a.s, b);
    const int32_t pos = in ? ld_i32(a.kept + ((int64_t)b * a.c.hkv + h) * keep + i) : -1;
    dst_page = in ? ld_i32(a.dst_table + (int64_t)b * a.dst_width + (i >> a.c.page_shift)) : -1;
    int32_t row = -1;
    float ks = 0.f, vs = 0.f;
    if (i < min(length, keep)) {
      const int32_t at = page_row(dst_page, a.c.n_pages, a.c.hkv, h, page_tokens);
      if (at < 0) mark_bad(a.c.status, FCP_CACHE_BAD_PAGE, b);
      else dst = at + (i & (page_tokens - 1));
      const int32_t src = ld_i32(a.s.page_table + (int64_t)b * a.s.table_width + (pos >> a.c.page_shift));
      row = page_row(src, a.c.n_pages, a.c.hkv, h, page_tokens);
      if (row >= 0) {
        ks = ld_f32(a.c.k_scale + src * a.c.hkv + h);
        vs = ld_f32(a.c.v_scale + src * a.c.hkv + h);
        row += (pos & (page_tokens - 1));
        weight = ld_f32(a.c.weight + row);
      }
    }
    src_row[tid] = row;
    dst_row[tid] = dst;
    __syncwarp();
    src_scale[0][tid] = ks;
    src_scale[1][tid] = vs;
  }
  __syncthreads();
  constexpr int C = D / 16, N = 2 * MOVE_TOKENS * C / MOVE_THREADS;
  uint4 x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {                       // codes before the scales are known to be usable
    const int e = i * MOVE_THREADS + tid, which = e / (MOVE_TOKENS * C), s = e / C % MOVE_TOKENS, c = e % C;
    x[i] = make_uint4(0, 0, 0, 0);
    if (src_row[s] >= 0 && dst_row[s] >= 0) x[i] = ld_v4((which ? a.c.v : a.c.k) + (int64_t)src_row[s] * D + c * 16);
  }
  if (tid < MOVE_TOKENS && src_row[tid] >= 0 && (!usable_scale(src_scale[0][tid]) || !usable_scale(src_scale[1][tid]))) {
    mark_bad(a.c.status, FCP_CACHE_BAD_SCALE, b);
    src_scale[0][tid] = src_scale[1][tid] = 0.f;
    weight = 0.f;
  } else if (tid < MOVE_TOKENS && dst >= 0 && src_row[tid] < 0) {
    mark_bad(a.c.status, FCP_CACHE_BAD_PAGE, b);
  }
  if (tid < MOVE_TOKENS && dst >= 0) a.c.weight[dst] = weight;
  __syncthreads();
  if (tid < 2 * MOVE_TOKENS) {                        // the largest scale of each new page: 16 threads a piece, then the page's
    const int which = tid / MOVE_TOKENS, s = tid % MOVE_TOKENS;
    float m = dst_row[s] >= 0 ? fmaxf(src_scale[which][s], FCP_CACHE_MIN_SCALE) : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (s % 16 == 0) top[which][s / 16] = m;
  }
  __syncthreads();
  {
    // what a token's codes are multiplied by: 256 threads, the keys' and the values' of 128 tokens
    const int which = tid / MOVE_TOKENS, s = tid % MOVE_TOKENS, pieces = page_tokens / 16, p = (s / 16) & ~(pieces - 1);
    float m = 0.f;
    for (int i = 0; i < pieces; ++i) m = fmaxf(m, top[which][p + i]);
    if (dst_row[s] >= 0) {
      if ((s & (page_tokens - 1)) == 0) (which ? a.c.v_scale : a.c.k_scale)[(dst_row[s] >> a.c.page_shift)] = m;
      src_scale[which][s] = __fdiv_rn(src_scale[which][s], m);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * MOVE_THREADS + tid, which = e / (MOVE_TOKENS * C), s = e / C % MOVE_TOKENS, c = e % C;
    if (dst_row[s] < 0) continue;
    const float ratio = src_scale[which][s];
    *reinterpret_cast<uint4*>((which ? a.c.v : a.c.k) + (int64_t)dst_row[s] * D + c * 16) = ratio == 0.f ? make_uint4(0, 0, 0, 0) : moved_codes<KIND>(x[i], ratio);
  }
}

}  // namespace fcp
