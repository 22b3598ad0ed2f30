// Kernels on a paged cache of 8-bit keys and values: append, attention of the newest tokens, the weights it leaves, eviction.
#pragma once
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
  int32_t n_pages, page_tokens, hkv;
};
struct BatchView {
  int32_t B, rows, max_new, table_width, capacity;     // capacity: tokens that a row of the page table can name
  const int32_t *page_table, *length, *row_offset;
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
  return seq_view(ld_i32(s.row_offset + b), ld_i32(s.row_offset + b + 1), ld_i32(s.length + b), s.rows, s.max_new, s.capacity);
}
__device__ __forceinline__ bool usable_scale(float x) { return x >= FCP_CACHE_MIN_SCALE && x <= FCP_CACHE_MAX_SCALE; }

// ---------------------------------------------------------------------------------------------
// Codes
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
// Two codes (the low or the high half of a word) -> two halves, exactly: e4m3 has 4 significant bits, int8 8, a half 11.
template <int KIND>
__device__ __forceinline__ uint32_t halves_lo(uint32_t w) {
  if (KIND == FCP_CACHE_E4M3) {
    __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xffffu), __NV_E4M3);
    return (uint32_t)r.x | ((uint32_t)r.y << 16);
  }
  // byte + 128 under the exponent of 1024 is the half 1024 + 128 + value
  const uint32_t h = __byte_perm(w ^ 0x80808080u, 0x64646464u, 0x4140);
  return h2_bits(__hsub2(*reinterpret_cast<const __half2*>(&h), __float2half2_rn(1152.f)));
}
template <int KIND>
__device__ __forceinline__ uint32_t halves_hi(uint32_t w) {
  if (KIND == FCP_CACHE_E4M3) {
    __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3);
    return (uint32_t)r.x | ((uint32_t)r.y << 16);
  }
  const uint32_t h = __byte_perm(w ^ 0x80808080u, 0x64646464u, 0x4342);
  return h2_bits(__hsub2(*reinterpret_cast<const __half2*>(&h), __float2half2_rn(1152.f)));
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
template <int KIND>
__device__ __forceinline__ uint32_t rescale_codes(uint32_t w, float ratio) {
  const uint32_t lo = halves_lo<KIND>(w), hi = halves_hi<KIND>(w);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  return to_codes<KIND>(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio);
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

// One block per (page touched, head, K or V): the page's new values stay in registers between the maximum and the codes.
constexpr int APPEND_THREADS = 128;
template <int D, int KIND, int N>                    // N: pieces of 16 values per thread
__global__ void __launch_bounds__(APPEND_THREADS) cache_append_kernel(const __grid_constant__ AppendArgs a) {
  __shared__ uint32_t warp_max[APPEND_THREADS / 32];
  grid_begin();
  const int w = blockIdx.x, h = blockIdx.y >> 1, tid = threadIdx.x;
  const bool is_v = blockIdx.y & 1;
  const int page_tokens = a.c.page_tokens;
  int b = 0;
  if (a.s.max_new == 1) {                            // one token, one page: a slot per sequence
    b = w;
  } else {                                           // the last b whose first slot is at most w
    int lo = 0, hi = a.s.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (append_slot(ld_i32(a.s.row_offset + mid), mid, page_tokens) <= w) lo = mid;
      else hi = mid - 1;
    }
    b = lo;
  }
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
  const int32_t row = page_row(page, a.c.n_pages, a.c.hkv, h, page_tokens);
  if (row < 0) {
    if (tid == 0) mark_bad(a.c.status, FCP_CACHE_BAD_PAGE, b);
    return;
  }
  const int held = sp.lo - sp.page * page_tokens, filled = sp.hi - sp.page * page_tokens;      // slots [held, filled) are new
  constexpr int C = D / 16;
  const __nv_bfloat16* x = (is_v ? a.v : a.k) + h * D;
  const int64_t stride = is_v ? a.v_stride : a.k_stride;
  const int64_t first = (int64_t)sv.row0 + sv.n - sv.length + (int64_t)sp.page * page_tokens;  // row of the page's slot 0
  uint4 r[N][2];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * APPEND_THREADS + tid, s = e / C, c = e % C;
    r[i][0] = r[i][1] = make_uint4(0, 0, 0, 0);
    if (s >= held && s < filled) {
      const __nv_bfloat16* p = x + (first + s) * stride + c * 16;
      r[i][0] = ld_v4(p);
      r[i][1] = ld_v4(p + 8);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(r[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, max(abs_bits(u[j]), abs_bits(u[j] >> 16)));
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if ((tid & 31) == 0) warp_max[tid >> 5] = most;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < APPEND_THREADS / 32; ++i) most = max(most, warp_max[i]);
  const int32_t cell = page * a.c.hkv + h;
  float* scales = is_v ? a.c.v_scale : a.c.k_scale;
  uint8_t* codes = (is_v ? a.c.v : a.c.k) + (int64_t)row * D;
  float scale = fresh_scale<KIND>(most), old = 0.f;
  if (held > 0) {
    old = ld_f32(scales + cell);
    scale = fmaxf(old, scale);
  }
  __syncthreads();                                   // every thread has read the old scale
  if (tid == 0 && !(held > 0 && scale == old)) scales[cell] = scale;
  const float inverse = 1.f / scale;                 // exact for powers of two; x / scale otherwise below
  const bool exact = (__float_as_uint(scale) & 0x7fffffu) == 0;
  if (!is_v && a.c.weight)
    for (int s = held + tid; s < filled; s += APPEND_THREADS) a.c.weight[(int64_t)row + s] = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * APPEND_THREADS + tid, s = e / C, c = e % C;
    if (s >= held && s < filled) {
      const uint32_t* u = reinterpret_cast<const uint32_t*>(r[i]);
      uint32_t out[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 f = make_float4(bf_lo(u[2 * j]), bf_hi(u[2 * j]), bf_lo(u[2 * j + 1]), bf_hi(u[2 * j + 1]));
        out[j] = exact ? to_codes<KIND>(f.x * inverse, f.y * inverse, f.z * inverse, f.w * inverse)
                       : to_codes<KIND>(__fdiv_rn(f.x, scale), __fdiv_rn(f.y, scale), __fdiv_rn(f.z, scale), __fdiv_rn(f.w, scale));
      }
      *reinterpret_cast<uint4*>(codes + s * D + c * 16) = make_uint4(out[0], out[1], out[2], out[3]);
    } else if (s < held && scale != old) {
      const float ratio = __fdiv_rn(old, scale);
      const uint4 u = ld_v4(codes + s * D + c * 16);
      *reinterpret_cast<uint4*>(codes + s * D + c * 16) =
          make_uint4(rescale_codes<KIND>(u.x, ratio), rescale_codes<KIND>(u.y, ratio), rescale_codes<KIND>(u.z, ratio), rescale_codes<KIND>(u.w, ratio));
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
// Products by mma.sync, not tcgen05: a decode step has 1 to 16 rows per KV head, tcgen05 wants 64 or 128, and codes
// have to pass through registers to become halves anyway.
constexpr int CT_KEYS = 128;                          // keys of a tile
constexpr int CT_STAGES = 4;
constexpr int CT_WARPS = 8;                           // consumer warps; one more loads
constexpr int CT_THREADS = (CT_WARPS + 1) * 32;

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
  float* part_o;                                      // workspace: [2 * CTAs][16 * WR][D], [2 * CTAs][16 * WR], [CTAs][8]
  float* part_lse;
  int32_t* split;
};

struct StageMeta {                                    // what a stage holds, for the consumers
  int32_t row0, n, length, head;                      // of the sequence and group
  int32_t row_tile, key0, flags, part;
  float ks[CT_KEYS / 16], vs[CT_KEYS / 16];           // per 16 keys; ks = 0: absent
};
enum { ST_FIRST = 1, ST_LAST = 2, ST_WHOLE = 4, ST_END = 8 };
enum { SP_COUNT = 0, SP_ROW0, SP_N, SP_HEAD, SP_ROW_TILE, SP_W = 8 };

template <int D>
struct AttnSmem {
  static constexpr int TILE = CT_KEYS * D;            // bytes of K or of V
  static constexpr int RING = CT_STAGES * 2 * TILE;
  static constexpr int JOIN = CT_WARPS * 16 * D * 4;  // the warps' partial outputs
  static constexpr int DYN_BYTES = RING + JOIN + 1024;
};

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"(m), "r"(bar), "r"(c0), "r"(c1)
               : "memory");
}
__device__ __forceinline__ uint4 lds_v4(uint32_t addr) {
  uint4 x;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(addr) : "memory");
  return x;
}
__device__ __forceinline__ uint2 lds_v2(uint32_t addr) {
  uint2 x;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(addr) : "memory");
  return x;
}
// D (fp32) += A (16 x 16 halves) * B (16 x 8 halves)
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) { return h2_bits(__floats2half2_rn(lo, hi)); }

// How the tiles of a batch lie in a row: sequence after sequence, its KV heads, their row tiles, their key tiles.
struct TileOrder {
  int32_t rows_per_tile, group, hkv;
  bool all_rows;                                      // one group per KV head, whatever its rows (the weights)
  __device__ __forceinline__ int32_t row_tiles(const SeqView& s) const {
    return s.n <= 0 ? 0 : all_rows ? 1 : (s.n * group + rows_per_tile - 1) / rows_per_tile;
  }
  __device__ __forceinline__ int32_t key_tiles(const SeqView& s) const { return s.length <= 0 ? 1 : (s.length + CT_KEYS - 1) / CT_KEYS; }
  __device__ __forceinline__ int64_t tiles(const SeqView& s) const { return (int64_t)row_tiles(s) * hkv * key_tiles(s); }
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

// The rows of a thread's fragments: thread (g, t) of a warp holds rows g and g + 8, and of them the head's columns
// [t * D / 4, (t + 1) * D / 4): the sum over columns may be taken in any order, as long as queries and keys agree.
template <int D>
struct QueryRows {
  static constexpr int KS = D / 16;                   // steps of 16 columns
  uint32_t a[KS][4];
  float factor[2];                                    // score of the product -> log2 units, without the key scale
  int32_t limit[2];                                   // keys in front of this position are seen
  int32_t least, most;                                // of the warp's 16 rows (least: of the existing ones)
  int32_t token[2], head[2];                          // packed row and query head; token -1: no such row

  __device__ __forceinline__ void fill(const AttnArgs& A, const StageMeta& m, int first_row, int lane) {
    const int g = lane >> 2, t = lane & 3, n_rows = m.n * A.group;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = first_row + g + 8 * i, j = r / A.group;
      const bool is = r < n_rows;
      token[i] = is ? m.row0 + j : -1;
      head[i] = m.head * A.group + r - j * A.group;
      limit[i] = is ? m.length - m.n + j + 1 : 0;
      uint32_t w[D / 8];
      if (is) {
        const __nv_bfloat16* p = A.q + (int64_t)token[i] * A.q_stride + head[i] * D + t * (D / 4);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const uint4 x = ld_v4(p + c * 8);
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
      const float up = __uint_as_float((uint32_t)(262 - e) << 23);            // 2^(8 - (e - 127)), e <= 255
      factor[i] = A.scale_log2 * __uint_as_float((uint32_t)(e - 8) << 23);    // 2^(e - 127 - 8)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        a[k][i] = pack_half(bf_lo(w[2 * k]) * up, bf_hi(w[2 * k]) * up);
        a[k][i + 2] = pack_half(bf_lo(w[2 * k + 1]) * up, bf_hi(w[2 * k + 1]) * up);
      }
    }
    const int last = min(first_row + 15, n_rows - 1);
    least = m.length - m.n + first_row / A.group + 1;
    most = first_row < n_rows ? m.length - m.n + last / A.group + 1 : 0;
  }
};

// Shared-memory address of 16 bytes `chunk` of key `key` of a tile, as TMA has swizzled them.
template <int D>
__device__ __forceinline__ uint32_t tile_addr(uint32_t tile, int key, int chunk) {
  return D == 128 ? tile + key * 128 + ((chunk ^ (key & 7)) << 4) : tile + key * 64 + ((chunk ^ ((key >> 1) & 3)) << 4);
}

// Scores of 16 keys (two blocks of 8 columns): S[i][..] = codes of key 8 i + g against the rows.
template <int D, int KIND>
__device__ __forceinline__ void key_codes(uint32_t tile, int key0, int lane, uint32_t (&w)[2][D / 16]) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const uint4 x = lds_v4(tile_addr<D>(tile, key0 + 8 * i + g, t * (D / 64) + c));
      w[i][4 * c] = x.x; w[i][4 * c + 1] = x.y; w[i][4 * c + 2] = x.z; w[i][4 * c + 3] = x.w;
    }
  }
}
template <int D, int KIND>
__device__ __forceinline__ void scores(const QueryRows<D>& q, const uint32_t (&w)[2][D / 16], float (&s)[2][4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
#pragma unroll
    for (int i = 0; i < 2; ++i) mma_f16(s[i], q.a[k][0], q.a[k][1], q.a[k][2], q.a[k][3], halves_lo<KIND>(w[i][k]), halves_hi<KIND>(w[i][k]));
}

// Loading warp: walks the CTA's tiles.  Lanes look 32 sub-blocks of 16 keys (four stages) ahead in page table and scales.
template <int D, bool WEIGHTS>
__device__ __forceinline__ void attn_producer(const AttnArgs& A, const CUtensorMap* tk, const CUtensorMap* tv, const TileOrder& order,
                                              const CtaRange& range, uint32_t ring, StageMeta* meta, uint32_t full, uint32_t empty,
                                              const WaitCtx& ctx) {
  constexpr int SUBS = CT_KEYS / 16;
  const int lane = threadIdx.x & 31, sub = lane & (SUBS - 1);
  const int page_tokens = A.c.page_tokens;
  const bool leads = (sub * 16) % A.box == 0;         // this lane's sub-block begins a box
  int64_t at = range.begin, seq_begin = range.seq_begin;
  int b = range.b, stage = 0;
  uint32_t phase = 0;
  int32_t split[SP_W] = {0, 0, 0, 0, 0, 0, 0, 0};
  bool ok = true;
  while (ok && at < range.end) {
    SeqView s = load_seq(A.s, b);
    int64_t n = order.tiles(s);
    while (at >= seq_begin + n) {                     // sequences without tiles
      seq_begin += n;
      s = load_seq(A.s, ++b);
      n = order.tiles(s);
    }
    const int kt = order.key_tiles(s), rt_n = order.row_tiles(s);
    const int64_t rel = at - seq_begin, grp = rel / kt;
    const int tile0 = (int)(rel - grp * kt), head = (int)(grp / rt_n), rt = (int)(grp - (int64_t)head * rt_n);
    const int tiles = (int)min((int64_t)(kt - tile0), range.end - at);
    const bool begins = tile0 == 0, ends = tile0 + tiles == kt;
    // keys that the last row of the row tile sees
    const int last_row = min((rt + 1) * order.rows_per_tile, s.n * A.group) - 1;
    const int seen = WEIGHTS ? s.length : s.length - s.n + last_row / A.group + 1;
    if (begins && !ends) {
      split[SP_COUNT] = (int)((seq_begin + (grp + 1) * kt - 1) / range.per) - (int)blockIdx.x;
      split[SP_ROW0] = s.row0; split[SP_N] = s.n; split[SP_HEAD] = head; split[SP_ROW_TILE] = rt;
    }
    for (int i0 = 0; ok && i0 < tiles; i0 += 4) {
      float ks = 0.f, vs = 0.f;
      int32_t row = -1;
      const int my_tile = i0 + lane / SUBS, key = (tile0 + my_tile) * CT_KEYS + sub * 16;
      if (my_tile < tiles && key < seen) {
        const int32_t page = ld_i32(A.s.page_table + (int64_t)b * A.s.table_width + key / page_tokens);
        row = page_row(page, A.c.n_pages, A.c.hkv, head, page_tokens);
        if (row >= 0) {
          ks = ld_f32(A.c.k_scale + page * A.c.hkv + head);
          vs = ld_f32(A.c.v_scale + page * A.c.hkv + head);
          row += key % page_tokens;
        }
        if (row < 0 || !usable_scale(ks) || !usable_scale(vs)) {
          mark_bad(A.c.status, row < 0 ? FCP_CACHE_BAD_PAGE : FCP_CACHE_BAD_SCALE, b);
          row = -1;
          ks = vs = 0.f;
        }
      }
      for (int i = i0; i < min(i0 + 4, tiles); ++i) {
        if (!mbar_wait_warp(empty + stage * 8, phase ^ 1, ctx, 911)) {
          ok = false;
          break;
        }
        const bool here = lane / SUBS == i - i0;
        const bool loads = here && leads && row >= 0;
        const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, loads));
        StageMeta& m = meta[stage];
        if (here) {
          m.ks[sub] = ks;
          m.vs[sub] = WEIGHTS ? __int_as_float(row) : vs;       // the weights' place is the codes' row
        }
        if (lane == 0) {
          m.row0 = s.row0; m.n = s.n; m.length = s.length; m.head = head;
          m.row_tile = rt;
          m.key0 = (tile0 + i) * CT_KEYS;
          m.flags = (i == 0 ? ST_FIRST : 0) | (i == tiles - 1 ? ST_LAST : 0) | (begins && ends ? ST_WHOLE : 0);
          m.part = 2 * (int)blockIdx.x + (begins ? 1 : 0);
        }
        __syncwarp();
        const uint32_t bar = full + stage * 8;
        if (lane == 0) {
          const uint32_t bytes = boxes * (uint32_t)(A.box * D) * (WEIGHTS ? 1u : 2u);
          if (bytes) mbar_expect_tx(bar, bytes);
          else mbar_arrive(bar);
        }
        __syncwarp();
        if (loads) {
          const uint32_t dst = ring + stage * 2 * AttnSmem<D>::TILE + sub * 16 * D;
          tma_load_2d(dst, tk, bar, 0, row);
          if (!WEIGHTS) tma_load_2d(dst + AttnSmem<D>::TILE, tv, bar, 0, row);
        }
        __syncwarp();
        if (++stage == CT_STAGES) {
          stage = 0;
          phase ^= 1;
        }
      }
    }
    at += tiles;
  }
  grid_launch_next();
  if (ok && mbar_wait_warp(empty + stage * 8, phase ^ 1, ctx, 912)) {
    if (lane == 0) {
      meta[stage].flags = ST_END;
      mbar_arrive(full + stage * 8);
    }
  }
  if (!WEIGHTS && lane < SP_W) {
    int32_t x = 0;
#pragma unroll
    for (int i = 0; i < SP_W; ++i) x = lane == i ? split[i] : x;
    A.split[blockIdx.x * SP_W + lane] = x;
  }
}

// WR warps side by side hold 16 * WR rows of a group; the 8 / WR warps behind each other take different keys of a tile.
template <int D, int KIND, int WR>
struct AttnConsumer {
  static constexpr int RT = 16 * WR, KG = CT_WARPS / WR, NT = D / 8;
  QueryRows<D> q;
  float o[NT][4];
  float m[2], l[2];

  // 16 keys from `key` (position) on, at `at` in the stage
  __device__ __forceinline__ void step(uint32_t ktile, uint32_t vtile, int at, int key, float ks, float vs, int lane) {
    const int g = lane >> 2, t = lane & 3;
    float s[2][4];
    {
      uint32_t w[2][D / 16];
      key_codes<D, KIND>(ktile, at, lane, w);
      scores<D, KIND>(q, w, s);
    }
    // In log2 units plus log2 of the value scale: w = 2^(a - m) are the weights of the value codes, and the sum of the
    // probabilities is that of w / vs.  The largest w is 2^14, which leaves a half 2^38 below it before it is rounded to 0.
    const float shift = __log2f(vs), f0 = q.factor[0] * ks, f1 = q.factor[1] * ks, inverse = 1.f / vs;
    const bool edge = key + 16 > q.least;
    float m0 = m[0], m1 = m[1];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        s[i][c] = fmaf(s[i][c], f0, shift);
        s[i][c + 2] = fmaf(s[i][c + 2], f1, shift);
        if (edge) {
          const int pos = key + 8 * i + 2 * t + c;
          if (pos >= q.limit[0]) s[i][c] = -INFINITY;
          if (pos >= q.limit[1]) s[i][c + 2] = -INFINITY;
        }
        m0 = fmaxf(m0, s[i][c]);
        m1 = fmaxf(m1, s[i][c + 2]);
      }
    m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 1));
    m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 1));
    m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 2));
    m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 2));
    if (__any_sync(0xffffffffu, m0 > m[0] || m1 > m[1])) {
      const float r0 = exp2_approx(m[0] - m0), r1 = exp2_approx(m[1] - m1);
      l[0] *= r0;
      l[1] *= r1;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        o[j][0] *= r0; o[j][1] *= r0;
        o[j][2] *= r1; o[j][3] *= r1;
      }
      m[0] = m0;
      m[1] = m1;
    }
    const float e0 = m0 - 14.f, e1 = m1 - 14.f;
    float z0 = 0.f, z1 = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        s[i][c] = exp2_approx(s[i][c] - e0);
        s[i][c + 2] = exp2_approx(s[i][c + 2] - e1);
        z0 += s[i][c];
        z1 += s[i][c + 2];
      }
    l[0] = fmaf(z0, inverse, l[0]);
    l[1] = fmaf(z1, inverse, l[1]);
    const uint32_t p0 = pack_half(s[0][0], s[0][1]), p1 = pack_half(s[0][2], s[0][3]);
    const uint32_t p2 = pack_half(s[1][0], s[1][1]), p3 = pack_half(s[1][2], s[1][3]);
    // value codes: thread (g, t) reads columns [g D/8, (g+1) D/8) of keys 2t, 2t+1, 2t+8, 2t+9; block j of 8 output columns
    // is then column g D/8 + j
    uint32_t v[4][D / 32];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int kk = 2 * t + (i & 1) + 8 * (i >> 1);
      if (D == 128) {
        const uint4 x = lds_v4(tile_addr<D>(vtile, at + kk, g));
        v[i][0] = x.x; v[i][1] = x.y; v[i][D / 32 - 2] = x.z; v[i][D / 32 - 1] = x.w;
      } else {
        const uint2 x = lds_v2(tile_addr<D>(vtile, at + kk, g >> 1) + (g & 1) * 8);
        v[i][0] = x.x; v[i][1] = x.y;
      }
    }
    bool careful = false;
    if (edge) {
      // what lies behind the last key that any row sees is whatever the page held: it must not meet a zero weight
      bool nan = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool past = key + 2 * t + (i & 1) + 8 * (i >> 1) >= q.most;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          if (past) v[i][c] = 0;
          if (KIND == FCP_CACHE_E4M3) nan |= __vcmpeq4(v[i][c] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
        }
      }
      careful = KIND == FCP_CACHE_E4M3 && __any_sync(0xffffffffu, nan);
    }
    if (KIND == FCP_CACHE_E4M3 && careful) {
      // a NaN that only some of the rows see: key by key, and only into the rows that see it
#pragma unroll 1
      for (int k = 0; k < 16; ++k) {
        const bool mine = t == ((k & 7) >> 1), odd = k & 1, high = k >> 3;
        const uint32_t keep = odd ? 0xffff0000u : 0x0000ffffu;
        const uint32_t a0 = mine && !high ? p0 & keep : 0, a1 = mine && !high ? p1 & keep : 0;
        const uint32_t a2 = mine && high ? p2 & keep : 0, a3 = mine && high ? p3 & keep : 0;
        const bool see0 = key + k < q.limit[0], see1 = key + k < q.limit[1];
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = mine && (i & 1) == odd && (i >> 1) == high ? v[i][c] : 0;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t b0 = __byte_perm(x[0], x[1], h ? 0x7362 : 0x5140), b1 = __byte_perm(x[2], x[3], h ? 0x7362 : 0x5140);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float d[4] = {0.f, 0.f, 0.f, 0.f};
              mma_f16(d, a0, a1, a2, a3, e ? halves_hi<KIND>(b0) : halves_lo<KIND>(b0), e ? halves_hi<KIND>(b1) : halves_lo<KIND>(b1));
              float (&acc)[4] = o[4 * c + 2 * h + e];
              if (see0) { acc[0] += d[0]; acc[1] += d[1]; }
              if (see1) { acc[2] += d[2]; acc[3] += d[3]; }
            }
          }
        }
      }
      return;
    }
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t b0 = __byte_perm(v[0][c], v[1][c], h ? 0x7362 : 0x5140), b1 = __byte_perm(v[2][c], v[3][c], h ? 0x7362 : 0x5140);
        mma_f16(o[4 * c + 2 * h], p0, p1, p2, p3, halves_lo<KIND>(b0), halves_lo<KIND>(b1));
        mma_f16(o[4 * c + 2 * h + 1], p0, p1, p2, p3, halves_hi<KIND>(b0), halves_hi<KIND>(b1));
      }
  }

  // Place of 16 bytes `i` of the thread column t's run (D / 16 of them) of a row, spread over the banks.
  __device__ static __forceinline__ int join_slot(int row, int t, int i) {
    return row * (D / 4) + t * (D / 16) + (D == 128 ? (i ^ (2 * t + (row & 1))) : (i ^ ((t >> 1) + 2 * (row & 1))));
  }

  // The end of a group's tiles on this CTA: joins the warps and writes the rows, or their partial result.
  __device__ __forceinline__ void finish(const AttnArgs& A, const StageMeta& meta, float4* join, float2 (*stats)[16], int warp, int lane) {
    const int g = lane >> 2, t = lane & 3, tid = warp * 32 + lane;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    }
    asm volatile("bar.sync 1, %0;" ::"n"(CT_WARPS * 32) : "memory");       // the join area's last readers are done
    float4* mine = join + warp * 16 * (D / 4);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (q.token[i] < 0) continue;
      const int row = g + 8 * i;
      if (t == 0) stats[warp][row] = make_float2(m[i], l[i]);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        const int j = 4 * (c % (D / 32)), e = 2 * i + c / (D / 32);
        mine[join_slot(row, t, c)] = make_float4(o[j][e], o[j + 1][e], o[j + 2][e], o[j + 3][e]);
      }
    }
    asm volatile("bar.sync 1, %0;" ::"n"(CT_WARPS * 32) : "memory");
    const int n_rows = min(RT, meta.n * A.group - meta.row_tile * RT);
    for (int e = tid; e < n_rows * (D / 4); e += CT_WARPS * 32) {
      const int r = e / (D / 4), f = e % (D / 4), wr = r / 16, row = r % 16;
      float top = -3e38f;
#pragma unroll
      for (int k = 0; k < KG; ++k) top = fmaxf(top, stats[k * WR + wr][row].x);
      float z = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < KG; ++k) {
        const float2 ml = stats[k * WR + wr][row];
        const float w = exp2_approx(ml.x - top);
        const float4 y = join[(k * WR + wr) * 16 * (D / 4) + join_slot(row, f / (D / 16), f % (D / 16))];
        z = fmaf(ml.y, w, z);
        x.x = fmaf(y.x, w, x.x); x.y = fmaf(y.y, w, x.y); x.z = fmaf(y.z, w, x.z); x.w = fmaf(y.w, w, x.w);
      }
      const float inverse = z == 0.f ? 0.f : 1.f / z;
      const float lse2 = z == 0.f ? -INFINITY : top - 14.f + __log2f(z);
      x.x *= inverse; x.y *= inverse; x.z *= inverse; x.w *= inverse;
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
  }

  __device__ __forceinline__ void run(const AttnArgs& A, uint32_t ring, StageMeta* metas, float4* join, float2 (*stats)[16], uint32_t full,
                                      uint32_t empty, const WaitCtx& ctx) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wr = warp % WR, kg = warp / WR;
    int stage = 0;
    uint32_t phase = 0;
    while (mbar_wait_warp(full + stage * 8, phase, ctx, 921)) {
      const StageMeta& meta = metas[stage];
      const int flags = meta.flags;
      if (flags & ST_END) break;
      if (flags & ST_FIRST) {
        q.fill(A, meta, meta.row_tile * RT + wr * 16, lane);
        m[0] = m[1] = -3e38f;
        l[0] = l[1] = 0.f;
#pragma unroll
        for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
      }
      const uint32_t ktile = ring + stage * 2 * AttnSmem<D>::TILE, vtile = ktile + AttnSmem<D>::TILE;
#pragma unroll 1
      for (int i = 0; i < WR; ++i) {
        const int sub = kg * WR + i, key = meta.key0 + sub * 16;
        const float ks = meta.ks[sub], vs = meta.vs[sub];
        if (key < q.most && ks != 0.f) step(ktile, vtile, sub * 16, key, ks, vs, lane);
      }
      if (flags & ST_LAST) finish(A, meta, join, stats, warp, lane);
      __syncwarp();
      if (lane == 0) mbar_arrive(empty + stage * 8);
      if (++stage == CT_STAGES) {
        stage = 0;
        phase ^= 1;
      }
    }
  }
};

// Weights of the cached keys: the scores once more, against the finished log-sum-exps.  A warp holds 16 keys and goes over
// the rows in tiles of 16, so that a key's sum is taken by one thread column in a fixed order.
template <int D, int KIND>
__device__ __forceinline__ void weight_consumer(const AttnArgs& A, uint32_t ring, StageMeta* metas, uint32_t full, uint32_t empty,
                                                const WaitCtx& ctx) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  int stage = 0;
  uint32_t phase = 0;
  QueryRows<D> q;
  float lse2[2] = {0.f, 0.f};
  while (mbar_wait_warp(full + stage * 8, phase, ctx, 931)) {
    const StageMeta& meta = metas[stage];
    if (meta.flags & ST_END) break;
    const int sub = warp, key = meta.key0 + sub * 16, n_rows = meta.n * A.group;
    const float ks = meta.ks[sub];
    auto rows_from = [&](int r) {
      q.fill(A, meta, r, lane);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        lse2[i] = q.token[i] >= 0 ? ld_f32(A.lse + (int64_t)q.token[i] * A.hq + q.head[i]) * 1.4426950408889634f : INFINITY;
    };
    if (n_rows <= 16 && (meta.flags & ST_FIRST)) rows_from(0);
    if (key < meta.length && ks != 0.f) {
      uint32_t w[2][D / 16];
      key_codes<D, KIND>(ring + stage * 2 * AttnSmem<D>::TILE, sub * 16, lane, w);
      float sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll 1
      for (int r = 0; r < n_rows; r += 16) {
        if (n_rows > 16) rows_from(r);
        float s[2][4];
        scores<D, KIND>(q, w, s);
        const float f0 = q.factor[0] * ks, f1 = q.factor[1] * ks;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int pos = key + 8 * i + 2 * t + c;
            if (pos < q.limit[0]) sum[i][c] += exp2_approx(fmaf(s[i][c], f0, -lse2[0]));
            if (pos < q.limit[1]) sum[i][c] += exp2_approx(fmaf(s[i][c + 2], f1, -lse2[1]));
          }
      }
#pragma unroll
      for (int o = 4; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int c = 0; c < 2; ++c) sum[i][c] += __shfl_xor_sync(0xffffffffu, sum[i][c], o);
      // lanes of thread row 0 and 1 write the two blocks of 8 keys
      const int pos = key + 8 * g + 2 * t;
      if (g < 2 && pos < meta.length) {
        float* dst = A.c.weight + (int64_t)__float_as_int(meta.vs[sub]) + 8 * g + 2 * t;
        dst[0] += g ? sum[1][0] : sum[0][0];
        if (pos + 1 < meta.length) dst[1] += g ? sum[1][1] : sum[0][1];
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty + stage * 8);
    if (++stage == CT_STAGES) {
      stage = 0;
      phase ^= 1;
    }
  }
}

// WR = 0: the weights.
template <int D, int KIND, int WR>
__global__ void __launch_bounds__(CT_THREADS, 1)
cache_attn_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv, const __grid_constant__ AttnArgs A) {
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[2 * CT_STAGES];
  __shared__ __align__(16) StageMeta metas[CT_STAGES];
  __shared__ float2 stats[CT_WARPS][16];
  __shared__ int64_t scratch[16];
  __shared__ int abort_flag;
  const int warp = threadIdx.x >> 5;
  const uint32_t full = smem_u32(bars), empty = full + CT_STAGES * 8;
  // the swizzle pattern repeats every 1024 bytes of address
  const uint32_t ring = (smem_u32(smem) + 1023u) & ~1023u;
  uint8_t* base = smem + (ring - smem_u32(smem));
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < CT_STAGES; ++i) {
      mbar_init(full + i * 8, 1);
      mbar_init(empty + i * 8, CT_WARPS);
    }
    fence_mbar_init();
    prefetch_tmap(&tk);
    prefetch_tmap(&tv);
  }
  grid_wait();
  __syncthreads();
  const WaitCtx ctx = {&abort_flag, A.c.status, (uint32_t)FCP_WAIT_NS};
  TileOrder order = {WR ? 16 * WR : 16, A.group, A.c.hkv, WR == 0};
  const CtaRange range = cta_range(A.s, order, A.c.status, scratch);
  if (warp == CT_WARPS) {
    attn_producer<D, WR == 0>(A, &tk, &tv, order, range, ring, metas, full, empty, ctx);
  } else if constexpr (WR == 0) {
    weight_consumer<D, KIND>(A, ring, metas, full, empty, ctx);
  } else {
    AttnConsumer<D, KIND, WR> consumer;
    consumer.run(A, ring, metas, reinterpret_cast<float4*>(base + AttnSmem<D>::RING), stats, full, empty, ctx);
  }
  __syncthreads();
  wait_teardown(ctx);
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
    float top = -INFINITY;
    for (int i = 0; i <= count; ++i) top = fmaxf(top, ld_f32(A.part_lse + (int64_t)part(i) * rows_per_tile + r));
    const float ref = top == -INFINITY ? 0.f : top;
    float z = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i <= count; ++i) {
      const int64_t at = (int64_t)part(i) * rows_per_tile + r;
      const float w = exp2_approx(ld_f32(A.part_lse + at) - ref);
      const float4 y = ld_stream_f4(A.part_o + at * D + f * 4);
      z += w;
      x.x = fmaf(y.x, w, x.x); x.y = fmaf(y.y, w, x.y); x.z = fmaf(y.z, w, x.z); x.w = fmaf(y.w, w, x.w);
    }
    const float inverse = z == 0.f ? 0.f : 1.f / z;
    const int gr = first + r, j = gr / A.group;
    const int64_t out = (int64_t)(row0 + j) * A.hq + head * A.group + gr - j * A.group;
    *reinterpret_cast<uint2*>(A.o + out * D + f * 4) = make_uint2(pack_bf16(x.x * inverse, x.y * inverse), pack_bf16(x.z * inverse, x.w * inverse));
    if (f == 0) A.lse[out] = z == 0.f ? -INFINITY : (ref + __log2f(z)) * 0.69314718055994531f;
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

// Weights as unsigned keys of the same order; NaN and what lies on a page that does not exist come last.
__device__ __forceinline__ uint32_t weight_key(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// Which tokens of a head stay: one block per (KV head, sequence).  The n_heavy largest weights by four counting passes over
// 8 bits of the keys, from the top; then one pass writes the kept positions in order.
constexpr int SELECT_THREADS = 1024;
constexpr int SELECT_KEYS = 49152;                    // as many keys stay in shared memory
constexpr int SELECT_COPIES = 8;                      // of the counters: fewer threads meet on one
constexpr int SELECT_BYTES = SELECT_KEYS * 4;
__global__ void __launch_bounds__(SELECT_THREADS) cache_select_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ uint32_t keys[];
  __shared__ uint32_t count[SELECT_COPIES][256];
  __shared__ uint32_t warp_count[32][2];
  __shared__ uint32_t chosen[2];                      // digit, how many are still wanted among the keys that have it
  grid_begin();
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int keep = a.n_sink + a.n_heavy + a.n_recent;
  const int length = usable_length(a.s, b);
  if (length < 0 && h == 0 && tid == 0) mark_bad(a.c.status, FCP_CACHE_BAD_LENGTH, b);
  int32_t* kept = a.kept + ((int64_t)b * a.c.hkv + h) * keep;
  if (h == 0 && tid == 0) a.new_length[b] = max(0, min(length, keep));
  if (length <= keep) {
    for (int i = tid; i < keep; i += SELECT_THREADS) kept[i] = i < length ? i : -1;
    return;
  }
  const int page_tokens = a.c.page_tokens, end = length - a.n_recent, n = end - a.n_sink;      // candidates [n_sink, end)
  auto key_at = [&](int pos) {
    const int32_t row = page_row(ld_i32(a.s.page_table + (int64_t)b * a.s.table_width + pos / page_tokens), a.c.n_pages, a.c.hkv, h, page_tokens);
    return row < 0 ? 0u : weight_key(ld_f32(a.c.weight + (int64_t)row + pos % page_tokens));
  };
  const bool in_smem = n <= SELECT_KEYS;
  if (in_smem)
    for (int i = tid; i < n; i += SELECT_THREADS) keys[i] = key_at(a.n_sink + i);
  uint32_t prefix = 0, wanted = (uint32_t)a.n_heavy;
  for (int shift = 24; shift >= 0 && a.n_heavy > 0; shift -= 8) {
    for (int i = tid; i < SELECT_COPIES * 256; i += SELECT_THREADS) (&count[0][0])[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += SELECT_THREADS) {
      const uint32_t k = in_smem ? keys[i] : key_at(a.n_sink + i);
      if (shift == 24 || k >> (shift + 8) == prefix) atomicAdd(&count[warp % SELECT_COPIES][(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (warp == 0) {                                  // from digit 255 down, 8 digits per lane
      uint32_t c[8], sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        c[j] = 0;
#pragma unroll
        for (int k = 0; k < SELECT_COPIES; ++k) c[j] += count[k][255 - (lane * 8 + j)];
        sum += c[j];
      }
      uint32_t upto = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      uint32_t before = upto - sum;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (before < wanted && wanted <= before + c[j]) {
          chosen[0] = (uint32_t)(255 - (lane * 8 + j));
          chosen[1] = wanted - before;
        }
        before += c[j];
      }
    }
    __syncthreads();
    prefix = prefix << 8 | chosen[0];
    wanted = chosen[1];
  }
  // prefix is the smallest kept key, `wanted` of its equals are kept: the first ones
  uint32_t above_base = 0, equal_base = 0;            // kept and equal keys in front of this trip
  for (int i = tid; i < a.n_sink; i += SELECT_THREADS) kept[i] = i;
  for (int i = tid; i < a.n_recent; i += SELECT_THREADS) kept[a.n_sink + a.n_heavy + i] = end + i;
  for (int i0 = 0; i0 < n && a.n_heavy > 0; i0 += SELECT_THREADS) {
    const int i = i0 + tid;
    const uint32_t k = i < n ? (in_smem ? keys[i] : key_at(a.n_sink + i)) : 0u;
    const bool above = i < n && k > prefix, equal = i < n && k == prefix;
    const uint32_t am = __ballot_sync(0xffffffffu, above), em = __ballot_sync(0xffffffffu, equal);
    if (lane == 0) {
      warp_count[warp][0] = __popc(am);
      warp_count[warp][1] = __popc(em);
    }
    __syncthreads();
    uint32_t av = warp_count[lane][0], ev = warp_count[lane][1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, av, o), y = __shfl_up_sync(0xffffffffu, ev, o);
      if (lane >= o) {
        av += x;
        ev += y;
      }
    }
    const uint32_t below = (1u << lane) - 1u;
    const uint32_t a_before = above_base + (warp ? __shfl_sync(0xffffffffu, av, warp - 1) : 0u) + __popc(am & below);
    const uint32_t e_before = equal_base + (warp ? __shfl_sync(0xffffffffu, ev, warp - 1) : 0u) + __popc(em & below);
    if (above || (equal && e_before < wanted)) kept[a.n_sink + a_before + min(e_before, wanted)] = a.n_sink + i;
    above_base += __shfl_sync(0xffffffffu, av, 31);
    equal_base += __shfl_sync(0xffffffffu, ev, 31);
    __syncthreads();
  }
}

// The kept tokens into their new pages: one block per (new page, KV head, sequence).
constexpr int MOVE_THREADS = 128;
template <int D, int KIND>
__global__ void __launch_bounds__(MOVE_THREADS) cache_move_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ int32_t src_row[128];                    // of every token; -1: none
  __shared__ float src_scale[2][128];
  __shared__ float top[2];
  grid_begin();
  const int page = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int keep = a.n_sink + a.n_heavy + a.n_recent, page_tokens = a.c.page_tokens;
  const int n = min(page_tokens, ld_i32(a.new_length + b) - page * page_tokens);
  if (n <= 0) return;
  const int32_t dst_page = ld_i32(a.dst_table + (int64_t)b * a.dst_width + page);
  const int32_t dst_row = page_row(dst_page, a.c.n_pages, a.c.hkv, h, page_tokens);
  if (dst_row < 0) {
    if (tid == 0) mark_bad(a.c.status, FCP_CACHE_BAD_PAGE, b);
    return;
  }
  if (tid < n) {
    const int pos = ld_i32(a.kept + ((int64_t)b * a.c.hkv + h) * keep + page * page_tokens + tid);
    const int32_t src = ld_i32(a.s.page_table + (int64_t)b * a.s.table_width + pos / page_tokens);
    int32_t row = page_row(src, a.c.n_pages, a.c.hkv, h, page_tokens);
    float ks = 0.f, vs = 0.f;
    if (row >= 0) {
      ks = ld_f32(a.c.k_scale + src * a.c.hkv + h);
      vs = ld_f32(a.c.v_scale + src * a.c.hkv + h);
    }
    if (row < 0 || !usable_scale(ks) || !usable_scale(vs)) {
      mark_bad(a.c.status, row < 0 ? FCP_CACHE_BAD_PAGE : FCP_CACHE_BAD_SCALE, b);
      row = -1;
      ks = vs = 0.f;
    } else {
      row += pos % page_tokens;
    }
    src_row[tid] = row;
    src_scale[0][tid] = ks;
    src_scale[1][tid] = vs;
    a.c.weight[(int64_t)dst_row + tid] = row < 0 ? 0.f : ld_f32(a.c.weight + row);
  }
  __syncthreads();
  if (tid < 64) {                                     // one warp for the keys' scale, one for the values'
    const int which = tid >> 5;
    float m = FCP_CACHE_MIN_SCALE;
    for (int i = tid & 31; i < n; i += 32) m = fmaxf(m, src_scale[which][i]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((tid & 31) == 0) {
      top[which] = m;
      (which ? a.c.v_scale : a.c.k_scale)[dst_page * a.c.hkv + h] = m;
    }
  }
  __syncthreads();
  constexpr int C = D / 16;
  for (int e = tid; e < 2 * n * C; e += MOVE_THREADS) {
    const int which = e / (n * C), r = e - which * n * C, s = r / C, c = r % C;
    uint8_t* codes = which ? a.c.v : a.c.k;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (src_row[s] >= 0) {
      x = ld_v4(codes + (int64_t)src_row[s] * D + c * 16);
      if (src_scale[which][s] != top[which]) {
        const float ratio = __fdiv_rn(src_scale[which][s], top[which]);
        x = make_uint4(rescale_codes<KIND>(x.x, ratio), rescale_codes<KIND>(x.y, ratio), rescale_codes<KIND>(x.z, ratio), rescale_codes<KIND>(x.w, ratio));
      }
    }
    *reinterpret_cast<uint4*>(codes + ((int64_t)dst_row + s) * D + c * 16) = x;
  }
}

}  // namespace fcp
