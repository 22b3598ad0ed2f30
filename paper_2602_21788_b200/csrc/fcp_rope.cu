// Rotary positions: table (host) and the kernel behind fcp_rope_fwd and fcp_rope_bwd.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "fcp_launch.cuh"
#include "sm100_ptx.cuh"

using namespace fcp;

// ---------------------------------------------------------------------------------------------
// Table
// ---------------------------------------------------------------------------------------------
extern "C" int fcp_rope_init(const fcp_rope_config* c, fcp_rope_table* t) {
  if (!c || !t) {
    fcp_set_error("fcp_rope_init: NULL argument");
    return FCP_ERR_INVALID_ARG;
  }
  if (c->head_dim != 64 && c->head_dim != 128) {
    fcp_set_error("fcp_rope_init: head_dim %d is not 64 or 128", c->head_dim);
    return FCP_ERR_UNSUPPORTED;
  }
  const int r = c->rotary_dim;
  const double b = c->base, s = c->factor, o = c->original_length;
  const bool by_length = c->scaling == FCP_ROPE_YARN || c->scaling == FCP_ROPE_WAVELENGTH;
  const double low = c->low > 0 ? c->low : 1.0;
  const double high = c->high > 0 ? c->high : c->scaling == FCP_ROPE_YARN ? 32.0 : 4.0;
  if (r < 2 || r % 2 != 0 || r > c->head_dim || (c->layout != FCP_ROPE_HALF && c->layout != FCP_ROPE_INTERLEAVED) ||
      c->scaling < FCP_ROPE_NONE || c->scaling > FCP_ROPE_WAVELENGTH) {
    fcp_set_error("fcp_rope_init: rotary_dim %d, layout %d or scaling %d", r, c->layout, c->scaling);
    return FCP_ERR_INVALID_ARG;
  }
  if (!(b > 1.0) || !std::isfinite(b) ||
      (c->scaling != FCP_ROPE_NONE && (!(s >= 1.0) || !std::isfinite(s) || (c->scaling == FCP_ROPE_NTK && r < 4))) ||
      (by_length && (!(o > 0.0) || !std::isfinite(o) || !(low < high) || !std::isfinite(high))) ||
      !std::isfinite(c->magnitude) || std::isnan(c->low) || std::isnan(c->high)) {
    fcp_set_error("fcp_rope_init: base %g, factor %g, original_length %g, low %g, high %g, magnitude %g", b, s, o, low, high,
                  c->magnitude);
    return FCP_ERR_INVALID_ARG;
  }
  const double two_pi = 6.283185307179586476925286766559;
  const double base = c->scaling == FCP_ROPE_NTK ? b * std::pow(s, r / (r - 2.0)) : b;
  double lo = 0.0, hi = 0.0;
  if (c->scaling == FCP_ROPE_YARN) {         // dimensions that turn `high` and `low` times within the original length
    lo = std::floor(r * std::log(o / (high * two_pi)) / (2.0 * std::log(b)));
    hi = std::ceil(r * std::log(o / (low * two_pi)) / (2.0 * std::log(b)));
    lo = std::fmin(std::fmax(lo, 0.0), r - 1.0);
    hi = std::fmin(std::fmax(hi, 0.0), r - 1.0);
  }
  t->head_dim = c->head_dim;
  t->rotary_dim = r;
  t->layout = c->layout;
  t->magnitude = c->magnitude > 0 ? (float)c->magnitude : c->scaling == FCP_ROPE_YARN ? (float)(0.1 * std::log(s) + 1.0) : 1.0f;
  for (int i = 0; i < 64; ++i) {
    double f = i < r / 2 ? std::pow(base, -2.0 * i / r) : 0.0;
    if (c->scaling == FCP_ROPE_LINEAR) f /= s;
    if (c->scaling == FCP_ROPE_YARN) {
      const double w = std::fmin(std::fmax((i - lo) / std::fmax(hi - lo, 1e-3), 0.0), 1.0);
      f = f / s * w + f * (1.0 - w);
    }
    if (c->scaling == FCP_ROPE_WAVELENGTH) {
      const double u = std::fmin(std::fmax((o * f / two_pi - low) / (high - low), 0.0), 1.0);
      f = f * u + f / s * (1.0 - u);
    }
    t->turn[i] = (uint64_t)((long double)f / 6.283185307179586476925286766559005768L * 18446744073709551616.0L + 0.5L);
  }
  return FCP_OK;
}

// ---------------------------------------------------------------------------------------------
// Kernel
// ---------------------------------------------------------------------------------------------
namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_TOKENS = 16;          // most tokens of one block
constexpr int ROPE_SLOTS = 1280;         // most slots of a block: 5 per thread
constexpr int ROPE_RESIDENT = 8;         // blocks of an SM

struct RopeArgs {
  const __nv_bfloat16 *q, *k;
  __nv_bfloat16 *q_out, *k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
  const int32_t *positions, *row_offset, *length;
  int32_t T, B, hq, hkv, D, rotary, tokens;          // tokens: per block
  float sign, magnitude;
  uint64_t turn[64];
};

__device__ __forceinline__ int32_t ld_i32(const int32_t* p) {
  int32_t x;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(x) : "l"(p));
  return x;
}

__device__ __forceinline__ void turn_pair(float& x, float& y, float2 cs) {
  const float a = x * cs.x - y * cs.y, b = y * cs.x + x * cs.y;
  x = a;
  y = b;
}
__device__ __forceinline__ float2 unpack(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// HBM bound.  A block takes a few tokens: one sine and cosine per (token, pair), shared by all heads through shared memory,
// then slots of 16 columns, heads fastest, so that neighbouring threads move neighbouring bytes.
// WIDE: rotary_dim is a multiple of 16 and everything 16-byte aligned; a slot is 8 pairs in two 16-byte pieces (or 16 copied
// columns).  Otherwise a slot is one pair, moved as two values.
template <bool WIDE, int LAYOUT>
__global__ void __launch_bounds__(ROPE_THREADS, ROPE_RESIDENT) rope_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ __align__(16) float2 cs[ROPE_TOKENS * 64];
  __shared__ int64_t pos[ROPE_TOKENS];
  __shared__ int32_t ok[ROPE_TOKENS];
  grid_begin();
  const int t0 = blockIdx.x * a.tokens, n = min(a.tokens, a.T - t0);
  const int tid = threadIdx.x;
  const int pairs = a.rotary / 2, turned = a.rotary / 16;
  // slots of a head's row: a power of two, so that a thread keeps its slot and steps over rows
  const int heads = a.hq + a.hkv, slots = WIDE ? a.D / 16 : a.D / 2;
  const int s = tid & (slots - 1), stride = ROPE_THREADS / slots;
  int t = 0, h = tid / slots;                        // token and head of the row to be fetched next
  auto settle = [&] {
    while (h >= heads) {
      h -= heads;
      ++t;
    }
  };
  settle();
  auto row = [&](const __nv_bfloat16*& src, __nv_bfloat16*& dst) {
    const int64_t tok = t0 + t;
    if (h < a.hq) {
      src = a.q + tok * a.q_stride + h * a.D;
      dst = a.q_out + tok * a.q_out_stride + h * a.D;
    } else {
      src = a.k + tok * a.k_stride + (h - a.hq) * a.D;
      dst = a.k_out + tok * a.k_out_stride + (h - a.hq) * a.D;
    }
  };
  // columns of a wide slot's two pieces
  const bool half = LAYOUT == FCP_ROPE_HALF && s < turned;
  const int cx = half ? s * 8 : s * 16, cy = half ? pairs + s * 8 : s * 16 + 8;
  uint4 x, y;
  __nv_bfloat16* dst;
  int at;                                            // token of the slot that was fetched; -1: none
  auto fetch = [&] {
    at = -1;
    if (t < n) {
      const __nv_bfloat16* src;
      row(src, dst);
      at = t;
      x = ld_v4(src + cx);
      y = ld_v4(src + cy);
      h += stride;
      settle();
    }
  };
  if (WIDE) fetch();                                 // the first values travel while positions and angles are found
  if (a.positions) {
    if (tid < n) {
      pos[tid] = ld_i32(a.positions + t0 + tid);
      ok[tid] = 1;
    }
  } else {
    // sequence of the block's first token: the last b with row_offset[b] <= t0, found by all threads, 256 offsets a round
    int lo = 0, hi = a.B;                            // row_offset[lo] <= t0 assumed; first b in (lo, hi] above t0
    while (lo < hi) {
      const int step = (hi - lo + ROPE_THREADS - 1) / ROPE_THREADS;
      const int at = lo + (tid + 1) * step;
      const int below = __syncthreads_count(at <= hi && ld_i32(a.row_offset + min(at, a.B)) <= t0);
      lo += below * step;
      hi = min(hi, lo + step - 1);
    }
    if (tid < n) {
      int b = lo;
      while (b < a.B && ld_i32(a.row_offset + b + 1) <= t0 + tid) ++b;
      const int first = b < a.B ? ld_i32(a.row_offset + b) : 0;
      int64_t p = (int64_t)(t0 + tid) - first;
      if (b < a.B && a.length) p += (int64_t)ld_i32(a.length + b) - ((int64_t)ld_i32(a.row_offset + b + 1) - first);
      pos[tid] = p;
      ok[tid] = b < a.B && first <= t0 + tid;
    }
  }
  __syncthreads();
  for (int i = tid; i < n * pairs; i += ROPE_THREADS) {
    const int t = i / pairs, p = i - t * pairs;
    const int32_t part = (int32_t)(((uint64_t)pos[t] * a.turn[p]) >> 32);      // fraction of a turn, two's complement
    float sine, cosine;
    sincospif((float)part * 0x1p-31f, &sine, &cosine);
    cs[t * 64 + p] = make_float2(cosine * a.magnitude, sine * a.magnitude * a.sign);
  }
  __syncthreads();
  if (WIDE) {
    for (; at >= 0; fetch()) {
      if (!ok[at]) continue;
      if (s < turned) {
        uint32_t wx[4] = {x.x, x.y, x.z, x.w}, wy[4] = {y.x, y.y, y.z, y.w};
        const float4* c4 = reinterpret_cast<const float4*>(cs + at * 64 + s * 8);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float2 u = unpack(wx[j]), v = unpack(wy[j]);
          if (LAYOUT == FCP_ROPE_HALF) {             // words j of both pieces: pairs 2j, 2j + 1
            const float4 c = c4[j];
            turn_pair(u.x, v.x, make_float2(c.x, c.y));
            turn_pair(u.y, v.y, make_float2(c.z, c.w));
          } else {                                   // word j of a piece is a pair
            const float4 c = c4[j >> 1], d = c4[2 + (j >> 1)];
            turn_pair(u.x, u.y, j & 1 ? make_float2(c.z, c.w) : make_float2(c.x, c.y));
            turn_pair(v.x, v.y, j & 1 ? make_float2(d.z, d.w) : make_float2(d.x, d.y));
          }
          wx[j] = pack_bf16(u.x, u.y);
          wy[j] = pack_bf16(v.x, v.y);
        }
        x = make_uint4(wx[0], wx[1], wx[2], wx[3]);
        y = make_uint4(wy[0], wy[1], wy[2], wy[3]);
      }
      *reinterpret_cast<uint4*>(dst + cx) = x;
      *reinterpret_cast<uint4*>(dst + cy) = y;
    }
  } else {
    const int c0 = LAYOUT == FCP_ROPE_HALF && s < pairs ? s : 2 * s, c1 = LAYOUT == FCP_ROPE_HALF && s < pairs ? s + pairs : 2 * s + 1;
    for (; t < n; h += stride, settle()) {
      const __nv_bfloat16* src;
      __nv_bfloat16* to;
      row(src, to);
      if (!ok[t]) continue;
      const volatile uint16_t* bits = reinterpret_cast<const volatile uint16_t*>(src);
      uint16_t o0 = bits[c0], o1 = bits[c1];
      if (s < pairs) {
        float u = __uint_as_float((uint32_t)o0 << 16), v = __uint_as_float((uint32_t)o1 << 16);
        turn_pair(u, v, cs[t * 64 + s]);
        o0 = __bfloat16_as_ushort(__float2bfloat16_rn(u));
        o1 = __bfloat16_as_ushort(__float2bfloat16_rn(v));
      }
      reinterpret_cast<uint16_t*>(to)[c0] = o0;
      reinterpret_cast<uint16_t*>(to)[c1] = o1;
    }
  }
}

int rope(const char* call, float sign, const fcp_rope_table* table, int64_t T, const void* q, int64_t q_stride, int32_t hq,
         const void* k, int64_t k_stride, int32_t hkv, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride,
         const int32_t* positions, const int32_t* row_offset, const int32_t* length, int32_t B, void* stream) {
  // the search for a row's sequence looks up to a block's threads behind the last one
  if (!table || T < 0 || T >= (int64_t(1) << 31) - 8 || hq < 0 || hkv < 0 || B < 0 || B >= (int64_t(1) << 31) - ROPE_THREADS || (int64_t)hq + hkv > 65536 ||
      (T > 0 && ((hq > 0 && (!q || !q_out)) || (hkv > 0 && (!k || !k_out)) || (!positions && !row_offset)))) {
    fcp_set_error("%s: NULL buffer or invalid size", call);
    return FCP_ERR_INVALID_ARG;
  }
  if ((table->head_dim != 64 && table->head_dim != 128) || table->rotary_dim < 2 || table->rotary_dim % 2 != 0 ||
      table->rotary_dim > table->head_dim || (table->layout != FCP_ROPE_HALF && table->layout != FCP_ROPE_INTERLEAVED)) {
    fcp_set_error("%s: the table was not filled by fcp_rope_init", call);
    return FCP_ERR_INVALID_ARG;
  }
  RopeArgs a;
  a.D = table->head_dim;
  a.q = (const __nv_bfloat16*)q;
  a.k = (const __nv_bfloat16*)k;
  a.q_out = (__nv_bfloat16*)q_out;
  a.k_out = (__nv_bfloat16*)k_out;
  a.q_stride = q_stride ? q_stride : (int64_t)hq * a.D;
  a.k_stride = k_stride ? k_stride : (int64_t)hkv * a.D;
  a.q_out_stride = q_out_stride ? q_out_stride : (int64_t)hq * a.D;
  a.k_out_stride = k_out_stride ? k_out_stride : (int64_t)hkv * a.D;
  if (a.q_stride < (int64_t)hq * a.D || a.q_out_stride < (int64_t)hq * a.D || a.k_stride < (int64_t)hkv * a.D ||
      a.k_out_stride < (int64_t)hkv * a.D) {
    fcp_set_error("%s: a stride is smaller than heads * head_dim", call);
    return FCP_ERR_INVALID_ARG;
  }
  if ((((uintptr_t)q | (uintptr_t)k | (uintptr_t)q_out | (uintptr_t)k_out) & 1) != 0) {
    fcp_set_error("%s: a tensor is not aligned to its 2-byte values", call);
    return FCP_ERR_INVALID_ARG;
  }
  if (T == 0 || hq + hkv == 0 || (!positions && B == 0)) return FCP_OK;
  a.positions = positions;
  a.row_offset = row_offset;
  a.length = length;
  a.T = (int32_t)T;
  a.B = B;
  a.hq = hq;
  a.hkv = hkv;
  a.rotary = table->rotary_dim;
  a.sign = sign;
  a.magnitude = table->magnitude;
  for (int i = 0; i < 64; ++i) a.turn[i] = table->turn[i];
  const uintptr_t bases = (uintptr_t)q | (uintptr_t)k | (uintptr_t)q_out | (uintptr_t)k_out;
  const int64_t strides = a.q_stride | a.k_stride | a.q_out_stride | a.k_out_stride;
  const bool wide = a.rotary % 16 == 0 && (bases & 15) == 0 && strides % 8 == 0;
  // As many tokens per block as let all blocks run at once, up to ROPE_SLOTS slots: finding the sequence and the angles costs a
  // thread as much as three slots.  16K tokens of 12/4 heads of 64: 14 tokens (0.99 rounds) 15.4 us, 10 (1.4) 16.4, 16 (0.87) 17.1; 4000: 4
  // tokens 6.4, 13 9.2; 64K tokens of 32/8 heads of 128: 4 tokens 211, 1 token 284.
  const int64_t per_token = (hq + hkv) * (wide ? a.D / 16 : a.D / 2), at_once = ROPE_RESIDENT * FCP_PLAN_SMS;
  a.tokens = (int)std::max<int64_t>(1, std::min<int64_t>({ROPE_TOKENS, ROPE_SLOTS / per_token, (T + at_once - 1) / at_once}));
  const unsigned grid = (unsigned)((T + a.tokens - 1) / a.tokens);
  cudaStream_t st = (cudaStream_t)stream;
  const bool half = table->layout == FCP_ROPE_HALF;
  void (*kernel)(const RopeArgs) = wide ? (half ? rope_kernel<true, FCP_ROPE_HALF> : rope_kernel<true, FCP_ROPE_INTERLEAVED>)
                                        : (half ? rope_kernel<false, FCP_ROPE_HALF> : rope_kernel<false, FCP_ROPE_INTERLEAVED>);
  FCP_CUDA_CHECK(launch(kernel, grid, ROPE_THREADS, 0, st, a));
  return FCP_OK;
}

}  // namespace

extern "C" int fcp_rope_fwd(const fcp_rope_table* table, int64_t T, const void* q, int64_t q_stride, int32_t hq, const void* k,
                            int64_t k_stride, int32_t hkv, void* q_out, int64_t q_out_stride, void* k_out,
                            int64_t k_out_stride, const int32_t* positions, const int32_t* row_offset, const int32_t* length,
                            int32_t B, void* stream) {
  return rope("fcp_rope_fwd", 1.f, table, T, q, q_stride, hq, k, k_stride, hkv, q_out, q_out_stride, k_out, k_out_stride,
              positions, row_offset, length, B, stream);
}

extern "C" int fcp_rope_bwd(const fcp_rope_table* table, int64_t T, const void* dq, int64_t dq_stride, int32_t hq, const void* dk,
                            int64_t dk_stride, int32_t hkv, void* dq_in, int64_t dq_in_stride, void* dk_in,
                            int64_t dk_in_stride, const int32_t* positions, const int32_t* row_offset, const int32_t* length,
                            int32_t B, void* stream) {
  return rope("fcp_rope_bwd", -1.f, table, T, dq, dq_stride, hq, dk, dk_stride, hkv, dq_in, dq_in_stride, dk_in, dk_in_stride,
              positions, row_offset, length, B, stream);
}
