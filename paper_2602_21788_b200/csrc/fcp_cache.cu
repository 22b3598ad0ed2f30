// The calls on a paged 8-bit cache: handle, checks, launches.
#include <algorithm>
#include <cstdint>
#include <mutex>
#include <new>

#include "fcp_cache.cuh"
#include "fcp_launch.cuh"

using namespace fcp;

// Whatever a call needs of the device is looked up at the handle's first compute call, so that a handle can be made, and its
// calls refused, on a machine without a GPU.
struct fcp_cache {
  fcp_cache_config config;
  mutable std::mutex mu;
  mutable int device = -1;
  mutable int sm_count = 0;
  mutable CUtensorMap k_map, v_map;
};

namespace {

// Row tiles in blocks of 8 rows: the smallest that holds a KV head's rows.  1, 2 and 4 blocks go by cache_attn_kernel, whose time grows
// with the rows, 16 by cache_tile_kernel, whose time does not.  16 sequences of 4K to 32K tokens, 40/8 heads, int8, us, the one against the
// other: 25 rows per KV head 178, 220; 35 rows (in tiles of 32) 325, 224; 100 rows 645, 237; e4m3 156, 214; 286, 218; 569, 235.
constexpr int kWeights = 0;
int row_blocks(int64_t rows) { return rows <= 8 ? 1 : rows <= 16 ? 2 : rows <= 32 ? 4 : TILE_ROWS / 8; }

int box_keys(const fcp_cache_config& c) { return std::min(c.page_tokens, CT_KEYS); }

CacheView view(const fcp_cache_config& c) {
  CacheView v;
  v.k = (uint8_t*)c.k;
  v.v = (uint8_t*)c.v;
  v.k_scale = c.k_scale;
  v.v_scale = c.v_scale;
  v.weight = c.weight;
  v.status = c.status;
  v.n_pages = c.n_pages;
  v.page_tokens = c.page_tokens;
  v.page_shift = c.page_tokens == 16 ? 4 : c.page_tokens == 32 ? 5 : c.page_tokens == 64 ? 6 : 7;
  v.hkv = c.hkv;
  return v;
}
BatchView view(const fcp_cache_config& c, const fcp_cache_batch& b) {
  BatchView v;
  v.B = b.B;
  v.rows = b.rows;
  v.max_new = b.max_new;
  v.table_width = b.table_width;
  v.capacity = b.table_width * c.page_tokens;
  v.page_table = b.page_table;
  v.length = b.length;
  v.row_offset = b.row_offset;
  v.only = nullptr;
  return v;
}

// One row of [hkv or hq][D] after the other: 16-byte pieces need aligned rows.
int check_rows(const char* call, const char* name, const void* p, int64_t& stride, int64_t width) {
  if (stride == 0) stride = width;
  if (!p || ((uintptr_t)p & 15) != 0 || stride < width || stride % 8 != 0) {
    fcp_set_error("%s: %s is NULL or not 16-byte aligned, or its stride %lld is below heads * head_dim = %lld or no multiple of 8",
                  call, name, (long long)stride, (long long)width);
    return FCP_ERR_INVALID_ARG;
  }
  return FCP_OK;
}

// `rows_used`: whether the call reads row_offset.
int check_batch(const char* call, const fcp_cache* cache, const fcp_cache_batch* b, bool rows_used) {
  if (!cache || !b) {
    fcp_set_error("%s: NULL cache or batch", call);
    return FCP_ERR_INVALID_ARG;
  }
  // positions, and those of the ends of the tiles that hold them, stay below 2^31
  if (b->B < 0 || b->table_width < 1 || (int64_t)b->table_width * cache->config.page_tokens > (int64_t(1) << 31) - 2 * CT_KEYS ||
      (b->B > 0 && (!b->page_table || !b->length))) {
    fcp_set_error("%s: B %d, table_width %d, or a NULL page_table or length", call, b->B, b->table_width);
    return FCP_ERR_INVALID_ARG;
  }
  if (rows_used && (b->rows < 0 || b->max_new < 0 || b->max_new > b->rows || (b->B > 0 && !b->row_offset) ||
                    (int64_t)b->rows + 2 * (int64_t)b->B >= int64_t(1) << 31)) {
    fcp_set_error("%s: rows %d, max_new %d, or a NULL row_offset", call, b->rows, b->max_new);
    return FCP_ERR_INVALID_ARG;
  }
  return FCP_OK;
}

int cache_map(CUtensorMap* m, const fcp_cache_config& c, void* base) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) {
    fcp_set_error("cuTensorMapEncodeTiled is not available from the driver");
    return FCP_ERR_CUDA;
  }
  const cuuint64_t dims[2] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.n_pages * c.hkv * c.page_tokens};
  const cuuint64_t strides[1] = {(cuuint64_t)c.head_dim};
  const cuuint32_t box[2] = {(cuuint32_t)c.head_dim, (cuuint32_t)box_keys(c)};
  const cuuint32_t estr[2] = {1, 1};
  CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  c.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    fcp_set_error("cuTensorMapEncodeTiled failed with %d", (int)r);
    return FCP_ERR_CUDA;
  }
  return FCP_OK;
}

typedef void (*AttnKernel)(const CUtensorMap, const CUtensorMap, const AttnArgs);
constexpr int kWeightBlocks = 16;
template <int D, int KIND>
AttnKernel attn_kernel(int blocks) {
  return blocks == kWeights ? cache_attn_kernel<D, KIND, kWeightBlocks, 0> : blocks == 1 ? cache_attn_kernel<D, KIND, 1, 1>
         : blocks == 2 ? cache_attn_kernel<D, KIND, 2, 1> : blocks == 4 ? cache_attn_kernel<D, KIND, 2, 2> : cache_tile_kernel<D, KIND>;
}
AttnKernel attn_kernel(const fcp_cache_config& c, int blocks) {
  if (c.head_dim == 128) return c.kind == FCP_CACHE_E4M3 ? attn_kernel<128, FCP_CACHE_E4M3>(blocks) : attn_kernel<128, FCP_CACHE_INT8>(blocks);
  return c.kind == FCP_CACHE_E4M3 ? attn_kernel<64, FCP_CACHE_E4M3>(blocks) : attn_kernel<64, FCP_CACHE_INT8>(blocks);
}
template <int D>
int attn_smem(int blocks) {
  return blocks == kWeights ? AttnSmem<D, kWeightBlocks, 0>::DYN_BYTES : blocks == 1 ? AttnSmem<D, 1, 1>::DYN_BYTES
         : blocks == 2 ? AttnSmem<D, 2, 1>::DYN_BYTES : blocks == 4 ? AttnSmem<D, 2, 2>::DYN_BYTES : TileSmem<D>::DYN_BYTES;
}
int attn_smem(const fcp_cache_config& c, int blocks) { return c.head_dim == 128 ? attn_smem<128>(blocks) : attn_smem<64>(blocks); }

// The first compute call of a handle: device, kernel attributes, tensor maps.  Later ones: the device is still the current one.
int ready(const char* call, const fcp_cache* cache) {
  int device = 0;
  FCP_CUDA_CHECK(cudaGetDevice(&device));
  std::lock_guard<std::mutex> lock(cache->mu);
  if (cache->device == device) return FCP_OK;
  if (cache->device >= 0) {
    fcp_set_error("%s: the cache lies on device %d, the current device is %d", call, cache->device, device);
    return FCP_ERR_INVALID_ARG;
  }
  cudaPointerAttributes where;
  FCP_CUDA_CHECK(cudaPointerGetAttributes(&where, cache->config.k));
  if (where.type != cudaMemoryTypeDevice && where.type != cudaMemoryTypeManaged) {
    fcp_set_error("%s: the cache is not in device memory", call);
    return FCP_ERR_INVALID_ARG;
  }
  if (where.device != device) {
    fcp_set_error("%s: the cache lies on device %d, the current device is %d", call, where.device, device);
    return FCP_ERR_INVALID_ARG;
  }
  int major = 0, sms = 0;
  FCP_CUDA_CHECK(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device));
  FCP_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
  if (major != 10) {
    fcp_set_error("device %d is not sm_100: this library is built for sm_100a only", device);
    return FCP_ERR_CUDA;
  }
  const fcp_cache_config& c = cache->config;
  for (int blocks : {kWeights, 1, 2, 4, TILE_ROWS / 8})
    FCP_CUDA_CHECK(cudaFuncSetAttribute(attn_kernel(c, blocks), cudaFuncAttributeMaxDynamicSharedMemorySize, attn_smem(c, blocks)));
  FCP_CUDA_CHECK(cudaFuncSetAttribute(cache_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SELECT_KEYS * 4));
  int rc = cache_map(&cache->k_map, c, c.k);
  if (rc == FCP_OK) rc = cache_map(&cache->v_map, c, c.v);
  if (rc != FCP_OK) return rc;
  cache->sm_count = std::min(sms, FCP_PLAN_SMS);
  cache->device = device;
  return FCP_OK;
}

int64_t chunk_stride(const fcp_cache_config& c, const fcp_cache_batch& b) {
  return ((int64_t)b.table_width * c.page_tokens + CT_KEYS - 1) / CT_KEYS * CT_KEYS;
}
// Whether a call goes through bf16 copies and the packed attention: where that takes less time by a third by what both were measured to
// take, in clk of the device per tile of 128 keys.  cache_tile_kernel: 4800 per KV head and 128 rows, spread over all SMs.  The other way:
// 5900 per KV head for the copies; fcp_fwd_kernel takes 1700 per query head and tile of 128 new tokens, 1270 where two run beside
// each other, and no item is cut along the keys.  4 sequences of 6K to 12K tokens, 32/8 heads, int8, us, copies against not: 512 new
// tokens 319, 535; 256 237, 291; 192 242, 228 (the rule takes the copies there, 6 % slower); 128 186, 174; 64 195, 110; one sequence, 256
// 163, 128.  The copies may take up to 8 GB; beyond that calls go without.  Every sequence counts as having max_new new tokens, and the
// copies are laid out for the table's width: one chunk beside single tokens is better two calls, as the header says.
constexpr int64_t kChunkBytes = int64_t(8) << 30;
bool in_chunks(const fcp_cache_config& c, const fcp_cache_batch& b, int32_t hq) {
  const int64_t tokens = b.B * chunk_stride(c, b), units = (int64_t)b.B * ((b.max_new + FCP_FWD_UNIT_ROWS - 1) / FCP_FWD_UNIT_ROWS);
  if (b.B < 1 || b.max_new < 2 || b.B > 65535 || tokens >= (int64_t(1) << 31) - CT_KEYS || tokens * c.hkv * c.head_dim * 4 > kChunkBytes ||
      2 * units * hq >= int64_t(1) << 31)
    return false;
  const int64_t rows = ((int64_t)b.max_new * (hq / c.hkv) + 127) / 128, items = b.B * ((b.max_new + 127) / 128) * (int64_t)hq;
  const int64_t direct = b.B * (int64_t)c.hkv * rows * 4800 / FCP_PLAN_SMS;
  const int64_t copied = std::max<int64_t>(1700, items * 1270 / FCP_PLAN_SMS) + b.B * (int64_t)c.hkv * 5900 / FCP_PLAN_SMS;
  return 3 * copied < 2 * direct;
}

// Workspace of fcp_cache_attn: partial outputs and log-sum-exps of two groups per CTA, and what each CTA shares; for chunks also
// the copies and the tables of the units.
struct AttnSpace {
  int64_t o, lse, split, k, v, careful, units, groups, row_limit, bytes;
  int32_t units_per_seq;
};
AttnSpace attn_space(const fcp_cache_config& c, const fcp_cache_batch& b, int32_t hq) {
  AttnSpace s = {};
  auto take = [&s](int64_t bytes) {
    const int64_t at = s.bytes;
    s.bytes += (bytes + 255) / 256 * 256;
    return at;
  };
  const int64_t parts = 2 * (int64_t)FCP_PLAN_SMS * 8 * row_blocks((int64_t)b.max_new * (hq / c.hkv));
  s.o = take(parts * c.head_dim * 4);
  s.lse = take(parts * 4);
  s.split = take(FCP_PLAN_SMS * SP_W * 4);
  if (!in_chunks(c, b, hq)) return s;
  const int64_t copy = b.B * chunk_stride(c, b) * c.hkv * c.head_dim * 2;
  s.units_per_seq = (b.max_new + FCP_FWD_UNIT_ROWS - 1) / FCP_FWD_UNIT_ROWS;
  s.k = take(copy);
  s.v = take(copy);
  s.careful = take((int64_t)b.B * 4);
  s.units = take((int64_t)b.B * s.units_per_seq * FCP_FWD_UNIT_W * 4);
  s.groups = take(FCP_WORK_GROUP_W * 4 + 4);
  s.row_limit = take((int64_t)b.rows * 4);
  return s;
}

int check_heads(const char* call, const fcp_cache_config& c, int32_t hq) {
  if (hq <= 0 || hq % c.hkv != 0 || hq > 65536) {
    fcp_set_error("%s: %d query heads over %d KV heads", call, hq, c.hkv);
    return hq > 0 && hq <= 65536 ? FCP_ERR_UNSUPPORTED : FCP_ERR_INVALID_ARG;
  }
  return FCP_OK;
}

}  // namespace

// ---------------------------------------------------------------------------------------------
// Handle
// ---------------------------------------------------------------------------------------------
extern "C" int fcp_cache_create(const fcp_cache_config* c, fcp_cache** cache) {
  if (!c || !cache) {
    fcp_set_error("fcp_cache_create: NULL argument");
    return FCP_ERR_INVALID_ARG;
  }
  *cache = nullptr;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->status || (((uintptr_t)c->k | (uintptr_t)c->v) & 15) != 0 ||
      ((uintptr_t)c->weight & 15) != 0 || (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale | (uintptr_t)c->status) & 3) != 0) {
    fcp_set_error("fcp_cache_create: a buffer is NULL or not aligned");
    return FCP_ERR_INVALID_ARG;
  }
  if (c->head_dim != 64 && c->head_dim != 128) {
    fcp_set_error("fcp_cache_create: head_dim %d is not 64 or 128", c->head_dim);
    return FCP_ERR_UNSUPPORTED;
  }
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) {
    fcp_set_error("fcp_cache_create: page_tokens %d is not 16, 32, 64 or 128", c->page_tokens);
    return FCP_ERR_UNSUPPORTED;
  }
  if (c->kind != FCP_CACHE_E4M3 && c->kind != FCP_CACHE_INT8) {
    fcp_set_error("fcp_cache_create: unknown kind %d", c->kind);
    return FCP_ERR_INVALID_ARG;
  }
  if (c->n_pages <= 0 || c->hkv <= 0 || c->hkv > 32767 ||
      (int64_t)c->n_pages * c->hkv >= ((int64_t(1) << 31) + c->page_tokens - 1) / c->page_tokens) {
    fcp_set_error("fcp_cache_create: %d pages of %d heads and %d tokens: not positive, or 2^31 rows and more", c->n_pages, c->hkv, c->page_tokens);
    return FCP_ERR_INVALID_ARG;
  }
  fcp_cache* h = new (std::nothrow) fcp_cache();
  if (!h) {
    fcp_set_error("fcp_cache_create: no host memory");
    return FCP_ERR_NO_MEMORY;
  }
  h->config = *c;
  *cache = h;
  return FCP_OK;
}

extern "C" int fcp_cache_destroy(fcp_cache* cache) {
  delete cache;
  return FCP_OK;
}

extern "C" int fcp_cache_device_status(const fcp_cache* cache, int32_t* status) {
  if (!cache || !status) {
    fcp_set_error("fcp_cache_device_status: NULL argument");
    return FCP_ERR_INVALID_ARG;
  }
  FCP_CUDA_CHECK(cudaDeviceSynchronize());
  FCP_CUDA_CHECK(cudaMemcpy(status, cache->config.status, 4 * sizeof(int32_t), cudaMemcpyDeviceToHost));
  return FCP_OK;
}

// ---------------------------------------------------------------------------------------------
// Compute calls
// ---------------------------------------------------------------------------------------------
namespace {
typedef void (*AppendKernel)(const AppendArgs);
constexpr int kPieces = 4;                            // of 16 values per thread: 32 registers
template <int D, int KIND>
AppendKernel append_kernel(int warps) {
  switch (warps) {
    case 1: return cache_append_kernel<D, KIND, kPieces, 1>;
    case 2: return cache_append_kernel<D, KIND, kPieces, 2>;
    case 4: return cache_append_kernel<D, KIND, kPieces, 4>;
    default: return cache_append_kernel<D, KIND, kPieces, 8>;
  }
}
AppendKernel append_kernel(const fcp_cache_config& c, int warps) {
  if (c.head_dim == 128) return c.kind == FCP_CACHE_E4M3 ? append_kernel<128, FCP_CACHE_E4M3>(warps) : append_kernel<128, FCP_CACHE_INT8>(warps);
  return c.kind == FCP_CACHE_E4M3 ? append_kernel<64, FCP_CACHE_E4M3>(warps) : append_kernel<64, FCP_CACHE_INT8>(warps);
}
}  // namespace

extern "C" int fcp_cache_append(const fcp_cache* cache, const fcp_cache_batch* batch, const void* k, int64_t k_stride,
                                const void* v, int64_t v_stride, void* stream) {
  const char* call = "fcp_cache_append";
  int rc = check_batch(call, cache, batch, true);
  if (rc != FCP_OK) return rc;
  const fcp_cache_config& c = cache->config;
  if (batch->B == 0 || batch->rows == 0 || batch->max_new == 0) return FCP_OK;
  if ((rc = check_rows(call, "k", k, k_stride, (int64_t)c.hkv * c.head_dim)) != FCP_OK) return rc;
  if ((rc = check_rows(call, "v", v, v_stride, (int64_t)c.hkv * c.head_dim)) != FCP_OK) return rc;
  if ((rc = ready(call, cache)) != FCP_OK) return rc;
  AppendArgs a;
  a.c = view(c);
  a.s = view(c, *batch);
  a.k = (const __nv_bfloat16*)k;
  a.v = (const __nv_bfloat16*)v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.slots = batch->max_new == 1 ? batch->B : append_slot(batch->rows, batch->B, c.page_tokens);
  const int warps = append_warps(c.page_tokens, c.head_dim, kPieces), threads = append_threads(warps), parts = threads / (32 * warps);
  const dim3 grid((unsigned)a.slots, (unsigned)((2 * c.hkv + parts - 1) / parts));
  FCP_CUDA_CHECK(launch(append_kernel(c, warps), grid, threads, 0, (cudaStream_t)stream, a));
  return FCP_OK;
}

extern "C" int fcp_cache_attn_workspace_bytes(const fcp_cache* cache, const fcp_cache_batch* batch, int32_t hq, int64_t* bytes) {
  const char* call = "fcp_cache_attn_workspace_bytes";
  if (!bytes) {
    fcp_set_error("%s: NULL argument", call);
    return FCP_ERR_INVALID_ARG;
  }
  int rc = check_batch(call, cache, batch, true);
  if (rc == FCP_OK) rc = check_heads(call, cache->config, hq);
  if (rc != FCP_OK) return rc;
  *bytes = attn_space(cache->config, *batch, hq).bytes;
  return FCP_OK;
}

namespace {
int attn_in_chunks(const fcp_cache* cache, const fcp_cache_batch& batch, const AttnArgs& a, const AttnSpace& space, char* ws, cudaStream_t st) {
  const fcp_cache_config& c = cache->config;
  ChunkArgs x;
  x.c = a.c;
  x.s = a.s;
  x.k = (__nv_bfloat16*)(ws + space.k);
  x.v = (__nv_bfloat16*)(ws + space.v);
  x.stride = (int32_t)chunk_stride(c, batch);
  x.careful = (int32_t*)(ws + space.careful);
  x.units = (int32_t*)(ws + space.units);
  x.groups = (int32_t*)(ws + space.groups);
  x.counter = x.groups + FCP_WORK_GROUP_W;
  x.row_limit = (int32_t*)(ws + space.row_limit);
  x.units_per_seq = space.units_per_seq;
  FCP_CUDA_CHECK(cudaMemsetAsync(x.careful, 0, (size_t)batch.B * 4, st));
  const dim3 grid((unsigned)(x.stride / CT_KEYS), (unsigned)c.hkv, (unsigned)batch.B);
  void (*unpack)(const ChunkArgs) = c.head_dim == 128 ? (c.kind == FCP_CACHE_E4M3 ? cache_unpack_kernel<128, FCP_CACHE_E4M3> : cache_unpack_kernel<128, FCP_CACHE_INT8>)
                                                      : (c.kind == FCP_CACHE_E4M3 ? cache_unpack_kernel<64, FCP_CACHE_E4M3> : cache_unpack_kernel<64, FCP_CACHE_INT8>);
  FCP_CUDA_CHECK(launch(unpack, grid, UNPACK_THREADS, 0, st, x));
  FCP_CUDA_CHECK(launch(cache_chunk_kernel, dim3((unsigned)space.units_per_seq, (unsigned)batch.B), CHUNK_THREADS, 0, st, x));
  FwdTables t;
  t.units = x.units;
  t.groups = x.groups;
  t.row_limit = x.row_limit;
  t.counter = x.counter;
  t.status = c.status;
  t.n_units = batch.B * space.units_per_seq;
  fcp_params p;
  p.hq = a.hq;
  p.hkv = c.hkv;
  p.head_dim = c.head_dim;
  p.scale = a.scale_log2 * 0.69314718055994531f;
  return launch_fwd_tables(t, p, a.q, a.q_stride, batch.rows, x.k, x.v, (int64_t)batch.B * x.stride, a.o, a.lse, st);
}
}  // namespace

extern "C" int fcp_cache_attn(const fcp_cache* cache, const fcp_cache_batch* batch, const void* q, int64_t q_stride, int32_t hq,
                              float scale, void* o, float* lse, int32_t accumulate, void* workspace, int64_t workspace_bytes,
                              void* stream) {
  const char* call = "fcp_cache_attn";
  int rc = check_batch(call, cache, batch, true);
  if (rc != FCP_OK) return rc;
  const fcp_cache_config& c = cache->config;
  if ((rc = check_heads(call, c, hq)) != FCP_OK) return rc;
  if (accumulate && !c.weight) {
    fcp_set_error("%s: accumulate without weights in the cache", call);
    return FCP_ERR_INVALID_ARG;
  }
  if (!(scale <= 3e38f)) {
    fcp_set_error("%s: scale is not finite", call);
    return FCP_ERR_INVALID_ARG;
  }
  const int group = hq / c.hkv;
  if ((int64_t)batch->max_new * group >= int64_t(1) << 30) {
    fcp_set_error("%s: %d new tokens of %d heads each", call, batch->max_new, group);
    return FCP_ERR_INVALID_ARG;
  }
  if (batch->B == 0 || batch->rows == 0 || batch->max_new == 0) return FCP_OK;
  if ((rc = check_rows(call, "q", q, q_stride, (int64_t)hq * c.head_dim)) != FCP_OK) return rc;
  if (!o || !lse || ((uintptr_t)o & 15) != 0 || ((uintptr_t)lse & 3) != 0) {
    fcp_set_error("%s: an output is NULL or not aligned", call);
    return FCP_ERR_INVALID_ARG;
  }
  const int blocks = row_blocks((int64_t)batch->max_new * group);
  const AttnSpace space = attn_space(c, *batch, hq);
  if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < space.bytes) {
    fcp_set_error("%s: workspace of %lld bytes (aligned to 256) needed, %lld given", call, (long long)space.bytes, (long long)workspace_bytes);
    return FCP_ERR_WORKSPACE;
  }
  if ((rc = ready(call, cache)) != FCP_OK) return rc;
  AttnArgs a;
  a.c = view(c);
  a.s = view(c, *batch);
  a.q = (const __nv_bfloat16*)q;
  a.q_stride = q_stride;
  a.o = (__nv_bfloat16*)o;
  a.lse = lse;
  a.scale_log2 = (scale > 0 ? scale : (c.head_dim == 128 ? 0.08838834764831845f : 0.125f)) * 1.4426950408889634f;
  a.hq = hq;
  a.group = group;
  a.box = box_keys(c);
  a.part_o = (float*)((char*)workspace + space.o);
  a.part_lse = (float*)((char*)workspace + space.lse);
  a.split = (int32_t*)((char*)workspace + space.split);
  cudaStream_t st = (cudaStream_t)stream;
  const int grid = cache->sm_count;
  const BatchView all = a.s;
  if (space.units_per_seq > 0) {
    if ((rc = attn_in_chunks(cache, *batch, a, space, (char*)workspace, st)) != FCP_OK) return rc;
    a.s.only = (const int32_t*)((char*)workspace + space.careful);       // what is left
  }
  FCP_CUDA_CHECK(launch(attn_kernel(c, blocks), grid, blocks > 4 ? TILE_THREADS : CT_THREADS, attn_smem(c, blocks), st, cache->k_map, cache->v_map, a));
  if (c.head_dim == 128) FCP_CUDA_CHECK(launch(cache_merge_kernel<128>, grid, MERGE_THREADS, 0, st, a, 8 * blocks));
  else FCP_CUDA_CHECK(launch(cache_merge_kernel<64>, grid, MERGE_THREADS, 0, st, a, 8 * blocks));
  a.s = all;
  if (accumulate)
    FCP_CUDA_CHECK(launch(attn_kernel(c, kWeights), WEIGHT_CTAS * grid, CT_THREADS, attn_smem(c, kWeights), st, cache->k_map, cache->v_map, a));
  return FCP_OK;
}

extern "C" int fcp_cache_evict(const fcp_cache* cache, const fcp_cache_batch* batch, int32_t n_sink, int32_t n_heavy, int32_t n_recent,
                               const int32_t* dst_table, int32_t dst_width, int32_t* new_length, int32_t* kept, void* stream) {
  const char* call = "fcp_cache_evict";
  int rc = check_batch(call, cache, batch, false);
  if (rc != FCP_OK) return rc;
  const fcp_cache_config& c = cache->config;
  const int64_t keep = (int64_t)n_sink + n_heavy + n_recent;
  if (!c.weight) {
    fcp_set_error("%s: the cache has no weights", call);
    return FCP_ERR_INVALID_ARG;
  }
  // positions of kept tokens are gone through in steps of up to SELECT_BLOCKS * SELECT_THREADS, in 32 bits
  if (n_sink < 0 || n_heavy < 0 || n_recent < 0 || keep < 1 || keep > (int64_t(1) << 31) - SELECT_BLOCKS * SELECT_THREADS || dst_width < 1 ||
      (int64_t)dst_width * c.page_tokens < keep) {
    fcp_set_error("%s: %d + %d + %d tokens to keep on %d pages of %d", call, n_sink, n_heavy, n_recent, dst_width, c.page_tokens);
    return FCP_ERR_INVALID_ARG;
  }
  if (batch->B > 65535) {
    fcp_set_error("%s: more than 65535 sequences", call);
    return FCP_ERR_UNSUPPORTED;
  }
  if (batch->B == 0) return FCP_OK;
  if (!dst_table || !new_length || !kept) {
    fcp_set_error("%s: NULL buffer", call);
    return FCP_ERR_INVALID_ARG;
  }
  if ((rc = ready(call, cache)) != FCP_OK) return rc;
  EvictArgs a;
  a.c = view(c);
  a.s = view(c, *batch);
  a.n_sink = n_sink;
  a.n_heavy = n_heavy;
  a.n_recent = n_recent;
  a.dst_table = dst_table;
  a.dst_width = dst_width;
  a.new_length = new_length;
  a.kept = kept;
  cudaStream_t st = (cudaStream_t)stream;
  // about 8 candidates per thread, as far as eight blocks go
  const int cluster = a.s.capacity > 32768 ? 8 : a.s.capacity > 16384 ? 4 : a.s.capacity > 8192 ? 2 : 1;
  const size_t smem = (size_t)std::min(SELECT_KEYS, (a.s.capacity + cluster - 1) / cluster + 8) * 4;        // whole fours at both ends
  FCP_CUDA_CHECK(launch_clusters(cluster, cache_select_kernel, dim3((unsigned)(c.hkv * cluster), (unsigned)batch->B), SELECT_THREADS, smem, st, a));
  const dim3 grid((unsigned)((keep + MOVE_TOKENS - 1) / MOVE_TOKENS), (unsigned)c.hkv, (unsigned)batch->B);
  if (c.head_dim == 128) {
    if (c.kind == FCP_CACHE_E4M3) FCP_CUDA_CHECK(launch(cache_move_kernel<128, FCP_CACHE_E4M3>, grid, MOVE_THREADS, 0, st, a));
    else FCP_CUDA_CHECK(launch(cache_move_kernel<128, FCP_CACHE_INT8>, grid, MOVE_THREADS, 0, st, a));
  } else {
    if (c.kind == FCP_CACHE_E4M3) FCP_CUDA_CHECK(launch(cache_move_kernel<64, FCP_CACHE_E4M3>, grid, MOVE_THREADS, 0, st, a));
    else FCP_CUDA_CHECK(launch(cache_move_kernel<64, FCP_CACHE_INT8>, grid, MOVE_THREADS, 0, st, a));
  }
  return FCP_OK;
}
