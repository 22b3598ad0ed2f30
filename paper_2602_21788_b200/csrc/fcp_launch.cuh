// Host-side plumbing that every file with launches shares: error checks, the driver's tensor-map encoder, launches that may
// begin before the kernel in front of them ends.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include "fcp_plan.hpp"

#define FCP_CUDA_CHECK(expr)                                                             \
  do {                                                                                   \
    cudaError_t e_ = (expr);                                                             \
    if (e_ != cudaSuccess) {                                                             \
      fcp_set_error("%s failed: %s (%s:%d)", #expr, cudaGetErrorString(e_), __FILE__, __LINE__); \
      return FCP_ERR_CUDA;                                                               \
    }                                                                                    \
  } while (0)

namespace fcp {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn get_encode_fn() {
  static EncodeTiledFn fn = nullptr;
  if (fn) return fn;
  void* p = nullptr;
  cudaDriverEntryPointQueryResult qres;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess ||
      qres != cudaDriverEntryPointSuccess)
    return nullptr;
  fn = (EncodeTiledFn)p;
  return fn;
}

// Launch that may begin while the kernel before it in the stream still runs (grid_begin of sm100_ptx.cuh); hides the
// launch latency and the set-up of barriers and tensor memory: 4K-token step, seven queue entries before and four launches now, 59 -> 50 us.
template <typename... P, typename... A>
cudaError_t launch_when(bool early, void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
// The same, early, in clusters of `cluster` blocks along x.
template <typename... P, typename... A>
cudaError_t launch_clusters(int cluster, void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
  return launch_when(true, kernel, grid, threads, smem, st, args...);
}

// The fused forward kernel over work units, one work group and row limits that a kernel before it on the stream has written
// (fcp_kernels.cu).  q [rows][hq][D] with q_stride elements between rows; k, v [kv_rows][hkv][D].
struct FwdTables {
  const int32_t *units, *groups, *row_limit;
  int32_t *counter, *status;                          // counter: zero
  int32_t n_units;
};
int launch_fwd_tables(const FwdTables& t, const fcp_params& p, const void* q, int64_t q_stride, int64_t rows, const void* k, const void* v,
                      int64_t kv_rows, void* o, float* lse, cudaStream_t st);

}  // namespace fcp
