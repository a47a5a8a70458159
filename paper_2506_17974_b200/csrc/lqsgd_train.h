// Host-side pieces shared by the training operators (lqsgd_act8.cu, lqsgd_norm.cu, lqsgd_linear.cu).
#pragma once
#include "../../include/lqsgd.h"

#include <cuda_runtime.h>
#include <stdint.h>

namespace lqsgd {

int record_cuda_failure(cudaError_t e, const char* what);   // lqsgd_api.cu: text for lqsgd_last_cuda_error()

inline bool train_dtype_ok(int32_t dtype) { return dtype == LQSGD_BF16 || dtype == LQSGD_F16 || dtype == LQSGD_F32; }
inline bool train_act_ok(int32_t act) { return act >= LQSGD_ACT_NONE && act <= LQSGD_ACT_SILU; }
inline int train_elem(int32_t dtype) { return dtype == LQSGD_F32 ? 4 : 2; }
inline bool train_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Checks of an 8-bit matrix argument whose codes are set.
inline int check_packed8(const lqsgd_packed8& p, int32_t cols) {
  if (!p.dev_codes || !p.dev_exps) return LQSGD_ERR_INVALID_ARG;
  if (p.ld_codes < cols || p.ld_exps < ceil_div64(cols, LQSGD_PACK8_GROUP)) return LQSGD_ERR_INVALID_ARG;
  return LQSGD_OK;
}

// SM count of the current device; asked once per device, 0 when it cannot be had.
int train_sm_count();

// Launch whose start may overlap the tail of the kernel in front of it in the stream; every kernel launched this way
// begins with griddepcontrol.wait before it touches memory.
template <typename... KArgs, typename... Args>
cudaError_t train_launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, int cluster, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cluster > 1) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}
#define TRAIN_CK(call, what)                                            \
  do {                                                                  \
    cudaError_t e__ = (call);                                           \
    if (e__ != cudaSuccess) return lqsgd::record_cuda_failure(e__, what); \
  } while (0)

}  // namespace lqsgd
