// Checks that the projections' entry points have in common.
#pragma once

#include "snn_handle.h"
#include "snn_products.h"

struct snn_conv_experts {
  snn::Products p;
};

namespace snn {

inline snn_status_t cuda_failed(cudaError_t e, const char* what) {
  cudaGetLastError();
  return api_fail(e == cudaErrorMemoryAllocation ? SNN_ERR_OOM : SNN_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}
inline bool act_ok(int type) { return type == SNN_ACT_F16 || type == SNN_ACT_BF16; }
inline bool out_ok(int type) { return type == SNN_OUT_F32 || type == SNN_OUT_F16 || type == SNN_OUT_BF16; }
inline size_t out_size(int type) { return type == SNN_OUT_F32 ? 4 : 2; }

inline snn_status_t select_device(int device) {
  int n = 0;
  if (cudaGetDeviceCount(&n) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return api_fail(SNN_ERR_CUDA, "no CUDA device available (this library has no CPU path)");
  }
  if (device < 0 || device >= n) return api_fail(SNN_ERR_INVALID_ARG, "device %d of %d", device, n);
  return SNN_OK;
}

// A bounded wait of an earlier launch that ran out, told once.
inline snn_status_t earlier_timeout(int* status) {
  if (!*status) return SNN_OK;
  const int code = *status;
  *status = 0;
  return api_fail(SNN_ERR_TIMEOUT, "an earlier launch gave up a bounded wait (code %d)", code);
}

}  // namespace snn
