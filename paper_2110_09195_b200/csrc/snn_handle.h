// The layer handle of the C ABI (include/snn_conv.h), as the entry points see it.
#pragma once

#include <cuda_runtime.h>

#include <map>
#include <mutex>
#include <tuple>

#include "snn_internal.h"

struct snn_conv {
  int C, K, tau, stride, pad, act_type, device;
  int ksize = 3;
  snn::LayerDev L;
  std::mutex mu;
  std::map<std::tuple<int, int, int>, int> tuned;        // (N,H,W) -> path measured fastest by snn_conv_tune
  // (N,H,W, packed-sign output?) -> tensor-core plan and weight operand (a group of one)
  std::map<std::tuple<int, int, int, int>, snn::GroupDev*> solo;
  // staging for snn_conv_forward_host
  void* stage_in = nullptr;
  void* stage_out = nullptr;
  size_t stage_in_bytes = 0, stage_out_bytes = 0;
  cudaStream_t host_stream = nullptr;
  int* tc_status_host = nullptr;  // pinned, written by the tensor-core kernel on a bounded-wait timeout
  int* tc_status_dev = nullptr;   // the same word as the device sees it
};

namespace snn {

// Makes a device current for the scope and the one before current again at its end.
struct DeviceGuard {
  int prev = -1;
  bool ok = false;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) return;
    ok = (prev == dev) || cudaSetDevice(dev) == cudaSuccess;
  }
  ~DeviceGuard() {
    int cur = -1;
    if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
  }
};

// The calling thread's last failure (snn_last_error) and the count of launches (snn_kernel_launches).
snn_status_t api_fail(snn_status_t st, const char* fmt, ...);
void api_count_launches(int n);

}  // namespace snn
