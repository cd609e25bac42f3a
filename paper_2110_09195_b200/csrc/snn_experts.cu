// Host side of the projections of language models in include/snn_conv.h: argument checks, handles and launches.
#include <new>

#include "snn_handle.h"
#include "snn_products.h"

using namespace snn;

struct snn_conv_experts {
  Products p;
};
struct snn_conv_adapters {
  Products p;
};

namespace {

snn_status_t cuda_failed(cudaError_t e, const char* what) {
  cudaGetLastError();
  return api_fail(e == cudaErrorMemoryAllocation ? SNN_ERR_OOM : SNN_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}
bool act_ok(int type) { return type == SNN_ACT_F16 || type == SNN_ACT_BF16; }
bool out_ok(int type) { return type == SNN_OUT_F32 || type == SNN_OUT_F16 || type == SNN_OUT_BF16; }
size_t out_size(int type) { return type == SNN_OUT_F32 ? 4 : 2; }

snn_status_t check_layers(snn_conv_t* const* layers, int count, const LayerDev** L) {
  for (int i = 0; i < count; ++i) {
    if (!layers[i]) return api_fail(SNN_ERR_INVALID_ARG, "layer %d is a null handle", i);
    if (layers[i]->ksize != 1 || layers[i]->stride != 1)
      return api_fail(SNN_ERR_INVALID_ARG, "layer %d is not a 1x1 layer of stride 1", i);
    if (layers[i]->C != layers[0]->C || layers[i]->K != layers[0]->K || layers[i]->device != layers[0]->device)
      return api_fail(SNN_ERR_INVALID_ARG, "layer %d differs from layer 0 in its channels or device", i);
    L[i] = &layers[i]->L;
  }
  return SNN_OK;
}

snn_status_t create(snn_conv_t* const* layers, int count, Products* p, const char* what) {
  const LayerDev** L = new (std::nothrow) const LayerDev*[count];
  if (!L) return api_fail(SNN_ERR_OOM, "host allocation failed");
  snn_status_t st = check_layers(layers, count, L);
  if (st == SNN_OK) {
    DeviceGuard guard(layers[0]->device);
    if (!guard.ok) st = api_fail(SNN_ERR_CUDA, "cannot select device %d", layers[0]->device);
    else {
      p->device = layers[0]->device;
      int launched = 0;
      const cudaError_t e = products_create(L, count, layers[0]->C, layers[0]->K, layers[0]->host_stream, p, &launched);
      api_count_launches(launched);
      if (e != cudaSuccess) {
        products_destroy(p);
        st = cuda_failed(e, what);
      }
    }
  }
  delete[] L;
  return st;
}

// What both forward calls have in common.
snn_status_t check_rows(const Products& p, const void* act, int act_type, int act_rows, int64_t ld_act, int rows, const void* out, int out_type,
                        int64_t ld_out) {
  if (!act_ok(act_type)) return api_fail(SNN_ERR_INVALID_ARG, "activations are SNN_ACT_F16 or SNN_ACT_BF16, not %d", act_type);
  if (!out_ok(out_type)) return api_fail(SNN_ERR_INVALID_ARG, "outputs are SNN_OUT_F32, SNN_OUT_F16 or SNN_OUT_BF16, not %d", out_type);
  if (act_rows < 0 || rows < 0) return api_fail(SNN_ERR_INVALID_ARG, "%d rows of activations, %d of outputs", act_rows, rows);
  if (ld_act < p.C || ld_act % 8 || ld_out < p.K)
    return api_fail(SNN_ERR_INVALID_ARG, "rows of %lld activations and %lld outputs (c_in %d, c_out %d; the former a multiple of 8)",
                    (long long)ld_act, (long long)ld_out, p.C, p.K);
  // (the kernels count pieces of rows times strips of channels in 32 bits, whatever the offsets say)
  if (rows > 1 << 30 || ((long long)rows / 8 + 1) * p.E >= (1ll << 31) || ((long long)rows / 8 + p.E) * ((p.K + 31) / 32) >= (1ll << 31))
    return api_fail(SNN_ERR_UNSUPPORTED, "%d rows of %d outputs over %d experts: split the call", rows, p.K, p.E);
  if (rows > 0 && (!out || (act_rows > 0 && !act))) return api_fail(SNN_ERR_INVALID_ARG, "null activation / output pointer");
  if (((uintptr_t)act & 15) || ((uintptr_t)out & (out_size(out_type) - 1)))
    return api_fail(SNN_ERR_INVALID_ARG, "activations must be 16-byte aligned, outputs aligned to their element");
  return SNN_OK;
}

snn_status_t forward(Products& p, const ProductCall& c, const ShrinkCall* first, const char* what) {
  DeviceGuard guard(p.device);
  if (!guard.ok) return api_fail(SNN_ERR_CUDA, "cannot select device %d", p.device);
  if (*p.status_host) {
    const int code = *p.status_host;
    *p.status_host = 0;
    return api_fail(SNN_ERR_TIMEOUT, "an earlier launch gave up a bounded wait (code %d)", code);
  }
  int launched = 0;
  cudaError_t e = first ? shrink_forward(*first, &launched) : cudaSuccess;
  if (e == cudaSuccess) e = products_forward(p, c, &launched);
  api_count_launches(launched);
  return e == cudaSuccess ? SNN_OK : cuda_failed(e, what);
}

snn_status_t select_device(int device) {
  int n = 0;
  if (cudaGetDeviceCount(&n) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return api_fail(SNN_ERR_CUDA, "no CUDA device available (this library has no CPU path)");
  }
  if (device < 0 || device >= n) return api_fail(SNN_ERR_INVALID_ARG, "device %d of %d", device, n);
  return SNN_OK;
}

}  // namespace

extern "C" {

snn_status_t snn_conv_experts_create(snn_conv_t* const* layers, int32_t count, snn_conv_experts_t** out) {
  if (!out) return api_fail(SNN_ERR_INVALID_ARG, "null output pointer");
  *out = nullptr;
  if (!layers) return api_fail(SNN_ERR_INVALID_ARG, "null argument");
  if (count < 1 || count > SNN_EXPERTS_MAX) return api_fail(SNN_ERR_INVALID_ARG, "1..%d experts, not %d", SNN_EXPERTS_MAX, count);
  snn_conv_experts* h = new (std::nothrow) snn_conv_experts();
  if (!h) return api_fail(SNN_ERR_OOM, "host allocation failed");
  const snn_status_t st = create(layers, count, &h->p, "snn_conv_experts_create");
  if (st != SNN_OK) {
    delete h;
    return st;
  }
  *out = h;
  return SNN_OK;
}

snn_status_t snn_conv_experts_forward(snn_conv_experts_t* h, const void* act_dev, int32_t act_type, int32_t act_rows, int64_t ld_act,
                                      const int32_t* rows_dev, const int32_t* offsets_dev, int32_t max_rows, void* out_dev, int32_t out_type,
                                      int64_t ld_out, void* cuda_stream) {
  if (!h) return api_fail(SNN_ERR_INVALID_ARG, "null handle");
  const snn_status_t st = check_rows(h->p, act_dev, act_type, act_rows, ld_act, max_rows, out_dev, out_type, ld_out);
  if (st != SNN_OK) return st;
  if (max_rows == 0) return SNN_OK;
  if (!offsets_dev) return api_fail(SNN_ERR_INVALID_ARG, "null offsets");
  if (((uintptr_t)offsets_dev & 3) || ((uintptr_t)rows_dev & 3)) return api_fail(SNN_ERR_INVALID_ARG, "misaligned offsets or rows");
  const ProductCall c{act_dev, act_type, act_rows, ld_act, rows_dev, offsets_dev, max_rows, out_dev, out_type, ld_out, Lowrank{}, (cudaStream_t)cuda_stream};
  return forward(h->p, c, nullptr, "snn_conv_experts_forward");
}

snn_status_t snn_conv_experts_destroy(snn_conv_experts_t* h) {
  if (!h) return SNN_OK;
  DeviceGuard guard(h->p.device);
  products_destroy(&h->p);
  delete h;
  return SNN_OK;
}

int64_t snn_conv_experts_route_work(int32_t tokens, int32_t experts) { return tokens < 1 || experts < 1 ? 0 : route_work_bytes(tokens, experts); }

snn_status_t snn_conv_experts_route(const void* logits_dev, int32_t type, int32_t tokens, int32_t experts, int64_t ld, int32_t top_k,
                                    int32_t normalise, int32_t* ids_dev, float* weights_dev, int32_t* offsets_dev, int32_t* rows_dev,
                                    int32_t* slots_dev, void* work_dev, int32_t device, void* cuda_stream) {
  if (!out_ok(type)) return api_fail(SNN_ERR_INVALID_ARG, "logits are SNN_OUT_F32, SNN_OUT_F16 or SNN_OUT_BF16, not %d", type);
  if (experts < 1 || experts > SNN_EXPERTS_MAX) return api_fail(SNN_ERR_INVALID_ARG, "1..%d experts, not %d", SNN_EXPERTS_MAX, experts);
  if (top_k < 1 || top_k > SNN_ROUTE_TOP_MAX || top_k > experts)
    return api_fail(SNN_ERR_INVALID_ARG, "top_k=%d of %d experts (at most %d)", top_k, experts, SNN_ROUTE_TOP_MAX);
  if (tokens < 0 || (long long)tokens * top_k >= (1ll << 31)) return api_fail(SNN_ERR_INVALID_ARG, "%d tokens of %d experts each", tokens, top_k);
  if (ld < experts) return api_fail(SNN_ERR_INVALID_ARG, "rows of %lld logits for %d experts", (long long)ld, experts);
  if (!offsets_dev || (tokens > 0 && (!logits_dev || !ids_dev || !weights_dev || !rows_dev || !slots_dev)))
    return api_fail(SNN_ERR_INVALID_ARG, "null device pointer");
  if (route_work_bytes(tokens, experts) > 0 && !work_dev) return api_fail(SNN_ERR_INVALID_ARG, "null workspace");
  if (((uintptr_t)logits_dev & (out_size(type) - 1)) ||
      (((uintptr_t)ids_dev | (uintptr_t)weights_dev | (uintptr_t)offsets_dev | (uintptr_t)rows_dev | (uintptr_t)slots_dev | (uintptr_t)work_dev) & 3))
    return api_fail(SNN_ERR_INVALID_ARG, "misaligned device pointer");
  const snn_status_t st = select_device(device);
  if (st != SNN_OK) return st;
  DeviceGuard guard(device);
  if (!guard.ok) return api_fail(SNN_ERR_CUDA, "cannot select device %d", device);
  const RouteCall c{logits_dev, type, tokens, experts, top_k, normalise != 0, ld, ids_dev, weights_dev, offsets_dev, rows_dev, slots_dev,
                    static_cast<int32_t*>(work_dev), (cudaStream_t)cuda_stream};
  int launched = 0;
  const cudaError_t e = route_forward(c, &launched);
  api_count_launches(launched);
  return e == cudaSuccess ? SNN_OK : cuda_failed(e, "snn_conv_experts_route");
}

snn_status_t snn_conv_experts_combine(const void* y_dev, int32_t y_type, int32_t y_rows, int64_t ld_y, const int32_t* slots_dev,
                                      const float* weights_dev, int32_t tokens, int32_t top_k, int32_t columns, void* out_dev, int32_t out_type,
                                      int64_t ld_out, int32_t device, void* cuda_stream) {
  if (!out_ok(y_type) || !out_ok(out_type))
    return api_fail(SNN_ERR_INVALID_ARG, "inputs and outputs are SNN_OUT_F32, SNN_OUT_F16 or SNN_OUT_BF16, not %d and %d", y_type, out_type);
  if (tokens < 0 || y_rows < 0 || columns < 1 || top_k < 1 || top_k > SNN_ROUTE_TOP_MAX)
    return api_fail(SNN_ERR_INVALID_ARG, "tokens=%d y_rows=%d columns=%d top_k=%d", tokens, y_rows, columns, top_k);
  if (ld_y < columns || ld_out < columns)
    return api_fail(SNN_ERR_INVALID_ARG, "rows of %lld and %lld for %d columns", (long long)ld_y, (long long)ld_out, columns);
  if ((long long)tokens * columns >= (1ll << 38)) return api_fail(SNN_ERR_UNSUPPORTED, "%d tokens of %d columns: split the call", tokens, columns);
  if (tokens == 0) return SNN_OK;
  if (!slots_dev || !weights_dev || !out_dev || (y_rows > 0 && !y_dev)) return api_fail(SNN_ERR_INVALID_ARG, "null device pointer");
  if (((uintptr_t)y_dev & (out_size(y_type) - 1)) || ((uintptr_t)out_dev & (out_size(out_type) - 1)) || (((uintptr_t)slots_dev | (uintptr_t)weights_dev) & 3))
    return api_fail(SNN_ERR_INVALID_ARG, "misaligned device pointer");
  const snn_status_t st = select_device(device);
  if (st != SNN_OK) return st;
  DeviceGuard guard(device);
  if (!guard.ok) return api_fail(SNN_ERR_CUDA, "cannot select device %d", device);
  const CombineCall c{y_dev, y_type, y_rows, ld_y, slots_dev, weights_dev, tokens, top_k, columns, out_dev, out_type, ld_out, (cudaStream_t)cuda_stream};
  int launched = 0;
  const cudaError_t e = combine_forward(c, &launched);
  api_count_launches(launched);
  return e == cudaSuccess ? SNN_OK : cuda_failed(e, "snn_conv_experts_combine");
}

snn_status_t snn_conv_adapters_create(snn_conv_t* layer, snn_conv_adapters_t** out) {
  if (!out) return api_fail(SNN_ERR_INVALID_ARG, "null output pointer");
  *out = nullptr;
  snn_conv_adapters* h = new (std::nothrow) snn_conv_adapters();
  if (!h) return api_fail(SNN_ERR_OOM, "host allocation failed");
  const snn_status_t st = create(&layer, 1, &h->p, "snn_conv_adapters_create");
  if (st != SNN_OK) {
    delete h;
    return st;
  }
  *out = h;
  return SNN_OK;
}

snn_status_t snn_conv_adapters_forward(snn_conv_adapters_t* h, const void* act_dev, int32_t act_type, int32_t rows, int64_t ld_act,
                                       const int32_t* adapter_dev, const void* a_dev, const void* b_dev, const float* scale_dev, int32_t adapters,
                                       int32_t rank, float* work_dev, void* out_dev, int32_t out_type, int64_t ld_out, void* cuda_stream) {
  if (!h) return api_fail(SNN_ERR_INVALID_ARG, "null handle");
  snn_status_t st = check_rows(h->p, act_dev, act_type, rows, ld_act, rows, out_dev, out_type, ld_out);
  if (st != SNN_OK) return st;
  if (adapters < 0) return api_fail(SNN_ERR_INVALID_ARG, "%d adapters", adapters);
  if (rank < 8 || rank > SNN_ADAPTERS_RANK_MAX || rank % 8)
    return api_fail(SNN_ERR_INVALID_ARG, "rank=%d is not a multiple of 8 in 8..%d", rank, SNN_ADAPTERS_RANK_MAX);
  if (rows == 0) return SNN_OK;
  if (!adapter_dev || !work_dev || (adapters > 0 && (!a_dev || !b_dev || !scale_dev))) return api_fail(SNN_ERR_INVALID_ARG, "null device pointer");
  if ((((uintptr_t)a_dev | (uintptr_t)b_dev | (uintptr_t)work_dev) & 15) || (((uintptr_t)adapter_dev | (uintptr_t)scale_dev) & 3))
    return api_fail(SNN_ERR_INVALID_ARG, "misaligned device pointer");
  const Products& p = h->p;
  const ShrinkCall first{act_dev, act_type, rows, p.C, ld_act, adapter_dev, a_dev, scale_dev, adapters, rank, work_dev, (cudaStream_t)cuda_stream};
  const Lowrank low{adapter_dev, work_dev, b_dev, adapters, rank};
  const ProductCall c{act_dev, act_type, rows, ld_act, nullptr, nullptr, rows, out_dev, out_type, ld_out, low, (cudaStream_t)cuda_stream};
  return forward(h->p, c, &first, "snn_conv_adapters_forward");
}

snn_status_t snn_conv_adapters_destroy(snn_conv_adapters_t* h) {
  if (!h) return SNN_OK;
  DeviceGuard guard(h->p.device);
  products_destroy(&h->p);
  delete h;
  return SNN_OK;
}

}  // extern "C"
