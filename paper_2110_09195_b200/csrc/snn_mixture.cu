// Host side of the whole mixture, the activation and the 8-bit projections in include/snn_conv.h: argument checks, handles and launches.
#include <new>

#include "snn_checks.h"

using namespace snn;

struct snn_conv_moe {
  const Products *gate, *up, *down;
  int fn;
};
struct snn_conv_scaled {
  Scaled p;
};

namespace {

bool fn_ok(int fn) { return fn >= SNN_FN_NONE && fn <= SNN_FN_GELU; }

// Inputs of the activation, with a gate or without.
snn_status_t check_between(const void* gate, int64_t ld_gate, const void* up, int64_t ld_up, int type, int rows, int columns, int fn) {
  if (!out_ok(type)) return api_fail(SNN_ERR_INVALID_ARG, "inputs are SNN_OUT_F32, SNN_OUT_F16 or SNN_OUT_BF16, not %d", type);
  if (!fn_ok(fn)) return api_fail(SNN_ERR_INVALID_ARG, "fn=%d is no SNN_FN_*", fn);
  if (rows < 0 || columns < 1) return api_fail(SNN_ERR_INVALID_ARG, "%d rows of %d columns", rows, columns);
  if (ld_up < columns || (gate && ld_gate < columns))
    return api_fail(SNN_ERR_INVALID_ARG, "rows of %lld and %lld for %d columns", (long long)ld_up, (long long)ld_gate, columns);
  if (((uintptr_t)gate | (uintptr_t)up) & (out_size(type) - 1)) return api_fail(SNN_ERR_INVALID_ARG, "misaligned device pointer");
  return SNN_OK;
}

}  // namespace

extern "C" {

snn_status_t snn_conv_experts_activate(const void* gate_dev, int64_t ld_gate, const void* up_dev, int64_t ld_up, int32_t type, int32_t rows, int32_t columns,
                                       int32_t fn, void* out_dev, int32_t out_type, int64_t ld_out, int32_t device, void* cuda_stream) {
  snn_status_t st = check_between(gate_dev, ld_gate, up_dev, ld_up, type, rows, columns, fn);
  if (st != SNN_OK) return st;
  if (!out_ok(out_type)) return api_fail(SNN_ERR_INVALID_ARG, "outputs are SNN_OUT_F32, SNN_OUT_F16 or SNN_OUT_BF16, not %d", out_type);
  if (ld_out < columns) return api_fail(SNN_ERR_INVALID_ARG, "rows of %lld outputs for %d columns", (long long)ld_out, columns);
  if ((long long)rows * columns >= (1ll << 34)) return api_fail(SNN_ERR_UNSUPPORTED, "%d rows of %d columns: split the call", rows, columns);
  if (rows == 0) return SNN_OK;
  if (!up_dev || !out_dev) return api_fail(SNN_ERR_INVALID_ARG, "null device pointer");
  if ((uintptr_t)out_dev & (out_size(out_type) - 1)) return api_fail(SNN_ERR_INVALID_ARG, "misaligned device pointer");
  st = select_device(device);
  if (st != SNN_OK) return st;
  DeviceGuard guard(device);
  if (!guard.ok) return api_fail(SNN_ERR_CUDA, "cannot select device %d", device);
  const ActivateCall c{gate_dev, up_dev, ld_gate, ld_up, type, rows, columns, fn, out_dev, out_type, ld_out, (cudaStream_t)cuda_stream};
  int launched = 0;
  const cudaError_t e = activate_forward(c, &launched);
  api_count_launches(launched);
  return e == cudaSuccess ? SNN_OK : cuda_failed(e, "snn_conv_experts_activate");
}

snn_status_t snn_conv_moe_create(snn_conv_experts_t* gate, snn_conv_experts_t* up, snn_conv_experts_t* down, int32_t fn, snn_conv_moe_t** out) {
  if (!out) return api_fail(SNN_ERR_INVALID_ARG, "null output pointer");
  *out = nullptr;
  if (!up || !down) return api_fail(SNN_ERR_INVALID_ARG, "null handle");
  if (!fn_ok(fn)) return api_fail(SNN_ERR_INVALID_ARG, "fn=%d is no SNN_FN_*", fn);
  const Products &u = up->p, &d = down->p;
  if (gate && (gate->p.E != u.E || gate->p.C != u.C || gate->p.K != u.K || gate->p.device != u.device))
    return api_fail(SNN_ERR_INVALID_ARG, "the gate's experts (%d of %d -> %d) differ from up's (%d of %d -> %d) or are on another device", gate->p.E, gate->p.C, gate->p.K, u.E,
                    u.C, u.K);
  if (d.E != u.E || d.C != u.K || d.device != u.device)
    return api_fail(SNN_ERR_INVALID_ARG, "down's experts (%d of %d -> %d) do not follow from up's (%d of %d -> %d) or are on another device", d.E, d.C, d.K, u.E, u.C, u.K);
  snn_conv_moe* h = new (std::nothrow) snn_conv_moe{gate ? &gate->p : nullptr, &u, &d, fn};
  if (!h) return api_fail(SNN_ERR_OOM, "host allocation failed");
  *out = h;
  return SNN_OK;
}

int64_t snn_conv_moe_work(const snn_conv_moe_t* m, int32_t tokens, int32_t top_k) {
  if (!m || tokens < 0 || tokens > SNN_MOE_TOKENS_MAX || top_k < 1 || top_k > SNN_ROUTE_TOP_MAX || top_k > m->up->E) return -1;
  return moe_work_bytes(*m->up, tokens, top_k);
}

snn_status_t snn_conv_moe_forward(snn_conv_moe_t* m, const void* act_dev, int32_t act_type, int32_t tokens, int64_t ld_act, const void* logits_dev,
                                  int32_t logits_type, int64_t ld_logits, int32_t top_k, int32_t normalise, void* work_dev, void* out_dev, int32_t out_type,
                                  int64_t ld_out, void* cuda_stream) {
  if (!m) return api_fail(SNN_ERR_INVALID_ARG, "null handle");
  const Products &up = *m->up, &down = *m->down;
  if (!act_ok(act_type)) return api_fail(SNN_ERR_INVALID_ARG, "activations are SNN_ACT_F16 or SNN_ACT_BF16, not %d", act_type);
  if (!out_ok(logits_type) || !out_ok(out_type))
    return api_fail(SNN_ERR_INVALID_ARG, "logits and outputs are SNN_OUT_F32, SNN_OUT_F16 or SNN_OUT_BF16, not %d and %d", logits_type, out_type);
  if (tokens < 0) return api_fail(SNN_ERR_INVALID_ARG, "%d tokens", tokens);
  if (tokens > SNN_MOE_TOKENS_MAX)
    return api_fail(SNN_ERR_UNSUPPORTED, "%d tokens, above %d: call the router, the experts, the activation and the weighted sum", tokens, SNN_MOE_TOKENS_MAX);
  if (top_k < 1 || top_k > SNN_ROUTE_TOP_MAX || top_k > up.E)
    return api_fail(SNN_ERR_INVALID_ARG, "top_k=%d of %d experts (at most %d)", top_k, up.E, SNN_ROUTE_TOP_MAX);
  if (ld_act < up.C || ld_act % 8 || ld_logits < up.E || ld_out < down.K)
    return api_fail(SNN_ERR_INVALID_ARG, "rows of %lld activations, %lld logits and %lld outputs (c_in %d, %d experts, c_out %d; the first a multiple of 8)",
                    (long long)ld_act, (long long)ld_logits, (long long)ld_out, up.C, up.E, down.K);
  if (tokens == 0) return SNN_OK;
  if (!act_dev || !logits_dev || !work_dev || !out_dev) return api_fail(SNN_ERR_INVALID_ARG, "null device pointer");
  if ((((uintptr_t)act_dev | (uintptr_t)work_dev) & 15) || ((uintptr_t)logits_dev & (out_size(logits_type) - 1)) || ((uintptr_t)out_dev & (out_size(out_type) - 1)))
    return api_fail(SNN_ERR_INVALID_ARG, "misaligned device pointer");
  DeviceGuard guard(up.device);
  if (!guard.ok) return api_fail(SNN_ERR_CUDA, "cannot select device %d", up.device);
  const MoeCall c{m->gate, &up, &down, m->fn, act_dev, act_type, tokens, ld_act, logits_dev, logits_type, ld_logits, top_k, normalise != 0, work_dev,
                  out_dev, out_type, ld_out, (cudaStream_t)cuda_stream};
  int launched = 0;
  const cudaError_t e = moe_forward(c, &launched);
  api_count_launches(launched);
  return e == cudaSuccess ? SNN_OK : cuda_failed(e, "snn_conv_moe_forward");
}

snn_status_t snn_conv_moe_destroy(snn_conv_moe_t* m) {
  delete m;
  return SNN_OK;
}

snn_status_t snn_conv_scaled_create(const void* weights_dev, const float* scales_dev, int32_t count, int32_t c_in, int32_t c_out, int32_t device,
                                    void* cuda_stream, snn_conv_scaled_t** out) {
  if (!out) return api_fail(SNN_ERR_INVALID_ARG, "null output pointer");
  *out = nullptr;
  if (!weights_dev || !scales_dev) return api_fail(SNN_ERR_INVALID_ARG, "null argument");
  if (count < 1 || count > SNN_EXPERTS_MAX) return api_fail(SNN_ERR_INVALID_ARG, "1..%d projections, not %d", SNN_EXPERTS_MAX, count);
  if (c_in < 16 || c_in % 16 || c_out < 1 || c_in > 1 << 24 || c_out > 1 << 24)
    return api_fail(SNN_ERR_INVALID_ARG, "c_in=%d (a multiple of 16), c_out=%d", c_in, c_out);
  if (((uintptr_t)weights_dev & 15) || ((uintptr_t)scales_dev & 3)) return api_fail(SNN_ERR_INVALID_ARG, "misaligned device pointer");
  snn_status_t st = select_device(device);
  if (st != SNN_OK) return st;
  DeviceGuard guard(device);
  if (!guard.ok) return api_fail(SNN_ERR_CUDA, "cannot select device %d", device);
  snn_conv_scaled* h = new (std::nothrow) snn_conv_scaled();
  if (!h) return api_fail(SNN_ERR_OOM, "host allocation failed");
  h->p.device = device;
  int launched = 0;
  const cudaError_t e = scaled_create(static_cast<const uint8_t*>(weights_dev), scales_dev, count, c_in, c_out, (cudaStream_t)cuda_stream, &h->p, &launched);
  api_count_launches(launched);
  if (e != cudaSuccess) {
    scaled_destroy(&h->p);
    delete h;
    return cuda_failed(e, "snn_conv_scaled_create");
  }
  *out = h;
  return SNN_OK;
}

snn_status_t snn_conv_scaled_forward(snn_conv_scaled_t* h, const void* act_dev, int64_t ld_act, const float* act_scales_dev, int64_t ld_scales,
                                     const int32_t* offsets_dev, int32_t act_rows, void* out_dev, int32_t out_type, int64_t ld_out, void* cuda_stream) {
  if (!h) return api_fail(SNN_ERR_INVALID_ARG, "null handle");
  const Scaled& p = h->p;
  if (!out_ok(out_type)) return api_fail(SNN_ERR_INVALID_ARG, "outputs are SNN_OUT_F32, SNN_OUT_F16 or SNN_OUT_BF16, not %d", out_type);
  if (act_rows < 0) return api_fail(SNN_ERR_INVALID_ARG, "%d rows", act_rows);
  if (ld_act < p.C || ld_act % 16 || ld_scales < p.n_kb || ld_out < p.K)
    return api_fail(SNN_ERR_INVALID_ARG, "rows of %lld values, %lld scales and %lld outputs (c_in %d, %d blocks, c_out %d; the first a multiple of 16)", (long long)ld_act,
                    (long long)ld_scales, (long long)ld_out, p.C, p.n_kb, p.K);
  // (the kernels count pieces of rows, and these times strips of channels, in 32 bits, whatever the offsets say)
  if (act_rows > 1 << 30 || ((long long)act_rows / 8 + 1) * p.E >= (1ll << 31) || ((long long)act_rows / 8 + p.E) * ((p.K + 15) / 16) >= (1ll << 31))
    return api_fail(SNN_ERR_UNSUPPORTED, "%d rows of %d outputs over %d projections: split the call", act_rows, p.K, p.E);
  if (act_rows == 0) return SNN_OK;
  if (!act_dev || !act_scales_dev || !out_dev) return api_fail(SNN_ERR_INVALID_ARG, "null device pointer");
  if (((uintptr_t)act_dev & 15) || (((uintptr_t)act_scales_dev | (uintptr_t)offsets_dev) & 3) || ((uintptr_t)out_dev & (out_size(out_type) - 1)))
    return api_fail(SNN_ERR_INVALID_ARG, "misaligned device pointer");
  DeviceGuard guard(p.device);
  if (!guard.ok) return api_fail(SNN_ERR_CUDA, "cannot select device %d", p.device);
  const snn_status_t st = earlier_timeout(p.status_host);
  if (st != SNN_OK) return st;
  const ScaledCall c{static_cast<const uint8_t*>(act_dev), ld_act, act_scales_dev, ld_scales, offsets_dev, act_rows, out_dev, out_type, ld_out, (cudaStream_t)cuda_stream};
  int launched = 0;
  const cudaError_t e = scaled_forward(p, c, &launched);
  api_count_launches(launched);
  return e == cudaSuccess ? SNN_OK : cuda_failed(e, "snn_conv_scaled_forward");
}

snn_status_t snn_conv_scaled_destroy(snn_conv_scaled_t* h) {
  if (!h) return SNN_OK;
  DeviceGuard guard(h->p.device);
  scaled_destroy(&h->p);
  delete h;
  return SNN_OK;
}

snn_status_t snn_conv_scaled_quantise(const void* gate_dev, int64_t ld_gate, const void* up_dev, int64_t ld_up, int32_t type, int32_t in_rows,
                                      const int32_t* rows_dev, int32_t out_rows, int32_t columns, int32_t fn, void* values_dev, int64_t ld_values,
                                      float* scales_dev, int64_t ld_scales, int32_t device, void* cuda_stream) {
  snn_status_t st = check_between(gate_dev, ld_gate, up_dev, ld_up, type, in_rows, columns, fn);
  if (st != SNN_OK) return st;
  if (out_rows < 0 || (!rows_dev && out_rows != in_rows)) return api_fail(SNN_ERR_INVALID_ARG, "%d rows of outputs for %d rows without an index", out_rows, in_rows);
  if (ld_values < columns || ld_scales < ((long long)columns + 127) / 128)
    return api_fail(SNN_ERR_INVALID_ARG, "rows of %lld values and %lld scales for %d columns", (long long)ld_values, (long long)ld_scales, columns);
  if ((long long)out_rows * columns >= (1ll << 34)) return api_fail(SNN_ERR_UNSUPPORTED, "%d rows of %d columns: split the call", out_rows, columns);
  if (out_rows == 0) return SNN_OK;
  if ((in_rows > 0 && !up_dev) || !values_dev || !scales_dev) return api_fail(SNN_ERR_INVALID_ARG, "null device pointer");
  if (((uintptr_t)rows_dev | (uintptr_t)scales_dev) & 3) return api_fail(SNN_ERR_INVALID_ARG, "misaligned device pointer");
  st = select_device(device);
  if (st != SNN_OK) return st;
  DeviceGuard guard(device);
  if (!guard.ok) return api_fail(SNN_ERR_CUDA, "cannot select device %d", device);
  const QuantiseCall c{gate_dev, up_dev, ld_gate, ld_up, type, in_rows, rows_dev, out_rows, columns, fn, static_cast<uint8_t*>(values_dev), ld_values, scales_dev, ld_scales,
                       (cudaStream_t)cuda_stream};
  int launched = 0;
  const cudaError_t e = quantise_forward(c, &launched);
  api_count_launches(launched);
  return e == cudaSuccess ? SNN_OK : cuda_failed(e, "snn_conv_scaled_quantise");
}

}  // extern "C"
