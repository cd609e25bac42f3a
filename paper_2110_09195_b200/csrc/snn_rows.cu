// Rows between two projections: activations, and the form of 8 bits with a scale for each 128 channels.
#include <cuda_fp8.h>

#include "snn_products.h"

#include "snn_products.cuh"
#include "snn_tc_common.cuh"

namespace snn {
namespace {

struct ActivateParams {
  const void *gate, *up;
  void* out;
  long long ld_gate, ld_up, ld_out;
  int rows, columns, groups, fn, type, out_type;
};

// A thread has 8 neighbouring columns.  Bound by memory: each value is read and written once, and leaves the caches first.
template <class Y, bool GATE>
__global__ void __launch_bounds__(256) activate_kernel(const ActivateParams p) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, r = i / p.groups;
  grid_dep_wait();
  grid_dep_launch();
  if (r >= p.rows) return;
  const int c = (int)(i - r * p.groups) * 8;
  using E = typename Element<Y>::type;
  Eight<Y> u, g;
  u.load(static_cast<const E*>(p.up) + r * p.ld_up + c);
  if (GATE) g.load(static_cast<const E*>(p.gate) + r * p.ld_gate + c);
  float2 v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float2 a = u.pair(q);
    if (GATE) {
      const float2 b = g.pair(q);
      v[q] = make_float2(activated(p.fn, b.x) * a.x, activated(p.fn, b.y) * a.y);
    } else {
      v[q] = make_float2(activated(p.fn, a.x), activated(p.fn, a.y));
    }
  }
  const long long at = r * p.ld_out + c;
  if (p.out_type == SNN_OUT_F32) {
    float4* const out = reinterpret_cast<float4*>(static_cast<float*>(p.out) + at);
    __stcs(out, make_float4(v[0].x, v[0].y, v[1].x, v[1].y));
    __stcs(out + 1, make_float4(v[2].x, v[2].y, v[3].x, v[3].y));
  } else {
    __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + at),
           make_uint4(pack_pair(p.out_type, v[0]), pack_pair(p.out_type, v[1]), pack_pair(p.out_type, v[2]), pack_pair(p.out_type, v[3])));
  }
}

// The same where columns, row lengths or pointers are not multiples of 8 values: one column a thread.
__global__ void __launch_bounds__(256) activate_odd_kernel(const ActivateParams p) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, r = i / p.columns;
  grid_dep_wait();
  grid_dep_launch();
  if (r >= p.rows) return;
  const int c = (int)(i - r * p.columns);
  const float u = value(p.up, p.type, r * p.ld_up + c);
  store_out(p.out, p.out_type, r * p.ld_out + c, p.gate ? activated(p.fn, value(p.gate, p.type, r * p.ld_gate + c)) * u : activated(p.fn, u));
}

struct QuantiseParams {
  const void *gate, *up;
  const int32_t* rows;
  uint8_t* values;
  float* scales;
  long long ld_gate, ld_up, ld_values, ld_scales;
  int in_rows, out_rows, columns, blocks, fn, type;
};

constexpr float kLargest = 448.f, kLeastScale = 0x1p-70f;

// 16 lanes have a block of 128 channels of a row, 8 each: the largest magnitude by four shuffles, one division for the scale and one for each value
// (by the scale, not times its reciprocal: 16-bit values often lie on a border between two of 8 bits, and go the way that the formula
// says).  ODD: columns, row lengths or pointers that are not multiples of 8 values.  Bound by memory.
template <class Y, bool GATE, bool ODD>
__global__ void __launch_bounds__(256) quantise_kernel(const QuantiseParams p) {
  const long long i = (long long)blockIdx.x * 16 + (threadIdx.x >> 4), r = i / p.blocks;
  grid_dep_wait();
  grid_dep_launch();
  // (whole half-warps; the shuffles name them alone)
  if (r >= p.out_rows) return;
  const int b = (int)(i - r * p.blocks), lane = threadIdx.x & 15, c = b * 128 + lane * 8;
  const long long from = p.rows ? p.rows[r] : r;
  const bool there = from >= 0 && from < p.in_rows;
  using E = typename Element<Y>::type;
  float v[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = 0.f;
  if (ODD) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (there && c + q < p.columns) {
        const float u = value(p.up, p.type, from * p.ld_up + c + q);
        v[q] = GATE ? activated(p.fn, value(p.gate, p.type, from * p.ld_gate + c + q)) * u : activated(p.fn, u);
      }
  } else if (there && c < p.columns) {
    Eight<Y> u, g;
    u.load(static_cast<const E*>(p.up) + from * p.ld_up + c);
    if (GATE) g.load(static_cast<const E*>(p.gate) + from * p.ld_gate + c);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float2 a = u.pair(q);
      if (GATE) {
        const float2 h = g.pair(q);
        v[2 * q] = activated(p.fn, h.x) * a.x;
        v[2 * q + 1] = activated(p.fn, h.y) * a.y;
      } else {
        v[2 * q] = activated(p.fn, a.x);
        v[2 * q + 1] = activated(p.fn, a.y);
      }
    }
  }
  float most = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const float m = fabsf(v[q]);
    most = m <= 3.402823466e38f ? fmaxf(most, m) : most;   // (infinities and NaN do not count)
  }
  const uint32_t mine = 0xffffu << (threadIdx.x & 16);
#pragma unroll
  for (int d = 8; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(mine, most, d));
  const float scale = fmaxf(most / kLargest, kLeastScale);
  uint32_t out[2] = {};
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const bool finite = fabsf(v[q]) <= 3.402823466e38f;
    const uint32_t bits = finite ? (uint32_t)__nv_cvt_float_to_fp8(v[q] / scale, __NV_SATFINITE, __NV_E4M3) : 0x7fu;
    out[q >> 2] |= bits << (8 * (q & 3));
  }
  uint8_t* const to = p.values + r * p.ld_values + c;
  if (ODD) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (c + q < p.columns) to[q] = (uint8_t)(out[q >> 2] >> (8 * (q & 3)));
  } else if (c < p.columns) {
    *reinterpret_cast<uint2*>(to) = make_uint2(out[0], out[1]);
  }
  if (lane == 0) p.scales[r * p.ld_scales + b] = scale;
}

template <class Y>
cudaError_t quantise_type(const QuantiseParams& p, bool odd, unsigned blocks, cudaStream_t s) {
  if (p.gate) return odd ? launch_dependent(quantise_kernel<Y, true, true>, blocks, 256, 0, s, p) : launch_dependent(quantise_kernel<Y, true, false>, blocks, 256, 0, s, p);
  return odd ? launch_dependent(quantise_kernel<Y, false, true>, blocks, 256, 0, s, p) : launch_dependent(quantise_kernel<Y, false, false>, blocks, 256, 0, s, p);
}
template <class Y>
cudaError_t activate_type(const ActivateParams& p, unsigned blocks, cudaStream_t s) {
  return p.gate ? launch_dependent(activate_kernel<Y, true>, blocks, 256, 0, s, p) : launch_dependent(activate_kernel<Y, false>, blocks, 256, 0, s, p);
}

}  // namespace

cudaError_t activate_forward(const ActivateCall& c, int* launched) {
  ActivateParams p{c.gate, c.up, c.out, c.ld_gate, c.ld_up, c.ld_out, c.rows, c.columns, c.columns / 8, c.fn, c.type, c.out_type};
  const bool eights = c.columns % 8 == 0 && c.ld_up % 8 == 0 && (!c.gate || c.ld_gate % 8 == 0) && c.ld_out % 8 == 0 &&
                      (((uintptr_t)c.up | (uintptr_t)c.gate | (uintptr_t)c.out) & 15) == 0;
  const long long blocks = ((long long)c.rows * (eights ? p.groups : c.columns) + 255) / 256;
  if (blocks >= (1ll << 31)) return cudaErrorInvalidValue;
  *launched += 1;
  if (!eights) return launch_dependent(activate_odd_kernel, (unsigned)blocks, 256, 0, c.stream, p);
  if (c.type == SNN_OUT_F32) return activate_type<float>(p, (unsigned)blocks, c.stream);
  return c.type == SNN_OUT_F16 ? activate_type<F16>(p, (unsigned)blocks, c.stream) : activate_type<BF16>(p, (unsigned)blocks, c.stream);
}

cudaError_t quantise_forward(const QuantiseCall& c, int* launched) {
  const QuantiseParams p{c.gate, c.up, c.rows, c.values, c.scales, c.ld_gate, c.ld_up, c.ld_values, c.ld_scales, c.in_rows, c.out_rows, c.columns, (c.columns + 127) / 128, c.fn, c.type};
  const bool odd = c.columns % 8 || c.ld_up % 8 || (c.gate && c.ld_gate % 8) || c.ld_values % 8 ||
                   (((uintptr_t)c.up | (uintptr_t)c.gate) & 15) || ((uintptr_t)c.values & 7);
  const long long blocks = ((long long)c.out_rows * p.blocks + 15) / 16;
  if (blocks >= (1ll << 31)) return cudaErrorInvalidValue;
  *launched += 1;
  if (c.type == SNN_OUT_F32) return quantise_type<float>(p, odd, (unsigned)blocks, c.stream);
  return c.type == SNN_OUT_F16 ? quantise_type<F16>(p, odd, (unsigned)blocks, c.stream) : quantise_type<BF16>(p, odd, (unsigned)blocks, c.stream);
}

}  // namespace snn
