// Rows between two projections: activations, and the form of 8 bits with a scale for each 128 channels.
#include <cuda_fp8.h>
#include <math_constants.h>

#include <type_traits>

#include "snn_products.h"

#include "snn_products.cuh"
#include "snn_tc_common.cuh"

namespace snn {
namespace {

// q / d for q below 2^31, by a multiplication.  (A division of 64 bits by each thread took as long as the activation.)
struct Divisor {
  uint32_t d, m, s;
  explicit Divisor(uint32_t by) : d(by), s(0) {
    while ((1ull << s) < d) ++s;
    m = (uint32_t)((1ull << (31 + s)) / d + 1);
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t q) const { return __umulhi(2u * q, m) >> s; }
};

struct ActivateParams {
  const void *gate, *up;
  void* out;
  long long ld_gate, ld_up, ld_out;
  int rows, columns, fn, type, out_type;
  Divisor each;   // eights of a row, or 256ths
};

// A thread has 8 neighbouring columns.  Bound by memory: each value is read and written once, and leaves the caches first (8191 x 8192 gated bf16 values behind SILU 66 us, 6.1 TB/s).
template <class Y, bool GATE>
__global__ void __launch_bounds__(256) activate_kernel(const ActivateParams p) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  const long long r = p.each(i);
  grid_dep_wait();
  grid_dep_launch();
  if (r >= p.rows) return;
  const int c = (int)(i - (uint32_t)r * p.each.d) * 8;
  using E = typename Element<Y>::type;
  Eight<Y> u, g;
  u.load(static_cast<const E*>(p.up) + r * p.ld_up + c);
  if (GATE) g.load(static_cast<const E*>(p.gate) + r * p.ld_gate + c);
  float2 v[4];
  auto all = [&](auto near) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float2 a = u.pair(q);
      const uint64_t w = pair_of(a.x, a.y);
      if (GATE) {
        const float2 b = g.pair(q);
        v[q] = floats_of(mul2(activated2<decltype(near)::value>(p.fn, pair_of(b.x, b.y)), w));
      } else {
        v[q] = floats_of(activated2<decltype(near)::value>(p.fn, w));
      }
    }
  };
  if (p.fn == SNN_FN_SILU && !((GATE ? g.lowest(g) : u.lowest(u)) < SILU_NEAR)) all(std::true_type{});
  else all(std::false_type{});
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
  const long long r = p.each(blockIdx.x);
  const int c = (int)(blockIdx.x - (uint32_t)r * p.each.d) * 256 + (int)threadIdx.x;
  grid_dep_wait();
  grid_dep_launch();
  if (c >= p.columns) return;
  const float u = value(p.up, p.type, r * p.ld_up + c);
  store_out(p.out, p.out_type, r * p.ld_out + c, p.gate ? activated(p.fn, value(p.gate, p.type, r * p.ld_gate + c)) * u : activated(p.fn, u));
}

struct QuantiseParams {
  const void *gate, *up;
  const int32_t* rows;
  uint8_t* values;
  float* scales;
  long long ld_gate, ld_up, ld_values, ld_scales;
  int in_rows, out_rows, columns, fn, type;
  Divisor blocks;   // of a row
};

constexpr float kLargest = 448.f, kLeastScale = 0x1p-70f;

// v / scale in fp32, by the scale's reciprocal (itself rounded once): the product is within 1.5 steps, and a correction of it within 2^-46 of the quotient before it is
// rounded; a second one then gives the quotient's nearest number (Markstein, IBM Journal of Research and Development 34, 1990).  ONCE: values of 16 bits.  One correction is
// then enough: what could go another way is a quotient that lies next to a number halfway between two fp32 numbers one of which is a border of the 8-bit values, and a value of
// 11 bits over one of 24 comes no nearer to it than 2^-35.  (Behind an activation the value itself is rounded.)  scale is at least 2^-70 and at most 2^120, so that
// nothing that reaches a step of the 8-bit value underflows; an infinity becomes NaN.  (Not v times the reciprocal: 16-bit values often lie on a border
// between two of 8 bits, and go the way that the formula says.)
template <bool ONCE>
__device__ __forceinline__ uint64_t quotients(uint64_t v, uint64_t minus_scale, uint64_t inverse) {
  uint64_t q = mul2(v, inverse);
  q = fma2(fma2(q, minus_scale, v), inverse, q);
  return ONCE ? q : fma2(fma2(q, minus_scale, v), inverse, q);
}

// 8 lanes have a block of 128 channels of a row, 8 neighbouring ones and the 8 that lie 64 behind them each: the largest magnitude by three shuffles, two divisions for the
// scale, three or five multiplications and additions for each value.  ODD: columns, row lengths or pointers that are not multiples of 8 values.  Bound by
// memory, nearly by the number of instructions (8191 x 4096 gated bf16 values behind SILU: 16 lanes a block, two corrections always and comparisons against infinity took 46 us, now 34: 5.0 TB/s, 74 % of the issue slots).
template <class Y, bool GATE, bool ODD>
__global__ void __launch_bounds__(256) quantise_kernel(const QuantiseParams p) {
  const uint32_t i = blockIdx.x * 32 + (threadIdx.x >> 3);
  const long long r = p.blocks(i);
  grid_dep_wait();
  grid_dep_launch();
  // (whole groups of 8 lanes; the shuffles name them alone)
  if (r >= p.out_rows) return;
  const int b = (int)(i - (uint32_t)r * p.blocks.d), lane = threadIdx.x & 7, c0 = b * 128 + lane * 8;
  const long long from = p.rows ? p.rows[r] : r;
  const bool there = from >= 0 && from < p.in_rows;
  using E = typename Element<Y>::type;
  float v[16];
#pragma unroll
  for (int q = 0; q < 16; ++q) v[q] = 0.f;
  if (ODD) {
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const int c = c0 + (q >> 3) * 64 + (q & 7);
      if (there && c < p.columns) {
        const float u = value(p.up, p.type, from * p.ld_up + c);
        v[q] = GATE ? activated(p.fn, value(p.gate, p.type, from * p.ld_gate + c)) * u : activated(p.fn, u);
      }
    }
  } else {
    Eight<Y> u[2], g[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = c0 + 64 * h;
      const bool have = there && c < p.columns;
      if (have) u[h].load(static_cast<const E*>(p.up) + from * p.ld_up + c);
      else u[h].zero();
      if (GATE) {
        if (have) g[h].load(static_cast<const E*>(p.gate) + from * p.ld_gate + c);
        else g[h].zero();
      }
    }
    auto all = [&](auto near) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float2 a = u[q >> 2].pair(q & 3);
        uint64_t w = pair_of(a.x, a.y);
        if (GATE) {
          const float2 h = g[q >> 2].pair(q & 3);
          w = mul2(activated2<decltype(near)::value>(p.fn, pair_of(h.x, h.y)), w);
        } else {
          w = activated2<decltype(near)::value>(p.fn, w);
        }
        const float2 f = floats_of(w);
        v[2 * q] = f.x;
        v[2 * q + 1] = f.y;
      }
    };
    if (p.fn == SNN_FN_SILU && !((GATE ? g[0].lowest(g[1]) : u[0].lowest(u[1])) < SILU_NEAR)) all(std::true_type{});
    else all(std::false_type{});
  }
  const uint32_t mine = 0xffu << (threadIdx.x & 24);
  float most = 0.f;
#pragma unroll
  for (int q = 0; q < 16; ++q) most = fmaxf(most, fabsf(v[q]));   // (NaN is nobody's larger)
#pragma unroll
  for (int d = 4; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(mine, most, d));
  if (most == CUDART_INF_F) {   // (the same in the 8 lanes)
    most = 0.f;
#pragma unroll
    for (int q = 0; q < 16; ++q) most = fabsf(v[q]) < CUDART_INF_F ? fmaxf(most, fabsf(v[q])) : most;
#pragma unroll
    for (int d = 4; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(mine, most, d));
  }
  const float scale = fmaxf(most / kLargest, kLeastScale), inverse = 1.f / scale;
  constexpr bool ONCE = !std::is_same<Y, float>::value;
  const uint64_t minus2 = pair_of(-scale, -scale), inverse2 = pair_of(inverse, inverse);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t out[2] = {};
#pragma unroll
    for (int q = 0; q < 8; q += 2)
      out[q >> 2] |= (uint32_t)__nv_cvt_float2_to_fp8x2(floats_of(quotients<ONCE>(pair_of(v[8 * h + q], v[8 * h + q + 1]), minus2, inverse2)), __NV_SATFINITE, __NV_E4M3) << (8 * (q & 3));
    const int c = c0 + 64 * h;
    uint8_t* const to = p.values + r * p.ld_values + c;
    if (ODD) {
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (c + q < p.columns) to[q] = (uint8_t)(out[q >> 2] >> (8 * (q & 3)));
    } else if (c < p.columns) {
      *reinterpret_cast<uint2*>(to) = make_uint2(out[0], out[1]);
    }
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
  const bool eights = c.columns % 8 == 0 && c.ld_up % 8 == 0 && (!c.gate || c.ld_gate % 8 == 0) && c.ld_out % 8 == 0 &&
                      (((uintptr_t)c.up | (uintptr_t)c.gate | (uintptr_t)c.out) & 15) == 0;
  const ActivateParams p{c.gate, c.up, c.out, c.ld_gate, c.ld_up, c.ld_out, c.rows, c.columns, c.fn, c.type, c.out_type, Divisor(eights ? c.columns / 8 : (c.columns + 255) / 256)};
  const long long units = (long long)c.rows * p.each.d, blocks = eights ? (units + 255) / 256 : units;
  if (units >= (1ll << 31)) return cudaErrorInvalidValue;
  *launched += 1;
  if (!eights) return launch_dependent(activate_odd_kernel, (unsigned)blocks, 256, 0, c.stream, p);
  if (c.type == SNN_OUT_F32) return activate_type<float>(p, (unsigned)blocks, c.stream);
  return c.type == SNN_OUT_F16 ? activate_type<F16>(p, (unsigned)blocks, c.stream) : activate_type<BF16>(p, (unsigned)blocks, c.stream);
}

cudaError_t quantise_forward(const QuantiseCall& c, int* launched) {
  const QuantiseParams p{c.gate, c.up, c.rows, c.values, c.scales, c.ld_gate, c.ld_up, c.ld_values, c.ld_scales, c.in_rows, c.out_rows, c.columns, c.fn, c.type, Divisor((c.columns + 127) / 128)};
  const bool odd = c.columns % 8 || c.ld_up % 8 || (c.gate && c.ld_gate % 8) || c.ld_values % 8 ||
                   (((uintptr_t)c.up | (uintptr_t)c.gate) & 15) || ((uintptr_t)c.values & 7);
  const long long units = (long long)c.out_rows * p.blocks.d, blocks = (units + 31) / 32;
  if (units >= (1ll << 31)) return cudaErrorInvalidValue;
  *launched += 1;
  if (c.type == SNN_OUT_F32) return quantise_type<float>(p, odd, (unsigned)blocks, c.stream);
  return c.type == SNN_OUT_F16 ? quantise_type<F16>(p, odd, (unsigned)blocks, c.stream) : quantise_type<BF16>(p, odd, (unsigned)blocks, c.stream);
}

}  // namespace snn
