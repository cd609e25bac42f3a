// Device helpers of the projections' kernels: 16-bit types, the warp's matrix instruction, +1 / -1 from bits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "snn_products.h"

namespace snn {
namespace {

// What differs between the two types of activations: +1.0 twice in a register, and conversions.
struct F16 {
  static constexpr uint32_t kOne = 0x3c003c00u;
  static __device__ __forceinline__ float2 unpack(uint32_t v) {
    __half2 h;
    memcpy(&h, &v, 4);
    return __half22float2(h);
  }
};
struct BF16 {
  static constexpr uint32_t kOne = 0x3f803f80u;
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
};

// D[16 x 8] += A[16 x 16] B[16 x 8], fp32 sums; g = lane / 4, t = lane % 4:
// a = rows g, g + 8, g, g + 8 at k = 2t, 2t, 2t + 8, 2t + 8; b = column g at k = 2t, 2t + 8; d = rows g, g, g + 8, g + 8 at columns 2t, 2t + 1.
// (The order of k is free as long as both operands have the same.)
template <class T>
__device__ __forceinline__ void mma_16x8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma_16x8<F16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma_16x8<BF16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 2, 4 and 8, from a kernel's parameters: a multiplication by a number that the compiler knows would become a shift.
struct Powers {
  uint32_t of[4];
};
inline Powers powers() { return Powers{{1, 2, 4, 8}}; }
__device__ __forceinline__ Powers in_registers(const Powers& p) {
  Powers r;
  r.of[0] = 1;
#pragma unroll
  for (int i = 1; i < 4; ++i) asm volatile("mov.u32 %0, %1;" : "=r"(r.of[i]) : "r"(p.of[i]));
  return r;
}
// The two weights whose bits lie at 15 - shift and 31 - shift, as 16-bit +1 / -1: a mask, and a multiplication that brings the bits to the
// signs and adds the ones (every fourth pair's bits come to the signs by a shift for four pairs).  One instruction of the integer units and
// one of the FMA units; a shift and an exclusive-or for each are two of the former, which bounded both kernels (65 % busy for 64
// tokens over 64 experts).
template <class T>
__device__ __forceinline__ uint32_t plus_minus(uint32_t w, int shift, const Powers& pow) {
  const uint32_t v = w << (shift & 12);
  const int rest = shift & 3;
  if (rest == 0) return (v & 0x80008000u) ^ T::kOne;
  uint32_t r;
  asm("mad.lo.u32 %0, %1, %2, %3;" : "=r"(r) : "r"(v & (0x80008000u >> rest)), "r"(pow.of[rest]), "r"(T::kOne));
  return r;
}

// 16 bytes that another kernel may have written while this one was being set up: no read-only path.
__device__ __forceinline__ uint4 ld16(const void* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// ... that nobody will read again
__device__ __forceinline__ uint4 ld16_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.cs.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ld8(const void* p) {
  uint2 v;
  asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// One value in an output type, rounded to nearest even.
__device__ __forceinline__ void store_out(void* out, int type, long long i, float v) {
  if (type == SNN_OUT_F32) static_cast<float*>(out)[i] = v;
  else if (type == SNN_OUT_F16) static_cast<__half*>(out)[i] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(out)[i] = __float2bfloat16_rn(v);
}

// B (A x) of one output: rank products in fp32.
template <class T>
__device__ __forceinline__ float lowrank_term(const Lowrank& low, int K, int row, int co) {
  const int a = low.adapter[row];
  if (a < 0 || a >= low.n) return 0.f;
  const uint16_t* b = static_cast<const uint16_t*>(low.b) + ((size_t)a * K + co) * low.rank;
  const float* h = low.h + (size_t)row * low.rank;
  float s = 0.f;
  for (int j = 0; j < low.rank; j += 8) {
    const uint4 v = ld16(b + j);
    const float4 h0 = *reinterpret_cast<const float4*>(h + j), h1 = *reinterpret_cast<const float4*>(h + j + 4);
    float2 f = T::unpack(v.x);
    s = fmaf(f.x, h0.x, fmaf(f.y, h0.y, s));
    f = T::unpack(v.y);
    s = fmaf(f.x, h0.z, fmaf(f.y, h0.w, s));
    f = T::unpack(v.z);
    s = fmaf(f.x, h1.x, fmaf(f.y, h1.y, s));
    f = T::unpack(v.w);
    s = fmaf(f.x, h1.z, fmaf(f.y, h1.w, s));
  }
  return s;
}

__device__ __forceinline__ int clamp_offset(int v, int most) { return min(max(v, 0), most); }

}  // namespace
}  // namespace snn
