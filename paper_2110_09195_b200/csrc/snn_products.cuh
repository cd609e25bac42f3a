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
  static __device__ __forceinline__ uint32_t lower(uint32_t a, uint32_t b) {   // (of either half)
    uint32_t r;
    asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
};
struct BF16 {
  static constexpr uint32_t kOne = 0x3f803f80u;
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
  static __device__ __forceinline__ uint32_t lower(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
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

// Pieces of at most `most` rows of an expert, counted over the experts in their order, by each warp for itself: every lane counts the
// pieces of a run of experts, and a scan over the lanes says whose run a piece is in.
struct Pieces {
  int upto, count, total;   // this lane's, and of all
};
__device__ __forceinline__ int pieces_of(const int32_t* offsets, int e, int R, int most, int* lo_out, int* hi_out) {
  const int lo = clamp_offset(offsets[e], R), hi = clamp_offset(offsets[e + 1], R);
  *lo_out = lo;
  *hi_out = hi;
  return (max(hi - lo, 0) + most - 1) / most;
}
__device__ __forceinline__ Pieces count_pieces(const int32_t* offsets, int E, int R, int most) {
  if (!offsets) return Pieces{0, 0, (R + most - 1) / most};
  const int lane = threadIdx.x & 31, per = (E + 31) >> 5, e0 = lane * per, e1 = min(E, e0 + per);
  Pieces r{0, 0, 0};
  int lo, hi;
  for (int e = e0; e < e1; ++e) r.count += pieces_of(offsets, e, R, most, &lo, &hi);
  r.upto = r.count;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, r.upto, d);
    if (lane >= d) r.upto += v;
  }
  r.total = __shfl_sync(0xffffffffu, r.upto, 31);
  return r;
}
// Expert, first row and rows of a piece below the total.
__device__ __forceinline__ void find_piece(const Pieces& all, const int32_t* offsets, int E, int R, int most, int piece, int* e_out, int* r_out, int* n_out) {
  if (!offsets) {
    *e_out = 0;
    *r_out = piece * most;
    *n_out = min(most, R - piece * most);
    return;
  }
  const int lane = threadIdx.x & 31, per = (E + 31) >> 5, e0 = lane * per, e1 = min(E, e0 + per);
  const int src = __ffs(__ballot_sync(0xffffffffu, piece < all.upto)) - 1;
  int e = 0, r = 0, n = 0;
  if (lane == src) {
    int left = piece - (all.upto - all.count), lo, hi;
    for (e = e0; e < e1; ++e) {
      const int pieces = pieces_of(offsets, e, R, most, &lo, &hi);
      if (left < pieces) {
        r = lo + left * most;
        n = min(most, hi - r);
        break;
      }
      left -= pieces;
    }
  }
  *e_out = __shfl_sync(0xffffffffu, e, src);
  *r_out = __shfl_sync(0xffffffffu, r, src);
  *n_out = __shfl_sync(0xffffffffu, n, src);
}

// 8 neighbouring values as fp32, and their 16 or 32 bytes: read once, so they are the first to leave the caches.
template <class Y>
struct Eight;
template <>
struct Eight<float> {
  uint4 lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = ld16_stream(p);
    hi = ld16_stream(p + 4);
  }
  __device__ __forceinline__ void zero() { lo = hi = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ float2 pair(int i) const {
    const uint4& v = i < 2 ? lo : hi;
    return i & 1 ? make_float2(__uint_as_float(v.z), __uint_as_float(v.w)) : make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
  }
  // the lowest of the values that are numbers, its own and `other`'s
  __device__ __forceinline__ float lowest(const Eight& other) const {
    float r = fminf(pair(0).x, other.pair(0).x);
#pragma unroll
    for (int i = 0; i < 4; ++i) r = fminf(fminf(r, fminf(pair(i).x, pair(i).y)), fminf(other.pair(i).x, other.pair(i).y));
    return r;
  }
};
template <class T>
struct Eight16 {
  uint4 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = ld16_stream(p); }
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ float2 pair(int i) const { return T::unpack(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
  __device__ __forceinline__ float lowest(const Eight16& other) const {
    const float2 r = T::unpack(T::lower(T::lower(T::lower(v.x, v.y), T::lower(v.z, v.w)),
                                        T::lower(T::lower(other.v.x, other.v.y), T::lower(other.v.z, other.v.w))));
    return fminf(r.x, r.y);
  }
};
template <>
struct Eight<F16> : Eight16<F16> {};
template <>
struct Eight<BF16> : Eight16<BF16> {};
template <class Y>
struct Element {
  using type = uint16_t;
};
template <>
struct Element<float> {
  using type = float;
};

__device__ __forceinline__ uint32_t pack_pair(int type, float2 v) {
  uint32_t r;
  if (type == SNN_OUT_F16) {
    const __half2 h = __floats2half2_rn(v.x, v.y);
    memcpy(&r, &h, 4);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
    memcpy(&r, &h, 4);
  }
  return r;
}

__device__ __forceinline__ float value(const void* y, int type, long long i) {
  if (type == SNN_OUT_F32) return static_cast<const float*>(y)[i];
  if (type == SNN_OUT_F16) return __half2float(static_cast<const __half*>(y)[i]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(y)[i]);
}

// Two fp32 operations an instruction, each rounded as by itself.
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 floats_of(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float exp2_approx(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float reciprocal_approx(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// v / (1 + exp(-v)), twice.  The exponential by powers of 2 with the product's rest (what the first number leaves of v / ln 2) in a second factor: within 2^-21.  Of v from
// SILU_NEAR up: from -87.34 down the reciprocal is 0, but the value a normal number to -91.9.
// (a thread asks once whether any of its values is below: for each pair of them, 8191 x 4096 gated bf16 values into 8 bits took 35.4 us and not 34.1; without asking 33.4)
constexpr float SILU_NEAR = -87.f;
__device__ __forceinline__ uint64_t silu2(uint64_t v) {
  constexpr float L = -1.44269504088896340736f, L_rest = -1.44269504088896340736 - (double)L, ln2 = 0.69314718055994530942f;
  const float2 f = floats_of(v);
  const uint64_t c = pair_of(fminf(fmaxf(f.x, -126.f), 126.f), fminf(fmaxf(f.y, -126.f), 126.f));   // (infinities would leave a rest that is none)
  const uint64_t h = mul2(c, pair_of(L, L));
  const float2 hs = floats_of(h);
  const uint64_t rest = fma2(c, pair_of(L, L), pair_of(-hs.x, -hs.y));
  const uint64_t e = pair_of(exp2_approx(hs.x), exp2_approx(hs.y));
  const uint64_t factor = fma2(fma2(c, pair_of(L_rest, L_rest), rest), pair_of(ln2, ln2), pair_of(1.f, 1.f));
  const float2 d = floats_of(fma2(e, factor, pair_of(1.f, 1.f)));
  return mul2(v, pair_of(reciprocal_approx(d.x), reciprocal_approx(d.y)));
}
// v exp(v), which v / (1 + exp(-v)) is below SILU_NEAR:  (v / 2^64) 2^(v / ln 2 + 64), so that nothing underflows but the result.
__device__ __forceinline__ float silu_far(float v) {
  constexpr float L = 1.44269504088896340736f, L_rest = 1.44269504088896340736 - (double)L, ln2 = 0.69314718055994530942f;
  const float c = fmaxf(v, -200.f), h = c * L, rest = fmaf(c, L_rest, fmaf(c, L, -h)), e = exp2_approx(h + 64.f);   // (h + 64 is exact: a multiple of h's last bit, and smaller)
  return v * 0x1p-64f * fmaf(e, rest * ln2, e);
}
__device__ __forceinline__ float silu(float v) { return v < SILU_NEAR ? silu_far(v) : floats_of(silu2(pair_of(v, v))).x; }

// The normal distribution's function.  For z = |v|:  exp(-z^2 / 2) times a smooth factor, which is P(u) / (z + k), u = 1 - 2 k / (z + k) in [-1, 1), with P fitted for the
// least relative error (2^-23 up to z = 13.3, from values of erfc in 64 bits); z^2 / 2 as a sum of two numbers.  Within 2^-20.4 of the value where that is a normal
// number, on both sides.  (normcdff takes 60 instructions; with them the activation of 8191 x 4096 gated bf16 values took 78 us.)
__device__ __forceinline__ float normal_cdf(float v) {
  constexpr float k = 4.25f, L = -0.72134752044448170368f, L_rest = -0.72134752044448170368 - (double)L;   // 1 / (2 ln 2)
  const float z = fminf(fabsf(v), 14.5f);   // (from there on 0; NaN is in the other factor)
  const float r = __fdividef(1.f, z + k), u = fmaf(-2.f * k, r, 1.f);
  float p = 0.0021056882105767727f;
  p = fmaf(p, u, -0.0010409007081761956f);
  p = fmaf(p, u, -0.01938452757894993f);
  p = fmaf(p, u, 0.08534717559814453f);
  p = fmaf(p, u, -0.22050929069519043f);
  p = fmaf(p, u, 0.41822102665901184f);
  p = fmaf(p, u, -0.6251299977302551f);
  p = fmaf(p, u, 0.7595543265342712f);
  const float square = z * z, h = square * L, rest = fmaf(square, L_rest, fmaf(fmaf(z, z, -square), L, fmaf(square, L, -h)));
  const float e = exp2_approx(h), lower = p * r * fmaf(e, rest * 0.69314718056f, e);
  return v < 0.f ? lower : 1.f - lower;
}

// What stands between two projections (SNN_FN_*): with a gate, fn(gate) * up.
__device__ __forceinline__ float activated(int fn, float v) {
  if (fn == SNN_FN_SILU) return silu(v);
  if (fn == SNN_FN_GELU) return v * normal_cdf(v);   // (no 1 + erf(v): that loses the digits of a negative v)
  if (fn == SNN_FN_RELU) return v < 0.f ? 0.f : v;   // (NaN stays)
  return v;
}
// (SILU_NEAR_ALL: it is SiLU, of values none of which is below SILU_NEAR)
template <bool SILU_NEAR_ALL>
__device__ __forceinline__ uint64_t activated2(int fn, uint64_t v) {
  if (SILU_NEAR_ALL) return silu2(v);
  const float2 f = floats_of(v);
  return pair_of(activated(fn, f.x), activated(fn, f.y));
}

}  // namespace
}  // namespace snn
