// Device helpers of the router: a token's choice by a warp, counts and places of the rows.
#pragma once
#include <math_constants.h>

#include <cstdint>

#include "snn_products.cuh"

namespace snn {
namespace {

struct RouteParams {
  const void* logits;
  long long ld;
  int type, T, E, k, normalise, direct;
  int32_t* ids;
  float* weights;
  int32_t *offsets, *rows, *slots, *work;
};

// A float as an unsigned number of the same order, above 0; -infinity and NaN, which are not chosen, as 0.
__device__ __forceinline__ uint32_t ordered(float v) {
  if (!(v > -CUDART_INF_F)) return 0u;
  const uint32_t u = __float_as_uint(v + 0.f);   // (-0 is +0: equal logits have to be equal)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

// exp(v - most), 1 where both are the same infinity
__device__ __forceinline__ float above(float v, float most) { return v == most ? 1.f : expf(v - most); }

// A warp's logits of a token, E <= 32 V: lane l holds experts l, l + 32, ...
template <int V>
__device__ __forceinline__ void load_logits(const RouteParams& p, int t, float (&v)[V]) {
  const int lane = threadIdx.x & 31;
  const long long at = t * p.ld + lane;
  if (p.type == SNN_OUT_F32) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = lane + 32 * i < p.E ? static_cast<const float*>(p.logits)[at + 32 * i] : -CUDART_INF_F;
  } else {
    uint16_t u[V];
#pragma unroll
    for (int i = 0; i < V; ++i) u[i] = lane + 32 * i < p.E ? static_cast<const uint16_t*>(p.logits)[at + 32 * i] : 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
      v[i] = lane + 32 * i >= p.E ? -CUDART_INF_F : p.type == SNN_OUT_F16 ? __half2float(__ushort_as_half(u[i])) : __uint_as_float((uint32_t)u[i] << 16);
  }
}

// One token by one warp.  k times the warp's largest is taken, the lowest expert that has it, and its lane goes on to its next: up to 8
// experts a lane are sorted before, so that the next is at hand; of more it is looked for.  Lane j keeps choice j.  Bound by the number
// of instructions, and with few tokens by their latency: the exponentials come at the end, for all choices at once.
template <int V>
__device__ __forceinline__ void choose(const RouteParams& p, int t, const float (&v)[V], uint32_t* mask, int local) {
  const int lane = threadIdx.x & 31;
  constexpr bool SORTED = V <= 8;
  uint32_t u[V];
  int x[V];   // where u was in v
#pragma unroll
  for (int i = 0; i < V; ++i) {
    u[i] = ordered(v[i]);
    x[i] = i;
  }
  if (SORTED) {
    // (neighbours change places only if the later one is larger: equal ones keep their order)
#pragma unroll
    for (int n = V - 1; n > 0; --n)
#pragma unroll
      for (int i = 0; i < n; ++i)
        if (u[i + 1] > u[i]) {
          const uint32_t w = u[i];
          u[i] = u[i + 1];
          u[i + 1] = w;
          const int y = x[i];
          x[i] = x[i + 1];
          x[i + 1] = y;
        }
  }
  uint32_t best = u[0];
  int at = x[0], id = -1;
  auto look = [&] {
    best = u[0];
    at = 0;
#pragma unroll
    for (int i = 1; i < V; ++i)
      if (u[i] > best) {
        best = u[i];
        at = i;
      }
  };
  if (!SORTED) look();
  const uint32_t top = __reduce_max_sync(0xffffffffu, best);
  uint32_t most = top, mine = 0;
  for (int j = 0; j < p.k && most; ++j) {   // (0: nothing left that can be chosen)
    const uint32_t me = (uint32_t)(lane + 32 * at), e = __reduce_min_sync(0xffffffffu, best == most ? me : 0xffffffffu);
    if (lane == j) {
      id = (int)e;
      mine = most;
    }
    if (e == me) {
      if (SORTED) {
#pragma unroll
        for (int i = 0; i + 1 < V; ++i) {
          u[i] = u[i + 1];
          x[i] = x[i + 1];
        }
        u[V - 1] = 0;
        best = u[0];
        at = x[0];
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i == at) u[i] = 0;
        look();
      }
    }
    most = __reduce_max_sync(0xffffffffu, best);
  }
  const float largest = unordered(top), w = id < 0 ? 0.f : above(unordered(mine), largest);
  float all = p.normalise ? w : 0.f;
  if (!p.normalise) {
#pragma unroll
    for (int i = 0; i < V; ++i) all += v[i] > -CUDART_INF_F ? above(v[i], largest) : 0.f;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
  if (lane < p.k) {
    p.ids[(size_t)t * p.k + lane] = id;
    p.weights[(size_t)t * p.k + lane] = id < 0 ? 0.f : w / all;
    if (mask && id >= 0) atomicOr(mask + 2 * id + (local >> 5), 1u << (local & 31));   // (bits: any order gives the same word)
  }
}

// Exclusive sums of count[0..E) in place, by the whole CTA; returns the total.
__device__ int scan_counts(int* count, int E, int* part) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = (int)blockDim.x, warps = n >> 5;
  int base = 0;
  for (int e0 = 0; e0 < E; e0 += n) {
    const int e = e0 + (int)threadIdx.x, v = e < E ? count[e] : 0;
    int upto = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += o;
    }
    if (lane == 31) part[warp] = upto;
    __syncthreads();
    int sums = lane < warps ? part[lane] : 0;   // (each warp adds up the warps' sums for itself)
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, sums, d);
      if (lane >= d) sums += o;
    }
    const int before = __shfl_sync(0xffffffffu, sums, max(warp - 1, 0));
    if (e < E) count[e] = base + (warp ? before : 0) + upto - v;
    base += __shfl_sync(0xffffffffu, sums, 31);
    __syncthreads();
  }
  return base;
}

// Rows and slots of the CTA's tokens: start[e] is the first row of the CTA's choices of expert e, the mask says which of its tokens
// come before.
__device__ __forceinline__ void place(const RouteParams& p, const uint32_t* mask, const int* start, int t0, int tokens) {
  for (int i = threadIdx.x; i < tokens * p.k; i += (int)blockDim.x) {
    const int local = i / p.k, id = p.ids[(size_t)t0 * p.k + i];
    int slot = -1;
    if (id >= 0) {
      const uint32_t lo = mask[2 * id], hi = mask[2 * id + 1];
      slot = start[id] + (local < 32 ? __popc(lo & ((1u << local) - 1u)) : __popc(lo) + __popc(hi & ((1u << (local - 32)) - 1u)));
      p.rows[slot] = t0 + local;
    }
    p.slots[(size_t)t0 * p.k + i] = slot;
  }
}

}  // namespace
}  // namespace snn
