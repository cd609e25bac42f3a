// Routing of tokens to experts: the choice, the order of the rows by expert, and the weighted sum that undoes it.
#include <math_constants.h>

#include "snn_products.h"

#include "snn_products.cuh"
#include "snn_tc_common.cuh"

namespace snn {
namespace {

constexpr int RT_BLOCK = 64;   // tokens of a CTA: two words of a mask for each expert
constexpr int RT_CHOOSE_WARPS = 32;   // two tokens a warp
constexpr int RT_WARPS = 16;
// CTAs up to which each adds up the others' counts by itself (128 experts, 8 each, 4000 tokens 9.4 us, with sums in a launch of their own 11.6; 6000
// tokens 10.7 and 12.1; 8191 tokens 16.9 and 12.7).
constexpr int RT_DIRECT = 96;

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
    if (id >= 0) atomicOr(mask + 2 * id + (local >> 5), 1u << (local & 31));   // (bits: any order gives the same word)
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

// First launch: each CTA's tokens choose, and the CTA counts its choices of each expert, in bytes where every CTA of the last launch reads all
// of them.  With one CTA that is all there is to count, and it goes on to place them.
template <int V>
__global__ void __launch_bounds__(RT_CHOOSE_WARPS * 32) route_choose_kernel(const RouteParams p) {
  const int threads = (int)blockDim.x;
  __shared__ uint32_t mask[2 * 32 * V];
  __shared__ int count[32 * V], part[RT_CHOOSE_WARPS];
  const int t0 = (int)blockIdx.x * RT_BLOCK, tokens = min(RT_BLOCK, p.T - t0), warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < 2 * p.E; i += threads) mask[i] = 0;
  grid_dep_wait();
  grid_dep_launch();
  __syncthreads();
  float v[V];
  if (warp < tokens) load_logits(p, t0 + warp, v);
  const int step = threads >> 5;
  for (int i = warp; i < tokens; i += step) {
    float next[V];
    const bool more = i + step < tokens;
    if (more) load_logits(p, t0 + i + step, next);
    choose<V>(p, t0 + i, v, mask, i);
#pragma unroll
    for (int q = 0; q < V; ++q)
      if (more) v[q] = next[q];
  }
  __syncthreads();
  const bool alone = gridDim.x == 1;
  auto chosen = [&](int e) { return e < p.E ? __popc(mask[2 * e]) + __popc(mask[2 * e + 1]) : 0; };   // (at most 64)
  if (!alone && p.direct) {
    for (int w = threadIdx.x; 4 * w < p.E; w += threads)
      p.work[(size_t)blockIdx.x * ((p.E + 3) / 4) + w] = chosen(4 * w) | chosen(4 * w + 1) << 8 | chosen(4 * w + 2) << 16 | chosen(4 * w + 3) << 24;
    return;
  }
  for (int e = threadIdx.x; e < p.E; e += threads) {
    if (alone) count[e] = chosen(e);
    else p.work[(size_t)blockIdx.x * p.E + e] = chosen(e);
  }
  if (!alone) return;
  __syncthreads();
  const int total = scan_counts(count, p.E, part);
  for (int e = threadIdx.x; e < p.E; e += threads) p.offsets[e] = count[e];
  if (threadIdx.x == 0) p.offsets[p.E] = total;
  place(p, mask, count, t0, tokens);
  for (int i = total + (int)threadIdx.x; i < p.T * p.k; i += threads) p.rows[i] = -1;
}

// Between the two with many CTAs: the counts become sums over the CTAs before, and the totals follow behind the last.  A CTA has 32
// experts, a lane one of them, each warp a run of the CTAs.
__global__ void __launch_bounds__(1024) route_sum_kernel(int32_t* work, int E, int blocks) {
  __shared__ int part[32][33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, e = (int)blockIdx.x * 32 + lane;
  const int each = (blocks + 31) / 32, b0 = min(blocks, warp * each), b1 = min(blocks, b0 + each);
  grid_dep_wait();
  grid_dep_launch();
  int sum = 0;
  if (e < E)
#pragma unroll 8
    for (int b = b0; b < b1; ++b) sum += work[(size_t)b * E + e];
  part[warp][lane] = sum;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < warp; ++w) before += part[w][lane];
  if (e < E) {
    for (int b = b0; b < b1; b += 8) {
      int v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = b + i < b1 ? work[(size_t)(b + i) * E + e] : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (b + i < b1) work[(size_t)(b + i) * E + e] = before;
        before += v[i];
      }
    }
    if (warp == 31) work[(size_t)blocks * E + e] = before;
  }
}

// Last launch: where the experts' rows begin, and where this CTA's begin among them (all CTAs' counts, added up here if `direct`), then its
// tokens' rows and slots.
__global__ void __launch_bounds__(RT_WARPS * 32) route_place_kernel(const RouteParams p) {
  extern __shared__ int sm[];
  int* const all = sm;                                                 // [E]
  int* const before = sm + p.E;                                        // [E]
  uint32_t* const mask = reinterpret_cast<uint32_t*>(sm + 2 * p.E);    // [E][2]
  __shared__ int part[RT_WARPS];
  const int t0 = (int)blockIdx.x * RT_BLOCK, tokens = min(RT_BLOCK, p.T - t0), n = RT_WARPS * 32;
  for (int i = threadIdx.x; i < 4 * p.E; i += n) sm[i] = 0;
  grid_dep_wait();
  grid_dep_launch();
  __syncthreads();
  for (int i = threadIdx.x; i < tokens * p.k; i += n) {
    const int id = p.ids[(size_t)t0 * p.k + i], local = i / p.k;
    if (id >= 0) atomicOr(mask + 2 * id + (local >> 5), 1u << (local & 31));
  }
  if (p.direct) {
    // a thread has four experts and every `turns`-th CTA, eight loads on their way, two sums in a register; the turns' sums meet (whole numbers:
    // any order gives the same)
    const int words = (p.E + 3) / 4, width = (words + 31) & ~31, turns = n / width, turn = (int)threadIdx.x / width, w = (int)threadIdx.x - turn * width;
    if (turn < turns && w < words) {
      uint32_t sum[2] = {}, mine[2] = {};   // experts 4w and 4w + 2, 4w + 1 and 4w + 3
      for (int b0 = turn; b0 < (int)gridDim.x; b0 += 8 * turns) {
        uint32_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = b0 + i * turns < (int)gridDim.x ? (uint32_t)p.work[(size_t)(b0 + i * turns) * words + w] : 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t two = (v[i] >> (8 * h)) & 0x00ff00ffu;
            sum[h] += two;
            if (b0 + i * turns < (int)blockIdx.x) mine[h] += two;
          }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * w + i < p.E) {
          atomicAdd(all + 4 * w + i, (int)((sum[i & 1] >> (8 * (i & 2))) & 0xffffu));
          atomicAdd(before + 4 * w + i, (int)((mine[i & 1] >> (8 * (i & 2))) & 0xffffu));
        }
    }
  } else {
    for (int e = threadIdx.x; e < p.E; e += n) {
      all[e] = p.work[(size_t)gridDim.x * p.E + e];
      before[e] = p.work[(size_t)blockIdx.x * p.E + e];
    }
  }
  __syncthreads();
  const int total = scan_counts(all, p.E, part);
  for (int e = threadIdx.x; e < p.E; e += n) {
    if (blockIdx.x == 0) p.offsets[e] = all[e];
    all[e] += before[e];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.E] = total;
  __syncthreads();
  place(p, mask, all, t0, tokens);
  // (behind the last row by a CTA's threads may be behind 2^31)
  for (long long i = total + (long long)blockIdx.x * n + (int)threadIdx.x; i < (long long)p.T * p.k; i += (long long)gridDim.x * n) p.rows[i] = -1;
}

// ---------------------------------------------------------------- combine

struct CombineParams {
  const void* y;
  const int32_t* slots;
  const float* weights;
  void* out;
  long long ld_y, ld_out;
  int y_type, y_rows, T, k, C, out_type, groups;
};

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
};
template <class T>
struct Eight16 {
  uint4 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = ld16_stream(p); }
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ float2 pair(int i) const { return T::unpack(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
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

// A thread sums 8 neighbouring columns of a token, 4 rows on their way at a time; neighbouring threads, neighbouring columns.  Bound by memory:
// each row is read once.
template <class Y>
__global__ void __launch_bounds__(256) combine_kernel(const CombineParams p) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long t = i / p.groups;
  grid_dep_wait();
  grid_dep_launch();
  const int c = (int)(i - t * p.groups) * 8;
  if (t >= p.T) return;
  const typename Element<Y>::type* const y = static_cast<const typename Element<Y>::type*>(p.y) + c;
  float2 s[4] = {};
  for (int j0 = 0; j0 < p.k; j0 += 4) {
    Eight<Y> v[4];
    float w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int slot = j0 + j < p.k ? p.slots[t * p.k + j0 + j] : -1;
      const bool there = slot >= 0 && slot < p.y_rows;
      w[j] = there ? p.weights[t * p.k + j0 + j] : 0.f;
      if (there) v[j].load(y + slot * p.ld_y);
      else v[j].zero();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 f = v[j].pair(q);
        s[q].x = fmaf(w[j], f.x, s[q].x);
        s[q].y = fmaf(w[j], f.y, s[q].y);
      }
  }
  const long long at = t * p.ld_out + c;
  if (p.out_type == SNN_OUT_F32) {
    float4* const out = reinterpret_cast<float4*>(static_cast<float*>(p.out) + at);
    __stcs(out, make_float4(s[0].x, s[0].y, s[1].x, s[1].y));
    __stcs(out + 1, make_float4(s[2].x, s[2].y, s[3].x, s[3].y));
  } else {
    __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + at),
           make_uint4(pack_pair(p.out_type, s[0]), pack_pair(p.out_type, s[1]), pack_pair(p.out_type, s[2]), pack_pair(p.out_type, s[3])));
  }
}

__device__ __forceinline__ float value(const void* y, int type, long long i) {
  if (type == SNN_OUT_F32) return static_cast<const float*>(y)[i];
  if (type == SNN_OUT_F16) return __half2float(static_cast<const __half*>(y)[i]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(y)[i]);
}

// The same where columns, row lengths or pointers are not multiples of 8 values: one column a thread.
__global__ void __launch_bounds__(256) combine_odd_kernel(const CombineParams p) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long t = i / p.C;
  grid_dep_wait();
  grid_dep_launch();
  const int c = (int)(i - t * p.C);
  if (t >= p.T) return;
  float s = 0.f;
  for (int j0 = 0; j0 < p.k; j0 += 4) {
    float v[4], w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int slot = j0 + j < p.k ? p.slots[t * p.k + j0 + j] : -1;
      const bool there = slot >= 0 && slot < p.y_rows;
      w[j] = there ? p.weights[t * p.k + j0 + j] : 0.f;
      v[j] = there ? value(p.y, p.y_type, slot * p.ld_y + c) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s = fmaf(w[j], v[j], s);
  }
  store_out(p.out, p.out_type, t * p.ld_out + c, s);
}

}  // namespace

long long route_work_bytes(int T, int E) {
  if (T <= RT_BLOCK) return 0;
  const long long blocks = (T + (long long)RT_BLOCK - 1) / RT_BLOCK;
  return (blocks <= RT_DIRECT ? blocks : blocks + 1) * E * 4;
}

cudaError_t route_forward(const RouteCall& c, int* launched) {
  // (no tokens: one CTA writes the offsets)
  const unsigned blocks = (unsigned)max(1ll, (c.T + (long long)RT_BLOCK - 1) / RT_BLOCK);
  const bool direct = blocks <= RT_DIRECT;
  const RouteParams p{c.logits, c.ld, c.type, c.T, c.E, c.k, c.normalise, direct, c.ids, c.weights, c.offsets, c.rows, c.slots, c.work};
  const int v = (c.E + 31) / 32, threads = 32 * min(RT_CHOOSE_WARPS, max(4, c.T));   // (few tokens: a small CTA begins sooner)
  cudaError_t e;
#define SNN_CHOOSE(V) e = launch_dependent(route_choose_kernel<V>, blocks, threads, 0, c.stream, p)
  if (v <= 1) SNN_CHOOSE(1);
  else if (v <= 2) SNN_CHOOSE(2);
  else if (v <= 4) SNN_CHOOSE(4);
  else if (v <= 8) SNN_CHOOSE(8);
  else if (v <= 16) SNN_CHOOSE(16);
  else SNN_CHOOSE(32);
#undef SNN_CHOOSE
  *launched += 1;
  if (e != cudaSuccess || blocks == 1) return e;
  if (!direct) {
    e = launch_dependent(route_sum_kernel, (unsigned)((c.E + 31) / 32), 1024, 0, c.stream, c.work, c.E, (int)blocks);
    *launched += 1;
    if (e != cudaSuccess) return e;
  }
  *launched += 1;
  return launch_dependent(route_place_kernel, blocks, RT_WARPS * 32, (size_t)c.E * 16, c.stream, p);
}

cudaError_t combine_forward(const CombineCall& c, int* launched) {
  CombineParams p{c.y, c.slots, c.weights, c.out, c.ld_y, c.ld_out, c.y_type, c.y_rows, c.T, c.k, c.C, c.out_type, c.C / 8};
  const bool eights = c.C % 8 == 0 && c.ld_y % 8 == 0 && c.ld_out % 8 == 0 && (((uintptr_t)c.y | (uintptr_t)c.out) & 15) == 0;
  const long long blocks = ((long long)c.T * (eights ? p.groups : c.C) + 255) / 256;
  if (blocks >= (1ll << 31)) return cudaErrorInvalidValue;
  *launched += 1;
  if (!eights) return launch_dependent(combine_odd_kernel, (unsigned)blocks, 256, 0, c.stream, p);
  if (c.y_type == SNN_OUT_F32) return launch_dependent(combine_kernel<float>, (unsigned)blocks, 256, 0, c.stream, p);
  if (c.y_type == SNN_OUT_F16) return launch_dependent(combine_kernel<F16>, (unsigned)blocks, 256, 0, c.stream, p);
  return launch_dependent(combine_kernel<BF16>, (unsigned)blocks, 256, 0, c.stream, p);
}

}  // namespace snn
