// Low-rank adapters beside a projection: the first factor, h = scale * (A x), for rows of many requests.
#include "snn_products.h"

#include "snn_products.cuh"

namespace snn {
namespace {

struct ShrinkParams {
  const uint16_t *act, *a;
  const int32_t* adapter;
  const float* scale;
  float* h;
  long long ld_act;
  int rows, C, n, rank;
};

// A CTA takes 8 neighbouring rows and 16 of the rank; its warps take different input channels, and their sums meet in shared
// memory.  One pass for each adapter that the rows have (rows of one request lie together: mostly one); the rows of other adapters are
// computed along and not written, since the instruction has 8 columns in any case.
template <class T>
__global__ void __launch_bounds__(256) shrink_kernel(const ShrinkParams p) {
  __shared__ float red[8][8][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int r0 = (int)blockIdx.x * 8, j0 = (int)blockIdx.y * 16;
  const int mine = r0 + g < p.rows ? p.adapter[r0 + g] : -1;   // of row g
  const uint16_t* x = p.act + (size_t)min(r0 + g, p.rows - 1) * (size_t)p.ld_act;
  for (int c = 0; c < 8; ++c) {
    const int a = __shfl_sync(0xffffffffu, mine, 4 * c);
    const unsigned same = __ballot_sync(0xffffffffu, mine == a);
    if (a < 0 || a >= p.n || (same & ((1u << (4 * c)) - 1u))) continue;   // none, or seen before
    const uint16_t* w0 = p.a + ((size_t)a * p.rank + j0 + g) * p.C;
    const uint16_t* w1 = w0 + (size_t)8 * p.C;
    const bool two = j0 + 8 < p.rank;
    float acc[4] = {};
    for (int k = warp * 64; k < p.C; k += 512) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = k + 16 * t + 8 * h;
        const bool in = i < p.C;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        const uint4 u = in ? ld16(w0 + i) : zero, v = in && two ? ld16(w1 + i) : zero, b = in ? ld16(x + i) : zero;
        mma_16x8<T>(acc, u.x, v.x, u.y, v.y, b.x, b.y);
        mma_16x8<T>(acc, u.z, v.z, u.w, v.w, b.z, b.w);
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) red[warp][2 * t + (q & 1)][g + 8 * (q >> 1)] = acc[q];
    __syncthreads();
    if (threadIdx.x < 128) {
      const int row = threadIdx.x >> 4, j = threadIdx.x & 15;
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) s += red[w][row][j];
      if ((same >> (4 * row)) & 1u && j0 + j < p.rank) p.h[(size_t)(r0 + row) * p.rank + j0 + j] = p.scale[a] * s;
    }
    __syncthreads();
  }
}

}  // namespace

cudaError_t shrink_forward(const ShrinkCall& c, int* launched) {
  const ShrinkParams p{static_cast<const uint16_t*>(c.act), static_cast<const uint16_t*>(c.a), c.adapter, c.scale, c.h, c.ld_act, c.rows, c.C, c.n, c.rank};
  const dim3 grid((unsigned)((c.rows + 7) / 8), (unsigned)((c.rank + 15) / 16));
  if (c.act_type == SNN_ACT_F16) shrink_kernel<F16><<<grid, 256, 0, c.stream>>>(p);
  else shrink_kernel<BF16><<<grid, 256, 0, c.stream>>>(p);
  *launched += 1;
  return cudaGetLastError();
}

}  // namespace snn
