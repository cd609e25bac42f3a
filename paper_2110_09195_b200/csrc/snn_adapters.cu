// Low-rank adapters beside a projection: the first factor, h = scale * (A x), for rows of many requests.
#include "snn_products.h"

#include "snn_products.cuh"
#include "snn_tc_common.cuh"

namespace snn {
namespace {

struct ShrinkParams {
  const uint16_t *act, *a;
  const int32_t* adapter;
  const float* scale;
  float* h;
  long long ld_act;
  int rows, C, n, rank, per_cta;
};

// A CTA takes up to 8 NT neighbouring rows and 16 MT of the rank; its warps take different input channels, and their sums meet in shared
// memory.  One pass for each adapter that the rows have (rows of one request lie together: mostly one); the rows of other adapters are
// computed along and not written.  The CTAs of a column of the grid have the same rows and take their adapters in turn: mostly only the first has
// any, and where two requests meet neither CTA takes twice as long as the rest (4096 rows of 4096, rank 32: 17.7 us, with one CTA after the other 25.3).
// Bound by reading A and x, each CTA both, mostly from L2 and 16 bytes a lane at a time.
template <class T, int NT, int MT, int U, int WARPS>
__global__ void __launch_bounds__(32 * WARPS) shrink_kernel(const ShrinkParams p) {
  constexpr int N = 8 * NT, M = 16 * MT;
  extern __shared__ float red_raw[];
  float (*const red)[N][M + 1] = reinterpret_cast<float (*)[N][M + 1]>(red_raw);   // [WARPS]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int r0 = (int)blockIdx.x * p.per_cta, n = min(p.per_cta, p.rows - r0), j0 = (int)blockIdx.y * M;
  grid_dep_wait();
  grid_dep_launch();   // (the projection's kernel begins with its own sums; it waits for these before it adds them)
  // (each warp for itself: lane i has row i's adapter, and a bit for each adapter's first row)
  int who = lane < n ? p.adapter[r0 + lane] : -1;
  if (who < 0 || who >= p.n) who = -1;
  const unsigned like_me = __match_any_sync(0xffffffffu, who);
  unsigned todo = __ballot_sync(0xffffffffu, who >= 0 && (int)__ffs(like_me) - 1 == lane);
  const uint16_t* x[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) x[i] = 8 * i + g < n ? p.act + (size_t)(r0 + 8 * i + g) * (size_t)p.ld_act + 8 * t : nullptr;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  for (int pass = 0; todo; ++pass) {
    if (pass % (int)gridDim.z != (int)blockIdx.z) {
      todo &= todo - 1;
      continue;
    }
    const int c = __ffs(todo) - 1, a = __shfl_sync(0xffffffffu, who, c);
    const unsigned same = __shfl_sync(0xffffffffu, like_me, c);
    todo &= todo - 1;
    const uint16_t* w[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) w[i] = j0 + 8 * i < p.rank ? p.a + ((size_t)a * p.rank + j0 + 8 * i + g) * p.C + 8 * t : nullptr;
    float acc[MT][NT][4] = {};
    // U blocks of 64 input channels on their way, then their products
    for (int k0 = warp * 64; k0 < p.C; k0 += 64 * WARPS * U) {
      uint4 b[U][NT][2], u[U][2 * MT][2];
#pragma unroll
      for (int v = 0; v < U; ++v)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = k0 + 64 * WARPS * v + 32 * h;
          const bool in = k + 8 * t < p.C;
#pragma unroll
          for (int i = 0; i < 2 * MT; ++i) u[v][i][h] = in && w[i] ? ld16(w[i] + k) : zero;
#pragma unroll
          for (int i = 0; i < NT; ++i) b[v][i][h] = in && x[i] ? ld16(x[i] + k) : zero;
        }
#pragma unroll
      for (int v = 0; v < U; ++v)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const uint4 &lo = u[v][2 * m][h], &hi = u[v][2 * m + 1][h], &r = b[v][i][h];
              mma_16x8<T>(acc[m][i], lo.x, hi.x, lo.y, hi.y, r.x, r.y);
              mma_16x8<T>(acc[m][i], lo.z, hi.z, lo.w, hi.w, r.z, r.w);
            }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) red[warp][8 * i + 2 * t + (q & 1)][16 * m + g + 8 * (q >> 1)] = acc[m][i][q];
    __syncthreads();
    for (int i = threadIdx.x; i < n * M; i += 32 * WARPS) {
      const int row = i / M, j = i % M;
      if (!((same >> row) & 1u) || j0 + j >= p.rank) continue;
      float s = 0.f;
#pragma unroll
      for (int v = 0; v < WARPS; ++v) s += red[v][row][j];
      p.h[(size_t)(r0 + row) * p.rank + j0 + j] = p.scale[a] * s;
    }
    __syncthreads();
  }
}

constexpr unsigned SH_TURNS = 4;

template <class T, int NT, int MT, int U, int WARPS>
cudaError_t shrink_launch(const ShrinkParams& p, cudaStream_t s) {
  static unsigned long long done = 0;
  const cudaError_t e = allow_max_smem(shrink_kernel<T, NT, MT, U, WARPS>, &done);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)((p.rows + p.per_cta - 1) / p.per_cta), (unsigned)((p.rank + 16 * MT - 1) / (16 * MT)), NT > 1 ? SH_TURNS : 1u);
  return launch_dependent(shrink_kernel<T, NT, MT, U, WARPS>, grid, 32 * WARPS, (size_t)WARPS * 8 * NT * (16 * MT + 1) * 4, s, p);
}

// How many rows and how much of the rank a CTA takes: the more, the less is read again; as long as there are CTAs for all SMs, so one row up to
// two for each SM.  (4096 rows of 4096 values, rank 64: 16 of the rank and 32 rows 36 us, 32 and 32 30 us, 64 and 32 26 us; 1000 rows: 16 and 6
// 19 us, 32 and 16 13 us, 16 and 32 16 us; 500 rows: 16 and 3 14.4 us, 32 and 16 8.5 us; rank 16 and 4096 rows, two blocks of input channels on their way 13.7 us,
// one 14.6.)
template <class T>
cudaError_t shrink_type(ShrinkParams p, cudaStream_t s) {
  const int sms = sm_count();
  if (p.rows >= 16 * sms) {
    p.per_cta = 32;
    if (p.rank > 32) return shrink_launch<T, 4, 4, 1, 8>(p, s);
    return p.rank > 16 ? shrink_launch<T, 4, 2, 1, 16>(p, s) : shrink_launch<T, 4, 1, 2, 16>(p, s);
  }
  if (p.rows >= 2 * sms) {
    p.per_cta = 16;
    return shrink_launch<T, 2, 2, 1, 16>(p, s);
  }
  p.per_cta = 1;   // (a CTA for each row still is less than two for each SM; its row is one of the instruction's eight columns)
  return shrink_launch<T, 1, 1, 4, 8>(p, s);
}

}  // namespace

cudaError_t shrink_forward(const ShrinkCall& c, int* launched) {
  const ShrinkParams p{static_cast<const uint16_t*>(c.act), static_cast<const uint16_t*>(c.a), c.adapter, c.scale, c.h, c.ld_act, c.rows, c.C, c.n, c.rank, 8};
  *launched += 1;
  return c.act_type == SNN_ACT_F16 ? shrink_type<F16>(p, c.stream) : shrink_type<BF16>(p, c.stream);
}

}  // namespace snn
