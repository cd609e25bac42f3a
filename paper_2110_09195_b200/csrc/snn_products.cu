// Projections of language models: rows of 16-bit activations times +1 / -1 weights, one bit each, grouped by expert.
#include "snn_products.h"

#include "snn_products.cuh"

namespace snn {
namespace {

// ---------------------------------------------------------------- layout of the weights

// One thread per word of one expert's bits (layout: snn_products.h), from the layer's bit-plane [word][channel].
__global__ void products_layout_kernel(const uint32_t* __restrict__ planes, uint32_t* __restrict__ bits, int C, int K, int n_mt, int n_kb) {
  const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (long long)n_mt * n_kb * 128) return;
  const int j = 2 * (int)(i & 1) + ((int)(i >> 3) & 1), t = (int)(i >> 1) & 3, g = (int)(i >> 4) & 7;
  const long long tile = i >> 7;
  const int kb = (int)(tile % n_kb), mt = (int)(tile / n_kb);
  const int c0 = kb * 256 + j * 64 + t * 16;
  uint32_t word = 0;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int k = mt * 16 + g + 8 * half;
    if (k >= K || c0 >= C) continue;
    uint32_t minus = ~(planes[(size_t)(c0 >> 5) * K + k] >> (c0 & 31)) & 0xffffu;
    if (C - c0 < 16) minus &= (1u << (C - c0)) - 1u;
#pragma unroll
    for (int p = 0; p < 8; ++p) word |= (((minus >> (2 * p)) & 1u) | (((minus >> (2 * p + 1)) & 1u) << 16)) << (p + 8 * half);
  }
  bits[i] = word;
}

// ---------------------------------------------------------------- few rows

struct SmallParams {
  const uint32_t* bits;
  const float* alpha;
  const void* act;
  const int32_t *rows, *offsets;
  void* out;
  long long ld_act, ld_out;
  int act_rows, max_rows, E, C, K, n_mt, n_kb, out_type, k_warps;
  Lowrank low;
};

// The chunk-th piece of at most `most` rows, counted over the experts in their order: expert, first row, rows.  Found by each warp for
// itself: every lane counts the pieces of a run of experts, a scan over the lanes says whose run holds it.
__device__ __forceinline__ bool find_chunk(const int32_t* offsets, int E, int R, int most, int chunk, int* e_out, int* r_out, int* n_out) {
  const int lane = threadIdx.x & 31;
  if (!offsets) {
    *e_out = 0;
    *r_out = chunk * most;
    *n_out = min(most, R - chunk * most);
    return *n_out > 0;
  }
  const int per = (E + 31) >> 5, e0 = lane * per, e1 = min(E, e0 + per);
  int count = 0;
  for (int e = e0; e < e1; ++e) {
    const int lo = clamp_offset(offsets[e], R), hi = clamp_offset(offsets[e + 1], R);
    count += (max(hi - lo, 0) + most - 1) / most;
  }
  int upto = count;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += v;
  }
  const unsigned who = __ballot_sync(0xffffffffu, chunk < upto);
  if (!who) return false;
  const int src = __ffs(who) - 1;
  int e = 0, r = 0, n = 0;
  if (lane == src) {
    int left = chunk - (upto - count);
    for (e = e0; e < e1; ++e) {
      const int lo = clamp_offset(offsets[e], R), hi = clamp_offset(offsets[e + 1], R);
      const int pieces = (max(hi - lo, 0) + most - 1) / most;
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
  return true;
}

// A warp computes 32 output channels times 8 NT rows over a share of the input channels: the weights, the M operand, are expanded from
// bits in registers, the rows, the N operand, come straight from memory as the instruction wants them (a lane's 16 neighbouring
// channels are four steps' operands).  The warps of a CTA take different input channels (k_warps of them) and different output
// channels; the former's sums meet in shared memory.
template <class T, int NT>
__global__ void __launch_bounds__(256) products_small_kernel(const SmallParams p) {
  constexpr int N = 8 * NT;
  __shared__ float red[8][N][33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kw = warp % p.k_warps, mw = warp / p.k_warps, m_warps = 8 / p.k_warps;
  int e, r0, n;
  if (!find_chunk(p.offsets, p.E, p.max_rows, N, (int)blockIdx.x, &e, &r0, &n)) return;
  const uint16_t* x[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int c = 8 * i + g;
    x[i] = nullptr;
    if (c < n) {
      const int row = p.rows ? p.rows[r0 + c] : r0 + c;
      if (row >= 0 && row < p.act_rows) x[i] = static_cast<const uint16_t*>(p.act) + (size_t)row * (size_t)p.ld_act;
    }
  }
  const int mt = 2 * ((int)blockIdx.y * m_warps + mw);
  float acc[2][NT][4] = {};
  if (mt < p.n_mt) {
    const uint2* w0 = reinterpret_cast<const uint2*>(p.bits) + ((size_t)(e * p.n_mt + mt) * p.n_kb) * 64 + 8 * g + t;
    const uint2* w1 = w0 + (size_t)p.n_kb * 64;
    for (int kb = kw; kb < p.n_kb; kb += p.k_warps) {
      const uint2 ue = ld8(w0 + (size_t)kb * 64), uo = ld8(w0 + (size_t)kb * 64 + 4);
      const uint2 ve = ld8(w1 + (size_t)kb * 64), vo = ld8(w1 + (size_t)kb * 64 + 4);
      const uint32_t ua[4] = {ue.x, uo.x, ue.y, uo.y}, ub[4] = {ve.x, vo.x, ve.y, vo.y};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = kb * 256 + j * 64 + t * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4 b[NT];
#pragma unroll
          for (int i = 0; i < NT; ++i) b[i] = x[i] && c + 8 * h < p.C ? ld16(x[i] + c + 8 * h) : make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int s = 2 * h + q;
            const uint32_t a0 = plus_minus<T>(ua[j], 15 - 2 * s), a2 = plus_minus<T>(ua[j], 14 - 2 * s);
            const uint32_t a1 = plus_minus<T>(ua[j], 7 - 2 * s), a3 = plus_minus<T>(ua[j], 6 - 2 * s);
            const uint32_t c0 = plus_minus<T>(ub[j], 15 - 2 * s), c2 = plus_minus<T>(ub[j], 14 - 2 * s);
            const uint32_t c1 = plus_minus<T>(ub[j], 7 - 2 * s), c3 = plus_minus<T>(ub[j], 6 - 2 * s);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
              const uint32_t b0 = q ? b[i].z : b[i].x, b1 = q ? b[i].w : b[i].y;
              mma_16x8<T>(acc[0][i], a0, a1, a2, a3, b0, b1);
              mma_16x8<T>(acc[1][i], c0, c1, c2, c3, b0, b1);
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) red[warp][8 * i + 2 * t + (q & 1)][16 * m + g + 8 * (q >> 1)] = acc[m][i][q];
  __syncthreads();
  const int width = 32 * m_warps, first = (int)blockIdx.y * width;
  for (int i = threadIdx.x; i < n * width; i += 256) {
    const int c = i / width, m = i % width, co = first + m;
    if (co >= p.K) continue;
    float s = 0.f;
    for (int k = 0; k < p.k_warps; ++k) s += red[(m >> 5) * p.k_warps + k][c][m & 31];
    float v = p.alpha[(size_t)e * p.n_mt * 16 + co] * s;
    if (p.low.adapter) v += lowrank_term<T>(p.low, p.K, r0 + c, co);
    store_out(p.out, p.out_type, (long long)(r0 + c) * p.ld_out + co, v);
  }
}

template <class T, int NT>
cudaError_t small_launch(const Products& p, const ProductCall& c, int* launched) {
  SmallParams q{p.bits, p.alpha, c.act, c.rows, c.offsets, c.out, c.ld_act, c.ld_out, c.act_rows, c.max_rows, p.E, p.C, p.K, p.n_mt, p.n_kb,
                c.out_type, 1, c.low};
  const int most = 8 * NT;
  const long long chunks = c.offsets ? ((long long)c.max_rows + (long long)min(p.E, c.max_rows) * (most - 1)) / most : (c.max_rows + most - 1) / most;
  // all warps on one strip of output channels until that gives every SM a CTA or the input channels are used up
  const int strips = (p.K + 31) / 32;
  int k_warps = 8;
  while (k_warps > 1 && (k_warps > p.n_kb || chunks * ((strips + 16 / k_warps - 1) / (16 / k_warps)) >= 4ll * sm_count())) k_warps /= 2;
  q.k_warps = k_warps;
  const int m_warps = 8 / k_warps;
  products_small_kernel<T, NT><<<dim3((unsigned)chunks, (unsigned)((strips + m_warps - 1) / m_warps)), 256, 0, c.stream>>>(q);
  *launched += 1;
  return cudaGetLastError();
}

template <class T>
cudaError_t small_forward(const Products& p, const ProductCall& c, int* launched) {
  const int per_expert = c.offsets ? c.max_rows / max(1, min(p.E, c.max_rows)) : c.max_rows;
  if (per_expert <= 6) return small_launch<T, 1>(p, c, launched);
  if (per_expert <= 12) return small_launch<T, 2>(p, c, launched);
  return small_launch<T, 4>(p, c, launched);
}

}  // namespace

cudaError_t products_create(const LayerDev* const* layers, int E, int C, int K, cudaStream_t s, Products* p, int* launched) {
  p->E = E;
  p->C = C;
  p->K = K;
  p->n_mt = (K + 255) / 256 * 16;
  p->n_kb = (C + 255) / 256;
  const size_t words = (size_t)p->n_mt * p->n_kb * 128, rows = (size_t)p->n_mt * 16;
  cudaError_t e = cudaMalloc((void**)&p->bits, words * 4 * E);
  if (e == cudaSuccess) e = cudaMalloc((void**)&p->alpha, rows * 4 * E);
  if (e == cudaSuccess) e = cudaHostAlloc((void**)&p->status_host, sizeof(int), cudaHostAllocMapped);
  if (e == cudaSuccess) {
    *p->status_host = 0;
    e = cudaHostGetDevicePointer((void**)&p->status_dev, p->status_host, 0);
  }
  if (e == cudaSuccess) e = cudaMemsetAsync(p->alpha, 0, rows * 4 * E, s);
  for (int i = 0; i < E && e == cudaSuccess; ++i) {
    products_layout_kernel<<<(unsigned)((words + 255) / 256), 256, 0, s>>>(layers[i]->wplanes, p->bits + words * i, C, K, p->n_mt, p->n_kb);
    *launched += 1;
    e = cudaGetLastError();
    if (e == cudaSuccess) e = cudaMemcpyAsync(p->alpha + rows * i, layers[i]->alpha, (size_t)K * 4, cudaMemcpyDeviceToDevice, s);
  }
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  return e;
}

void products_destroy(Products* p) {
  cudaFree(p->bits);
  cudaFree(p->alpha);
  if (p->status_host) cudaFreeHost(p->status_host);
}

cudaError_t products_forward(const Products& p, const ProductCall& c, int* launched) {
  const int per_expert = c.offsets ? c.max_rows / max(1, min(p.E, c.max_rows)) : c.max_rows;
  if (per_expert >= 48 && c.act_rows > 0) return products_tall(p, c, launched);
  return c.act_type == SNN_ACT_F16 ? small_forward<F16>(p, c, launched) : small_forward<BF16>(p, c, launched);
}

}  // namespace snn
