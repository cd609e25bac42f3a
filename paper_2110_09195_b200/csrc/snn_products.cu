// Projections of language models: rows of 16-bit activations times +1 / -1 weights, one bit each, grouped by expert.
#include <cstdlib>
#include <cstring>

#include "snn_products.h"

#include "snn_products.cuh"
#include "snn_tc_common.cuh"

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
  uint32_t word = 0;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int k = mt * 16 + g + 8 * half;
    if (k >= K) continue;
    uint32_t minus = 0;   // (channels come in eights)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int c = kb * 256 + j * 64 + 32 * q + 8 * t;
      if (c < C) minus |= (~(planes[(size_t)(c >> 5) * K + k] >> (8 * t)) & 0xffu) << (8 * q);
    }
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
  Powers pow;
};

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

// A warp computes 32 MP output channels times 8 rows over a share of the input channels: the weights, the M operand, are expanded from
// bits in registers, the rows, the N operand, come straight from memory as the instruction wants them (a lane's 16
// channels are four steps' operands) and stay in registers for all of the warp's output channels (loaded for every 32 of them, they took
// as many cycles of the L1 cache as the rest).  The warps of a CTA take different input channels (k_warps of them) and different output
// channels; the former's sums meet in shared memory.  The work, pieces of rows times strips of output channels, is counted on the device and
// shared out evenly: a CTA has a run of strips, mostly of one piece.  Bound by latency where there are few weights, else mostly by the
// expansion: 16 masks and 15 multiplications, at half rate each, for four of the instructions (64 tokens over 64 experts of 2048 x 2048, 4
// each, 31 us: 52 % of the issue slots and 47 % of the integer units used, none of them full; the rest is waits, a barrier and a sum over the warps for
// each strip among them).  With adapters of many rows the second term is more than all else: a row's adapter, then its B, eight of the rank at a time
// one behind the other (419 rows of 400 x 1912, rank 32, runs of 2 rows 42 us, 9 where no row has an adapter).  16 rows a warp were no faster for any number of rows (16 experts of 4096 x 4096, 128 rows: 47 us
// against 41, 256 rows: 76 against 65).
constexpr int SM_N = 8;
template <class T, int MP>
__global__ void __launch_bounds__(256, 2) products_small_kernel(const SmallParams p) {
  constexpr int M = 32 * MP;
  __shared__ float red_both[2][8][SM_N][M + 1];
  int turn = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kw = warp % p.k_warps, mw = warp / p.k_warps, m_warps = 8 / p.k_warps, n_groups = (p.K + M * m_warps - 1) / (M * m_warps);
  // The kernel before may be the one that writes A x: it has waited for what came before it, and so for the rows and all else that is read
  // or overwritten here.  Else this waits for whatever came before.
  if (!p.low.adapter) grid_dep_wait();
  const Powers pow = in_registers(p.pow);
  const Pieces pieces = count_pieces(p.offsets, p.E, p.max_rows, SM_N);
  const long long items = (long long)pieces.total * n_groups;
  long long item = items * blockIdx.x / gridDim.x;
  const long long last = items * (blockIdx.x + 1) / gridDim.x;
  bool waited = !p.low.adapter;
  grid_dep_launch();
  while (item < last) {
    const int piece = (int)(item / n_groups), group0 = (int)(item - (long long)piece * n_groups);
    const int group1 = (int)min((long long)n_groups, group0 + (last - item));
    item += group1 - group0;
    int e, r0, n;
    find_piece(pieces, p.offsets, p.E, p.max_rows, SM_N, piece, &e, &r0, &n);
    const uint16_t* x = nullptr;
    if (g < n) {
      const int row = p.rows ? p.rows[r0 + g] : r0 + g;
      if (row >= 0 && row < p.act_rows) x = static_cast<const uint16_t*>(p.act) + (size_t)row * (size_t)p.ld_act + 8 * t;
    }
    const uint2* const bits = reinterpret_cast<const uint2*>(p.bits) + (size_t)e * p.n_mt * p.n_kb * 64 + 8 * g + t;
    uint2 w[2][2];   // [tile][odd blocks of 64]
    auto load_bits = [&](int group, int pair, int kb) {
      // (tiles behind the last: the sums of the last pair there is, which nobody writes)
      const int mt = min(2 * MP * (group * m_warps + mw) + 2 * pair, p.n_mt - 2);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int o = 0; o < 2; ++o) w[m][o] = ld8(bits + ((size_t)(mt + m) * p.n_kb + kb) * 64 + 4 * o);
    };
    uint4 b[4][2];
    auto load_rows = [&](int kb) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int c = kb * 256 + j * 64 + 32 * h;
          b[j][h] = x && c + 8 * t < p.C ? ld16(x + c) : make_uint4(0, 0, 0, 0);
        }
    };
    if (kw < p.n_kb) {   // (few items: some warps only help with the outputs)
      load_bits(group0, 0, kw);
      load_rows(kw);
    }
    for (int group = group0; group < group1; ++group) {
      float acc[2 * MP][4] = {};
      for (int kb = kw; kb < p.n_kb; kb += p.k_warps) {
        const bool last_kb = kb + p.k_warps >= p.n_kb;
#pragma unroll
        for (int pair = 0; pair < MP; ++pair) {
          const uint32_t u[2][4] = {{w[0][0].x, w[0][1].x, w[0][0].y, w[0][1].y}, {w[1][0].x, w[1][1].x, w[1][0].y, w[1][1].y}};
          if (pair + 1 < MP) load_bits(group, pair + 1, kb);
          else if (!last_kb) load_bits(group, 0, kb + p.k_warps);
          else if (group + 1 < group1) load_bits(group + 1, 0, kw);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
              const uint4& v = b[j][s >> 1];
#pragma unroll
              for (int m = 0; m < 2; ++m) {
                const uint32_t a0 = plus_minus<T>(u[m][j], 15 - 2 * s, pow), a1 = plus_minus<T>(u[m][j], 7 - 2 * s, pow);
                const uint32_t a2 = plus_minus<T>(u[m][j], 14 - 2 * s, pow), a3 = plus_minus<T>(u[m][j], 6 - 2 * s, pow);
                mma_16x8<T>(acc[2 * pair + m], a0, a1, a2, a3, s & 1 ? v.z : v.x, s & 1 ? v.w : v.y);
              }
            }
        }
        // the next input channels', or, before the sums meet, the next strip's
        if (!last_kb) load_rows(kb + p.k_warps);
        else if (group + 1 < group1 && p.n_kb > p.k_warps) load_rows(kw);
      }
      float (*const red)[SM_N][M + 1] = red_both[turn];
      turn ^= 1;
#pragma unroll
      for (int m = 0; m < 2 * MP; ++m)
#pragma unroll
        for (int q = 0; q < 4; ++q) red[warp][2 * t + (q & 1)][16 * m + g + 8 * (q >> 1)] = acc[m][q];
      __syncthreads();   // (the other half of the buffer is for the next strip)
      if (!waited) grid_dep_wait();
      waited = true;
      // a thread has a channel (or two), and every 256 / width-th row
      const int width = M * m_warps, columns = min(width, 256), first = group * width;
      for (int m = (int)threadIdx.x & (columns - 1); m < width; m += 256) {
        const int co = first + m;
        if (co >= p.K) break;
        const float alpha = p.alpha[(size_t)e * p.n_mt * 16 + co];
#pragma unroll 2
        for (int c = (int)threadIdx.x / columns; c < n; c += 256 / columns) {
          float s = 0.f;
          for (int k = 0; k < p.k_warps; ++k) s += red[(m / M) * p.k_warps + k][c][m % M];
          float v = alpha * s;
          if (p.low.adapter) v += lowrank_term<T>(p.low, p.K, r0 + c, co);
          store_out(p.out, p.out_type, (long long)(r0 + c) * p.ld_out + co, v);
        }
      }
    }
  }
  if (!waited) grid_dep_wait();   // (no CTA ends before what came before has)
}

// Pieces of 8 rows that the experts have at most (the host does not know how the rows are spread).
long long most_pieces(const Products& p, const ProductCall& c) {
  return c.offsets ? ((long long)c.max_rows + (long long)min(p.E, c.max_rows) * (SM_N - 1)) / SM_N : (c.max_rows + SM_N - 1) / SM_N;
}

template <class T, int MP>
cudaError_t small_launch(const Products& p, const ProductCall& c, int k_warps, unsigned ctas, int* launched) {
  const SmallParams q{p.bits, p.alpha, c.act, c.rows, c.offsets, c.out, c.ld_act, c.ld_out, c.act_rows, c.max_rows, p.E, p.C, p.K, p.n_mt, p.n_kb,
                      c.out_type, k_warps, c.low, powers()};
  *launched += 1;
  return launch_dependent(products_small_kernel<T, MP>, ctas, 256, 0, c.stream, q);
}

template <class T>
cudaError_t small_forward(const Products& p, const ProductCall& c, int* launched) {
  // all warps on one strip of output channels, unless there are not so many blocks of 256 input channels, and more strips than CTAs (the warps that have
  // no input channels still help with the outputs: 40 rows of 584 x 130 with adapters of rank 64 6.5 us, with two warps for each block 12.8; 33
  // rows of 368 x 91 and rank 8 4.6 and 6.9)
  const long long ctas = 2ll * sm_count(), pieces = most_pieces(p, c);
  int k_warps = 8;
  while (k_warps > p.n_kb && pieces * ((p.K + 8 / k_warps * 32 - 1) / (8 / k_warps * 32)) > ctas) k_warps /= 2;
  // 32 or 64 output channels a warp: a strip of 64 takes 1.86 times as long as one of 32, and what counts is how many of them a CTA has one
  // after the other (one expert of 4096 x 4096: 16 rows 6.7 us with 32, 32 rows 10.5 and 9.8, 48 rows 14.2 and 16.3, 64 rows 17.7 and
  // 16.4; 64 tokens over 64 experts of 2048 x 2048 39 and 33)
  auto items = [&](int m) { return pieces * ((p.K + 8 / k_warps * m - 1) / (8 / k_warps * m)); };
  auto turns = [&](int m) { return (items(m) + ctas - 1) / ctas; };
  if (186 * turns(64) <= 100 * turns(32)) return small_launch<T, 2>(p, c, k_warps, (unsigned)min(ctas, items(64)), launched);
  return small_launch<T, 1>(p, c, k_warps, (unsigned)min(ctas, items(32)), launched);
}

// Which kernel, by the time that each would take on 148 SMs (us).  Few rows: each piece of 8 expands all of its expert's weights, 11 G
// weights a ms, and with few input channels each strip of outputs takes a time of its own.  Many rows: tiles of 256 output channels in turns of a
// tile for each pair of SMs, 0.16 to 0.24 us for 64 input channels, whatever the number of rows up to 192.  (140 calls of drawn sizes took 0.8 %
// longer than with the better kernel for each, geometric mean.  The worst: 419 rows of 400 x 1912, 16 adapters of rank 32 in runs of 2 rows, 42.0 us by
// the kernel taken, few rows, and 26.5 by the other; 2860 rows of 160 x 253 with one adapter of rank 8, 20.2 and 14.1; the other 138 at most
// 13 % longer.  The number of adapters is not used, nor is the time of their first factor.  Measured both ways: one expert of 4096 x 4096, 32 rows 9.8 and 15.6 us, 64 rows 15 and 16; 16
// of them, 128 rows 41 and 51, 256 rows 65 and 51; 64 of 2048 x 2048, 512 rows 48 and 53, 1024 rows 78 and 54.  With adapters the
// time of many rows depends on how many adapters the rows of a tile have, which the host does not know: 16 adapters on 4096 x 4096, requests of
// 50 rows, rank 16, 64 rows 22 and 21, 128 rows 37 and 25, rank 64 31 and 26, 56 and 35; an adapter for each row, rank 16 21 and 30, 36 and 35,
// rank 64 31 and 56, 55 and 69.)
// SNN_FORCE_ROWS=few or many in the environment takes one of them wherever it can run.
bool many_rows(const Products& p, const ProductCall& c) {
  if (c.act_rows < 1) return false;   // (no tensor to describe)
  if (const char* f = getenv("SNN_FORCE_ROWS")) {
    if (!strcmp(f, "few")) return false;
    if (!strcmp(f, "many")) return true;
  }
  const double pairs = sm_count() / 2.0, used = c.offsets ? min(p.E, c.max_rows) : 1, blocks = (p.C + 63) / 64, rows = fmin(192.0, c.max_rows / used);
  double few = 3.0 + (c.max_rows / 8.0 + (c.offsets ? 0.5 * used : 0.5)) * p.K * (double)p.C / 11e6;
  if (p.n_kb < 8) few += 3.0 * (1 - p.n_kb / 8.0) * (c.max_rows / 8.0) * ((p.K + 255) / 256) / (2 * sm_count());
  const double tiles = (c.max_rows < 192 * used ? used : c.max_rows / 192.0) * ((p.K + 255) / 256);
  double many = 5.5 + blocks * (tiles <= pairs ? 0.16 + 0.0002 * rows : tiles / pairs * (0.2 + 0.0002 * rows));
  if (c.low.adapter) {
    few += 8.5e-7 * c.max_rows * c.low.rank * p.K;
    many += 2.0 + (0.02 + (4.2e-4 + 5.5e-7 * p.C) * c.low.rank) * rows;
  }
  return many < few;
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
  if (many_rows(p, c)) return products_tall(p, c, launched);
  return c.act_type == SNN_ACT_F16 ? small_forward<F16>(p, c, launched) : small_forward<BF16>(p, c, launched);
}

}  // namespace snn
