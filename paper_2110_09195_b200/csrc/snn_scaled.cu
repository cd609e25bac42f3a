// Projections in 8-bit floating point with a scale for each block of 128: layout of the weights, and the kernel for few rows.
#include <cmath>
#include <cstdlib>
#include <cstring>

#include "snn_products.h"

#include "snn_products.cuh"
#include "snn_tc_common.cuh"

namespace snn {
namespace {

// ---------------------------------------------------------------- layout of the weights

// One thread per 16 bytes of the tiles (layout: snn_products.h).
__global__ void scaled_layout_kernel(const uint8_t* __restrict__ weights, uint4* __restrict__ tiles, int C, int K, int n_kt, int n_kb, long long pieces) {
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < pieces; i += (long long)gridDim.x * blockDim.x) {
    const int piece = (int)(i & 7), r = (int)(i >> 3) & 127;
    const long long tile = i >> 10;
    const int kb = (int)(tile % n_kb), kt = (int)(tile / n_kb % n_kt);
    const long long e = tile / n_kb / n_kt;
    const int k = kt * 128 + r, c = kb * 128 + piece * 16;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (k < K && c < C) v = *reinterpret_cast<const uint4*>(weights + ((size_t)e * K + k) * C + c);
    tiles[(tile << 10) + (r << 3) + (piece ^ (r & 7))] = v;
  }
}

// ---------------------------------------------------------------- few rows

struct FewParams {
  const uint8_t *tiles, *act;
  const float *w_scales, *x_scales;
  const int32_t* offsets;
  void* out;
  long long ld_act, ld_scales, ld_out;
  int rows, E, C, K, n_kt, n_kb, out_type, k_warps;
  int* status;
};

// D[16 x 8] += A[16 x 32] B[32 x 8] of e4m3 values, fp32 sums; g = lane / 4, t = lane % 4: a = rows g, g + 8, g, g + 8 at k = 4t, 4t, 4t + 16,
// 4t + 16, four each; b = column g at k = 4t, 4t + 16; d as of mma_16x8.
__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float ld_float(const float* p) {
  float v;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}

// A warp computes 16 output channels, the M operand, times 8 NT rows over its share of the blocks of 128 input channels; the warps' sums meet in shared
// memory.  Bound by reading the weights, once: each warp has a ring of blocks (16 channels x 128 bytes, 2 KB and one bulk copy each) that are on their way
// across the ends of strips and pieces, so that no sum, barrier or output stops the reading.  The rows come straight from memory, 16 bytes a
// lane (the order of k within a block is free as long as both operands have the same), the next block's while this one is multiplied.  Lane group g has
// channel 4 (g mod 2) + g / 2 of eight: the 16-byte pieces that eight lanes read at a time then lie in different banks.  One row of 4096 x 4096 5.0 us (3.4 TB/s),
// of 4096 x 8192 9.1 (3.7): the latencies of a launch and of the first block, then the reading.
constexpr int SC_BLOCK = 2048;
template <int NT>
struct FewShape {
  static constexpr int kRows = 8 * NT;
  static constexpr int kDepth = NT == 1 ? 6 : NT == 2 ? 5 : 4;   // blocks on their way for each warp, so that two CTAs fit
  static constexpr int kRing = 8 * kDepth * SC_BLOCK, kRed = 2 * 8 * kRows * 17 * 4;
  static constexpr int kBytes = 128 + kRing + kRed + 8 * kDepth * 8;
};
template <int NT>
__global__ void __launch_bounds__(256, 2) scaled_few_kernel(const FewParams p) {
  using S = FewShape<NT>;
  constexpr int N = S::kRows, DEPTH = S::kDepth;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
  float (*const red_both)[8][N][17] = reinterpret_cast<float (*)[8][N][17]>(smem + S::kRing);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kw = warp % p.k_warps, mw = warp / p.k_warps, m_warps = 8 / p.k_warps, n_groups = (p.K + 16 * m_warps - 1) / (16 * m_warps);
  const uint32_t ring = smem_u32(smem) + warp * DEPTH * SC_BLOCK, bars = smem_u32(smem + S::kRing + S::kRed) + warp * DEPTH * 8;
  if (lane < DEPTH) mbar_init(bars + 8 * lane, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  fence_proxy_async();
  __syncwarp();
  if (p.offsets) grid_dep_wait();   // (else the weights, which nobody writes, may come while the kernel before ends)
  const Pieces pieces = count_pieces(p.offsets, p.E, p.rows, N);
  const long long items = (long long)pieces.total * n_groups;
  const long long first = items * blockIdx.x / gridDim.x, last = items * (blockIdx.x + 1) / gridDim.x;

  // the next block to ask for
  struct Next {
    long long item;
    int piece, group, kb, e;
  } next{first, (int)(first / n_groups), (int)(first % n_groups), kw, 0};
  bool more = first < last && kw < p.n_kb, ok = true;
  int r_unused, n_unused;
  if (more) find_piece(pieces, p.offsets, p.E, p.rows, N, next.piece, &next.e, &r_unused, &n_unused);
  int issued = 0, taken = 0;
  auto issue = [&] {
    const int slot = issued % DEPTH, strip = min(next.group * m_warps + mw, p.n_kt * 8 - 1);
    if (lane == 0) {
      const uint8_t* const src = p.tiles + ((((size_t)next.e * p.n_kt + (strip >> 3)) * p.n_kb + next.kb) << 14) + (strip & 7) * SC_BLOCK;
      mbar_expect_tx(bars + 8 * slot, SC_BLOCK);
      bulk_g2s(ring + slot * SC_BLOCK, src, SC_BLOCK, bars + 8 * slot);
    }
    __syncwarp();
    ++issued;
    next.kb += p.k_warps;
    if (next.kb >= p.n_kb) {
      next.kb = kw;
      if (++next.item >= last) more = false;
      else if (++next.group == n_groups) {
        next.group = 0;
        ++next.piece;
        find_piece(pieces, p.offsets, p.E, p.rows, N, next.piece, &next.e, &r_unused, &n_unused);
      }
    }
  };
  for (int i = 0; i < DEPTH && more; ++i) issue();
  if (!p.offsets) grid_dep_wait();
  grid_dep_launch();

  int turn = 0;
  const int row_a = (g >> 1) | ((g & 1) << 2);
  const uint32_t lds_at[2] = {(uint32_t)(row_a * 128 + ((t ^ (row_a & 7)) << 4)), (uint32_t)(row_a * 128 + (((4 + t) ^ (row_a & 7)) << 4))};
  int piece = -1, e = 0, r0 = 0, n = 0;
  for (long long item = first; item < last; ++item) {
    const int now = (int)(item / n_groups), group = (int)(item - (long long)now * n_groups);
    if (now != piece) {
      piece = now;
      find_piece(pieces, p.offsets, p.E, p.rows, N, piece, &e, &r0, &n);
    }
    const int strip = min(group * m_warps + mw, p.n_kt * 8 - 1);
    const float* const ws = p.w_scales + ((size_t)e * p.n_kt + (strip >> 3)) * p.n_kb;
    uint4 x[NT][2];
    float xs[NT][2], w_scale;
    auto load = [&](int kb) {
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int row = 8 * i + g;
        const uint8_t* const from = p.act + (size_t)(r0 + row) * (size_t)p.ld_act;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int c = kb * 128 + 64 * h + 16 * t;
          x[i][h] = row < n && c < p.C ? ld16(from + c) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int column = 8 * i + 2 * t + q;
          xs[i][q] = column < n ? ld_float(p.x_scales + (size_t)(r0 + column) * (size_t)p.ld_scales + kb) : 0.f;
        }
      }
      w_scale = ld_float(ws + kb);
    };
    float acc[NT][4] = {};
    if (kw < p.n_kb) load(kw);
    for (int kb = kw; kb < p.n_kb; kb += p.k_warps) {
      const int slot = taken % DEPTH;
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * slot, (uint32_t)(taken / DEPTH) & 1u));
      if (!ok) break;
      ++taken;
      const uint32_t block = ring + slot * SC_BLOCK;
      uint4 w[2][2];   // [rows from 0, from 8][first, second 64]
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < 2; ++u) w[u][h] = lds16(block + 1024 * u + lds_at[h]);
      __syncwarp();
      if (more) issue();
      float part[NT][4] = {}, f[NT][2];
#pragma unroll
      for (int i = 0; i < NT; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          mma_e4m3(part[i], w[0][h].x, w[1][h].x, w[0][h].y, w[1][h].y, x[i][h].x, x[i][h].y);
          mma_e4m3(part[i], w[0][h].z, w[1][h].z, w[0][h].w, w[1][h].w, x[i][h].z, x[i][h].w);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) f[i][q] = xs[i][q] * w_scale;
      }
      if (kb + p.k_warps < p.n_kb) load(kb + p.k_warps);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[i][q] = fmaf(part[i][q], f[i][q & 1], acc[i][q]);
    }
    float (*const red)[N][17] = red_both[turn];
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) red[warp][8 * i + 2 * t + (q & 1)][row_a + 8 * (q >> 1)] = acc[i][q];
    __syncthreads();   // (the other half of the buffer is for the next strip)
    const int width = 16 * m_warps;
    for (int i = threadIdx.x; i < width * n; i += 256) {
      const int m = i & (width - 1), c = i / width, co = group * width + m;
      if (co >= p.K) continue;
      float s = 0.f;
      for (int k = 0; k < p.k_warps; ++k) s += red[(m >> 4) * p.k_warps + k][c][m & 15];
      store_out(p.out, p.out_type, (long long)(r0 + c) * p.ld_out + co, s);
    }
  }
  // (after a wait that ran out: copies on their way land before the CTA ends)
  if (!ok) {
    for (; taken < issued; ++taken) mbar_wait(bars + 8 * (taken % DEPTH), (uint32_t)(taken / DEPTH) & 1u);
    if (lane == 0) raise_status(p.status, 30);
  }
}

template <int NT>
cudaError_t few_launch(const Scaled& p, const ScaledCall& c, int* launched) {
  static unsigned long long done = 0;
  const cudaError_t e = allow_max_smem(scaled_few_kernel<NT>, &done);
  if (e != cudaSuccess) return e;
  // all warps on one strip of output channels, unless there are not so many blocks of 128 input channels
  int k_warps = 8;
  while (k_warps > p.n_kb) k_warps /= 2;
  const long long pieces = c.offsets ? ((long long)c.rows + (long long)min(p.E, c.rows) * (8 * NT - 1)) / (8 * NT) : (c.rows + 8 * NT - 1) / (8 * NT);
  const long long items = pieces * ((p.K + 16 * (8 / k_warps) - 1) / (16 * (8 / k_warps)));
  const FewParams q{p.tiles, c.act, p.scales, c.scales, c.offsets, c.out, c.ld_act, c.ld_scales, c.ld_out, c.rows, p.E, p.C, p.K, p.n_kt, p.n_kb, c.out_type, k_warps, p.status_dev};
  *launched += 1;
  return launch_dependent(scaled_few_kernel<NT>, (unsigned)min(items, 2ll * sm_count()), 256, FewShape<NT>::kBytes, c.stream, q);
}

// Which kernel, by the time that each would take (us), where the experts have equal numbers of rows.  Few rows: the weights' bytes, once for each 8, 16 or 32 rows, or what a
// CTA's turns take; many rows: each block of 128 input channels takes a tile's CTA 0.14 to 0.28 us (a pair's 0.34 to 0.48: 256 rows and channels), a launch 4, a join of two
// or four CTAs 1.75; or the weights' bytes.  On 214 calls (dense 256 x 256 to 4096 x 8192 and 8192 x 1024 with 1 to 8192 rows, 8 to 64 experts with 1 to 512 rows each) the
// kernel taken was 0.7 % slower than the best (geometric mean), 1.24 times at worst (16 experts of 1104 x 1003, 512 rows each: 29.5 us by pairs, 23.7 by tiles of 64
// channels).  Both sides: one row of 4096 x 4096 5.1 (few rows) and 8.7 us, 16 rows 7.2 and 8.7, 24 rows 11.5 and 8.7; 64 experts of 2048 x 2048, 4 rows each 78 and 49;
// 24 rows of 8192 x 1024 8.0 by four CTAs a tile and 13.3 by one; 192 rows of 4096 x 8192 15.5 by tiles of 64 channels and 11.8 by 128; 4096 rows 135 by tiles of 128
// channels and 112 by pairs.
// SNN_FORCE_ROWS=few, many, 64 (with /2 or /4 behind it: CTAs that share a tile), 128 or 256 in the environment takes that wherever it can run.
struct Way {
  int tile, split;   // output channels of a tile, and CTAs that share one of 64; or 0: few rows, and eights of rows of a piece
};
Way choose_way(const Scaled& p, const ScaledCall& c) {
  const auto up = [](double a, double b) { return ceil(a / b); };
  const double used = c.offsets ? min(p.E, c.rows) : 1, each = up(c.rows, used), sms = sm_count(), nk = p.n_kb, mb = used * p.n_kt * nk * 16384e-6;
  const long long row_tiles = c.offsets ? c.rows / 128 + (long long)min(p.E, c.rows) : (c.rows + 127ll) / 128;   // at most
  const int nt = each <= 8 ? 1 : each <= 16 ? 2 : 4;
  const char* const force = getenv("SNN_FORCE_ROWS");
  const auto can_share = [&](int split) { return row_tiles * ((p.K + 63) / 64) * split <= (long long)sms && p.n_kb >= 2 * split; };
  if (force) {
    if (!strcmp(force, "few")) return {0, nt};
    for (int tile = 64; tile <= 256; tile *= 2) {
      char* end;
      if (strtol(force, &end, 10) != tile) continue;
      int split = *end == '/' && tile == 64 ? atoi(end + 1) : 1;
      while (split > 1 && (split != 2 && split != 4 || !can_share(split))) split /= 2;
      return {tile, max(split, 1)};
    }
  }
  const double turns = up(up(each, 8 * nt) * used * up(p.K, 16), 2 * sms);
  Way best{0, nt};
  double least = 1.55 + (nt == 4 ? 1.6 : 0.0) + 0.34 * turns +
                 fmax(mb * (nt == 1 ? 0.24 : nt == 2 ? 0.37 : 0.66) * up(nk, 8) * 8 / fmax(nk, 8) * up(each, 8 * nt), turns * up(nk, 8) * (nt == 1 ? 0.45 : nt == 2 ? 0.79 : 1.16));
  if (force && !strcmp(force, "many")) least = 1e30;
  const auto offer = [&](int tile, int split, double time) {
    if (time < least) {
      least = time;
      best = Way{tile, split};
    }
  };
  for (int split = 1; split <= 4 && (split == 1 || can_share(split)); split *= 2) {
    const double around = up(used * up(each, 128) * up(p.K, 64) * split, sms);
    offer(64, split, fmax(3.75 + around * (up(nk, split) * (around > 1 ? 0.194 : 0.141) + 0.5) + (split > 1 ? 1.75 : 0.0), 3.3 + mb / 4.8));
  }
  double around = up(used * up(each, 128) * up(p.K, 128), sms);
  offer(128, 1, fmax(3.75 + around * (nk * (around > 1 ? 0.283 : c.rows <= 64 ? 0.2 : 0.208) + 0.23), 3.3 + mb / 5.2));
  around = up(used * up(each, 256) * up(p.K, 256), fmax(1.0, floor(sms / 2)));
  offer(256, 1, fmax(4.5 + around * (nk * (around > 1 ? 0.477 : 0.339) + 0.77), 4.5 + mb / 4.1));
  return best;
}

}  // namespace

cudaError_t scaled_create(const uint8_t* weights, const float* scales, int E, int C, int K, cudaStream_t s, Scaled* p, int* launched) {
  p->E = E;
  p->C = C;
  p->K = K;
  p->n_kt = (K + 127) / 128;
  p->n_kb = (C + 127) / 128;
  const size_t tiles = (size_t)E * p->n_kt * p->n_kb;
  cudaError_t e = cudaMalloc((void**)&p->tiles, tiles << 14);
  if (e == cudaSuccess) e = cudaMalloc((void**)&p->scales, tiles * 4);
  if (e == cudaSuccess) e = cudaHostAlloc((void**)&p->status_host, sizeof(int), cudaHostAllocMapped);
  if (e == cudaSuccess) {
    *p->status_host = 0;
    e = cudaHostGetDevicePointer((void**)&p->status_dev, p->status_host, 0);
  }
  if (e == cudaSuccess) {
    const long long pieces = (long long)tiles << 10;
    scaled_layout_kernel<<<(unsigned)min((pieces + 255) / 256, 1ll << 20), 256, 0, s>>>(weights, reinterpret_cast<uint4*>(p->tiles), C, K, p->n_kt, p->n_kb, pieces);
    *launched += 1;
    e = cudaGetLastError();
  }
  if (e == cudaSuccess) e = cudaMemcpyAsync(p->scales, scales, tiles * 4, cudaMemcpyDeviceToDevice, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  return e;
}

void scaled_destroy(Scaled* p) {
  cudaFree(p->tiles);
  cudaFree(p->scales);
  if (p->status_host) cudaFreeHost(p->status_host);
}

cudaError_t scaled_forward(const Scaled& p, const ScaledCall& c, int* launched) {
  const Way way = choose_way(p, c);
  if (way.tile) return scaled_tall(p, c, way.tile, way.split, launched);
  return way.split == 1 ? few_launch<1>(p, c, launched) : way.split == 2 ? few_launch<2>(p, c, launched) : few_launch<4>(p, c, launched);
}

}  // namespace snn
