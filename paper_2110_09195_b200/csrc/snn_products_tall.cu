// Projections of language models, many rows: the 5th-generation tensor cores, the weights expanded from bits into tensor memory.
#include <cuda.h>

#include <type_traits>

#include "snn_products.h"

#include "snn_products.cuh"
#include "snn_tc_common.cuh"

namespace snn {
namespace {

// out[row, co] = alpha * sum_k W[co, k] x[row, k] as D[256 channels x up to 192 rows] = W (M operand) * x^T (N operand), by a pair of
// CTAs (a cluster of two, one instruction for both): each has 128 of the channels and half of the rows.
//
// The weights come as bits (snn_products.h): in each CTA two warpgroups in turn expand 128 channels x 64 input channels at a time into
// 16-bit +1 / -1, two instructions for two weights, and store them to tensor memory, from where the instruction takes its M operand.
// Shared memory then holds and feeds the rows alone, and no 16-bit weight is ever read from memory.  A single CTA with all the rows
// waited for them 40 % of the time: 64 bytes a cycle and SM at the instructions' full rate, from L2 and through shared memory; a pair needs
// half.  TMA brings the rows; rows named by an index come by 16-byte asynchronous copies of three warps (TMA's gather of four rows an
// instruction took 2900 cycles for 192 rows of 128 bytes, seven times the instructions that they feed).
// 512 columns: four stages of weights (32 columns each) and two accumulators of 192, so that one is written out while the next is
// being summed.
constexpr int TL_N = 192;             // rows of a tile, at most
constexpr int TL_A_STAGES = 4;
constexpr int TL_A_COLS = 32;         // 64 input channels, two to a column
constexpr int TL_D0 = TL_A_STAGES * TL_A_COLS;
constexpr int TL_HALF = TL_N / 2;      // rows of a CTA
constexpr int TL_B_BYTES = TL_HALF * 128;
constexpr int TL_BOX = 32;            // rows of one TMA box
// warps: 0 rows (with an index: 0, 2 and 3), 1 MMA, 2 tensor memory, 4-11 weights, 12-15 outputs (with adapters: 12-19)
constexpr int TL_PENDING = 3;         // stages of copied rows on their way, for each of the three warps that copy
// Stages of rows, and bytes of the tile's rows' A x and of an adapter's B kept beside them (RANK: 0 without adapters, else a bound of
// their rank).
template <int RANK>
struct TallShape {
  static constexpr int kStages = RANK == 128 ? 4 : RANK == 64 ? 7 : RANK == 32 ? 12 : RANK == 16 ? 14 : 16;
  static constexpr int kOutWarps = RANK ? 8 : 4;
  static constexpr int kThreads = 384 + 32 * kOutWarps;
  static constexpr int kH = RANK ? TL_N * (RANK + 4) * 4 : 0;       // fp32, rows in different banks
  static constexpr bool kWide = RANK <= 64;                          // B as fp32, too; else there is no room
  static constexpr int kB = RANK ? 256 * (kWide ? (RANK + 4) * 4 : (RANK + 8) * 2) : 0;   // the same; each warp its own
};

// The same value in all lanes, known to be so
__device__ __forceinline__ int uni(int x) { return __shfl_sync(0xffffffffu, x, 0); }

struct TallParams {
  const uint32_t* bits;
  const float* alpha;
  const uint16_t* act;
  const int32_t *rows, *offsets;
  void* out;
  long long ld_act, ld_out;
  int act_rows, max_rows, E, C, K, n_mt, n_kb, out_type, n_cp;
  int* status;
  Lowrank low;
  Powers pow;
};

struct TallBars {
  uint64_t b_full[16], b_empty[16], a_full[TL_A_STAGES], a_empty[TL_A_STAGES], d_full[2], d_empty[2], drain;
  uint32_t tmem, pad;
  int who[TL_N];         // adapters of the tile's rows, below 0: none
  int group[TL_N / 8];   // of eight rows
};

// Issued by the lanes for which `on` is not 0: D[256 x N] (+)= A[256 x 64] * B[N x 64]^T in four steps of 16, A in tensor memory, then the
// commits to both CTAs' barriers.  One statement, under a predicate: four statements with a branch on the lane around them took 700 cycles a
// stage, with a predicate each 400, this one 70.
__device__ __forceinline__ void stage_ts_f16(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate, uint32_t bar0, uint32_t bar1, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 d1, d2, d3;\n\t.reg .b32 a1, a2, a3;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
      "add.u64 d1, %2, 2;\n\tadd.u64 d2, %2, 4;\n\tadd.u64 d3, %2, 6;\n\t"
      "add.u32 a1, %1, 8;\n\tadd.u32 a2, %1, 16;\n\tadd.u32 a3, %1, 24;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f16 [%0], [a1], d1, %3, 1;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f16 [%0], [a2], d2, %3, 1;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f16 [%0], [a3], d3, %3, 1;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%5], %8;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%6], %8;\n\t}" ::"r"(d),
      "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(bar0), "r"(bar1), "r"(on), "h"((uint16_t)3)
      : "memory");
}
__device__ __forceinline__ void commit_on(uint32_t bar, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %2;\n\t}" ::"r"(bar),
      "r"(on), "h"((uint16_t)3)
      : "memory");
}
// 32 columns of the warp's 32 lanes; they are there after tmem_st_wait
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]),
      "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]),
      "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 8 columns of the warp's 32 lanes, a thread (g = lane / 4, t = lane % 4): columns 2t and 2t + 1 of lanes g and g + 8 (first four values),
// g + 16 and g + 24.  Loads and wait are one statement.
__device__ __forceinline__ void tmem_ld_16x8(uint32_t taddr, float (&v)[2][4]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%8];\n\t"
      "tcgen05.ld.sync.aligned.16x256b.x1.b32 {%4,%5,%6,%7}, [%9];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0][0]), "=f"(v[0][1]), "=f"(v[0][2]), "=f"(v[0][3]), "=f"(v[1][0]), "=f"(v[1][1]), "=f"(v[1][2]), "=f"(v[1][3])
      : "r"(taddr), "r"(taddr + (16u << 16))
      : "memory");
}
// (the barrier: the pair's first CTA's)
__device__ __forceinline__ void tma_rows(uint32_t dst, const void* map, int c, int row, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(c),
               "r"(row), "r"(bar)
               : "memory");
}
// 16 bytes, or zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// The address of the pair's first CTA's copy of a variable in shared memory, and an arrival there.  What the arrival stands for is in tensor
// memory or in the SM's own shared memory, after wait::st, wait::ld or a proxy fence, and is read by the MMA unit: no wider release is needed
// (one of cluster scope, with waits that acquire at that scope, made every stage take 900 cycles, whatever its size).
__device__ __forceinline__ uint32_t at_first(uint32_t addr) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
__device__ __forceinline__ void arrive_at_first(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(at_first(bar)) : "memory");
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// Barrier ID among THREADS of the CTA's threads, whole warps; whether all of them say so.
template <int ID, int THREADS>
__device__ __forceinline__ bool bar_all(bool v) {
  uint32_t r;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.and.pred p, %2, %3, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)v), "n"(ID), "n"(THREADS)
      : "memory");
  return r != 0;
}

// The experts' ranges in shared memory: end[e] counts the row tiles up to and with expert e.
struct Ranges {
  int *lo, *n, *end;
};
struct Tile {
  int e, r0, n, ct;   // expert, first row, rows, the CTA's channel tile
};
// Tile `index` of the launch, channels of the same rows one after the other; `t.e` is where the search begins (indices rise).
__device__ __forceinline__ bool tall_tile(const Ranges& R, int E, int n_cp, int index, int rank, Tile& t) {
  const int q = index / n_cp;
  int e = t.e;
  while (e < E && q >= R.end[e]) ++e;
  t.e = uni(e);
  if (t.e >= E) return false;
  const int n = R.n[t.e], tiles = (n + TL_N - 1) / TL_N, per = ((n + tiles - 1) / tiles + 31) & ~31;   // about the same rows in each
  const int k = q - (t.e ? R.end[t.e - 1] : 0);
  t.ct = 2 * (index - q * n_cp) + rank;
  t.r0 = uni(R.lo[t.e] + k * per);
  t.n = uni(min(per, n - k * per));
  return true;
}

// A channel's outputs of up to 32 rows.
__device__ __forceinline__ void to_out(float* p, float v) { *p = v; }
__device__ __forceinline__ void to_out(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void to_out(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
template <class O>
__device__ __forceinline__ void store_column(O* out, long long ld, int n, float alpha, const uint32_t (&v)[32]) {
#pragma unroll
  for (int c = 0; c < 32; ++c, out += ld)
    if (c < n) to_out(out, alpha * __uint_as_float(v[c]));
}

// 32 channels from co0, up to 8 rows from r0, in the layout of tmem_ld_16x8.  16-bit outputs change hands first: a thread then has four
// neighbouring channels of a row (twice), eight threads a row's 32 bytes.
__device__ __forceinline__ uint32_t pack_out(int type, float lo, float hi) {
  uint32_t r;
  if (type == SNN_OUT_F16) {
    const __half2 h = __floats2half2_rn(lo, hi);
    memcpy(&r, &h, 4);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    memcpy(&r, &h, 4);
  }
  return r;
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void store_16x8(const TallParams& p, int r0, int n, int co0, const float (&v)[2][4]) {
  const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  if (p.out_type == SNN_OUT_F32) {
    float* const out = static_cast<float*>(p.out) + (long long)(r0 + 2 * q) * p.ld_out + co0 + g;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (2 * q + (i & 1) < n && co0 + g + 8 * (i >> 1) < p.K) out[(i & 1) * p.ld_out + 8 * (i >> 1)] = v[i >> 2][i & 3];
    return;
  }
  uint32_t w[4];   // row g, channels 8 i + 2 q and the next
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = transpose_8x8(pack_out(p.out_type, v[i >> 1][2 * (i & 1)], v[i >> 1][2 * (i & 1) + 1]));
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    // an even q gives its pair of the second eight for its neighbour's of the first
    const uint32_t other = __shfl_xor_sync(0xffffffffu, q & 1 ? w[i] : w[i + 1], 1);
    const uint32_t lo = q & 1 ? other : w[i], hi = q & 1 ? w[i + 1] : other;
    const int co = co0 + 8 * (i + (q & 1)) + 2 * (q & 2);
    if (g < n && co < p.K) {
      uint16_t* const out = static_cast<uint16_t*>(p.out) + (long long)(r0 + g) * p.ld_out + co;
      if (co + 4 <= p.K && ((uintptr_t)out & 7) == 0) {
        *reinterpret_cast<uint2*>(out) = make_uint2(lo, hi);
      } else {
        const uint16_t part[4] = {(uint16_t)lo, (uint16_t)(lo >> 16), (uint16_t)hi, (uint16_t)(hi >> 16)};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (co + k < p.K) out[k] = part[k];
      }
    }
  }
}

// B (A x) in fp32 on the FMA units, two of the rank at a time, in the layout of tmem_ld_16x8: a thread has four channels and two rows of
// eight, so that a value from shared memory serves two or four products.  Two warps for each 32 channels, which take turns at eight rows: one
// alone is bound by latency, 142 us for 4096 rows of 4096 x 4096 and rank 32.  (On the warp's matrix instruction, with A x in three 16-bit or
// two tf32 parts, each instruction waited for one of the pair's: 72 to 96 cycles.  With a channel a thread, and a load of A x for every two
// products: 163 us.)
__device__ __forceinline__ void fma2(uint64_t& d, uint64_t a, uint64_t b) { asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(d) : "l"(a), "l"(b)); }
__device__ __forceinline__ uint64_t pack2(float2 v) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
  return r;
}
__device__ __forceinline__ float sum2(uint64_t v) {
  float a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
  return a + b;
}
// 8 of the rank: b, of channels g, g + 8, g + 16, g + 24 (16-bit values, or pairs of fp32 values as they are in shared memory, which saves
// as many instructions as the products take); h, of rows 2t and 2t + 1, h_row floats apart
template <class T>
__device__ __forceinline__ void lowrank_step(uint64_t (&d)[2][4], const uint4 (&b)[4], const float* h, int h_row) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    ulonglong2 x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = *reinterpret_cast<const ulonglong2*>(h + i * h_row + 4 * half);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint64_t w0 = pack2(T::unpack(half ? b[c].z : b[c].x)), w1 = pack2(T::unpack(half ? b[c].w : b[c].y));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fma2(d[i][c], w0, x[i].x);
        fma2(d[i][c], w1, x[i].y);
      }
    }
  }
}
__device__ __forceinline__ ulonglong2 lds16(uint32_t addr) {
  ulonglong2 v;
  asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(v.x), "=l"(v.y) : "r"(addr));
  return v;
}
// (addresses in shared memory; all loads before the first product: beside the pair's MMAs a load takes over a hundred cycles)
__device__ __forceinline__ void lowrank_step_wide(uint64_t (&d)[2][4], uint32_t b, uint32_t b_row, uint32_t h, uint32_t h_row) {
  ulonglong2 x[2][2], w[4][2];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i][half] = lds16(h + i * h_row + 16 * half);
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c][half] = lds16(b + 8 * c * b_row + 16 * half);
  }
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fma2(d[i][c], w[c][half].x, x[i][half].x);
        fma2(d[i][c], w[c][half].y, x[i][half].y);
      }
}
// ... added to the outputs of the rows whose bit is set
__device__ __forceinline__ void add_lowrank(float (&v)[2][4], const uint64_t (&d)[2][4], uint32_t which) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if ((which >> (i & 1)) & 1u) v[i >> 2][i & 3] += sum2(d[i & 1][i >> 1]);
}

// RANK: 0 without adapters, else a bound of their rank.
template <class T, bool GATHER, int RANK>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(TallShape<RANK>::kThreads, 1) products_tall_kernel(const TallParams p, const __grid_constant__ CUtensorMap map) {
  constexpr int STAGES = TallShape<RANK>::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  TallBars* const bars = reinterpret_cast<TallBars*>(smem + STAGES * TL_B_BYTES + TallShape<RANK>::kH + TallShape<RANK>::kB);
  Ranges R;
  R.lo = reinterpret_cast<int*>(bars + 1);
  R.n = R.lo + p.E;
  R.end = R.n + p.E;
  const int warp = uni(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t b_smem = smem_u32(smem);
  const int rank = (int)(blockIdx.x & 1), first_tile = (int)(blockIdx.x >> 1), n_pairs = (int)(gridDim.x >> 1);
  // As in the kernel for few rows: after the one that writes A x, only the warps that read it wait.
  if (warp == 0) {
    if (!RANK) grid_dep_wait();
    // tiles of each expert, summed up: every lane a run of experts
    const int per = (p.E + 31) >> 5, e0 = lane * per, e1 = min(p.E, e0 + per);
    int count = 0;
    for (int e = e0; e < e1; ++e) {
      const int lo = p.offsets ? clamp_offset(p.offsets[e], p.max_rows) : 0;
      const int n = p.offsets ? max(clamp_offset(p.offsets[e + 1], p.max_rows) - lo, 0) : p.max_rows;
      R.lo[e] = lo;
      R.n[e] = n;
      count += (n + TL_N - 1) / TL_N;
    }
    int upto = count;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += v;
    }
    int end = upto - count;
    for (int e = e0; e < e1; ++e) R.end[e] = end += (R.n[e] + TL_N - 1) / TL_N;
  } else if (warp == 1 && lane == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(smem_u32(&bars->b_full[i]), GATHER ? 2 : 1);
      mbar_init(smem_u32(&bars->b_empty[i]), 1);
    }
    for (int i = 0; i < TL_A_STAGES; ++i) {
      mbar_init(smem_u32(&bars->a_full[i]), 8);
      mbar_init(smem_u32(&bars->a_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bars->d_full[i]), 1);
      mbar_init(smem_u32(&bars->d_empty[i]), 2 * TallShape<RANK>::kOutWarps);
    }
    mbar_init(smem_u32(&bars->drain), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  } else if (warp == 2) {
    // (not before the kernel before has ended: it may still have to get tensor memory of its own)
    if (!RANK) grid_dep_wait();
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars->tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (!RANK || warp >= 12) grid_dep_wait();
  tc_fence_before();
  __syncthreads();
  pair_sync();
  tc_fence_after();
  grid_dep_launch();   // (only now: a dependent that has tensor memory before this pair does would wait for it for good)
  const uint32_t tmem = bars->tmem;
  const int nk = (p.C + 63) >> 6;
  bool ok = true;
  Tile t{};

  if (GATHER && (warp == 0 || warp == 2 || warp == 3)) {
    // ------------------------------------------------------------ rows by an index: 8 lanes copy 128 bytes of a row
    // Each of the three warps has every third stage: what a stage costs beside its copies is a third of the time for each.
    const int first = lane >> 3, chunk = lane & 7, turn = warp ? warp - 1 : 0;   // rows first, first + 4, ... of the CTA's
    const uint32_t dst = b_smem + (uint32_t)first * 128u;
    const uint32_t swizzled[2] = {(uint32_t)((chunk ^ first) << 4), (uint32_t)((chunk ^ (first + 4)) << 4)};
    uint32_t seq = 0;   // stages of the tiles before
    int issued = 0;
    uint32_t mine[TL_PENDING + 1] = {};   // the last stages this warp issued, the oldest first
    for (int index = first_tile; ok && tall_tile(R, p.E, p.n_cp, index, rank, t); index += n_pairs, seq += (uint32_t)nk) {
      const int half = ((t.n + 31) & ~31) / 2, r0 = t.r0 + rank * half, n = min(t.n - rank * half, half);
      int who[TL_HALF / 4];
#pragma unroll
      for (int i = 0; i < TL_HALF / 4; ++i) {
        const int c = first + 4 * i;
        who[i] = c < n ? p.rows[r0 + c] : -1;
        if (who[i] >= p.act_rows) who[i] = -1;   // (outside: zeros)
      }
      for (int kb = (int)((turn + 3u - seq % 3u) % 3u); kb < nk; kb += 3) {
        const uint32_t at = seq + (uint32_t)kb, s = at % STAGES;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->b_empty[s]), (at / STAGES & 1u) ^ 1u));
        if (!ok) break;
        const int k = kb * 64 + chunk * 8;
        const uint16_t* const x = p.act + k;
        const bool in = k < p.C;
#pragma unroll
        for (int i = 0; i < TL_HALF / 4; ++i) {
          const bool there = in && who[i] >= 0;
          if (4 * i < half) copy16(dst + s * TL_B_BYTES + i * 512 + swizzled[i & 1], there ? x + (size_t)who[i] * (size_t)p.ld_act : p.act, there);
        }
        copy_commit();
#pragma unroll
        for (int i = 0; i < TL_PENDING; ++i) mine[i] = mine[i + 1];
        mine[TL_PENDING] = s;
        if (++issued > TL_PENDING) {   // the oldest stage on its way has landed
          copy_wait<TL_PENDING>();
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) arrive_at_first(smem_u32(&bars->b_full[mine[0]]));
        }
      }
    }
    copy_wait<0>();
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
#pragma unroll
      for (int i = 1; i <= TL_PENDING; ++i)
        if (TL_PENDING - i < issued) arrive_at_first(smem_u32(&bars->b_full[mine[i]]));
    }
    if (!ok && lane == 0) raise_status(p.status, 20);
  } else if (!GATHER && warp == 0) {
    // ------------------------------------------------------------ rows: one stage is 64 input channels of the tile's rows
    int s = 0, filled = 0;
    uint32_t phase = 0;
    for (int index = first_tile; ok && tall_tile(R, p.E, p.n_cp, index, rank, t); index += n_pairs) {
      const int half = ((t.n + 31) & ~31) / 2, r0 = t.r0 + rank * half;
      const uint32_t bytes = (uint32_t)((half + TL_BOX - 1) / TL_BOX * TL_BOX) * 256u;   // of both CTAs
      for (int kb = 0; kb < nk; ++kb) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->b_empty[s]), phase ^ 1u));
        if (!ok) break;
        const uint32_t full = smem_u32(&bars->b_full[s]), dst = b_smem + s * TL_B_BYTES;
        if (rank == 0 && lane == 0) mbar_expect_tx(full, bytes);
        __syncwarp();
        if (lane * TL_BOX < half) tma_rows(dst + lane * TL_BOX * 128, &map, kb * 64, r0 + lane * TL_BOX, at_first(full));
        filled = min(filled + 1, STAGES);
        if (++s == STAGES) {
          s = 0;
          phase ^= 1u;
        }
      }
    }
    // both CTAs' copies in flight land before the pair ends, whatever became of the other warps
    for (int i = 0; rank == 0 && i < filled; ++i) {
      if (--s < 0) {
        s = STAGES - 1;
        phase ^= 1u;
      }
      ok = mbar_wait(smem_u32(&bars->b_full[s]), phase) && ok;
    }
    if (!ok && lane == 0) raise_status(p.status, 21);
  } else if (warp == 1 && rank == 0) {
    // ------------------------------------------------------------ MMA, for both CTAs
    int s = 0, a = 0, d = 0;
    uint32_t b_phase = 0, a_phase = 0, d_phase = 0;
    const uint32_t type = std::is_same<T, BF16>::value ? 1u : 0u, leader = elect_one(), tmem_u = (uint32_t)uni((int)tmem);
    for (int index = first_tile; ok && tall_tile(R, p.E, p.n_cp, index, rank, t); index += n_pairs) {
      const uint32_t n32 = (uint32_t)(t.n + 31) & ~31u;   // (a pair's instructions take multiples of 32)
      const uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | ((n32 >> 3) << 17) | ((256u >> 4) << 24);
      const uint32_t acc = tmem_u + TL_D0 + d * TL_N;
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->d_empty[d]), d_phase ^ 1u));
      for (int kb = 0; ok && kb < nk; ++kb) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->b_full[s]), b_phase) && mbar_wait(smem_u32(&bars->a_full[a]), a_phase));
        if (!ok) break;
        tc_fence_after();
        const uint64_t desc = ((uint64_t)2 << 61) | ((uint64_t)1 << 46) | ((uint64_t)64 << 32) | ((uint64_t)1 << 16) | ((b_smem + s * TL_B_BYTES) >> 4);
        stage_ts_f16(acc, tmem_u + a * TL_A_COLS, desc, idesc, kb ? 1u : 0u, smem_u32(&bars->b_empty[s]), smem_u32(&bars->a_empty[a]), leader);
        __syncwarp();
        if (++s == STAGES) {
          s = 0;
          b_phase ^= 1u;
        }
        if (++a == TL_A_STAGES) {
          a = 0;
          a_phase ^= 1u;
        }
      }
      if (!ok) break;
      commit_on(smem_u32(&bars->d_full[d]), leader);
      __syncwarp();
      if ((d ^= 1) == 0) d_phase ^= 1u;
    }
    commit_on(smem_u32(&bars->drain), leader);
    __syncwarp();
    ok = mbar_wait(smem_u32(&bars->drain), 0) && ok;
    if (!ok && lane == 0) raise_status(p.status, 22);
  } else if (warp >= 4 && warp < 12) {
    // ------------------------------------------------------------ weights: thread m of a warpgroup is channel m of the tile
    const int m = ((int)threadIdx.x - 128) & 127, group = (warp - 4) >> 2;   // blocks group, group + 2, ... of a tile
    const int shift = (m >> 3) & 1 ? 8 : 0;
    const Powers pow = in_registers(p.pow);
    const uint32_t dst = tmem + ((uint32_t)(m & ~31) << 16);
    uint32_t base = 0;      // blocks of the tiles before
    uint32_t stored = ~0u;  // a block that is on its way to tensor memory; it is waited for when the next one has been expanded
    for (int index = first_tile; ok && tall_tile(R, p.E, p.n_cp, index, rank, t); index += n_pairs, base += (uint32_t)nk) {
      const uint4* src = reinterpret_cast<const uint4*>(p.bits) + ((size_t)(t.e * p.n_mt + t.ct * 8 + (m >> 4)) * p.n_kb) * 32 + 4 * (m & 7) + 2 * group;
      uint4 next[2] = {ld16(src), ld16(src + 1)};
      for (int kb = 0; ok && kb < p.n_kb; ++kb) {
        const uint32_t w[2][4] = {{next[0].x >> shift, next[0].z >> shift, next[1].x >> shift, next[1].z >> shift},
                                  {next[0].y >> shift, next[0].w >> shift, next[1].y >> shift, next[1].w >> shift}};
        if (kb + 1 < p.n_kb) {
          next[0] = ld16(src + (size_t)(kb + 1) * 32);
          next[1] = ld16(src + (size_t)(kb + 1) * 32 + 1);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int block = 4 * kb + 2 * i + group;
          if (block >= nk) break;
          uint32_t v[32];
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[(j < 4 ? 0 : 12) + 4 * q + j] = plus_minus<T>(w[i][q], 15 - j, pow);
          if (stored != ~0u) {
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at_first(smem_u32(&bars->a_full[stored]));
          }
          const uint32_t at = base + (uint32_t)block;
          stored = at % TL_A_STAGES;
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->a_empty[stored]), (at / TL_A_STAGES & 1u) ^ 1u));
          if (!ok) break;
          tc_fence_after();
          tmem_st32(dst + stored * TL_A_COLS, v);
        }
      }
    }
    if (stored != ~0u) {
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (ok && lane == 0) arrive_at_first(smem_u32(&bars->a_full[stored]));
    }
    if (!ok && lane == 0) raise_status(p.status, 23);
  } else if (warp >= 12) {
    // ------------------------------------------------------------ outputs: thread m is channel m of the tile, a column is a row
    const int m = ((int)threadIdx.x - 384) & 127, turn = (warp - 12) >> 2;
    constexpr int OUTS = 32 * TallShape<RANK>::kOutWarps;
    constexpr bool WIDE = TallShape<RANK>::kWide;
    const int h_row = p.low.rank + 4, b_row = p.low.rank + (WIDE ? 4 : 8);   // (elements)
    float* const h_smem = reinterpret_cast<float*>(smem + STAGES * TL_B_BYTES);
    uint8_t* const b_smem_warp = smem + STAGES * TL_B_BYTES + TallShape<RANK>::kH + (warp - 12) * 32 * b_row * (WIDE ? 4 : 2);
    float* const b_wide = reinterpret_cast<float*>(b_smem_warp);
    uint16_t* const b_narrow = reinterpret_cast<uint16_t*>(b_smem_warp);
    int *const who = bars->who, *const group = bars->group;
    constexpr int MIXED = -2;
    int d = 0;
    uint32_t phase = 0;
    for (int index = first_tile; ok && tall_tile(R, p.E, p.n_cp, index, rank, t); index += n_pairs) {
      const int co = t.ct * 128 + m;
      const float alpha = p.alpha[(size_t)t.e * p.n_mt * 16 + co];
      int held = -1;
      if (RANK) {   // the rows' adapters and A x, while the sums are under way
        const int quads = p.low.rank / 4;
        for (int i = (int)threadIdx.x - 384; i < t.n * quads; i += OUTS)
          copy16(smem_u32(h_smem + (i / quads) * h_row + 4 * (i % quads)), p.low.h + (size_t)t.r0 * p.low.rank + 4 * i, true);
        copy_commit();
        for (int i = (int)threadIdx.x - 384; i < TL_N; i += OUTS) {
          const int a = i < t.n ? p.low.adapter[t.r0 + i] : -1, one = a >= 0 && a < p.low.n ? a : -1;
          who[i] = one;
          // the adapter that the eight rows around this one have (those behind the last count with it)
          const int lead = __shfl_sync(0xffffffffu, one, lane & 24);
          const unsigned same = __ballot_sync(0xffffffffu, one == lead || i >= t.n);
          if ((i & 7) == 0) group[i >> 3] = ((same >> (lane & 24)) & 255u) == 255u ? lead : MIXED;
        }
        copy_wait<0>();
      }
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->d_full[d]), phase));
      if (RANK) ok = bar_all<1, OUTS>(ok);   // (everybody's part of A x has landed; the warps go on, or give up, together)
      if (!ok) break;
      tc_fence_after();
      const uint32_t src = tmem + ((uint32_t)(m & ~31) << 16) + TL_D0 + d * TL_N;
      const long long first = (long long)t.r0 * p.ld_out + co;
      if (RANK == 0) {
        for (int c0 = 0; c0 < t.n; c0 += 32) {
          uint32_t v[32];
          tmem_ld32(src + c0, v);
          const int n = co < p.K ? min(32, t.n - c0) : 0;
          const long long at = first + c0 * p.ld_out;
          if (p.out_type == SNN_OUT_F32) store_column(static_cast<float*>(p.out) + at, p.ld_out, n, alpha, v);
          else if (p.out_type == SNN_OUT_F16) store_column(static_cast<__half*>(p.out) + at, p.ld_out, n, alpha, v);
          else store_column(static_cast<__nv_bfloat16*>(p.out) + at, p.ld_out, n, alpha, v);
          __syncwarp();
        }
      } else {
        // Eight rows at a time.  Rows of one request lie together, so they mostly have one adapter: its B stays in shared memory until the
        // next one's.  Else there is a pass for each of their adapters.
        const int n_rank = p.low.rank, g = lane >> 2, q = lane & 3, co0 = t.ct * 128 + (m & ~31);
        float scale[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) scale[i] = __shfl_sync(0xffffffffu, alpha, 8 * i + g);
        const uint16_t* const b_all = static_cast<const uint16_t*>(p.low.b);
        const size_t b_size = (size_t)p.K * n_rank;
        for (int c0 = 8 * turn; c0 < t.n; c0 += 16) {
          float v[2][4];
          tmem_ld_16x8(src + c0, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] *= scale[i >> 1];
          const float* const h = h_smem + (c0 + 2 * q) * h_row;
          const int a = group[c0 >> 3];   // (the same for the whole warp)
          if (a >= 0) {
            if (a != held) {
              held = a;
              __syncwarp();
              const int chunks = n_rank / 8, all = min(32, p.K - co0) * chunks;
              for (int i = lane; i < all; i += 32) {
                const uint4 u = ld16(b_all + a * b_size + (size_t)co0 * n_rank + 8 * i);
                const int at = (i / chunks) * b_row + 8 * (i % chunks);
                if (WIDE) {
                  const float2 f0 = T::unpack(u.x), f1 = T::unpack(u.y), f2 = T::unpack(u.z), f3 = T::unpack(u.w);
                  *reinterpret_cast<float4*>(b_wide + at) = make_float4(f0.x, f0.y, f1.x, f1.y);
                  *reinterpret_cast<float4*>(b_wide + at + 4) = make_float4(f2.x, f2.y, f3.x, f3.y);
                } else {
                  *reinterpret_cast<uint4*>(b_narrow + at) = u;
                }
              }
              __syncwarp();
            }
            uint64_t low[2][4] = {};
#pragma unroll 1
            for (int j = 0; j < n_rank; j += 8) {
              if (WIDE) {
                lowrank_step_wide(low, smem_u32(b_wide + g * b_row + j), 4u * (uint32_t)b_row, smem_u32(h + j), 4u * (uint32_t)h_row);
              } else {
                uint4 b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = *reinterpret_cast<const uint4*>(b_narrow + (8 * i + g) * b_row + j);
                lowrank_step<T>(low, b, h + j, h_row);
              }
            }
            add_lowrank(v, low, 3u);
          } else if (a == MIXED) {
            const int mine = lane < 8 ? who[c0 + lane] : -1;
            unsigned left = __ballot_sync(0xffffffffu, mine >= 0);
            while (left) {
              const int one = __shfl_sync(0xffffffffu, mine, __ffs(left) - 1);
              const unsigned same = __ballot_sync(0xffffffffu, mine == one);
              left &= ~same;
              uint64_t low[2][4] = {};
#pragma unroll 2
              for (int j = 0; j < n_rank; j += 8) {
                uint4 b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = ld16(b_all + one * b_size + (size_t)min(co0 + 8 * i + g, p.K - 1) * n_rank + j);
                lowrank_step<T>(low, b, h + j, h_row);
              }
              // (rows are apart: what other rows' A x gives with this B goes nowhere)
              add_lowrank(v, low, (same >> (2 * q)) & 3u);
            }
          }
          store_16x8(p, t.r0 + c0, t.n - c0, co0, v);
        }
        bar_sync_some<1, OUTS>();   // (everybody has read A x)
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_at_first(smem_u32(&bars->d_empty[d]));
      if ((d ^= 1) == 0) phase ^= 1u;
    }
    if (!ok && lane == 0) raise_status(p.status, 24);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 2) mbar_wait(smem_u32(&bars->drain), 0);   // (the last arrival here from the pair's MMAs)
  __syncwarp();
  pair_sync();
  tc_fence_after();
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

using MapEncoder = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
// The driver's tensor-map encoder, looked up once (the library does not link the driver).
MapEncoder map_encoder() {
  static const MapEncoder f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<MapEncoder>(p);
  }();
  return f;
}

template <class T, bool GATHER, int RANK>
cudaError_t tall_launch(const Products& p, const ProductCall& c, const CUtensorMap& map, int* launched) {
  static unsigned long long done = 0;
  cudaError_t e = allow_max_smem(products_tall_kernel<T, GATHER, RANK>, &done);
  if (e != cudaSuccess) return e;
  const TallParams q{p.bits, p.alpha, static_cast<const uint16_t*>(c.act), c.rows, c.offsets, c.out, c.ld_act, c.ld_out, c.act_rows, c.max_rows, p.E, p.C, p.K, p.n_mt, p.n_kb, c.out_type,
                     (p.K + 255) / 256, p.status_dev, c.low, powers()};
  const long long tiles = ((long long)c.max_rows / TL_N + (c.offsets ? min(p.E, c.max_rows) : 1)) * q.n_cp;
  const size_t smem = 1024 + TallShape<RANK>::kStages * TL_B_BYTES + TallShape<RANK>::kH + TallShape<RANK>::kB + sizeof(TallBars) + (size_t)p.E * 12;
  *launched += 1;
  return launch_dependent(products_tall_kernel<T, GATHER, RANK>, 2u * (unsigned)min(tiles, (long long)max(1, sm_count() / 2)), TallShape<RANK>::kThreads, smem,
                          c.stream, q, map);
}

template <class T>
cudaError_t tall_kind(const Products& p, const ProductCall& c, const CUtensorMap& map, int* launched) {
  if (!c.low.adapter) return c.rows ? tall_launch<T, true, 0>(p, c, map, launched) : tall_launch<T, false, 0>(p, c, map, launched);
  if (c.low.rank <= 16) return tall_launch<T, false, 16>(p, c, map, launched);
  if (c.low.rank <= 32) return tall_launch<T, false, 32>(p, c, map, launched);
  if (c.low.rank <= 64) return tall_launch<T, false, 64>(p, c, map, launched);
  return tall_launch<T, false, 128>(p, c, map, launched);
}

}  // namespace

cudaError_t products_tall(const Products& p, const ProductCall& c, int* launched) {
  const MapEncoder encode = map_encoder();
  if (!encode) return cudaErrorNotSupported;
  CUtensorMap map;
  const bool bf16 = c.act_type != SNN_ACT_F16;
  const cuuint64_t dims[2] = {(cuuint64_t)p.C, (cuuint64_t)c.act_rows}, strides[1] = {(cuuint64_t)c.ld_act * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)TL_BOX}, steps[2] = {1, 1};
  if (encode(&map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(c.act), dims, strides, box, steps,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  return bf16 ? tall_kind<BF16>(p, c, map, launched) : tall_kind<F16>(p, c, map, launched);
}

}  // namespace snn
