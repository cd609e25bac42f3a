// Projections of language models, many rows: the 5th-generation tensor cores, the weights expanded from bits into tensor memory.
#include <cuda.h>

#include <type_traits>

#include "snn_products.h"

#include "snn_pairs.cuh"
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
// being summed.  (Times here are a call's in a graph of twelve, a run too short for the power limit; among seconds of calls the clock is lower and the
// long ones take up to 1.17 times as long.  4096 rows, one expert of 4096 x 4096, bf16: 90 us, 1530 TFLOP/s; 8192 rows by an index, 8
// experts of 2048 x 8192, 200 us, 1380 TFLOP/s, and 233 us.)
//
// With adapters, D = alpha S + B (A x), A x in fp32 from the kernel before: the warps of the outputs multiply the sums by alpha in place, in
// tensor memory, and the matrix instructions add the second term, as tf32: B's 16-bit values are such numbers, and A x is the sum of three (11
// bits each, so that nothing is rounded).  A pass adds 32 of the rank, of one adapter or of several small ones, to the rows between the first and the
// last that have them; rows of others have zeros there.  Two slots: the warps write the next pass's operands while this one is being added.  On
// the FMA units, from shared memory, the same took longer than the sums themselves (4096 rows of 4096 x 4096 and rank 32 141 us, now 105, among
// seconds of calls 121; rank 64 208 and 125, rank 128 312 and 153); as 16-bit or tf32 products of the warps' own matrix instruction each waited for one of the
// pair's, 72 to 96 cycles.  Tiles with more than TL_LOW_MOST adapters, nearly one for each row, take the FMA units all the same (4096 rows, an adapter of
// 48 for each row, rank 16 483 and 628 us, rank 64 1006 and 1191; of 100, 669 and 669, 1515 and 1328).
constexpr int TL_N = 192;             // rows of a tile, at most
constexpr int TL_A_STAGES = 4;
constexpr int TL_A_COLS = 32;         // 64 input channels, two to a column
constexpr int TL_D0 = TL_A_STAGES * TL_A_COLS;
constexpr int TL_HALF = TL_N / 2;      // rows of a CTA
constexpr int TL_B_BYTES = TL_HALF * 128;
constexpr int TL_BOX = 32;            // rows of one TMA box
// warps: 0 rows (with an index: 0, 2 and 3), 1 MMA, 2 tensor memory, 4-11 weights, 12-15 outputs (with adapters: 3 the MMAs of their terms, and 12-19 outputs where there
// are many passes)
constexpr int TL_PENDING = 3;         // stages of copied rows on their way, for each of the three warps that copy
// With adapters, for 32 of the rank: their B, [128 channels][32], and three parts of A x, [96 rows][32] each, as 32-bit values; twice, so
// that the next are written while the matrix instructions read these.
constexpr int TL_LOW_A = 128 * 128, TL_LOW_B = TL_HALF * 128, TL_LOW_PARTS = 3, TL_LOW_BYTES = TL_LOW_A + TL_LOW_PARTS * TL_LOW_B;
constexpr int TL_LOW_MOST = 72;       // different adapters in a tile, up to which the matrix instructions add them
// What stands for an infinity or NaN of B in the matrix instructions, with its sign: the rows of other adapters have 0 there and get 0, an infinite
// A x gives its infinity (a 0 here would make it NaN, which nothing added later takes back), and a finite one at most 2^28, beside
// the infinity or NaN that is added to this output afterwards.
constexpr float TL_LOW_ODD = 0x1p-100f;
template <int LOW>   // 0, or with adapters the number of warps that write the outputs
struct TallShape {
  static constexpr int kStages = LOW ? 10 : 16;
  static constexpr int kOutWarps = LOW ? LOW : 4;
  static constexpr int kThreads = 384 + 32 * kOutWarps;
  static constexpr int kLow = LOW ? 2 * TL_LOW_BYTES : 0;   // bytes
};

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
  uint64_t b_full[16], b_empty[16], a_full[TL_A_STAGES], a_empty[TL_A_STAGES], d_full[2], d_empty[2], drain, low_full[2], low_done[2];
  uint32_t tmem;
  int odd;   // some adapter's B had an infinity or NaN
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
// Up to four steps of 8 of the rank: D[256 x N] += B[256 x 8 steps] * H[N x 8 steps]^T, both 32-bit values of 10 bits (tf32) in shared memory.
__device__ __forceinline__ void low_ss_tf32(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t steps, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q, q1, q2, q3;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "setp.ne.u32 q, %5, 0;\n\tsetp.gt.and.u32 q1, %4, 1, q;\n\tsetp.gt.and.u32 q2, %4, 2, q;\n\tsetp.gt.and.u32 q3, %4, 3, q;\n\t"
      "add.u64 a1, %1, 2;\n\tadd.u64 a2, %1, 4;\n\tadd.u64 a3, %1, 6;\n\t"
      "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::tf32 [%0], %1, %2, %3, 1;\n\t"
      "@q1 tcgen05.mma.cta_group::2.kind::tf32 [%0], a1, b1, %3, 1;\n\t"
      "@q2 tcgen05.mma.cta_group::2.kind::tf32 [%0], a2, b2, %3, 1;\n\t"
      "@q3 tcgen05.mma.cta_group::2.kind::tf32 [%0], a3, b3, %3, 1;\n\t}" ::"r"(d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(steps), "r"(on)
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
// 4 columns; load and wait are one statement
__device__ __forceinline__ void tmem_ld4(uint32_t taddr, uint32_t (&v)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];\n\ttcgen05.wait::ld.sync.aligned;"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t (&v)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
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

// The adapters of a tile's rows, by a warp: lane l has rows l, l + 32, ...; -1 for none.
constexpr int NO_MORE = 0x7fffffff;
struct Adapters {
  int of[TL_N / 32];
  __device__ __forceinline__ void load(const Lowrank& low, const Tile& t) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < TL_N / 32; ++i) {
      const int a = lane + 32 * i < t.n ? low.adapter[t.r0 + lane + 32 * i] : -1;
      of[i] = a < low.n ? a : -1;
    }
  }
  // the least above `a` (-1: the first), or NO_MORE
  __device__ __forceinline__ int after(int a) const {
    int least = NO_MORE;
#pragma unroll
    for (int i = 0; i < TL_N / 32; ++i)
      if (of[i] > a) least = min(least, of[i]);
    return __reduce_min_sync(0xffffffffu, least);
  }
  // how many there are, up to TL_LOW_MOST + 1
  __device__ __forceinline__ int count() const {
    int n = 0;
    for (int a = after(-1); a != NO_MORE && n <= TL_LOW_MOST; a = after(a)) ++n;
    return n;
  }
};

// The passes in which the adapters' terms are added: 32 of an adapter's rank at a time, or, of ranks up to 16, as many adapters as fit into 32;
// for the rows from the first to the last that has one of them, in 32s.
struct Passes {
  int rank, each, a[4], n, j, row0, rows;
  __device__ __forceinline__ bool take(const Adapters& who, int after) {
    j = n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = i < each && after != NO_MORE ? who.after(after) : NO_MORE;
      after = a[i];
      if (after != NO_MORE) ++n;
    }
    const int lane = threadIdx.x & 31;
    int lo = TL_N, hi = -1;
#pragma unroll
    for (int i = 0; i < TL_N / 32; ++i) {
      const int o = who.of[i];
      if (o >= 0 && (o == a[0] || o == a[1] || o == a[2] || o == a[3])) {
        lo = min(lo, lane + 32 * i);
        hi = lane + 32 * i;
      }
    }
    row0 = __reduce_min_sync(0xffffffffu, lo) & ~31;
    rows = ((__reduce_max_sync(0xffffffffu, hi) + 32) & ~31) - row0;
    return n > 0;
  }
  __device__ __forceinline__ bool begin(const Adapters& who, int r) {
    rank = r;
    each = r <= 16 ? 32 / r : 1;
    return take(who, -1);
  }
  __device__ __forceinline__ bool next(const Adapters& who) {
    if (each == 1 && j + 32 < rank) {
      j += 32;
      return true;
    }
    return take(who, each == 1 ? a[0] : each == 2 ? a[1] : a[3]);
  }
  // eights of the rank in this pass, and the adapter and place of one of them
  __device__ __forceinline__ int eights() const { return each == 1 ? min(4, (rank - j) / 8) : n * rank / 8; }
  __device__ __forceinline__ int adapter(int c) const {
    const int i = each == 1 ? 0 : each == 2 ? c >> 1 : c;
    return i == 0 ? a[0] : i == 1 ? a[1] : i == 2 ? a[2] : a[3];
  }
  __device__ __forceinline__ int place(int c) const { return each == 1 ? j + 8 * c : each == 2 ? 8 * (c & 1) : 0; }
};

// B (A x) of one output, of the rank's places where B is an infinity or NaN.
template <class T>
__device__ float lowrank_odd_term(const Lowrank& low, int K, int row, int co) {
  const int a = low.adapter[row];
  if (a < 0 || a >= low.n) return 0.f;
  const uint16_t* b = static_cast<const uint16_t*>(low.b) + ((size_t)a * K + co) * low.rank;
  const float* h = low.h + (size_t)row * low.rank;
  float s = 0.f;
  for (int j = 0; j < low.rank; ++j) {
    const float v = T::unpack(b[j]).x;
    if (!isfinite(v)) s = fmaf(v, h[j], s);
  }
  return s;
}

template <class T, bool GATHER, int LOW>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(TallShape<LOW>::kThreads, 1) products_tall_kernel(const TallParams p, const __grid_constant__ CUtensorMap map) {
  constexpr int STAGES = TallShape<LOW>::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* const low_smem = smem + STAGES * TL_B_BYTES;
  TallBars* const bars = reinterpret_cast<TallBars*>(low_smem + TallShape<LOW>::kLow);
  Ranges R;
  R.lo = reinterpret_cast<int*>(bars + 1);
  R.n = R.lo + p.E;
  R.end = R.n + p.E;
  const int warp = uni(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t b_smem = smem_u32(smem);
  const int rank = (int)(blockIdx.x & 1), first_tile = (int)(blockIdx.x >> 1), n_pairs = (int)(gridDim.x >> 1);
  // As in the kernel for few rows: after the one that writes A x, only the warps that read it wait.
  if (warp == 0) {
    if (!LOW) grid_dep_wait();
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
      mbar_init(smem_u32(&bars->d_empty[i]), 2 * TallShape<LOW>::kOutWarps + (LOW ? 1 : 0));
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bars->low_full[i]), 2 * TallShape<LOW>::kOutWarps);
      mbar_init(smem_u32(&bars->low_done[i]), 1);
    }
    bars->odd = 0;
    mbar_init(smem_u32(&bars->drain), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  } else if (warp == 2) {
    // (not before the kernel before has ended: it may still have to get tensor memory of its own)
    if (!LOW) grid_dep_wait();
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars->tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (!LOW || warp >= 12 || warp == 3) grid_dep_wait();
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
        stage_ts_f16(acc, tmem_u + a * TL_A_COLS, rows_desc(b_smem + s * TL_B_BYTES), idesc, kb ? 1u : 0u, smem_u32(&bars->b_empty[s]), smem_u32(&bars->a_empty[a]), leader);
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
  } else if (LOW && warp == 3 && rank == 0) {
    // ------------------------------------------------------------ MMA of the adapters' terms, for both CTAs
    int d = 0;
    uint32_t d_phase = 0, passes = 0;
    const uint32_t leader = elect_one(), low_u = (uint32_t)uni((int)smem_u32(low_smem)), tmem_u = (uint32_t)uni((int)tmem);
    Adapters who;
    Passes pass;
    for (int index = first_tile; ok && tall_tile(R, p.E, p.n_cp, index, rank, t); index += n_pairs) {
      who.load(p.low, t);
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->d_full[d]), d_phase));
      if (who.count() <= TL_LOW_MOST) {
        for (bool more = pass.begin(who, p.low.rank); ok && more; more = pass.next(who), ++passes) {
          const uint32_t slot = passes & 1u, b = low_u + slot * TL_LOW_BYTES;
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->low_full[slot]), passes >> 1 & 1u));
          if (!ok) break;
          tc_fence_after();
          const uint32_t idesc = (1u << 4) | (2u << 7) | (2u << 10) | ((uint32_t)(pass.rows >> 3) << 17) | ((256u >> 4) << 24);
#pragma unroll
          for (int part = 0; part < TL_LOW_PARTS; ++part)
            low_ss_tf32(tmem_u + TL_D0 + d * TL_N + pass.row0, rows_desc(b), rows_desc(b + TL_LOW_A + part * TL_LOW_B), idesc, (uint32_t)pass.eights(), leader);
          commit_on(smem_u32(&bars->low_done[slot]), leader);
          __syncwarp();
        }
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) arrive_at_first(smem_u32(&bars->d_empty[d]));
      if ((d ^= 1) == 0) d_phase ^= 1u;
    }
    if (passes) ok = mbar_wait(smem_u32(&bars->low_done[(passes - 1) & 1u]), (passes - 1) >> 1 & 1u) && ok;
    if (!ok && lane == 0) raise_status(p.status, 25);
  } else if (warp >= 4 && warp < 12) {
    // ------------------------------------------------------------ weights: thread m of a warpgroup is channel m of the tile
    const int m = ((int)threadIdx.x - 128) & 127, group = (warp - 4) >> 2;   // blocks group, group + 2, ... of a tile
    const int shift = (m >> 3) & 1 ? 8 : 0;
    const Powers pow = in_registers(p.pow);
    const uint32_t dst = tmem + ((uint32_t)(m & ~31) << 16);
    uint32_t base = 0;      // blocks of the tiles before
    uint32_t stored = ~0u;  // a block that is on its way to tensor memory; it is waited for when the next one has been expanded
    const uint4* src = nullptr;
    uint4 next[2];
    int index = first_tile;
    // A tile's first words are asked for while the tile before has its last expanded (840 tiles of 504 input channels and 29 rows 29.3 us; asked for
    // when the tile begins 35.7).
    auto begin_tile = [&] {
      if (!tall_tile(R, p.E, p.n_cp, index, rank, t)) return false;
      index += n_pairs;
      src = reinterpret_cast<const uint4*>(p.bits) + ((size_t)(t.e * p.n_mt + t.ct * 8 + (m >> 4)) * p.n_kb) * 32 + 4 * (m & 7) + 2 * group;
      next[0] = ld16(src);
      next[1] = ld16(src + 1);
      return true;
    };
    for (bool more = begin_tile(); ok && more; base += (uint32_t)nk) {
      for (int kb = 0; ok && kb < p.n_kb; ++kb) {
        const uint32_t w[2][4] = {{next[0].x >> shift, next[0].z >> shift, next[1].x >> shift, next[1].z >> shift},
                                  {next[0].y >> shift, next[0].w >> shift, next[1].y >> shift, next[1].w >> shift}};
        if (kb + 1 < p.n_kb) {
          next[0] = ld16(src + (size_t)(kb + 1) * 32);
          next[1] = ld16(src + (size_t)(kb + 1) * 32 + 1);
        } else {
          more = begin_tile();
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
    const int thread = (int)threadIdx.x - 384, m = thread & 127, turn = (warp - 12) >> 2;
    constexpr int OUTS = 32 * TallShape<LOW>::kOutWarps, STEP = OUTS / 4;   // columns: 32 for each set of four warps in turn
    int d = 0;
    uint32_t phase = 0, passes = 0;
    // A pass's B, of this CTA's channels, and A x, of its half of the rows (zeros: those of other adapters): from memory, and as the instruction
    // wants them.
    uint4 u[128 * 4 / OUTS], h[TL_HALF * 8 / OUTS];
    auto load = [&](const Passes& pass) {
      const int eights = pass.eights(), half = pass.rows / 2;
#pragma unroll
      for (int i = 0; i < 128 * 4 / OUTS; ++i) {
        const int row = (thread + i * OUTS) >> 2, c = thread & 3, co = t.ct * 128 + row;
        u[i] = make_uint4(0, 0, 0, 0);
        if (c < eights && co < p.K) u[i] = ld16(static_cast<const uint16_t*>(p.low.b) + ((size_t)pass.adapter(c) * p.K + co) * pass.rank + pass.place(c));
      }
#pragma unroll
      for (int i = 0; i < TL_HALF * 8 / OUTS; ++i) {
        const int row = (thread + i * OUTS) >> 3, c = thread & 7, at = pass.row0 + rank * half + row;
        h[i] = make_uint4(0, 0, 0, 0);
        if (row < half && at < t.n && (c >> 1) < eights && p.low.adapter[t.r0 + at] == pass.adapter(c >> 1))
          h[i] = ld16(p.low.h + (size_t)(t.r0 + at) * pass.rank + pass.place(c >> 1) + 4 * (c & 1));
      }
    };
    auto store = [&](int half, uint32_t slot) {
      uint8_t* const to = low_smem + slot * TL_LOW_BYTES;
#pragma unroll
      for (int i = 0; i < 128 * 4 / OUTS; ++i) {
        const int row = (thread + i * OUTS) >> 2, c = thread & 3;
        const float2 f[4] = {T::unpack(u[i].x), T::unpack(u[i].y), T::unpack(u[i].z), T::unpack(u[i].w)};
        float v[8];
        bool fine = true;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          v[q] = q & 1 ? f[q >> 1].y : f[q >> 1].x;
          if (!isfinite(v[q])) {   // (would reach the rows of other adapters; added by itself afterwards)
            v[q] = copysignf(TL_LOW_ODD, v[q]);
            fine = false;
          }
        }
        if (!fine) bars->odd = 1;
        *reinterpret_cast<float4*>(to + row * 128 + (((2 * c) ^ (row & 7)) << 4)) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(to + row * 128 + (((2 * c + 1) ^ (row & 7)) << 4)) = make_float4(v[4], v[5], v[6], v[7]);
      }
#pragma unroll
      for (int i = 0; i < TL_HALF * 8 / OUTS; ++i) {
        const int row = (thread + i * OUTS) >> 3, c = thread & 7;
        if (row >= half) break;
        uint32_t v[4] = {h[i].x, h[i].y, h[i].z, h[i].w};
        // 11 bits of each value at a time (the differences are exact); an infinity or NaN in the first
#pragma unroll
        for (int part = 0; part < TL_LOW_PARTS; ++part) {
          uint32_t top[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            top[q] = v[q] & 0xffffe000u;
            const float rest = __uint_as_float(v[q]) - __uint_as_float(top[q]);
            v[q] = isfinite(rest) ? __float_as_uint(rest) : 0u;
          }
          *reinterpret_cast<uint4*>(to + TL_LOW_A + part * TL_LOW_B + row * 128 + ((c ^ (row & 7)) << 4)) = make_uint4(top[0], top[1], top[2], top[3]);
        }
      }
    };
    // (the slot is free once the pass before the last has been added)
    auto slot_free = [&] { return __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->low_done[passes & 1u]), (passes >> 1 & 1u) ^ 1u)); };
    for (int index = first_tile; ok && tall_tile(R, p.E, p.n_cp, index, rank, t); index += n_pairs) {
      const int co = t.ct * 128 + m;
      float alpha = p.alpha[(size_t)t.e * p.n_mt * 16 + co];
      Adapters who;
      Passes pass;
      int n_low = 0;
      if (LOW) {   // while the sums are under way
        who.load(p.low, t);
        n_low = who.count();
        if (n_low && n_low <= TL_LOW_MOST) {
          pass.begin(who, p.low.rank);
          load(pass);
          ok = slot_free();
          if (ok) store(pass.rows / 2, passes & 1u);
        }
      }
      ok = __all_sync(0xffffffffu, ok && mbar_wait(smem_u32(&bars->d_full[d]), phase));
      tc_fence_after();
      const uint32_t src = tmem + ((uint32_t)(m & ~31) << 16) + TL_D0 + d * TL_N;
      if (LOW) {
        if (ok && n_low) {   // alpha S, back in place
          for (int c0 = 32 * turn; c0 < t.n; c0 += STEP) {
            uint32_t v[32];
            tmem_ld32(src + c0, v);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(alpha * __uint_as_float(v[i]));
            tmem_st32(src + c0, v);
          }
          tmem_st_wait();
        }
        if (n_low) alpha = 1.f;
        if (n_low && n_low <= TL_LOW_MOST) {
          for (bool more = true; ok && more;) {   // (this pass is in its slot)
            const uint32_t slot = passes++ & 1u;
            fence_proxy_async();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at_first(smem_u32(&bars->low_full[slot]));
            more = pass.next(who);
            if (more) {
              load(pass);
              ok = slot_free();
              if (ok) store(pass.rows / 2, passes & 1u);
            }
          }
          ok = __all_sync(0xffffffffu, ok && mbar_wait(smem_u32(&bars->low_done[(passes - 1) & 1u]), (passes - 1) >> 1 & 1u));
          tc_fence_after();
        }
        ok = bar_all<1, OUTS>(ok);   // (the warps go on, or give up, together; and all have said what is odd)
        if (ok && n_low && (n_low > TL_LOW_MOST || *reinterpret_cast<volatile int*>(&bars->odd))) {
          for (int c0 = 32 * turn; c0 < t.n; c0 += STEP)
            for (int c = c0; c < min(c0 + 32, t.n); c += 4) {
              uint32_t v[4];
              tmem_ld4(src + c, v);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (co < p.K && c + i < t.n) {
                  const int row = t.r0 + c + i;
                  const float term = n_low > TL_LOW_MOST ? lowrank_term<T>(p.low, p.K, row, co) : lowrank_odd_term<T>(p.low, p.K, row, co);
                  v[i] = __float_as_uint(__uint_as_float(v[i]) + term);
                }
              __syncwarp();
              tmem_st4(src + c, v);
            }
          tmem_st_wait();
        }
      }
      if (!ok) break;
      const long long to = (long long)t.r0 * p.ld_out + co;
      for (int c0 = 32 * turn; c0 < t.n; c0 += STEP) {
        uint32_t v[32];
        tmem_ld32(src + c0, v);
        const int n = co < p.K ? min(32, t.n - c0) : 0;
        const long long at = to + c0 * p.ld_out;
        if (p.out_type == SNN_OUT_F32) store_column(static_cast<float*>(p.out) + at, p.ld_out, n, alpha, v);
        else if (p.out_type == SNN_OUT_F16) store_column(static_cast<__half*>(p.out) + at, p.ld_out, n, alpha, v);
        else store_column(static_cast<__nv_bfloat16*>(p.out) + at, p.ld_out, n, alpha, v);
        __syncwarp();
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

template <class T, bool GATHER, int LOW>
cudaError_t tall_launch(const Products& p, const ProductCall& c, const CUtensorMap& map, int* launched) {
  static unsigned long long done = 0;
  cudaError_t e = allow_max_smem(products_tall_kernel<T, GATHER, LOW>, &done);
  if (e != cudaSuccess) return e;
  const TallParams q{p.bits, p.alpha, static_cast<const uint16_t*>(c.act), c.rows, c.offsets, c.out, c.ld_act, c.ld_out, c.act_rows, c.max_rows, p.E, p.C, p.K, p.n_mt, p.n_kb, c.out_type,
                     (p.K + 255) / 256, p.status_dev, c.low, powers()};
  const long long tiles = ((long long)c.max_rows / TL_N + (c.offsets ? min(p.E, c.max_rows) : 1)) * q.n_cp;
  const size_t smem = 1024 + TallShape<LOW>::kStages * TL_B_BYTES + TallShape<LOW>::kLow + sizeof(TallBars) + (size_t)p.E * 12;
  *launched += 1;
  return launch_dependent(products_tall_kernel<T, GATHER, LOW>, 2u * (unsigned)min(tiles, (long long)max(1, sm_count() / 2)), TallShape<LOW>::kThreads, smem,
                          c.stream, q, map);
}

template <class T>
cudaError_t tall_kind(const Products& p, const ProductCall& c, const CUtensorMap& map, int* launched) {
  // Four warps of outputs leave the weights' more of the SM, eight are faster at the operands of the passes (4096 rows of 4096 x 4096, four requests, rank
  // 16 101 and 106 us, rank 64 119 and 122, rank 128 161 and 149; an adapter of 16 for each row, rank 16 264 and 237, rank 64 616 and 518).
  if (c.low.adapter) return c.low.rank <= 32 ? tall_launch<T, false, 4>(p, c, map, launched) : tall_launch<T, false, 8>(p, c, map, launched);
  return c.rows ? tall_launch<T, true, 0>(p, c, map, launched) : tall_launch<T, false, 0>(p, c, map, launched);
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
