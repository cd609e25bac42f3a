// Projections in 8-bit floating point with a scale for each block of 128, many rows: the 5th-generation tensor cores.
#include "snn_products.h"

#include "snn_pairs.cuh"
#include "snn_products.cuh"
#include "snn_tc_common.cuh"

namespace snn {
namespace {

// out[row, co] = sum over blocks of 128 input channels of  xs[row, b] ws[co / 128, b] (x w)[row, co, b]:  D[128 or 256 rows x N channels] = x (M operand) * w^T (N
// operand) for one block at a time, each into a buffer of its own in tensor memory, from where eight warps add it, times its scales, to sums in
// registers (fp32).  Rows are the M operand so that a thread has one row: one factor for all of its channels of a block.  While they add one block up,
// the next ones are multiplied: two to four buffers.  Both operands come by TMA, the weights in the layout that they are kept in.
//   CG = 2, N = 256: a pair of CTAs (one instruction for both), 128 rows and half of the channels' weights in each.  An SM then reads 64 bytes a cycle of
//   operands, and as many arrive; alone with 128 x 256 it would be 96 and 96, more than shared memory gives.
//   CG = 1, N = 128 or 64: fewer rows, more tiles, for problems that would leave SMs without any; of 64 a tile may be shared by two or four CTAs of a cluster, each a
//   run of the input channels.  What bounds these is a block's waits, issues and commits: 300 to 400 cycles of one warp, so two warps do that in turns (one row of 4096 x
//   4096 11.0 and 10.7 us), and of narrow stages two blocks go together (8.7).
// 4096 rows of 4096 x 8192 take 112 us in a short run (2.45 PFLOP/s), 136 to 138 among other calls, each with inputs that the caches do not hold (2.0); 8192 rows 222 in a long run at the power
// limit (2.48).
constexpr int ST_ROWS = 128;          // of a CTA's tile
constexpr int ST_MAX_STAGES = 16;
constexpr int ST_OUT_WARPS = 8;
constexpr int ST_STAGING = 4096;      // of a warp: 32 rows of 128 bytes
// Scales: of four blocks at a time, of a tile's rows and of its two halves' channels; a warp brings them.  (Each four cost an L2 latency; where the warps of the sums
// waited for it themselves, that was 22 of 131 us on 4096 rows of 4096 x 8192.)
constexpr int ST_SCALES = 4, ST_SCALE_BYTES = ST_ROWS * 16 + 32;
// warps: 0 copies, 1 and 2 MMA (in turns: one takes 350 cycles for a block's waits, instructions and commits), 2 tensor memory, 3 scales, 4-11 sums and outputs

struct TallScaledParams {
  const float *w_scales, *x_scales;
  const int32_t* offsets;
  void* out;
  long long ld_scales, ld_out;
  int rows, E, C, K, n_kt, n_kb, out_type, n_ct, stages, stage, staging, region, box, split, fours, eights;   // rows of x in a stage and of a box; CTAs that share a tile; scales and outputs by 16 bytes
  int* status;
};
struct TallScaledBars {
  uint64_t full[ST_MAX_STAGES], empty[ST_MAX_STAGES], d_full[4], d_empty[4], scales_full[ST_SCALES], scales_empty[ST_SCALES], drain[2];
  uint32_t tmem;
};
template <int CG, int N, int BLOCKS>   // BLOCKS go through the stages and buffers together
struct TallScaledShape {
  static constexpr int kParts = CG;                                // instructions of N / CG channels for a block, each with buffers of its own
  static constexpr int kN = N / kParts, kBRows = kN / CG;          // channels of an instruction, and rows of the weights that each CTA has of them
  // A block's rows (a region of as many as a tile can have: the instruction reads 128, and what it makes of those behind them, other operands or outputs of before, is nobody's),
  // and its weights
  static int stage(int region) { return BLOCKS * (region * 128 + kParts * kBRows * 128); }
  static constexpr int kBuffers = BLOCKS == 2 ? 2 : 4, kColumns = kN * BLOCKS * kBuffers;   // of tensor memory
  static constexpr int kWarps = ST_OUT_WARPS / kParts;             // that read a buffer, in each CTA
  static constexpr int kFixed = 1024 + ST_SCALES * ST_SCALE_BYTES + (int)sizeof(TallScaledBars);
};

// Issued by the lanes for which `on` is not 0: D = A * B^T over 128 input channels in four steps of 32, then the commits: the stage is free (if `frees`), the buffer is
// full (if `fills`).
template <int CG>
__device__ __forceinline__ void block_e4m3(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t bar0, uint32_t bar1, uint32_t on, uint32_t frees, uint32_t fills);
template <>
__device__ __forceinline__ void block_e4m3<2>(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t bar0, uint32_t bar1, uint32_t on, uint32_t frees, uint32_t fills) {
  asm volatile(
      "{\n\t.reg .pred q, y, z;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "setp.ne.b32 q, %6, 0;\n\tsetp.ne.and.b32 z, %8, 0, q;\n\tsetp.ne.and.b32 y, %9, 0, q;\n\t"
      "add.u64 a1, %1, 2;\n\tadd.u64 a2, %1, 4;\n\tadd.u64 a3, %1, 6;\n\t"
      "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, 0;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a1, b1, %3, 1;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a2, b2, %3, 1;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a3, b3, %3, 1;\n\t"
      "@z tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%4], %7;\n\t"
      "@y tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%5], %7;\n\t}" ::"r"(d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(bar0), "r"(bar1), "r"(on), "h"((uint16_t)3), "r"(frees), "r"(fills)
      : "memory");
}
template <>
__device__ __forceinline__ void block_e4m3<1>(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t bar0, uint32_t bar1, uint32_t on, uint32_t frees, uint32_t fills) {
  asm volatile(
      "{\n\t.reg .pred q, y, z;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "setp.ne.b32 q, %6, 0;\n\tsetp.ne.and.b32 z, %7, 0, q;\n\tsetp.ne.and.b32 y, %8, 0, q;\n\t"
      "add.u64 a1, %1, 2;\n\tadd.u64 a2, %1, 4;\n\tadd.u64 a3, %1, 6;\n\t"
      "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a1, b1, %3, 1;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a2, b2, %3, 1;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a3, b3, %3, 1;\n\t"
      "@z tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%4];\n\t"
      "@y tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t}" ::"r"(d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(bar0), "r"(bar1), "r"(on), "r"(frees), "r"(fills)
      : "memory");
}
template <int CG>
__device__ __forceinline__ void commit_drain(uint32_t bar, uint32_t on) {
  if (CG == 2) commit_on(bar, on);
  else if (on) tc_commit(bar);
}
template <int CG>
__device__ __forceinline__ void copy_box(uint32_t dst, const void* map, int c, int row, uint32_t bar) {
  if (CG == 2) tma_rows(dst, map, c, row, at_first(bar));
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(c), "r"(row), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ uint4 lds16_at(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// Four neighbouring numbers, of which `n` are there, by one load if `whole`.  (One statement: where the two ways meet in code, the registers are moved, and
// the warp waits for the load.)
__device__ __forceinline__ void ld_four(const float* p, int n, int whole, float (&v)[4]) {
  asm volatile(
      "{\n\t.reg .pred a, b, c, d, e;\n\t"
      "setp.ne.s32 a, %6, 0;\n\tsetp.eq.s32 b, %6, 0;\n\t"
      "setp.gt.and.s32 c, %5, 1, b;\n\tsetp.gt.and.s32 d, %5, 2, b;\n\tsetp.gt.and.s32 e, %5, 3, b;\n\t"
      "@a ld.global.v4.f32 {%0, %1, %2, %3}, [%4];\n\t"
      "@b ld.global.f32 %0, [%4];\n\t"
      "@c ld.global.f32 %1, [%4 + 4];\n\t"
      "@d ld.global.f32 %2, [%4 + 8];\n\t"
      "@e ld.global.f32 %3, [%4 + 12];\n\t}"
      : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3])
      : "l"(p), "r"(n), "r"(whole));
}

// W columns of the warp's 32 lanes; load and wait are one statement.
template <int W>
__device__ __forceinline__ void tmem_ld_some(uint32_t taddr, uint32_t (&v)[W]);
template <>
__device__ __forceinline__ void tmem_ld_some<32>(uint32_t taddr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
        "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
        "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr)
      : "memory");
}
template <>
__device__ __forceinline__ void tmem_ld_some<64>(uint32_t taddr, uint32_t (&v)[64]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n\ttcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
        "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
        "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31]),
        "=r"(v[32]), "=r"(v[33]), "=r"(v[34]), "=r"(v[35]), "=r"(v[36]), "=r"(v[37]), "=r"(v[38]), "=r"(v[39]),
        "=r"(v[40]), "=r"(v[41]), "=r"(v[42]), "=r"(v[43]), "=r"(v[44]), "=r"(v[45]), "=r"(v[46]), "=r"(v[47]),
        "=r"(v[48]), "=r"(v[49]), "=r"(v[50]), "=r"(v[51]), "=r"(v[52]), "=r"(v[53]), "=r"(v[54]), "=r"(v[55]),
        "=r"(v[56]), "=r"(v[57]), "=r"(v[58]), "=r"(v[59]), "=r"(v[60]), "=r"(v[61]), "=r"(v[62]), "=r"(v[63])
      : "r"(taddr)
      : "memory");
}
// Two at a time, or one: of 128 sums a thread the former move registers about (4096 rows of 4096 x 8192 126 us and, one at a time, 112), of 64 and 32 the latter are slower
// (147 and 137, 192 and 183 us).
template <int W, bool TWO>
__device__ __forceinline__ void add_some(float* acc, const uint32_t (&v)[W], float f) {
  if (TWO) {
    const uint64_t g = pair_of(f, f);
#pragma unroll
    for (int i = 0; i < W; i += 2)
      asm("{\n\t.reg .b64 t, a;\n\tmov.b64 t, {%2, %3};\n\tmov.b64 a, {%0, %1};\n\tfma.rn.f32x2 a, t, %4, a;\n\tmov.b64 {%0, %1}, a;\n\t}" : "+f"(acc[i]), "+f"(acc[i + 1]) : "r"(v[i]), "r"(v[i + 1]), "l"(g));
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) acc[i] = fmaf(__uint_as_float(v[i]), f, acc[i]);
  }
}

// 16 bytes to the shared memory of a CTA of the cluster.
__device__ __forceinline__ void st_shared_of(uint32_t addr, int rank, float4 v) {
  uint32_t there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(there), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
struct ScaledTile {
  int e, r0, n, ct;   // expert, first row, rows, channel tile
};
struct ScaledRanges {
  int *lo, *n, *end;   // end[e] counts the row tiles up to and with expert e
};
// Tile `index` of the launch, channels of the same rows one after the other; `t.e` is where the search begins (indices rise).
template <int CG>
__device__ __forceinline__ bool scaled_tile(const ScaledRanges& R, int E, int n_ct, int index, ScaledTile& t) {
  const int q = index / n_ct;
  int e = t.e;
  while (e < E && q >= R.end[e]) ++e;
  t.e = uni(e);
  if (t.e >= E) return false;
  const int k = q - (t.e ? R.end[t.e - 1] : 0);
  t.ct = index - q * n_ct;
  t.r0 = uni(R.lo[t.e] + k * CG * ST_ROWS);
  t.n = uni(min(CG * ST_ROWS, R.n[t.e] - k * CG * ST_ROWS));
  return true;
}

template <int CG, int N, int BLOCKS>
__device__ __forceinline__ void scaled_tall_body(const TallScaledParams& p, const CUtensorMap& x_map, const CUtensorMap& w_map) {
  using S = TallScaledShape<CG, N, BLOCKS>;
  constexpr int NB = S::kBuffers, PARTS = S::kParts;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* const staging = smem + p.stages * p.stage;   // of the outputs, or what is received of the sums
  const uint32_t scales = smem_u32(staging) + p.staging;
  TallScaledBars* const bars = reinterpret_cast<TallScaledBars*>(staging + p.staging + ST_SCALES * ST_SCALE_BYTES);
  ScaledRanges R;
  R.lo = reinterpret_cast<int*>(bars + 1);
  R.n = R.lo + p.E;
  R.end = R.n + p.E;
  const int warp = uni(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t base = (uint32_t)uni((int)smem_u32(smem)), received = smem_u32(staging);
  const int rank = CG == 2 ? (int)(blockIdx.x & 1) : 0, shared_by = CG * p.split, first_tile = (int)blockIdx.x / shared_by, step = (int)gridDim.x / shared_by;
  if (warp == 0) {
    grid_dep_wait();
    // tiles of each expert, summed up: every lane a run of experts
    const int per = (p.E + 31) >> 5, e0 = lane * per, e1 = min(p.E, e0 + per);
    int count = 0;
    for (int e = e0; e < e1; ++e) {
      const int lo = p.offsets ? clamp_offset(p.offsets[e], p.rows) : 0;
      const int n = p.offsets ? max(clamp_offset(p.offsets[e + 1], p.rows) - lo, 0) : e ? 0 : p.rows;
      R.lo[e] = lo;
      R.n[e] = n;
      count += (n + CG * ST_ROWS - 1) / (CG * ST_ROWS);
    }
    int upto = count;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += v;
    }
    int end = upto - count;
    for (int e = e0; e < e1; ++e) R.end[e] = end += (R.n[e] + CG * ST_ROWS - 1) / (CG * ST_ROWS);
  } else if (warp == 1 && lane == 0) {
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(smem_u32(&bars->full[i]), 1);
      mbar_init(smem_u32(&bars->empty[i]), 1);
    }
    for (int i = 0; i < NB; ++i) {
      mbar_init(smem_u32(&bars->d_full[i]), 1);
      mbar_init(smem_u32(&bars->d_empty[i]), CG * S::kWarps);
    }
    for (int i = 0; i < ST_SCALES; ++i) {
      mbar_init(smem_u32(&bars->scales_full[i]), 1);
      mbar_init(smem_u32(&bars->scales_empty[i]), ST_OUT_WARPS);
    }
    mbar_init(smem_u32(&bars->drain[0]), 1);
    mbar_init(smem_u32(&bars->drain[1]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  } else if (warp == 2) {
    // (not before the kernel before has ended: it may still have to get tensor memory of its own)
    grid_dep_wait();
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem)), "n"(S::kColumns) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem)), "n"(S::kColumns) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  if (warp > 2 || warp == 1) grid_dep_wait();
  tc_fence_before();
  __syncthreads();
  if (CG == 2 || (N == 64 && p.split > 1)) pair_sync();
  tc_fence_after();
  grid_dep_launch();   // (only now: a dependent that has tensor memory before this CTA does would wait for it for good)
  const uint32_t tmem = bars->tmem;
  // blocks of input channels: all, or this CTA's share of them
  const int nk = p.n_kb, part = N == 64 ? (int)blockIdx.x % p.split : 0, kb_first = nk * part / p.split, kb_last = nk * (part + 1) / p.split;
  bool ok = true;
  ScaledTile t{};

  if (warp < 4) {
    if (N == 256) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0) {
      // ------------------------------------------------------------ copies: a stage is BLOCKS times 128 input channels of the rows and of the weights
      int s = 0, filled = 0;
      uint32_t phase = 0;
      const bool leader = elect_one();
      for (int index = first_tile; ok && scaled_tile<CG>(R, p.E, p.n_ct, index, t); index += step) {
        auto boxes = [&](int r) { return (min(max(t.n - r * ST_ROWS, 0), ST_ROWS) + p.box - 1) / p.box; };
        const int mine = boxes(rank);
        const uint32_t bytes = (uint32_t)(CG * PARTS * S::kBRows + (boxes(0) + (CG == 2 ? boxes(1) : 0)) * p.box) * 128u;   // of a block, of both CTAs
        // the weights: 64 rows of each of two tiles, one, or half of one
        const int kt = N == 256 ? 2 * t.ct : N == 128 ? t.ct : t.ct >> 1, w_half = CG == 2 ? rank * 64 : N == 64 ? (t.ct & 1) * 64 : 0;
        for (int kb = kb_first; kb < kb_last; kb += BLOCKS) {
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->empty[s]), phase ^ 1u));
          if (!ok) break;
          const uint32_t full = smem_u32(&bars->full[s]), dst = base + s * p.stage;
          const int blocks = min(BLOCKS, kb_last - kb);
          if (leader) {   // (one lane: copies of several lanes are issued one after the other, 100 cycles each)
            if (rank == 0) mbar_expect_tx(full, blocks * bytes);
#pragma unroll
            for (int u = 0; u < BLOCKS; ++u) {
              if (u >= blocks) break;
              for (int i = 0; i < mine; ++i)
                copy_box<CG>(dst + (u * p.region + i * p.box) * 128, &x_map, (kb + u) * 128, t.r0 + rank * ST_ROWS + i * p.box, full);
#pragma unroll
              for (int i = 0; i < PARTS; ++i)
                copy_box<CG>(dst + (BLOCKS * p.region + (u * PARTS + i) * S::kBRows) * 128, &w_map, 0, ((t.e * p.n_kt + min(kt + i, p.n_kt - 1)) * nk + kb + u) * 128 + w_half, full);
            }
          }
          __syncwarp();
          filled = min(filled + 1, p.stages);
          if (++s == p.stages) {
            s = 0;
            phase ^= 1u;
          }
        }
      }
      // both CTAs' copies in flight land before the pair ends, whatever became of the other warps
      for (int i = 0; rank == 0 && i < filled; ++i) {
        if (--s < 0) {
          s = p.stages - 1;
          phase ^= 1u;
        }
        ok = mbar_wait(smem_u32(&bars->full[s]), phase) && ok;
      }
      if (!ok && lane == 0) raise_status(p.status, 31);
    } else if (warp == 3) {
      // ------------------------------------------------------------ scales
      int s = 0;
      uint32_t phase = 0;
      for (int index = first_tile; ok && scaled_tile<CG>(R, p.E, p.n_ct, index, t); index += step) {
        const float* const ws = p.w_scales + (size_t)t.e * p.n_kt * nk;
        for (int kb = kb_first; kb < kb_last; kb += 4) {
          const int whole = p.fours && kb % 4 == 0 && kb + 4 <= kb_last;
          float v[4][4] = {}, w[4] = {};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = min(rank * ST_ROWS + 32 * i + lane, t.n - 1);
            ld_four(p.x_scales + (size_t)(t.r0 + row) * (size_t)p.ld_scales + kb, kb_last - kb, whole, v[i]);
          }
          if (lane < 2) ld_four(ws + (size_t)min((t.ct * N + lane * (N / 2)) >> 7, p.n_kt - 1) * nk + kb, kb_last - kb, whole, w);
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->scales_empty[s]), phase ^ 1u));
          if (!ok) break;
          const uint32_t to = scales + s * ST_SCALE_BYTES;
#pragma unroll
          for (int i = 0; i < 4; ++i) sts16(to + (32 * i + lane) * 16, make_uint4(__float_as_uint(v[i][0]), __float_as_uint(v[i][1]), __float_as_uint(v[i][2]), __float_as_uint(v[i][3])));
          if (lane < 2) sts16(to + ST_ROWS * 16 + lane * 16, make_uint4(__float_as_uint(w[0]), __float_as_uint(w[1]), __float_as_uint(w[2]), __float_as_uint(w[3])));
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&bars->scales_full[s]));
          if (++s == ST_SCALES) {
            s = 0;
            phase ^= 1u;
          }
        }
      }
      if (!ok && lane == 0) raise_status(p.status, 34);
    } else if (rank == 0) {
      // ------------------------------------------------------------ MMA, for both CTAs: every second stage
      const int turn = warp - 1;
      int s = turn, d = turn * PARTS, mine = turn;   // (the next of this warp's in the tile)
      uint32_t phase = 0, d_phase = 0;
      const uint32_t leader = elect_one(), tmem_u = (uint32_t)uni((int)tmem);
      const uint32_t idesc = (1u << 4) | ((uint32_t)(S::kN >> 3) << 17) | ((uint32_t)(CG * ST_ROWS >> 4) << 24);   // fp32 sums of e4m3 values
      const int units = (kb_last - kb_first + BLOCKS - 1) / BLOCKS;
      for (int index = first_tile; ok && scaled_tile<CG>(R, p.E, p.n_ct, index, t); index += step) {
        int unit = mine;
        for (; unit < units; unit += 2) {
          const int kb = kb_first + unit * BLOCKS;
          const uint32_t a = base + s * p.stage;
#pragma unroll
          for (int i = 0; i < PARTS; ++i) {
            // First the buffer: what was in it has been added up, and all before it, the stage's last contents among them (there are no fewer stages than buffers).  The
            // stage's barrier is then in the phase before or past it, whichever warp has waited for it in between; parities tell no more apart.
            ok = __all_sync(0xffffffffu, ok && mbar_wait(smem_u32(&bars->d_empty[d + i]), d_phase ^ 1u));
            if (i == 0) ok = __all_sync(0xffffffffu, ok && mbar_wait(smem_u32(&bars->full[s]), phase));
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int u = 0; u < BLOCKS; ++u) {
              if (kb + u >= kb_last) break;
              const uint32_t last = u + 1 == BLOCKS || kb + u + 1 == kb_last;
              block_e4m3<CG>(tmem_u + ((d + i) * BLOCKS + u) * S::kN, rows_desc(a + u * p.region * 128), rows_desc(a + (BLOCKS * p.region + (u * PARTS + i) * S::kBRows) * 128), idesc,
                             smem_u32(&bars->empty[s]), smem_u32(&bars->d_full[d + i]), leader, last && i + 1 == PARTS, last);
              __syncwarp();
            }
          }
          if (!ok) break;
          s += 2;
          if (s >= p.stages) {
            s -= p.stages;
            phase ^= 1u;
          }
          d += 2 * PARTS;
          if (d >= NB) {
            d -= NB;
            d_phase ^= 1u;
          }
        }
        mine = unit - units;
      }
      commit_drain<CG>(smem_u32(&bars->drain[turn]), leader);
      __syncwarp();
      ok = mbar_wait(smem_u32(&bars->drain[turn]), 0) && ok;
      if (!ok && lane == 0) raise_status(p.status, 32);
    }
  } else {
    // ------------------------------------------------------------ sums: a thread has a row and half of the tile's channels
    if (N == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    constexpr int A = N / 2;
    const int quarter = warp & 3, half = (warp - 4) >> 2, row = quarter * 32 + lane;
    const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16) + (PARTS == 1 ? half * A : 0), stage = smem_u32(staging) + (warp - 4) * ST_STAGING;
    int d = PARTS == 2 ? half : 0, g = 0;
    uint32_t d_phase = 0, g_phase = 0;
    for (int index = first_tile; ok && scaled_tile<CG>(R, p.E, p.n_ct, index, t); index += step) {
      const int n = t.n - rank * ST_ROWS, co0 = t.ct * N + half * A;   // rows of this CTA's (0 or less: none), first channel
      float acc[A];
#pragma unroll
      for (int i = 0; i < A; ++i) acc[i] = 0.f;
      for (int kb = kb_first; ok && kb < kb_last; kb += 4) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->scales_full[g]), g_phase));
        if (!ok) break;
        const uint32_t from = scales + g * ST_SCALE_BYTES;
        const uint4 xs = lds16_at(from + row * 16), ws = lds16_at(from + ST_ROWS * 16 + half * 16);
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->scales_empty[g]));
        if (++g == ST_SCALES) {
          g = 0;
          g_phase ^= 1u;
        }
        const float f[4] = {__uint_as_float(xs.x) * __uint_as_float(ws.x), __uint_as_float(xs.y) * __uint_as_float(ws.y), __uint_as_float(xs.z) * __uint_as_float(ws.z),
                            __uint_as_float(xs.w) * __uint_as_float(ws.w)};
#pragma unroll
        for (int i = 0; i < 4; i += BLOCKS) {
          if (kb + i >= kb_last) break;
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->d_full[d]), d_phase));
          if (!ok) break;
          tc_fence_after();
          constexpr int W = A < 64 ? A : 64;
#pragma unroll
          for (int u = 0; u < BLOCKS; ++u) {
            const bool last = u + 1 == BLOCKS || kb + i + u + 1 == kb_last;
#pragma unroll
            for (int c = 0; c < A; c += W) {
              uint32_t v[W];
              tmem_ld_some<W>(src + (d * BLOCKS + u) * S::kN + c, v);
              if (last && c + W == A) {   // (all of the buffer has been read)
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                  if (CG == 2) arrive_at_first(smem_u32(&bars->d_empty[d]));
                  else mbar_arrive(smem_u32(&bars->d_empty[d]));
                }
              }
              add_some<W, A < 128>(acc + c, v, f[i + u]);
            }
            if (last) break;
          }
          d += PARTS;
          if (d >= NB) {
            d -= NB;
            d_phase ^= 1u;
          }
        }
      }
      if (!ok) break;
      if (N == 64 && p.split > 1) {
        // This CTA's share of the sums goes to the CTAs that have the channels: [CTA from][fours of channels][row], 16 bytes each.
        const int fours = N / 4 / p.split;
#pragma unroll
        for (int i = 0; i < A / 4; ++i) {
          const int four = half * (A / 4) + i, to = four / fours;
          st_shared_of(received + (uint32_t)((part * fours + four - to * fours) * ST_ROWS + row) * 16u, to, make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]));
        }
        continue;
      }
      // Outputs through shared memory, 128 bytes of each row at a time (16-byte pieces, their order by the row: no bank twice), so that whole lines go out.
      const long long to = (long long)(t.r0 + rank * ST_ROWS + quarter * 32) * p.ld_out;
      const int rows = min(n - quarter * 32, 32);
      constexpr int PIECES = A < 64 ? 4 : 8;   // of 16-bit outputs
      auto pass = [&](auto words, int co, int each, int pieces) {   // `each` values in 16 bytes
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 8; ++q) sts16(stage + lane * 128 + ((q ^ (lane & 7)) << 4), words(q));
        __syncwarp();
        const int size = 16 / each;
        uint8_t* const first = static_cast<uint8_t*>(p.out) + (to + co) * size;
        if (p.eights && co + pieces * each <= p.K) {
          const int piece = lane & 7;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (lane >> 3);
            const uint4 v = lds16_at(stage + r * 128 + ((piece ^ (r & 7)) << 4));
            if (r < rows && piece < pieces) *reinterpret_cast<uint4*>(first + (long long)r * p.ld_out * size + piece * 16) = v;
          }
        } else {   // (neighbouring lanes, neighbouring values)
          for (int r = 0; r < rows; ++r)
            for (int e = lane; e < pieces * each && co + e < p.K; e += 32) {
              const uint32_t at = stage + r * 128 + ((e / each ^ (r & 7)) << 4) + e % each * size;
              if (size == 4) {
                uint32_t v;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
                reinterpret_cast<uint32_t*>(first + (long long)r * p.ld_out * 4)[e] = v;
              } else {
                uint16_t v;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
                reinterpret_cast<uint16_t*>(first + (long long)r * p.ld_out * 2)[e] = v;
              }
            }
        }
      };
      if (rows > 0 && co0 < p.K) {   // (the same for all lanes)
        if (p.out_type == SNN_OUT_F32) {
#pragma unroll
          for (int c = 0; c < A; c += 32)
            pass([&](int q) {
              const float* const a = acc + c + 4 * q;
              return make_uint4(__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(a[2]), __float_as_uint(a[3]));
            }, co0 + c, 4, 8);
        } else if (A >= 64) {
#pragma unroll
          for (int c = 0; c < A; c += 64)
            pass([&](int q) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) w[j] = pack_pair(p.out_type, make_float2(acc[c + 8 * q + 2 * j], acc[c + 8 * q + 2 * j + 1]));
              return make_uint4(w[0], w[1], w[2], w[3]);
            }, co0 + c, 8, PIECES);
        } else {   // (32 channels: half of a pass, the other half is not there)
          pass([&](int q) {
            uint32_t w[4] = {};
            if (q < 4)
#pragma unroll
              for (int j = 0; j < 4; ++j) w[j] = pack_pair(p.out_type, make_float2(acc[(8 * q + 2 * j) % A], acc[(8 * q + 2 * j + 1) % A]));
            return make_uint4(w[0], w[1], w[2], w[3]);
          }, co0, 8, PIECES);
        }
      }
    }
    if (!ok && lane == 0) raise_status(p.status, 33);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 2) {   // (the last arrivals here from the pair's MMAs)
    mbar_wait(smem_u32(&bars->drain[0]), 0);
    mbar_wait(smem_u32(&bars->drain[1]), 0);
  }
  __syncwarp();
  if (CG == 2) pair_sync();
  if (N == 64 && p.split > 1) {
    pair_sync();
    // the sums over the CTAs in their order; a thread has a row and every second four of this CTA's channels
    t = ScaledTile{};
    if (warp >= 4 && scaled_tile<CG>(R, p.E, p.n_ct, first_tile, t)) {
      const int row = ((int)threadIdx.x - 128) & 127, fours = N / 4 / p.split;
      for (int four = ((int)threadIdx.x - 128) >> 7; four < fours; four += 2) {
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < p.split; ++k) {
          const uint4 v = lds16_at(received + (uint32_t)((k * fours + four) * ST_ROWS + row) * 16u);
          sum.x += __uint_as_float(v.x), sum.y += __uint_as_float(v.y), sum.z += __uint_as_float(v.z), sum.w += __uint_as_float(v.w);
        }
        const int co = t.ct * N + (part * fours + four) * 4;
        const long long to = (long long)(t.r0 + row) * p.ld_out + co;
        if (row >= t.n) continue;
        if (p.eights && co + 4 <= p.K) {
          if (p.out_type == SNN_OUT_F32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to) = sum;
          else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + to) = make_uint2(pack_pair(p.out_type, make_float2(sum.x, sum.y)), pack_pair(p.out_type, make_float2(sum.z, sum.w)));
        } else {
          const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (co + j < p.K) store_out(p.out, p.out_type, to + j, v[j]);
        }
      }
    }
  }
  tc_fence_after();
  if (warp == 2) {
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kColumns) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kColumns) : "memory");
  }
}
constexpr int ST_THREADS = 128 + 32 * ST_OUT_WARPS;
__global__ void __launch_bounds__(ST_THREADS, 1)
    scaled_pair_kernel(const TallScaledParams p, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map) {
  scaled_tall_body<2, 256, 1>(p, x_map, w_map);
}
template <int N, int BLOCKS>
__global__ void __launch_bounds__(ST_THREADS, 1) scaled_single_kernel(const TallScaledParams p, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map) {
  scaled_tall_body<1, N, BLOCKS>(p, x_map, w_map);
}

bool rows_map(CUtensorMap* map, const void* base, long long columns, long long rows, long long ld, int box_rows, bool swizzled) {
  const MapEncoder encode = map_encoder();
  const cuuint64_t dims[2] = {(cuuint64_t)columns, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, steps[2] = {1, 1};
  return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG, int N, int BLOCKS, class Kernel>
cudaError_t tall_launch(Kernel kernel, unsigned long long* done, const Scaled& p, const ScaledCall& c, int split, int* launched) {
  using S = TallScaledShape<CG, N, BLOCKS>;
  cudaError_t e = allow_max_smem(kernel, done);
  if (e != cudaSuccess) return e;
  CUtensorMap x_map, w_map;
  // (few rows: no more than there are)
  const long long each = c.offsets ? ((long long)c.rows + min(p.E, c.rows) - 1) / min(p.E, c.rows) : c.rows;
  const auto pieces = [](long long rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : ST_ROWS; };
  const int region = pieces(c.rows), box = pieces(each);
  if (!rows_map(&x_map, c.act, p.C, c.rows, c.ld_act, box, true) ||
      !rows_map(&w_map, p.tiles, 128, (long long)p.E * p.n_kt * p.n_kb * 128, 128, S::kBRows, false))
    return cudaErrorInvalidValue;
  static_assert(N != 64 || ST_ROWS * N * 4 <= ST_OUT_WARPS * ST_STAGING, "what is received of the sums fits the staging");
  const int size = c.out_type == SNN_OUT_F32 ? 4 : 2, staging = ST_OUT_WARPS * ST_STAGING,
            fixed = S::kFixed + staging + p.E * 12;
  const TallScaledParams q{p.scales, c.scales, c.offsets, c.out, c.ld_scales, c.ld_out, c.rows, p.E, p.C, p.K, p.n_kt, p.n_kb, c.out_type, (p.K + N - 1) / N,
                           min(ST_MAX_STAGES, (kMaxDynSmem - fixed) / S::stage(region)), S::stage(region), staging, region, box, split, p.n_kb % 4 == 0 && c.ld_scales % 4 == 0 && ((uintptr_t)c.scales & 15) == 0,
                           c.ld_out * size % 16 == 0 && ((uintptr_t)c.out & 15) == 0, p.status_dev};
  if (q.stages < S::kBuffers / S::kParts || (split > 1 && N != 64)) return cudaErrorInvalidConfiguration;   // (the warps of the MMAs count on it; the first never happens up to 1024 experts)
  const long long tiles = ((long long)c.rows / (CG * ST_ROWS) + (c.offsets ? min(p.E, c.rows) : 1)) * q.n_ct;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)(CG * split);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.stream = c.stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cfg.gridDim = dim3((unsigned)(CG * split * min(tiles, (long long)max(1, sm_count() / (CG * split)))));
  cfg.blockDim = dim3(ST_THREADS);
  cfg.dynamicSmemBytes = (size_t)(fixed + q.stages * q.stage);
  *launched += 1;
  return cudaLaunchKernelEx(&cfg, kernel, q, x_map, w_map);
}

}  // namespace

cudaError_t scaled_tall(const Scaled& p, const ScaledCall& c, int shape, int split, int* launched) {
  static unsigned long long done[4] = {0, 0, 0, 0};
  if (shape == 256) return tall_launch<2, 256, 1>(scaled_pair_kernel, done, p, c, 1, launched);
  if (shape == 64) return tall_launch<1, 64, 2>(scaled_single_kernel<64, 2>, done + 1, p, c, split, launched);
  // Two blocks at a time save waits, but of more than 64 rows they leave two stages only (a row of 4096 x 4096 9.6 and 11.0 us, 4096 rows of 4096 x 8192 149 and 139).
  if (c.rows <= 64) return tall_launch<1, 128, 2>(scaled_single_kernel<128, 2>, done + 2, p, c, split, launched);
  return tall_launch<1, 128, 1>(scaled_single_kernel<128, 1>, done + 3, p, c, split, launched);
}

}  // namespace snn
