// A whole mixture of experts for a few tokens: router, first projections and activation in one launch, second projection and weighted sum in another.
#include "snn_products.h"

#include "snn_products.cuh"
#include "snn_route.cuh"
#include "snn_tc_common.cuh"

namespace snn {
namespace {

constexpr int MO_N = 8;    // rows of a piece
constexpr int MO_M = 32;   // output channels of a warp

// What lies in the workspace.
struct MoeWork {
  int32_t *offsets, *rows;   // [E + 1], [slots]
  float* shares;             // [slots]: the weight of each row in its token's sum
  int32_t *ids, *slots;      // [tokens][top_k], of a router in a launch of its own
  float* weights;
  uint16_t* h;               // [parts][slots][hidden], bf16
};
long long carve(void* base, int E, int slots, int hidden, MoeWork* w) {
  long long at = 0;
  auto take = [&](long long bytes) {
    void* const p = static_cast<uint8_t*>(base) + at;
    at += (bytes + 15) & ~15ll;
    return p;
  };
  MoeWork m;
  m.offsets = static_cast<int32_t*>(take((E + 1) * 4ll));
  m.rows = static_cast<int32_t*>(take(slots * 4ll));
  m.shares = static_cast<float*>(take(slots * 4ll));
  m.ids = static_cast<int32_t*>(take(slots * 4ll));
  m.slots = static_cast<int32_t*>(take(slots * 4ll));
  m.weights = static_cast<float*>(take(slots * 4ll));
  m.h = static_cast<uint16_t*>(take(6ll * slots * hidden));
  if (w) *w = m;
  return at;
}

// Products of 256 input channels: 32 output channels (two tiles) times 8 rows; bits and rows as in the kernel for few rows.
struct Bits32 {
  uint2 w[2][2];   // [tile][odd blocks of 64]
  __device__ __forceinline__ void load(const uint2* bits, int mt, int n_kb, int kb) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int o = 0; o < 2; ++o) w[m][o] = ld8(bits + ((size_t)(mt + m) * n_kb + kb) * 64 + 4 * o);
  }
  // word j: the 64 input channels from 64 j on
  __device__ __forceinline__ uint32_t word(int m, int j) const { return j < 2 ? w[m][j & 1].x : w[m][j & 1].y; }
};
template <class T>
__device__ __forceinline__ void multiply64(float (&acc)[2][4], const Bits32& bits, int j, const uint4 (&b)[2], const Powers& pow) {
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const uint4& v = b[s >> 1];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const uint32_t u = bits.word(m, j);
      const uint32_t a0 = plus_minus<T>(u, 15 - 2 * s, pow), a1 = plus_minus<T>(u, 7 - 2 * s, pow);
      const uint32_t a2 = plus_minus<T>(u, 14 - 2 * s, pow), a3 = plus_minus<T>(u, 6 - 2 * s, pow);
      mma_16x8<T>(acc[m], a0, a1, a2, a3, s & 1 ? v.z : v.x, s & 1 ? v.w : v.y);
    }
  }
}

struct UpParams {
  const uint32_t* bits[2];   // gate (or null), up
  const float* alpha[2];
  const void* act;
  long long ld_act;
  int tokens, E, C, H, n_mt, n_kb, k_warps, fn, parts, fused;
  RouteParams route;   // ids, weights and slots: of a router in a launch of its own, else unused
  MoeWork work;
  Powers pow;
};

// First launch.  Up to SNN_MOE_FUSED_TOKENS tokens, every CTA routes for itself (a token a warp): less than a launch in front.  Then as in the kernel for few rows: 8 rows
// of an expert times 32 output channels a warp, of both the gate and the other projection, input channels split over the warps; the sums meet in shared memory,
// and what comes of them behind the activation goes out as the sum of `parts` bf16 numbers.
template <class T, bool GATE>
__global__ void __launch_bounds__(256, 2) moe_up_kernel(const UpParams p) {
  constexpr int WIDE = (GATE ? 2 : 1) * MO_M;
  __shared__ float red_both[2][8][MO_N][WIDE + 1];
  __shared__ int s_ids[SNN_MOE_FUSED_TOKENS * SNN_ROUTE_TOP_MAX], s_rows[SNN_MOE_FUSED_TOKENS * SNN_ROUTE_TOP_MAX], s_slots[SNN_MOE_FUSED_TOKENS * SNN_ROUTE_TOP_MAX];
  __shared__ float s_weights[SNN_MOE_FUSED_TOKENS * SNN_ROUTE_TOP_MAX];
  __shared__ int part[8];
  extern __shared__ int s_experts[];   // offsets [E + 1], mask [E][2]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kw = warp % p.k_warps, mw = warp / p.k_warps, m_warps = 8 / p.k_warps, n_groups = (p.H + MO_M * m_warps - 1) / (MO_M * m_warps);
  const int *offsets = p.work.offsets, *rows = p.work.rows;
  const int choices = p.tokens * p.route.k;
  if (p.fused) {
    uint32_t* const mask = reinterpret_cast<uint32_t*>(s_experts + p.E + 1);
    for (int i = threadIdx.x; i < 2 * p.E; i += 256) mask[i] = 0;
    RouteParams r = p.route;
    r.ids = s_ids;
    r.weights = s_weights;
    r.rows = s_rows;
    r.slots = s_slots;
    __syncthreads();
    grid_dep_wait();
    if (warp < p.tokens) {
      if (p.E <= 64) {
        float v[2];
        load_logits(r, warp, v);
        choose<2>(r, warp, v, mask, warp);
      } else if (p.E <= 256) {
        float v[8];
        load_logits(r, warp, v);
        choose<8>(r, warp, v, mask, warp);
      } else {
        float v[32];
        load_logits(r, warp, v);
        choose<32>(r, warp, v, mask, warp);
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.E; e += 256) s_experts[e] = __popc(mask[2 * e]);
    __syncthreads();
    const int total = scan_counts(s_experts, p.E, part);
    if (threadIdx.x == 0) s_experts[p.E] = total;
    place(r, mask, s_experts, 0, p.tokens);
    __syncthreads();
    if (blockIdx.x == 0) {
      for (int e = threadIdx.x; e <= p.E; e += 256) p.work.offsets[e] = s_experts[e];
      for (int i = threadIdx.x; i < choices; i += 256)
        if (s_slots[i] >= 0) {
          p.work.rows[s_slots[i]] = i / p.route.k;
          p.work.shares[s_slots[i]] = s_weights[i];
        }
    }
    offsets = s_experts;
    rows = s_rows;
  } else {
    grid_dep_wait();
    if (blockIdx.x == 0)
      for (int i = threadIdx.x; i < choices; i += 256) {
        const int slot = p.work.slots[i];
        if (slot >= 0) p.work.shares[slot] = p.work.weights[i];
      }
  }
  grid_dep_launch();
  const Powers pow = in_registers(p.pow);
  const Pieces pieces = count_pieces(offsets, p.E, choices, MO_N);
  const long long items = (long long)pieces.total * n_groups;
  long long item = items * blockIdx.x / gridDim.x;
  const long long last = items * (blockIdx.x + 1) / gridDim.x;
  int turn = 0;
  while (item < last) {
    const int piece = (int)(item / n_groups), group0 = (int)(item - (long long)piece * n_groups);
    const int group1 = (int)min((long long)n_groups, group0 + (last - item));
    item += group1 - group0;
    int e, r0, n;
    find_piece(pieces, offsets, p.E, choices, MO_N, piece, &e, &r0, &n);
    const uint16_t* x = nullptr;
    if (g < n) x = static_cast<const uint16_t*>(p.act) + (size_t)rows[r0 + g] * (size_t)p.ld_act + 8 * t;
    const size_t expert = (size_t)e * p.n_mt * p.n_kb * 64 + 8 * g + t;
    for (int group = group0; group < group1; ++group) {
      float acc[GATE ? 2 : 1][2][4] = {};
      const int mt = min(2 * (group * m_warps + mw), p.n_mt - 2);
      for (int kb = kw; kb < p.n_kb; kb += p.k_warps) {
        Bits32 bits[GATE ? 2 : 1];
#pragma unroll
        for (int i = 0; i < (GATE ? 2 : 1); ++i) bits[i].load(reinterpret_cast<const uint2*>(p.bits[GATE ? i : 1]) + expert, mt, p.n_kb, kb);
        uint4 b[4][2];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int c = kb * 256 + j * 64 + 32 * h;
            b[j][h] = x && c + 8 * t < p.C ? ld16(x + c) : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
        for (int i = 0; i < (GATE ? 2 : 1); ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) multiply64<T>(acc[i], bits[i], j, b[j], pow);
      }
      float (*const red)[MO_N][WIDE + 1] = red_both[turn];
      turn ^= 1;
#pragma unroll
      for (int i = 0; i < (GATE ? 2 : 1); ++i)
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int q = 0; q < 4; ++q) red[warp][2 * t + (q & 1)][MO_M * i + 16 * m + g + 8 * (q >> 1)] = acc[i][m][q];
      __syncthreads();   // (the other half of the buffer is for the next strip)
      const int width = MO_M * m_warps;
      for (int i = threadIdx.x; i < width * n; i += 256) {
        const int m = i & (width - 1), c = i / width, co = group * width + m;
        if (co >= p.H) continue;
        float s[2] = {};
        for (int k = 0; k < p.k_warps; ++k) {
          const float* const from = red[(m / MO_M) * p.k_warps + k][c] + m % MO_M;
          s[0] += from[0];
          if (GATE) s[1] += from[MO_M];
        }
        const size_t of = (size_t)e * p.n_mt * 16 + co;
        const float v = GATE ? activated(p.fn, p.alpha[0][of] * s[0]) * (p.alpha[1][of] * s[1]) : activated(p.fn, p.alpha[1][of] * s[0]);
        // 8 bits at a time, cut (the rests are exact), the last part rounded; an infinity or NaN in the first
        uint16_t* const to = p.work.h + (size_t)(r0 + c) * p.H + co;
        const size_t step = (size_t)choices * p.H;
        float rest = v;
        const bool finite = fabsf(v) <= 3.402823466e38f;
        for (int k = 0; k < p.parts; ++k) {
          const bool whole = k + 1 == p.parts || !finite;
          const __nv_bfloat16 b = whole ? __float2bfloat16_rn(rest) : __ushort_as_bfloat16((unsigned short)(__float_as_uint(rest) >> 16));
          to[k * step] = __bfloat16_as_ushort(b);
          rest = finite ? rest - __bfloat162float(b) : 0.f;
        }
      }
    }
  }
}

struct DownParams {
  const uint32_t* bits;
  const float* alpha;
  const uint16_t* h;
  const int32_t *offsets, *rows;
  const float* shares;
  void* out;
  long long ld_out;
  int tokens, choices, E, C, K, n_mt, n_kb, out_type, cluster;
  Powers pow;
};

__device__ __forceinline__ float ld_cluster(uint32_t addr, int rank) {
  uint32_t there;
  float v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(there) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Second launch.  A cluster has 32 output channels; its warps share out all pieces of all experts, 256 input channels at a time, evenly: a run of them
// each.  The outputs are linear in what the pieces give, so a warp adds its run's products, times the scale and the row's share, to a table of its own [tokens][32],
// and the tables are added up at the end, warp by warp, CTA by CTA (through distributed shared memory).  No atomics, no partial sums in memory, and
// no waiting until then.
constexpr int MO_LD = MO_M + 1;
template <int PARTS>
__global__ void __launch_bounds__(256, 2) moe_down_kernel(const DownParams p) {
  extern __shared__ float sums[];   // [8][tokens][MO_LD]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int strip = (int)blockIdx.x / p.cluster, rank = (int)blockIdx.x % p.cluster, table = p.tokens * MO_LD;
  float* const mine = sums + warp * table;
  for (int i = lane; i < table; i += 32) mine[i] = 0.f;
  __syncwarp();
  const Powers pow = in_registers(p.pow);
  grid_dep_wait();
  grid_dep_launch();
  const Pieces pieces = count_pieces(p.offsets, p.E, p.choices, MO_N);
  const long long units = (long long)pieces.total * p.n_kb;
  const int w = rank * 8 + warp, warps = p.cluster * 8;
  long long unit = units * w / warps;
  const long long last = units * (w + 1) / warps;
  const size_t step = (size_t)p.choices * p.C;
  while (unit < last) {
    const int piece = (int)(unit / p.n_kb), kb0 = (int)(unit - (long long)piece * p.n_kb);
    const int kb1 = (int)min((long long)p.n_kb, kb0 + (last - unit));
    unit += kb1 - kb0;
    int e, r0, n;
    find_piece(pieces, p.offsets, p.E, p.choices, MO_N, piece, &e, &r0, &n);
    const uint2* const bits = reinterpret_cast<const uint2*>(p.bits) + (size_t)e * p.n_mt * p.n_kb * 64 + 8 * g + t;
    const uint16_t* const x = p.h + (size_t)(r0 + g) * p.C + 8 * t;
    float acc[2][4] = {};
    for (int kb = kb0; kb < kb1; ++kb) {
      Bits32 b32;
      b32.load(bits, 2 * strip, p.n_kb, kb);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint4 b[PARTS][2];
#pragma unroll
        for (int k = 0; k < PARTS; ++k)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int c = kb * 256 + j * 64 + 32 * h;
            b[k][h] = g < n && c + 8 * t < p.C ? ld16(x + k * step + c) : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
        for (int k = 0; k < PARTS; ++k) multiply64<BF16>(acc, b32, j, b[k], pow);
      }
    }
    // (a piece's rows are of different tokens)
    const float* const alpha = p.alpha + (size_t)e * p.n_mt * 16 + strip * MO_M;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int c = 2 * t + q;
      if (c < n) {
        const float share = p.shares[r0 + c];
        float* const to = mine + p.rows[r0 + c] * MO_LD;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int ch = 16 * m + 8 * u + g;
            to[ch] = fmaf(share, alpha[ch] * acc[m][2 * u + q], to[ch]);
          }
      }
    }
    __syncwarp();
  }
  __syncthreads();
  for (int i = threadIdx.x; i < table; i += 256) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += sums[k * table + i];
    sums[i] = s;   // (read by this thread alone before)
  }
  if (p.cluster > 1) cluster_sync();
  else __syncthreads();
  for (int i = rank * 256 + (int)threadIdx.x; i < p.tokens * MO_M; i += p.cluster * 256) {
    const int token = i / MO_M, ch = i % MO_M, co = strip * MO_M + ch;
    float s = 0.f;
    for (int k = 0; k < p.cluster; ++k) s += p.cluster > 1 ? ld_cluster(smem_u32(sums + token * MO_LD + ch), k) : sums[token * MO_LD + ch];
    if (co < p.K) store_out(p.out, p.out_type, token * p.ld_out + co, s);
  }
  if (p.cluster > 1) cluster_sync();   // (nobody ends while its table is read)
}

template <int PARTS>
cudaError_t down_launch(const DownParams& p, unsigned strips, cudaStream_t s) {
  static unsigned long long done = 0;
  const cudaError_t e = allow_max_smem(moe_down_kernel<PARTS>, &done);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cfg.gridDim = dim3(strips * (unsigned)p.cluster);
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = (size_t)8 * p.tokens * MO_LD * 4;
  return cudaLaunchKernelEx(&cfg, moe_down_kernel<PARTS>, p);
}

template <class T>
cudaError_t up_launch(const UpParams& p, bool gate, unsigned ctas, cudaStream_t s) {
  const size_t smem = p.fused ? (size_t)(3 * p.E + 1) * 4 : 0;
  return gate ? launch_dependent(moe_up_kernel<T, true>, ctas, 256, smem, s, p) : launch_dependent(moe_up_kernel<T, false>, ctas, 256, smem, s, p);
}

}  // namespace

long long moe_work_bytes(const Products& up, int tokens, int top_k) { return carve(nullptr, up.E, tokens * top_k, up.K, nullptr); }

cudaError_t moe_forward(const MoeCall& c, int* launched) {
  const Products &up = *c.up, &down = *c.down;
  const int choices = c.tokens * c.top_k, E = up.E;
  UpParams u{};
  carve(c.work, E, choices, up.K, &u.work);
  u.fused = c.tokens <= SNN_MOE_FUSED_TOKENS;
  u.route = RouteParams{c.logits, c.ld_logits, c.logits_type, c.tokens, E, c.top_k, c.normalise, 0, u.work.ids, u.work.weights, u.work.offsets, u.work.rows, u.work.slots, nullptr};
  cudaError_t e = cudaSuccess;
  if (!u.fused) {
    const RouteCall r{c.logits, c.logits_type, c.tokens, E, c.top_k, c.normalise, c.ld_logits, u.work.ids, u.work.weights, u.work.offsets, u.work.rows, u.work.slots, nullptr, c.stream};
    e = route_forward(r, launched);
    if (e != cudaSuccess) return e;
  }
  u.bits[0] = c.gate ? c.gate->bits : nullptr;
  u.alpha[0] = c.gate ? c.gate->alpha : nullptr;
  u.bits[1] = up.bits;
  u.alpha[1] = up.alpha;
  u.act = c.act;
  u.ld_act = c.ld_act;
  u.tokens = c.tokens;
  u.E = E;
  u.C = up.C;
  u.H = up.K;
  u.n_mt = up.n_mt;
  u.n_kb = up.n_kb;
  u.fn = c.fn;
  u.parts = c.out_type == SNN_OUT_F32 ? 3 : 2;
  u.pow = powers();
  // (as in the kernel for few rows: all warps on one strip, unless there are not so many blocks of input channels, and more strips than CTAs)
  const long long ctas = 2ll * sm_count(), pieces = ((long long)choices + (long long)min(E, choices) * (MO_N - 1)) / MO_N;
  auto items = [&](int k) { return pieces * ((up.K + 8 / k * MO_M - 1) / (8 / k * MO_M)); };
  u.k_warps = 8;
  while (u.k_warps > up.n_kb && items(u.k_warps) > ctas) u.k_warps /= 2;
  const unsigned grid = (unsigned)min(ctas, items(u.k_warps));
  e = c.act_type == SNN_ACT_F16 ? up_launch<F16>(u, c.gate != nullptr, grid, c.stream) : up_launch<BF16>(u, c.gate != nullptr, grid, c.stream);
  *launched += 1;
  if (e != cudaSuccess) return e;
  DownParams d{down.bits, down.alpha, u.work.h, u.work.offsets, u.work.rows, u.work.shares, c.out, c.ld_out, c.tokens, choices, E, down.C, down.K, down.n_mt, down.n_kb, c.out_type, 1, powers()};
  const int strips = (down.K + MO_M - 1) / MO_M;
  while (d.cluster < 8 && strips * d.cluster * 2 <= ctas && d.cluster * 8 < pieces * down.n_kb) d.cluster *= 2;
  *launched += 1;
  return u.parts == 3 ? down_launch<3>(d, (unsigned)strips, c.stream) : down_launch<2>(d, (unsigned)strips, c.stream);
}

}  // namespace snn
