// A whole mixture of experts for a few tokens: router, first projections and activation in one launch, second projection and weighted sum in another.
#include "snn_products.h"

#include "snn_products.cuh"
#include "snn_route.cuh"
#include "snn_tc_common.cuh"

namespace snn {
namespace {

constexpr int MO_N = 8;    // rows of a piece
constexpr int MO_M = 32;   // output channels of a warp
constexpr int MO_FEW = SNN_MOE_FUSED_TOKENS * SNN_ROUTE_TOP_MAX;
constexpr int MO_PARTS = 3;   // bf16 numbers whose sum is a value between the projections: all of its 24 bits

// What lies in the workspace.
struct MoeWork {
  int32_t* total;            // pieces that there are
  int4* pieces;              // [slots]: expert, first row, rows
  int32_t* rows;             // [slots]: the token of each row
  float* shares;             // [slots]: the weight of each row in its token's sum
  int32_t *offsets, *ids, *slots;   // of a router in a launch of its own
  float* weights;
  uint16_t* h;               // [MO_PARTS][slots][hidden], bf16
};
long long carve(void* base, int E, int slots, int hidden, MoeWork* w) {
  long long at = 0;
  auto take = [&](long long bytes) {
    void* const p = static_cast<uint8_t*>(base) + at;
    at += (bytes + 15) & ~15ll;
    return p;
  };
  MoeWork m;
  m.total = static_cast<int32_t*>(take(4));
  m.pieces = static_cast<int4*>(take(slots * 16ll));
  m.rows = static_cast<int32_t*>(take(slots * 4ll));
  m.shares = static_cast<float*>(take(slots * 4ll));
  m.offsets = static_cast<int32_t*>(take((E + 1) * 4ll));
  m.ids = static_cast<int32_t*>(take(slots * 4ll));
  m.slots = static_cast<int32_t*>(take(slots * 4ll));
  m.weights = static_cast<float*>(take(slots * 4ll));
  m.h = static_cast<uint16_t*>(take(2ll * MO_PARTS * slots * hidden));
  if (w) *w = m;
  return at;
}

// Bits of two tiles of 16 output channels times 256 input channels (layout: snn_products.h).
struct TileBits {
  uint2 w[2][2];   // [tile][odd blocks of 64]
  __device__ __forceinline__ void load(const uint2* bits, int mt, int n_kb, int kb) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int o = 0; o < 2; ++o) w[m][o] = ld8(bits + ((size_t)(mt + m) * n_kb + kb) * 64 + 4 * o);
  }
  // the word of the 64 input channels from 64 j on
  __device__ __forceinline__ uint32_t word(int m, int j) const { return j < 2 ? w[m][j & 1].x : w[m][j & 1].y; }
};
// 64 input channels' products with P parts of 8 rows: the weights, expanded once, are the M operand.  The first part's go to `acc`, the others' to `low`.
template <class T, int P>
__device__ __forceinline__ void multiply64(float (&acc)[2][4], float (&low)[2][4], const TileBits& bits, int j, const uint4 (&b)[P][2], const Powers& pow) {
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const uint32_t u = bits.word(m, j);
      const uint32_t a0 = plus_minus<T>(u, 15 - 2 * s, pow), a1 = plus_minus<T>(u, 7 - 2 * s, pow);
      const uint32_t a2 = plus_minus<T>(u, 14 - 2 * s, pow), a3 = plus_minus<T>(u, 6 - 2 * s, pow);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const uint4& v = b[k][s >> 1];
        mma_16x8<T>(k ? low[m] : acc[m], a0, a1, a2, a3, s & 1 ? v.z : v.x, s & 1 ? v.w : v.y);
      }
    }
}

struct UpParams {
  const uint32_t* bits[2];   // gate (or null), up
  const float* alpha[2];
  const void* act;
  long long ld_act;
  int tokens, E, C, H, n_mt, n_kb, k_warps, fn, fused;
  RouteParams route;   // ids, weights and slots: of a router in a launch of its own, else unused
  MoeWork work;
  Powers pow;
};

__device__ __forceinline__ int ld_int(const int32_t* p) {
  int v;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ float ld_number(const float* p) {
  float v;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}
// A team of warps and nobody else (one warp: the barrier is its own).
__device__ __forceinline__ void team_sync(int team, int warps) {
  __syncwarp();
  if (warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(warps * 32) : "memory");
}

// First launch.  Up to SNN_MOE_FUSED_TOKENS tokens, every CTA routes for itself (a token a warp, then each choice finds its place among at most 128): less than a launch in
// front.  Then 8 rows of an expert times 32 output channels, of both the gate and the other projection, are an item of a team of warps, which share the input channels;
// a team has a run of items.  A team of one warp holds whole sums and needs nobody; larger ones, where there are few items, meet in shared memory.  What comes out
// behind the activation goes to memory as the sum of three bf16 numbers, whatever the outputs' type: with two, outputs of 16 bits are as near to the formula, but other ones than the
// rounded fp32 outputs wherever those lie next to a border.
// ANEW: sums begin anew every 256 channels, as in the second launch; for warps with more than two blocks of these.  The others' sums are cut 32 times at most; to begin anew
// costs them 2 to 4 % (64 tokens, 4 of 64 experts, 2048 -> 1024 -> 2048: 66.7 and 68.8 us).  3 tokens, 16384 channels, activations of sizes from 1 to 2^-12: fp32 outputs 3.0e-7 off, and
// 3.0e-6 in sums that go on; 64 tokens, 4096 channels, two blocks a warp: 3.1e-7 and 6.2e-7.
template <class T, bool GATE, bool ANEW>
__global__ void __launch_bounds__(256, 2) moe_up_kernel(const UpParams p) {
  constexpr int G = GATE ? 2 : 1, WIDE = G * MO_M;
  __shared__ float red_both[2][8][MO_N][WIDE + 1];
  __shared__ int s_ids[MO_FEW], s_rows[MO_FEW], s_first[MO_FEW], s_total;
  __shared__ float s_weights[MO_FEW];
  __shared__ int4 s_pieces[MO_FEW];
  __shared__ int s_offsets[SNN_EXPERTS_MAX + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int choices = p.tokens * p.route.k;
  Pieces counted{0, 0, 0};
  if (p.fused) {
    if (threadIdx.x == 0) s_total = 0;
    grid_dep_wait();
    if (warp < p.tokens) {
      RouteParams r = p.route;
      r.ids = s_ids;
      r.weights = s_weights;
      if (p.E <= 64) {
        float v[2];
        load_logits(r, warp, v);
        choose<2>(r, warp, v, nullptr, warp);
      } else if (p.E <= 256) {
        float v[8];
        load_logits(r, warp, v);
        choose<8>(r, warp, v, nullptr, warp);
      } else {
        float v[32];
        load_logits(r, warp, v);
        choose<32>(r, warp, v, nullptr, warp);
      }
    }
    __syncthreads();
    // An expert's choices are one piece (it has no more than 8); pieces in the order of their first choices, rows in that of the choices.
    auto place_choice = [&](int i, int id, int piece, int before, int same, int lower) {
      s_rows[lower + before] = i / p.route.k;
      if (before == 0) s_pieces[piece] = make_int4(id, lower, same, 0);
      if (blockIdx.x == 0) {
        p.work.rows[lower + before] = i / p.route.k;
        p.work.shares[lower + before] = s_weights[i];
        if (before == 0) p.work.pieces[piece] = make_int4(id, lower, same, 0);
      }
    };
    if (choices <= 32) {   // a lane has a choice
      if (warp == 0) {
        const int id = lane < choices ? s_ids[lane] : -1;
        const unsigned like = __match_any_sync(0xffffffffu, id), firsts = __ballot_sync(0xffffffffu, id >= 0 && __ffs(like) - 1 == lane);
        const int first = __ffs(like) - 1, before = __popc(like & ((1u << lane) - 1u)), same = __popc(like);
        int lower = 0;   // rows of the pieces before
        for (unsigned left = firsts; left; left &= left - 1) {
          const int q = __ffs(left) - 1, n = __shfl_sync(0xffffffffu, same, q);
          if (q < first) lower += n;
        }
        if (id >= 0) place_choice(lane, id, __popc(firsts & ((1u << first) - 1u)), before, same, lower);
        if (lane == 0) s_total = __popc(firsts);
      }
    } else {
      for (int i = threadIdx.x; i < choices; i += 256) {
        int first = 0;
        while (s_ids[first] != s_ids[i]) ++first;
        s_first[i] = first;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < choices; i += 256) {
        const int first = s_first[i];
        int before = 0, same = 0, lower = 0, piece = 0;
        for (int q = 0; q < choices; ++q) {
          const int f = s_first[q];
          same += f == first;
          before += f == first && q < i;
          lower += f < first && s_ids[f] >= 0;
          piece += f == q && q < first && s_ids[f] >= 0;
        }
        if (s_ids[i] >= 0) {
          place_choice(i, s_ids[i], piece, before, same, lower);
          if (before == 0) atomicAdd(&s_total, 1);   // (a count)
        }
      }
    }
    __syncthreads();
    counted.total = s_total;
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.work.total = s_total;
  } else {
    grid_dep_wait();
    for (int i = threadIdx.x; i <= p.E; i += 256) s_offsets[i] = ld_int(p.work.offsets + i);
    __syncthreads();
    counted = count_pieces(s_offsets, p.E, choices, MO_N);
    if (blockIdx.x == 0) {
      for (int i = threadIdx.x; i < choices; i += 256) {
        const int slot = p.work.slots[i];
        if (slot >= 0) p.work.shares[slot] = p.work.weights[i];
      }
      for (int i = warp; i < counted.total; i += 8) {
        int e, r0, n;
        find_piece(counted, s_offsets, p.E, choices, MO_N, i, &e, &r0, &n);
        if (lane == 0) p.work.pieces[i] = make_int4(e, r0, n, 0);
      }
      if (threadIdx.x == 0) *p.work.total = counted.total;
    }
  }
  grid_dep_launch();
  const Powers pow = in_registers(p.pow);
  const int team = warp / p.k_warps, kw = warp - team * p.k_warps, teams = 8 / p.k_warps, strips = (p.H + MO_M - 1) / MO_M;
  const long long items = (long long)counted.total * strips, all = (long long)gridDim.x * teams, me = (long long)blockIdx.x * teams + team;
  const int* const rows = p.fused ? s_rows : p.work.rows;
  const size_t step = (size_t)choices * p.H;
  // An item's rows and weights, as they are asked for: a block of input channels ahead, across the ends of items.
  struct Place {
    int piece, strip, e, r0, n;
    const uint16_t* x;
  };
  auto find = [&](Place& at) {
    if (p.fused) {
      const int4 v = s_pieces[at.piece];
      at.e = v.x, at.r0 = v.y, at.n = v.z;
    } else {
      find_piece(counted, s_offsets, p.E, choices, MO_N, at.piece, &at.e, &at.r0, &at.n);
    }
    at.x = g < at.n ? static_cast<const uint16_t*>(p.act) + (size_t)rows[at.r0 + g] * (size_t)p.ld_act + 8 * t : nullptr;
  };
  const long long first = items * me / all, last = items * (me + 1) / all;
  if (first >= last) return;
  TileBits bits[G], more[G];
  uint4 b[4][1][2];   // the rows of four blocks of 64: each is asked for again as soon as it has been used
  auto load_bits = [&](const Place& at, int kb) {
    const size_t expert = (size_t)at.e * p.n_mt * p.n_kb * 64 + 8 * g + t;
#pragma unroll
    for (int i = 0; i < G; ++i) more[i].load(reinterpret_cast<const uint2*>(p.bits[GATE ? i : 1]) + expert, 2 * at.strip, p.n_kb, kb);
  };
  auto load_rows = [&](const Place& at, int kb, int j) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = kb * 256 + j * 64 + 32 * h;
      b[j][0][h] = at.x && c + 8 * t < p.C ? ld16(at.x + c) : make_uint4(0, 0, 0, 0);
    }
  };
  Place now{(int)(first / strips), (int)(first % strips), 0, 0, 0, nullptr};
  find(now);
  load_bits(now, kw);
#pragma unroll
  for (int j = 0; j < 4; ++j) load_rows(now, kw, j);
  int turn = 0;
  for (long long item = first; item < last; ++item) {
    // the scales of the channels whose outputs this lane writes
    const size_t of = (size_t)now.e * p.n_mt * 16 + now.strip * MO_M;
    float alpha[G][4];
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q == 0 || p.k_warps == 1) alpha[i][q] = ld_number(p.alpha[GATE ? i : 1] + of + (p.k_warps == 1 ? g + 8 * q : lane));
    float acc[G][2][4] = {};
    Place then = now;
    for (int kb = kw; kb < p.n_kb; kb += p.k_warps) {
#pragma unroll
      for (int i = 0; i < G; ++i) bits[i] = more[i];
      int next = kb + p.k_warps;
      bool another = true;
      if (next >= p.n_kb) {   // the next item's
        next = kw;
        another = item + 1 < last;
        if (another && ++then.strip == strips) {
          then.strip = 0;
          ++then.piece;
          find(then);
        }
      }
      if (another) load_bits(then, next);
      float anew[G][2][4] = {};
      float (&part)[G][2][4] = ANEW ? anew : acc;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int i = 0; i < G; ++i) multiply64<T, 1>(part[i], part[i], bits[i], j, b[j], pow);
        if (another) load_rows(then, next, j);
      }
      if (ANEW)
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[i][m][q] += anew[i][m][q];
    }
    // 8 bits at a time, cut (the rests are exact), the last part rounded; an infinity or NaN in the first
    auto write = [&](int c, int co, float v) {
      uint16_t* const to = p.work.h + (size_t)(now.r0 + c) * p.H + co;
      float rest = v;
      const bool finite = fabsf(v) <= 3.402823466e38f;
#pragma unroll
      for (int k = 0; k < MO_PARTS; ++k) {
        const bool whole = k + 1 == MO_PARTS || !finite;
        const __nv_bfloat16 part = whole ? __float2bfloat16_rn(rest) : __ushort_as_bfloat16((unsigned short)(__float_as_uint(rest) >> 16));
        to[k * step] = __bfloat16_as_ushort(part);
        rest = finite ? rest - __bfloat162float(part) : 0.f;
      }
    };
    if (p.k_warps == 1) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = 2 * t + (q & 1), ch = 2 * m + (q >> 1), co = now.strip * MO_M + g + 8 * ch;
          const float v = activated(p.fn, alpha[0][ch] * acc[0][m][q]);
          if (c < now.n && co < p.H) write(c, co, GATE ? v * (alpha[G - 1][ch] * acc[G - 1][m][q]) : v);
        }
    } else {
      float (*const red)[MO_N][WIDE + 1] = red_both[turn] + team * p.k_warps;
      turn ^= 1;
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int q = 0; q < 4; ++q) red[kw][2 * t + (q & 1)][MO_M * i + 16 * m + g + 8 * (q >> 1)] = acc[i][m][q];
      team_sync(team, p.k_warps);   // (the other half of the buffer is for the next strip)
      const int co = now.strip * MO_M + lane;
      for (int c = kw; c < now.n; c += p.k_warps) {
        float sum[2] = {};
        for (int k = 0; k < p.k_warps; ++k) {
          sum[0] += red[k][c][lane];
          if (GATE) sum[1] += red[k][c][MO_M + lane];
        }
        const float v = activated(p.fn, alpha[0][0] * sum[0]);
        if (co < p.H) write(c, co, GATE ? v * (alpha[G - 1][0] * sum[1]) : v);
      }
    }
    now = then;
  }
}

struct DownParams {
  const uint32_t* bits;
  const float* alpha;
  const uint16_t* h;
  const int32_t *total, *rows;
  const int4* pieces;
  const float* shares;
  void* out;
  long long ld_out;
  int tokens, choices, C, K, n_mt, n_kb, out_type, cluster;
  Powers pow;
};

__device__ __forceinline__ void st_cluster(uint32_t addr, int rank, float v) {
  uint32_t there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ int4 ld_piece(const int4* p) {
  const uint4 v = ld16(p);
  return make_int4((int)v.x, (int)v.y, (int)v.z, (int)v.w);
}

// Second launch.  A cluster has 32 output channels; its warps share out all pieces of all experts, 256 input channels at a time, evenly: a run of them
// each.  The outputs are linear in what the pieces give, so a warp adds its run's products, times the scale and the row's share, to a table of its own [tokens][channels],
// and the tables are added up at the end, warp by warp, then CTA by CTA: each CTA sends every other one the outputs that that one writes (one barrier; read from there they took
// two, and 5 tokens with 3 of 60 experts of 1000 -> 1003 17.4 us instead of 16.3).  No atomics, no partial sums in memory, and
// no waiting until then.  The matrix instructions cut what they add: sums begin anew every 256 channels, and the lower two parts, which lie below what a sum of the first would keep of
// them, have sums of their own (fp32 outputs of 5 tokens, 1096 -> 1000 -> 1003, 1.8e-7 off, and 8.6e-7 where all three went into one; no slower).
// What bounds it, and the first launch, is no single unit: 64 tokens with 4 of 64 experts (2048 -> 1024 -> 2048) take 38 and 36 us with cold caches at 44 to 46 % of the issue slots, 34 to
// 41 % of the integer units, 20 and 33 % of the tensor pipe and 6 to 11 % of the memory rate.  The four warps of a scheduler wait for fixed latencies (1.5 to 1.7 of a warp's cycles
// for each that it issues), the multiplications' pipe (1.1 to 1.5), memory (0.9 to 1.2) and, in the first launch, instructions (1.5).  A lone warp takes 17.5 cycles for 256 weights and
// 8 rows in one part, 26 in two.  The same on the 5th-generation tensor cores (weights expanded into tensor memory, 128 channels a CTA, clusters of four to eight), then in two parts,
// took 0.5 us for 128 x 256 weights and came out even: 60.3 and 59.3 us for those 64 tokens, 18.5 and 18.3 for one (2 of 8, 4096): not kept.
constexpr int MO_LD = MO_M + 1, MO_TABLES = 9;
__global__ void __launch_bounds__(256, 2) moe_down_kernel(const DownParams p) {
  constexpr int LD = MO_LD, RING = 2;
  extern __shared__ int4 pieces[];
  int* const tokens = reinterpret_cast<int*>(pieces + p.choices);   // of the rows
  float* const shares = reinterpret_cast<float*>(tokens + p.choices);
  float* const sums = shares + p.choices;   // [8 warps][tokens][LD], then what the cluster's CTAs send (no more than one table: its sizes divide 32)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int strip = (int)blockIdx.x / p.cluster, rank = (int)blockIdx.x % p.cluster, table = p.tokens * LD;
  float* const mine = sums + warp * table;
  for (int i = lane; i < table; i += 32) mine[i] = 0.f;
  __syncwarp();
  if (p.cluster > 1) cluster_arrive();
  const Powers pow = in_registers(p.pow);
  grid_dep_wait();
  grid_dep_launch();
  // All at once, and more than there may be: one latency.
  const int total = ld_int(p.total);
  for (int i = threadIdx.x; i < p.choices; i += 256) {
    pieces[i] = ld_piece(p.pieces + i);
    tokens[i] = ld_int(p.rows + i);
    shares[i] = ld_number(p.shares + i);
  }
  __syncthreads();
  const long long units = (long long)total * p.n_kb;
  const int w = rank * 8 + warp, warps = p.cluster * 8;
  const long long first = units * w / warps, last = units * (w + 1) / warps;
  const size_t step = (size_t)p.choices * p.C;
  TileBits bits, more;
  uint4 b[RING][MO_PARTS][2];   // the rows of the next blocks of 64, as in the first launch
  struct Place {
    int piece, kb, e, r0, n;
    const uint16_t* x;
  };
  auto find = [&](Place& at) {
    const int4 v = pieces[at.piece];
    at.e = v.x, at.r0 = v.y, at.n = v.z;
    at.x = p.h + (size_t)(at.r0 + g) * p.C + 8 * t;
  };
  auto load_bits = [&](const Place& at) {
    more.load(reinterpret_cast<const uint2*>(p.bits) + (size_t)at.e * p.n_mt * p.n_kb * 64 + 8 * g + t, 2 * strip, p.n_kb, at.kb);
  };
  auto load_rows = [&](const Place& at, int j) {
#pragma unroll
    for (int k = 0; k < MO_PARTS; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = at.kb * 256 + j * 64 + 32 * h;
        b[j % RING][k][h] = g < at.n && c + 8 * t < p.C ? ld16(at.x + k * step + c) : make_uint4(0, 0, 0, 0);
      }
  };
  Place now{};
  if (first < last) {
    now.piece = (int)(first / p.n_kb);
    now.kb = (int)(first % p.n_kb);
    find(now);
    load_bits(now);
#pragma unroll
    for (int j = 0; j < RING; ++j) load_rows(now, j);
  }
  float acc[2][4] = {}, low[2][4] = {}, alpha[4];
  bool begins = true;
  for (long long unit = first; unit < last; ++unit) {
    if (begins) {   // the scales that its outputs need
#pragma unroll
      for (int q = 0; q < 4; ++q) alpha[q] = ld_number(p.alpha + (size_t)now.e * p.n_mt * 16 + strip * MO_M + g + 8 * q);
    }
    bits = more;
    Place then = now;
    const bool another = unit + 1 < last;
    if (++then.kb == p.n_kb) {
      then.kb = 0;
      ++then.piece;
      if (another) find(then);
    }
    if (another) load_bits(then);
    float part[2][4] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      multiply64<BF16, MO_PARTS>(part, low, bits, j, b[j % RING], pow);
      if (j + RING < 4) load_rows(now, j + RING);
      else if (another) load_rows(then, j + RING - 4);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[m][q] += part[m][q];
    begins = then.kb == 0 || !another;
    if (begins) {   // (a piece's rows are of different tokens)
#pragma unroll
      for (int q = 0; q < 2; ++q)
        if (2 * t + q < now.n) {
          const float share = shares[now.r0 + 2 * t + q];
          float* const to = mine + tokens[now.r0 + 2 * t + q] * LD + g;
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              float* const at = to + 16 * m + 8 * u;
              *at = fmaf(share, alpha[2 * m + u] * (acc[m][2 * u + q] + low[m][2 * u + q]), *at);
              acc[m][2 * u + q] = low[m][2 * u + q] = 0.f;
            }
        } else {
#pragma unroll
          for (int m = 0; m < 2; ++m) acc[m][q] = acc[m][2 + q] = low[m][q] = low[m][2 + q] = 0.f;
        }
      __syncwarp();
    }
    now = then;
  }
  __syncthreads();
  // A CTA adds its warps' tables up and sends every CTA of the cluster its share of the outputs, [CTA from][the share's place]; each then adds up what it has received.
  const int outputs = p.tokens * MO_M, most = (outputs + p.cluster - 1) / p.cluster;
  float* const received = sums + 8 * table;
  if (p.cluster > 1) cluster_wait();   // (they have all begun)
  for (int i = threadIdx.x; i < outputs; i += 256) {
    const float* const from = sums + i / MO_M * LD + i % MO_M;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += from[k * table];
    const int to = i / most;
    if (p.cluster > 1) st_cluster(smem_u32(received + rank * most + i - to * most), to, s);
    else received[i] = s;
  }
  if (p.cluster > 1) {
    cluster_arrive();
    cluster_wait();
  }
  for (int i = rank * most + (int)threadIdx.x; i < min(outputs, (rank + 1) * most); i += 256) {   // (in a cluster of one: what this thread has left there)
    const int token = i / MO_M, co = strip * MO_M + i % MO_M;
    float s = 0.f;
    for (int k = 0; k < p.cluster; ++k) s += received[k * most + i - rank * most];
    if (co < p.K) store_out(p.out, p.out_type, token * p.ld_out + co, s);
  }
}

cudaError_t down_launch(const DownParams& p, unsigned strips, cudaStream_t s) {
  static unsigned long long done = 0;
  const cudaError_t e = allow_max_smem(moe_down_kernel, &done);
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
  cfg.dynamicSmemBytes = (size_t)MO_TABLES * p.tokens * MO_LD * 4 + (size_t)p.choices * 24;
  return cudaLaunchKernelEx(&cfg, moe_down_kernel, p);
}

template <class T, bool ANEW>
cudaError_t up_launch(const UpParams& p, bool gate, unsigned ctas, cudaStream_t s) {
  return gate ? launch_dependent(moe_up_kernel<T, true, ANEW>, ctas, 256, 0, s, p) : launch_dependent(moe_up_kernel<T, false, ANEW>, ctas, 256, 0, s, p);
}
template <class T>
cudaError_t up_launch(const UpParams& p, bool gate, unsigned ctas, cudaStream_t s) {
  return p.n_kb > 2 * p.k_warps ? up_launch<T, true>(p, gate, ctas, s) : up_launch<T, false>(p, gate, ctas, s);
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
  u.pow = powers();
  // Pieces that the choices make at most: each expert of theirs has one that is not full.
  const long long ctas = 2ll * sm_count(), pieces = ((long long)choices + (long long)min(E, choices) * (MO_N - 1)) / MO_N, items = pieces * ((up.K + MO_M - 1) / MO_M);
  // Warps of a team: as many as have input channels, evenly, while all items run at once; and no fewer than four of two blocks each where they do not, whose loads hide one another's
  // latency.  Both sides (us, teams of 1, 2, 4 and 8; with two parts in place of three): one token, 2 of 8 experts of 4096: 42, 34, 23, 18; 16 tokens, 2 of 32, 4096 -> 2048: 85, 75, 68, 68; 64 tokens, 4 of 64, 2048 -> 1024:
  // 60.7, 61.2, 60.0, 61.3; 8 tokens, 2 of 64, 1024 -> 2048: 25.7, 18.9, 19.5; 5 tokens, 3 of 60, 1096 -> 1000, five blocks: 19.2, 14.5, 16.0.
  u.k_warps = 1;
  for (int k = 2; k <= min(8, up.n_kb); k *= 2)
    if (2 * ((up.n_kb + k - 1) / k) * k <= 3 * up.n_kb && (items * k <= 8 * ctas || k <= min(4, up.n_kb / 2))) u.k_warps = k;
  const unsigned grid = (unsigned)min(ctas, (items + 8 / u.k_warps - 1) / (8 / u.k_warps));
  e = c.act_type == SNN_ACT_F16 ? up_launch<F16>(u, c.gate != nullptr, grid, c.stream) : up_launch<BF16>(u, c.gate != nullptr, grid, c.stream);
  *launched += 1;
  if (e != cudaSuccess) return e;
  DownParams d{down.bits, down.alpha, u.work.h, u.work.total, u.work.rows, u.work.pieces, u.work.shares, c.out, c.ld_out, c.tokens, choices, down.C, down.K, down.n_mt, down.n_kb,
               c.out_type, 1, powers()};
  const int strips = (down.K + MO_M - 1) / MO_M;
  while (d.cluster < 8 && strips * d.cluster * 2 <= ctas && d.cluster * 8 < pieces * down.n_kb) d.cluster *= 2;
  *launched += 1;
  return down_launch(d, (unsigned)strips, c.stream);
}

}  // namespace snn
