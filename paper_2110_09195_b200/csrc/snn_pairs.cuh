// Helpers of the kernels that run on pairs of CTAs (a cluster of two, one matrix instruction for both), and the tensor maps of their rows.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "snn_tc_common.cuh"

namespace snn {
namespace {

// The same value in all lanes, known to be so
__device__ __forceinline__ int uni(int x) { return __shfl_sync(0xffffffffu, x, 0); }

__device__ __forceinline__ void commit_on(uint32_t bar, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %2;\n\t}" ::"r"(bar),
      "r"(on), "h"((uint16_t)3)
      : "memory");
}
// Rows of 128 bytes, the 16-byte pieces of eight rows in turn (the layout that TMA writes the rows of activations in)
__device__ __forceinline__ uint64_t rows_desc(uint32_t addr) {
  return ((uint64_t)2 << 61) | ((uint64_t)1 << 46) | ((uint64_t)64 << 32) | ((uint64_t)1 << 16) | (addr >> 4);
}
// (the barrier: the pair's first CTA's)
__device__ __forceinline__ void tma_rows(uint32_t dst, const void* map, int c, int row, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(c),
               "r"(row), "r"(bar)
               : "memory");
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

}  // namespace
}  // namespace snn
