// Projections of language models (include/snn_conv.h: experts, adapters): device form of the weights and the launches.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "snn_internal.h"

namespace snn {

// Weights of E projections [K x C], one bit each (set: -1), for both product kernels:
//   bits [E][n_mt][n_kb][8 g][2 o][4 t][2 i]:  a tile of 16 output channels times 256 input channels is 512 bytes.
//   Word (g, o, t, i): rows g and g + 8 of the tile, of the 64 input channels from 256 kb + 64 (2 i + o) those from 8 t on and from
//   32 + 8 t on, eight each, as eight pairs of neighbouring channels: pair p of row g in bits p (the even one) and 16 + p, of row
//   g + 8 in bits 8 + p and 24 + p.  (Four lanes that load 16 bytes of activations each for their words then read 64 neighbouring bytes: whole
//   sectors.)
// (A lane 4g + t of the small kernel's warps reads two times 8 bytes, a thread of the tall kernel's two warpgroups, which take odd and
// even blocks of 64, twice 16.)
// A shift and a masked exclusive-or turn a pair into two 16-bit +1 / -1 in one register.  Rows and channels that do not
// exist have bit 0; the former's sums are not stored, the latter meet zeros.
struct Products {
  int device = 0, E = 0, C = 0, K = 0;
  int n_mt = 0;   // tiles of 16 output channels, a multiple of 16
  int n_kb = 0;   // blocks of 256 input channels
  uint32_t* bits = nullptr;
  float* alpha = nullptr;       // [E][16 n_mt], zeros behind K
  int* status_host = nullptr;   // pinned, written by a kernel that gave up a bounded wait
  int* status_dev = nullptr;
};
cudaError_t products_create(const LayerDev* const* layers, int E, int C, int K, cudaStream_t s, Products* out, int* launched);
void products_destroy(Products* p);

// A term added to the rows' outputs: scale * B (A x) of each row's adapter.
struct Lowrank {
  const int32_t* adapter = nullptr;   // [rows]
  const float* h = nullptr;           // [rows][rank]: scale * (A x), of rows with an adapter
  const void* b = nullptr;            // [n][K][rank], 16-bit
  int n = 0, rank = 0;
};
struct ProductCall {
  const void* act;
  int act_type, act_rows;
  long long ld_act;
  const int32_t* rows;      // or null
  const int32_t* offsets;   // or null: all max_rows rows are expert 0's
  int max_rows;
  void* out;
  int out_type;
  long long ld_out;
  Lowrank low;              // adapter null: none
  cudaStream_t stream;
};
cudaError_t products_forward(const Products& p, const ProductCall& c, int* launched);
cudaError_t products_tall(const Products& p, const ProductCall& c, int* launched);   // (snn_products_tall.cu: many rows)

// h[r][0..rank) = scale[a] * (A[a] x[r]) for the rows with an adapter; the others' are not written.
struct ShrinkCall {
  const void* act;
  int act_type, rows, C;
  long long ld_act;
  const int32_t* adapter;
  const void* a;
  const float* scale;
  int n, rank;
  float* h;
  cudaStream_t stream;
};
cudaError_t shrink_forward(const ShrinkCall& c, int* launched);

struct RouteCall {
  const void* logits;
  int type, T, E, k, normalise;
  long long ld;
  int32_t* ids;
  float* weights;
  int32_t *offsets, *rows, *slots;
  int32_t* work;
  cudaStream_t stream;
};
long long route_work_bytes(int T, int E);
cudaError_t route_forward(const RouteCall& c, int* launched);

struct CombineCall {
  const void* y;
  int y_type, y_rows;
  long long ld_y;
  const int32_t* slots;
  const float* weights;
  int T, k, C;
  void* out;
  int out_type;
  long long ld_out;
  cudaStream_t stream;
};
cudaError_t combine_forward(const CombineCall& c, int* launched);

}  // namespace snn
