// What the translation units of the gated feed-forward block share: activations, and the matrix products as the host sees them.
#pragma once

#include <algorithm>
#include <type_traits>

#include "buffer_access.h"
#include "layer_ops.h"

namespace bsr {

// ---- activations ----

__device__ __forceinline__ float logistic(float g) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * g)); }

// act(g) and its derivative.
struct Activation {
  float value, slope;
};
template <int ACT>
__device__ __forceinline__ Activation activation(float g) {
  if constexpr (ACT == BSR_ACT_SILU) {
    const float p = logistic(g);
    return {g * p, p * (1.0f + g * (1.0f - p))};
  } else if constexpr (ACT == BSR_ACT_GELU) {
    const float p = 0.5f * (1.0f + erff(g * 0.70710678118654752f));
    return {g * p, p + g * __builtin_amdgcn_exp2f(-0.72134752044448170f * g * g) * 0.39894228040143268f};
  } else if constexpr (ACT == BSR_ACT_GELU_TANH) {
    // (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
    const float p = logistic(1.59576912160573071f * (g + 0.044715f * g * g * g));
    return {g * p, p + g * p * (1.0f - p) * 1.59576912160573071f * (1.0f + 0.134145f * fminf(g * g, 0x1p100f))};
  } else {
    return {g != g ? g : fmaxf(g, 0.0f), g > 0.0f ? 1.0f : 0.0f};
  }
}

__device__ __forceinline__ float activation_value(int act, float g) {
  return act == BSR_ACT_SILU ? activation<BSR_ACT_SILU>(g).value
         : act == BSR_ACT_GELU ? activation<BSR_ACT_GELU>(g).value
         : act == BSR_ACT_GELU_TANH ? activation<BSR_ACT_GELU_TANH>(g).value : activation<BSR_ACT_RELU>(g).value;
}

// ---- the products ----

template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);          // elements of 16 bytes

constexpr uint32_t kBeyond = 0xFFFF0000u;          // a byte offset no buffer reaches: reads as zeros
constexpr uint32_t kRange = 0x80000000u;           // bytes that a tile's offsets may span

struct ProductArgs {
  const void *A, *B;
  int64_t M, N, K, lda, ldb;       // N: columns of the result; of the gated product, of H
  int64_t up, cols;                // gated: column of B from which U's weights are, columns of B
  void *out, *gu;                  // result (H); GU or null
  float *partial;                  // split: [splits][M][N or 2N] binary32
  int64_t ldo, ldgu;
  int64_t pitch;                   // of a row of `partial`: N or 2N, each in whole vectors
  int32_t tiles_m, tiles_n, splits, stages_per_split, act;
};

// How a product is computed: the tile of a workgroup, and how many workgroups share the contraction of a tile.
enum Tile { kTile256, kTileWide, kTile128, kTile128Alone, kTile96Alone, kTile64, kTile32 };
struct TileSize {
  int rows, cols, row_bytes;
};
constexpr TileSize kTiles[] = {{256, 256, 128}, {128, 256, 64}, {128, 128, 128}, {128, 128, 128}, {96, 128, 128}, {64, 128, 128}, {32, 256, 64}};
struct Plan {
  Tile tile;
  int32_t tiles_n, splits, stages_per_split;
  double us;                       // estimated
};

// Floats between the rows of a part of a split contraction.
inline int64_t partial_pitch(int64_t N, bool gated) { return ceil_div(N, (int64_t)4) * (gated ? 8 : 4); }

constexpr int64_t kMostGrid = int64_t(1) << 20;
inline int32_t blocks_for(int64_t threads) { return (int32_t)std::min(ceil_div(threads, (int64_t)256), kMostGrid); }

// gated_bf16.hip, gated_f32.hip: the product and, of a split contraction, the sum of the parts.
int launch_product_bf16(const Plan &p, const ProductArgs &a, bool gated, hipStream_t s);
// (M <= 32)
int launch_gated_rows_bf16(const GatedArgs &g, void *H, int64_t ldh, void *GU, int64_t ldgu, hipStream_t s);
int launch_product_f32(const Plan &p, const ProductArgs &a, bool gated, hipStream_t s);

}  // namespace bsr
