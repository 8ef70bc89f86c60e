// Gated feed-forward block, forward and backward: two matrix products with what surrounds them fused in.
//
//   forward   [G | U] = X W,  H = act(G) * U         (W as it is stored, [D x 2F]: the contraction is its slow axis)
//   backward  dGU from GU and dH, then dX = dGU W^T  (both operands contiguous along the contraction)
//
// Tiles of the product are computed by workgroups of 4 or 8 waves, a wave 32 .. 128 rows x 64 columns; the forward pass gives a wave 32 columns of
// the gate and the same 32 of the other projection, so that activation and product happen in its registers.  Operands go from global
// memory into LDS by the texture path (buffer_load ... lds, 16 bytes a lane), in stages of 64 bytes of the contraction (32 bfloat16, 16
// binary32), through a ring of four stages: three are on their way while one is multiplied.  A stage is multiplied in two halves, the
// fragments of one requested while the other is multiplied, across the barrier between stages too; there is one barrier a stage.
// LDS rows of X are 64 bytes, their 16-byte chunks permuted by the row (chosen by the lane that fetches them) so that the reads of a
// fragment touch every bank once; W's are 128 bytes of 64 columns, read by transposing loads.
// The matrix instructions take W's fragment first: a lane then holds four consecutive columns of one row of the result, and
// two exchanges between the halves of a wave make 16-byte stores of them.
//
// Operands whose rows are not whole 16-byte vectors are copied into the workspace first, rows padded; then so is the contraction,
// with zeros.  Where there are few tiles the contraction is split and a second kernel adds the parts up, in order.
#include <algorithm>
#include <type_traits>

#include "buffer_access.h"
#include "layer_ops.h"

namespace bsr {

namespace {

typedef __attribute__((ext_vector_type(4))) short v4s;
typedef __attribute__((ext_vector_type(8))) short v8s;
typedef __attribute__((ext_vector_type(8))) __bf16 v8bf;
typedef __attribute__((ext_vector_type(4))) float v4f;
typedef __attribute__((ext_vector_type(16))) float v16f;

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

// ---- the product ----

constexpr int kRing = 4;
constexpr uint32_t kBeyond = 0xFFFF0000u;          // a byte offset no buffer reaches: reads as zeros
constexpr uint32_t kRange = 0x80000000u;           // bytes that a tile's offsets may span

template <typename T>
constexpr int kStageK = 64 / (int)sizeof(T);       // contraction of a stage
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

// One global -> LDS copy: lane l's 16 bytes land at lds_addr + 16 * l.  Inline assembly, so that the compiler keeps no account of
// it (it would wait for all copies in front of the next LDS read); the waits are explicit.
__device__ __forceinline__ void copy_to_lds(__amdgpu_buffer_rsrc_t rsrc, uint32_t lds_addr, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
               "buffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(lds_addr), "v"(voff), "s"(rsrc) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}

struct ProductArgs {
  const void *A, *B;
  int64_t M, N, K, lda, ldb;       // N: columns of the result; of the gated product, of H
  int64_t up;                      // gated: column of B from which U's weights are
  void *out, *gu;                  // result (H); GU or null
  float *partial;                  // split: [splits][M][N or 2N] binary32
  int64_t ldo, ldgu;
  int32_t tiles_m, tiles_n, splits, stages_per_split;
};

// A result tile of 32 x 32 in a wave's registers (lane: row lane % 32, columns 8 a + 4 (lane / 32) + b in v[4 a + b]) to memory.
template <typename T>
__device__ __forceinline__ void store_tile(T *out, int64_t ld, int64_t m, int64_t M, int64_t n0, int64_t N, const float (&v)[16]) {
  const int half = (threadIdx.x >> 5) & 1;
  if constexpr (sizeof(T) == 2) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    // the halves exchange: then a lane has 16 consecutive columns, from 16 * half on
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto r = __builtin_amdgcn_permlane32_swap(w[i], w[i + 4], false, false);
      w[i] = r[0];
      w[i + 4] = r[1];
    }
    // w[0], w[1] | w[4], w[5]: columns 0 .. 7; w[2], w[3] | w[6], w[7]: columns 8 .. 15
    if (m >= M) return;
    T *dst = out + m * ld + n0 + 16 * half;
    const int64_t left = N - n0 - 16 * half;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const Words4 x = {w[2 * i], w[2 * i + 1], w[2 * i + 4], w[2 * i + 5]};
      if (left >= 8 * i + 8) RowVec<T, 8>::store(dst + 8 * i, x);
      else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (8 * i + q < left) dst[8 * i + q] = (T)(q % 2 ? x[q / 2] >> 16 : x[q / 2] & 0xFFFFu);
      }
    }
  } else {
    if (m >= M) return;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int64_t n = n0 + 8 * a + 4 * half;
      T *dst = out + m * ld + n;
      if (n + 4 <= N) RowVec<T, 4>::store(dst, Words4{__float_as_uint(v[4 * a]), __float_as_uint(v[4 * a + 1]),
                                                      __float_as_uint(v[4 * a + 2]), __float_as_uint(v[4 * a + 3])});
      else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (n + q < N) dst[q] = v[4 * a + q];
      }
    }
  }
}

// GATED: B is W [K x 2N], contraction the slow axis, and the result act(G) * U; otherwise B is [N x K] and the result A B^T.
// A wave's tile is TM x TN fragments of 32 x 32; WM x WN waves.
template <typename T, bool GATED, int ACT, int TM, int TN, int WM, int WN, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN, 2) void product_kernel(ProductArgs a) {
  constexpr int kWaves = WM * WN;
  constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN;            // BN: columns of B in a tile; of a gated tile half belong to G
  constexpr int kStageBytes = (BM + BN) * 64;
  constexpr int kCopiesA = BM / 16, kCopiesB = BN / 16, kCopies = kCopiesA + kCopiesB;
  constexpr int kMine = (kCopies + kWaves - 1) / kWaves;         // copies of a wave per stage; the last waves have one less
  constexpr int kLess = kMine * kWaves - kCopies;
  constexpr int SK = kStageK<T>, VE = kVec<T>;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[kRing * kStageBytes];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int wm = wave / WN, wn = wave % WN;

  // tiles: every XCD (blockIdx % 8) takes a contiguous part of them, eight rows of tiles at a time column by column
  const uint32_t tiles = (uint32_t)a.tiles_m * (uint32_t)a.tiles_n;
  const uint32_t items = tiles * (uint32_t)a.splits, per_xcd = (items + 7) / 8;
  const uint32_t item = (blockIdx.x & 7u) * per_xcd + (blockIdx.x >> 3);
  if (item >= items || (blockIdx.x >> 3) >= per_xcd) return;
  const uint32_t split = item / tiles, tile = item % tiles;
  constexpr uint32_t kBand = 8;
  const uint32_t band = tile / (kBand * a.tiles_n), in_band = tile % (kBand * a.tiles_n);
  const uint32_t rows = min(kBand, a.tiles_m - band * kBand);
  const int64_t m0 = (int64_t)(band * kBand + in_band % rows) * BM;
  const int64_t n0 = (int64_t)(in_band / rows) * (GATED ? BN / 2 : BN);
  const int64_t first_stage = (int64_t)split * a.stages_per_split;
  const int64_t all_stages = (a.K + SK - 1) / SK;
  const int stages = (int)max((int64_t)0, min((int64_t)a.stages_per_split, all_stages - first_stage));

  // ---- this wave's copies: 1 KB each, the first kCopiesA of a stage for A ----
  const uint8_t *const baseA = static_cast<const uint8_t *>(a.A) + (m0 * a.lda + first_stage * SK) * (int64_t)sizeof(T);
  const uint8_t *const baseB = static_cast<const uint8_t *>(a.B) +
                               (GATED ? first_stage * SK * a.ldb + n0 : n0 * a.ldb + first_stage * SK) * (int64_t)sizeof(T);
  const int64_t stepA = SK * (int64_t)sizeof(T), stepB = GATED ? SK * a.ldb * (int64_t)sizeof(T) : SK * (int64_t)sizeof(T);
  uint32_t voff[kMine];          // per-lane offset of a copy
  int32_t kfirst[kMine];         // first index of the contraction (within the stage) that the lane's chunk belongs to
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int c = wave + i * kWaves;
    if (c < kCopiesA || !GATED) {
      // 16 rows x 64 bytes
      const bool isA = c < kCopiesA;
      const int64_t row = 16 * (isA ? c : c - kCopiesA) + (lane >> 2);
      const int64_t last = (isA ? a.M - m0 : a.N - n0) - 1;
      const int chunk = (lane & 3) ^ ((lane >> 4) & 3);
      voff[i] = (uint32_t)(min(row, last) * (isA ? a.lda : a.ldb) * (int64_t)sizeof(T)) + (uint32_t)chunk * 16u;
      kfirst[i] = chunk * VE;
    } else {
      // 8 rows x 128 bytes of a panel: the first half of the panels from G's columns, the others from U's
      constexpr int kPanelCols = 128 / (int)sizeof(T), kPanels = BN / kPanelCols, kPerPanel = SK / 8;
      const int p = (c - kCopiesA) / kPerPanel, r = ((c - kCopiesA) % kPerPanel) * 8 + (lane >> 3);
      const int chunk = sizeof(T) == 2 ? (lane & 7) ^ (4 * ((lane >> 4) & 1)) : lane & 7;
      const int64_t col = (p % (kPanels / 2)) * kPanelCols + chunk * VE;
      const bool there = n0 + col < a.N;
      voff[i] = there ? (uint32_t)((r * a.ldb + (p >= kPanels / 2 ? a.up : 0) + col) * (int64_t)sizeof(T)) : kBeyond;
      kfirst[i] = r;
    }
  }
  const uint32_t ring_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)ring;
  const int32_t k_all = (int32_t)(a.K - first_stage * SK);       // contraction from the first stage on
  auto issue = [&](int stage, uint32_t slot) {
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(baseA + stage * stepA, kRange), rb = make_rsrc(baseB + stage * stepB, kRange);
    const int32_t left = k_all - stage * SK;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int c = wave + i * kWaves;
      const uint32_t v = kfirst[i] < left ? voff[i] : kBeyond;
      const uint32_t to = ring_lds + slot * kStageBytes + (uint32_t)c * 1024u;
      if (kLess != 0 && i == kMine - 1 && c >= kCopies) continue;
      if (c < kCopiesA) copy_to_lds(ra, to, v);
      else copy_to_lds(rb, to, v);
    }
  };
  // the copies of all but the last `STAGES` stages that this wave issued have landed
  auto wait_for = [&](auto stages_c) {
    constexpr int N = decltype(stages_c)::value;
    if (kLess != 0 && wave + (kMine - 1) * kWaves >= kCopies) wait_copies<N * (kMine - 1)>();
    else wait_copies<N * kMine>();
  };

  // ---- fragments ----
  struct Frags {
    Words4 a[TM], b[TN];
  };
  const int g4 = lane >> 4, L = lane & 15, half = lane >> 5;
  // 16-byte chunk `2 * ks + half` of row lane % 32
  uint32_t offRow[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) offRow[ks] = (uint32_t)((lane & 31) * 64 + (((2 * ks + half) ^ ((lane >> 2) & 3)) * 16));
  const uint32_t offB = !GATED ? 0u
                        : sizeof(T) == 2
                            ? (uint32_t)((8 * (g4 >> 1) + (L >> 2)) * 128 + ((2 * (g4 & 1) + ((L & 3) >> 1)) ^ (4 * ((L >> 3) & 1))) * 16 + 8 * (L & 1))
                            : (uint32_t)(4 * half * 128 + (lane & 31) * 4);
  auto load_frags = [&](Frags &f, uint32_t slot, auto ks_c) {
    constexpr int ks = decltype(ks_c)::value;
    const uint8_t *st = ring + slot * kStageBytes;
#pragma unroll
    for (int i = 0; i < TM; ++i) f.a[i] = *reinterpret_cast<const Words4 *>(st + (wm * TM + i) * 2048 + offRow[ks]);
    const uint8_t *sb = st + BM * 64;
    if constexpr (!GATED) {
#pragma unroll
      for (int j = 0; j < TN; ++j) f.b[j] = *reinterpret_cast<const Words4 *>(sb + (wn * TN + j) * 2048 + offRow[ks]);
    } else if constexpr (sizeof(T) == 2) {
      typedef v4s __attribute__((address_space(3))) * lds_v4s;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        // strip of 32 columns: of G for the first half of the wave's fragments, of U for the others
        const int strip = wn * (TN / 2) + j % (TN / 2) + (j >= TN / 2 ? BN / 64 : 0);
        const uint8_t *p = sb + (strip >> 1) * 4096 + (offB ^ ((strip & 1) * 64u)) + ks * 2048;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)p);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(p + 512));
        const v8s r = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        f.b[j] = __builtin_bit_cast(Words4, r);
      }
    } else {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int strip = wn * (TN / 2) + j % (TN / 2) + (j >= TN / 2 ? BN / 64 : 0);
        const uint8_t *p = sb + strip * 2048 + offB + ks * 1024;
#pragma unroll
        for (int q = 0; q < 4; ++q) f.b[j][q] = *reinterpret_cast<const uint32_t *>(p + q * 128);
      }
    }
  };
  v16f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  auto multiply = [&](const Frags &f) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, f.b[j]), __builtin_bit_cast(v8bf, f.a[i]), acc[i][j], 0, 0, 0);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(f.b[j][q]), __uint_as_float(f.a[i][q]), acc[i][j], 0, 0, 0);
    }
  };

  // ---- stages ----
  typedef std::integral_constant<int, 0> K0;
  typedef std::integral_constant<int, 1> K1;
  if (stages > 0) {
    for (int s = 0; s < kRing; ++s) issue(s, (uint32_t)s);
    wait_for(std::integral_constant<int, kRing - 1>());
    asm volatile("s_barrier" ::: "memory");
    Frags f0, f1;
    load_frags(f0, 0, K0());
    uint32_t slot = 0;
    for (int s = 0; s < stages; ++s) {
      load_frags(f1, slot, K1());
      multiply(f0);
      // everybody's copies of the next stage have landed, and everybody has the fragments of this one
      wait_for(std::integral_constant<int, kRing - 2>());
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      issue(s + kRing, slot);
      slot = slot == kRing - 1 ? 0 : slot + 1;
      load_frags(f0, slot, K0());
      multiply(f1);
    }
    // no copy may be on its way when the workgroup gives its LDS back
    wait_copies<0>();
  }

  // ---- results ----
  const int64_t mw = m0 + wm * 32 * TM + (lane & 31);
  if constexpr (SPLIT) {
    const int64_t width = GATED ? 2 * a.N : a.N;
    float *out = a.partial + (int64_t)split * a.M * width;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        float v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = acc[i][j][r];
        if constexpr (GATED) {
          const int64_t n = n0 + (wn * (TN / 2) + j % (TN / 2)) * 32;
          store_tile<float>(out + (j >= TN / 2 ? a.N : 0), width, mw + 32 * i, a.M, n, a.N, v);
        } else {
          store_tile<float>(out, width, mw + 32 * i, a.M, n0 + (wn * TN + j) * 32, a.N, v);
        }
      }
  } else if constexpr (GATED) {
    T *const H = static_cast<T *>(a.out), *const GU = static_cast<T *>(a.gu);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN / 2; ++j) {
        float g[16], u[16], h[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          g[r] = acc[i][j][r];
          u[r] = acc[i][j + TN / 2][r];
          h[r] = activation<ACT>(g[r]).value * u[r];
        }
        const int64_t n = n0 + (wn * (TN / 2) + j) * 32;
        store_tile<T>(H, a.ldo, mw + 32 * i, a.M, n, a.N, h);
        if (GU != nullptr) {
          store_tile<T>(GU, a.ldgu, mw + 32 * i, a.M, n, a.N, g);
          store_tile<T>(GU + a.N, a.ldgu, mw + 32 * i, a.M, n, a.N, u);
        }
      }
  } else {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        float v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = acc[i][j][r];
        store_tile<T>(static_cast<T *>(a.out), a.ldo, mw + 32 * i, a.M, n0 + (wn * TN + j) * 32, a.N, v);
      }
  }
}

// The parts of a split contraction added up: four columns to a thread.
template <typename T, bool GATED, int ACT>
__global__ __launch_bounds__(256) void join_kernel(const float *__restrict__ partial, int splits, int64_t M, int64_t N, T *__restrict__ out,
                                                   int64_t ldo, T *__restrict__ gu, int64_t ldgu) {
  const int64_t quads = (N + 3) / 4, width = GATED ? 2 * N : N;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * quads; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / quads, n = i % quads * 4;
    const int there = N - n >= 4 ? 4 : (int)(N - n);
    float g[4] = {0.0f, 0.0f, 0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
      const float *p = partial + ((int64_t)s * M + m) * width + n;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q < there) {
          g[q] += p[q];
          if constexpr (GATED) u[q] += p[N + q];
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q >= there) continue;
      if constexpr (GATED) {
        out[m * ldo + n + q] = from_float<T>(activation<ACT>(g[q]).value * u[q]);
        if (gu != nullptr) {
          gu[m * ldgu + n + q] = from_float<T>(g[q]);
          gu[m * ldgu + N + n + q] = from_float<T>(u[q]);
        }
      } else out[m * ldo + n + q] = from_float<T>(g[q]);
    }
  }
}

// dGU from GU and dH, a vector of columns to a thread; `also`: a second copy with rows of `pitch` elements, or null.
template <typename T, int VE, int ACT>
__global__ __launch_bounds__(256) void gated_slope_kernel(const T *GU, int64_t M, int64_t F, int64_t ldgu, const T *__restrict__ dH,
                                                          int64_t lddh, T *dGU, int64_t lddgu, T *__restrict__ also, int64_t pitch) {
  typedef RowVec<T, VE> R;
  const int64_t vecs = F / VE;                       // whole vectors
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * vecs; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / vecs, f = i % vecs * VE;
    const typename R::Raw g = R::load(GU + m * ldgu + f), u = R::load(GU + m * ldgu + F + f), d = R::load(dH + m * lddh + f);
    float a[VE], b[VE];
#pragma unroll
    for (int q = 0; q < VE; ++q) {
      const Activation x = activation<ACT>(R::elem(g, q));
      const float dh = R::elem(d, q);
      a[q] = dh * R::elem(u, q) * x.slope;
      b[q] = dh * x.value;
    }
    const typename R::Raw pa = pack_row<T, VE>(a), pb = pack_row<T, VE>(b);
    R::store(dGU + m * lddgu + f, pa);
    R::store(dGU + m * lddgu + F + f, pb);
    if (also != nullptr) {
      R::store(also + m * pitch + f, pa);
      R::store(also + m * pitch + F + f, pb);
    }
  }
  if (also != nullptr) {                             // zeros behind the last column
    const int64_t pad = pitch - 2 * F;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * pad; i += (int64_t)gridDim.x * 256)
      also[i / pad * pitch + 2 * F + i % pad] = (T)0;
  }
  if constexpr (VE > 1) {
    const int64_t rest = F - vecs * VE;
    if (rest == 0) return;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * rest; i += (int64_t)gridDim.x * 256) {
      const int64_t m = i / rest, f = vecs * VE + i % rest;
      const Activation x = activation<ACT>(elem_to_float<T>(GU[m * ldgu + f]));
      const float u = elem_to_float<T>(GU[m * ldgu + F + f]), dh = elem_to_float<T>(dH[m * lddh + f]);
      const T a = from_float<T>(dh * u * x.slope), b = from_float<T>(dh * x.value);
      dGU[m * lddgu + f] = a;
      dGU[m * lddgu + F + f] = b;
      if (also != nullptr) {
        also[m * pitch + f] = a;
        also[m * pitch + F + f] = b;
      }
    }
  }
}

// Columns [from, from + cols) of a matrix into rows of `pitch` elements from column `to` on, zeros up to column `to + padded`.
template <typename T>
__global__ __launch_bounds__(256) void pack_rows_kernel(const T *__restrict__ src, int64_t rows, int64_t ld, int64_t from, int64_t cols,
                                                        T *__restrict__ dst, int64_t pitch, int64_t to, int64_t padded) {
  constexpr int VE = kVec<T>;
  const int64_t vecs = padded / VE;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * vecs; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / vecs, c = i % vecs * VE;
    const T *p = src + r * ld + from + c;
    Words4 v = {0, 0, 0, 0};
    if (c + VE <= cols) v = RowVec<T, VE>::load(p);
    else {
      T e[VE];
#pragma unroll
      for (int q = 0; q < VE; ++q) e[q] = c + q < cols ? p[q] : (T)0;
      __builtin_memcpy(&v, e, 16);
    }
    *reinterpret_cast<Words4 *>(dst + r * pitch + to + c) = v;
  }
}

// ---- host ----

template <typename F>
void with_act(int act, F f) {
  if (act == BSR_ACT_SILU) f(std::integral_constant<int, BSR_ACT_SILU>());
  else if (act == BSR_ACT_GELU) f(std::integral_constant<int, BSR_ACT_GELU>());
  else if (act == BSR_ACT_GELU_TANH) f(std::integral_constant<int, BSR_ACT_GELU_TANH>());
  else f(std::integral_constant<int, BSR_ACT_RELU>());
}

constexpr int kCus = 256;
constexpr int64_t kMostGrid = int64_t(1) << 20;

dim3 grid_for(int64_t threads) { return dim3((uint32_t)std::min(ceil_div(threads, (int64_t)256), kMostGrid)); }

int64_t padded(int64_t n, int dtype) {
  const int64_t ve = 16 / elem_bytes(dtype);
  return ceil_div(n, ve) * ve;
}

// Whether the product can take an operand as it is: rows of whole vectors at 16 bytes, offsets of a tile within its range.
bool in_place(const void *p, int dtype, int64_t ld, int64_t inner) {
  const int64_t e = elem_bytes(dtype);
  return (uintptr_t)p % 16 == 0 && ld * e % 16 == 0 && inner * e % 16 == 0 && ld * e * 256 < (int64_t)kRange;
}

// Tile of a product and how its contraction is split.
enum TileShape { kTile256, kTile128, kTile32 };
struct Plan {
  TileShape shape;
  int32_t tiles_n, splits, stages_per_split;
};
Plan plan_product(int64_t M, int64_t N, int64_t K, int dtype, bool gated) {
  auto tiles = [&](int bm, int bn) { return ceil_div(M, (int64_t)bm) * ceil_div(N, (int64_t)(gated ? bn / 2 : bn)); };
  Plan p;
  int bm, bn;
  if (M <= 32) { p.shape = kTile32; bm = 32; bn = 256; }
  else if (tiles(256, 256) >= 192) { p.shape = kTile256; bm = 256; bn = 256; }
  else { p.shape = kTile128; bm = 128; bn = 128; }
  p.tiles_n = (int32_t)ceil_div(N, (int64_t)(gated ? bn / 2 : bn));
  const int64_t stages = std::max<int64_t>(1, ceil_div(K, (int64_t)(64 / elem_bytes(dtype))));
  const int64_t all = ceil_div(M, (int64_t)bm) * p.tiles_n;
  int64_t splits = 1;
  if (p.shape != kTile256 && all < 2 * kCus) splits = std::min(2 * kCus / all, std::max<int64_t>(1, stages / 4));
  p.stages_per_split = (int32_t)ceil_div(stages, splits);
  p.splits = (int32_t)ceil_div(stages, (int64_t)p.stages_per_split);
  return p;
}

size_t partial_bytes(const Plan &p, int64_t M, int64_t N, bool gated) {
  return p.splits > 1 ? align_up((size_t)p.splits * (size_t)M * (size_t)(gated ? 2 * N : N) * 4, 256) : 0;
}

template <typename T, bool GATED, int ACT>
int run_product(const Plan &p, ProductArgs a, hipStream_t s) {
  a.tiles_n = p.tiles_n;
  a.splits = p.splits;
  a.stages_per_split = p.stages_per_split;
  // a launch's lanes are counted in 32 bits: more tiles than that go by parts of the rows
  constexpr int64_t kMostItems = int64_t(1) << 22;
  const int64_t height = p.shape == kTile256 ? 256 : p.shape == kTile128 ? 128 : 32;
  const int64_t rows_at_once = p.splits > 1 ? a.M : std::max<int64_t>(1, kMostItems / p.tiles_n) * height;
  const ProductArgs whole = a;
  for (int64_t r = 0; r < whole.M; r += rows_at_once) {
    a.M = std::min(whole.M - r, rows_at_once);
    a.A = static_cast<const T *>(whole.A) + r * whole.lda;
    a.out = static_cast<T *>(whole.out) + r * whole.ldo;
    a.gu = whole.gu != nullptr ? static_cast<T *>(whole.gu) + r * whole.ldgu : nullptr;
    a.tiles_m = (int32_t)ceil_div(a.M, height);
    const dim3 grid((uint32_t)(ceil_div((int64_t)a.tiles_m * a.tiles_n * a.splits, (int64_t)8) * 8));
    if (p.splits > 1) {
      if (p.shape == kTile128) product_kernel<T, GATED, 0, 2, 2, 2, 2, true><<<grid, 256, 0, s>>>(a);
      else product_kernel<T, GATED, 0, 1, 2, 1, 4, true><<<grid, 256, 0, s>>>(a);
      if (const int rc = check_launch(); rc != BSR_OK) return rc;
      join_kernel<T, GATED, ACT><<<grid_for(a.M * ceil_div(a.N, (int64_t)4)), 256, 0, s>>>(
          a.partial, p.splits, a.M, a.N, static_cast<T *>(a.out), a.ldo, static_cast<T *>(a.gu), a.ldgu);
    } else {
      if (p.shape == kTile256) product_kernel<T, GATED, ACT, 4, 2, 2, 4, false><<<grid, 512, 0, s>>>(a);
      else if (p.shape == kTile128) product_kernel<T, GATED, ACT, 2, 2, 2, 2, false><<<grid, 256, 0, s>>>(a);
      else product_kernel<T, GATED, ACT, 1, 2, 1, 4, false><<<grid, 256, 0, s>>>(a);
    }
    if (const int rc = check_launch(); rc != BSR_OK) return rc;
  }
  return BSR_OK;
}

// What goes into the workspace, in this order.
struct Layout {
  Plan plan;
  size_t a = 0, b = 0, partial = 0, all = 0;         // bytes of the packed operands (0: taken in place), of the parts, together
};

Layout forward_layout(const GatedArgs &g) {
  Layout l;
  l.plan = plan_product(g.M, g.F, g.D, g.dtype, true);
  const size_t e = (size_t)elem_bytes(g.dtype);
  if (g.D > 0 && !in_place(g.X, g.dtype, g.ldx, g.D)) l.a = align_up((size_t)g.M * (size_t)padded(g.D, g.dtype) * e, 256);
  if (g.D > 0 && !in_place(g.W, g.dtype, g.ldw, g.F)) l.b = align_up((size_t)g.D * 2 * (size_t)padded(g.F, g.dtype) * e, 256);
  l.partial = partial_bytes(l.plan, g.M, g.F, true);
  l.all = l.a + l.b + l.partial;
  return l;
}

Layout backward_layout(const GatedArgs &g, const void *dGU, int64_t lddgu) {
  Layout l;
  l.plan = plan_product(g.M, g.D, 2 * g.F, g.dtype, false);
  const size_t e = (size_t)elem_bytes(g.dtype);
  const int64_t pitch = padded(2 * g.F, g.dtype);
  if (g.F > 0 && !in_place(dGU, g.dtype, lddgu, 2 * g.F)) l.a = align_up((size_t)g.M * (size_t)pitch * e, 256);
  if (g.F > 0 && !in_place(g.W, g.dtype, g.ldw, 2 * g.F)) l.b = align_up((size_t)g.D * (size_t)pitch * e, 256);
  l.partial = partial_bytes(l.plan, g.M, g.D, false);
  l.all = l.a + l.b + l.partial;
  return l;
}

template <typename T>
int forward(const GatedArgs &g, void *H, int64_t ldh, void *GU, int64_t ldgu, void *ws, hipStream_t s) {
  const Layout l = forward_layout(g);
  uint8_t *const at = static_cast<uint8_t *>(ws);
  ProductArgs a = {};
  a.A = g.X;
  a.lda = g.ldx;
  a.B = g.W;
  a.ldb = g.ldw;
  a.M = g.M;
  a.N = g.F;
  a.K = g.D;
  if (l.a != 0) {
    T *dst = reinterpret_cast<T *>(at);
    const int64_t pitch = padded(g.D, g.dtype);
    pack_rows_kernel<T><<<grid_for(g.M * pitch / kVec<T>), 256, 0, s>>>(static_cast<const T *>(g.X), g.M, g.ldx, 0, g.D, dst, pitch, 0, pitch);
    a.A = dst;
    a.lda = pitch;
  }
  a.up = g.F;
  if (l.b != 0) {
    T *dst = reinterpret_cast<T *>(at + l.a);
    const int64_t half = padded(g.F, g.dtype);
    for (int i = 0; i < 2; ++i)
      pack_rows_kernel<T><<<grid_for(g.D * half / kVec<T>), 256, 0, s>>>(static_cast<const T *>(g.W), g.D, g.ldw, i * g.F, g.F, dst, 2 * half,
                                                                        i * half, half);
    a.B = dst;
    a.ldb = 2 * half;
    a.up = half;
  }
  if (const int rc = check_launch(); rc != BSR_OK) return rc;
  a.out = H;
  a.ldo = ldh;
  a.gu = GU;
  a.ldgu = ldgu;
  a.partial = reinterpret_cast<float *>(at + l.a + l.b);
  int rc = BSR_OK;
  with_act(g.act, [&](auto act) { rc = run_product<T, true, decltype(act)::value>(l.plan, a, s); });
  return rc;
}

template <typename T>
int backward(const GatedArgs &g, const void *GU, int64_t ldgu, const void *dH, int64_t lddh, void *dGU, int64_t lddgu, void *dX,
             int64_t lddx, void *ws, hipStream_t s) {
  const bool product = dX != nullptr && g.D > 0;
  const Layout l = product ? backward_layout(g, dGU, lddgu) : Layout();
  uint8_t *const at = static_cast<uint8_t *>(ws);
  const int64_t pitch = padded(2 * g.F, g.dtype);
  T *const also = l.a != 0 ? reinterpret_cast<T *>(at) : nullptr;
  if (g.M > 0 && g.F > 0) {
    with_act(g.act, [&](auto act) {
      gated_slope_kernel<T, kVec<T>, decltype(act)::value><<<grid_for(g.M * ceil_div(g.F, (int64_t)kVec<T>)), 256, 0, s>>>(
          static_cast<const T *>(GU), g.M, g.F, ldgu, static_cast<const T *>(dH), lddh, static_cast<T *>(dGU), lddgu, also, pitch);
    });
    if (const int rc = check_launch(); rc != BSR_OK) return rc;
  }
  if (!product) return BSR_OK;
  ProductArgs a = {};
  a.A = also != nullptr ? also : dGU;
  a.lda = also != nullptr ? pitch : lddgu;
  a.B = g.W;
  a.ldb = g.ldw;
  if (l.b != 0) {
    T *dst = reinterpret_cast<T *>(at + l.a);
    pack_rows_kernel<T><<<grid_for(g.D * pitch / kVec<T>), 256, 0, s>>>(static_cast<const T *>(g.W), g.D, g.ldw, 0, 2 * g.F, dst, pitch, 0, pitch);
    if (const int rc = check_launch(); rc != BSR_OK) return rc;
    a.B = dst;
    a.ldb = pitch;
  }
  a.M = g.M;
  a.N = g.D;
  a.K = 2 * g.F;
  a.out = dX;
  a.ldo = lddx;
  a.partial = reinterpret_cast<float *>(at + l.a + l.b);
  return run_product<T, false, 0>(l.plan, a, s);
}

}  // namespace

size_t gated_ff_ws_bytes(const GatedArgs &a) { return forward_layout(a).all; }

int launch_gated_ff(const GatedArgs &a, void *H, int64_t ldh, void *GU, int64_t ldgu, void *ws, hipStream_t s) {
  return a.dtype == BSR_F32 ? forward<float>(a, H, ldh, GU, ldgu, ws, s) : forward<uint16_t>(a, H, ldh, GU, ldgu, ws, s);
}

size_t gated_ff_grad_ws_bytes(const GatedArgs &a, const void *dGU, int64_t lddgu) { return backward_layout(a, dGU, lddgu).all; }

int launch_gated_ff_grad(const GatedArgs &a, const void *GU, int64_t ldgu, const void *dH, int64_t lddh, void *dGU, int64_t lddgu,
                         void *dX, int64_t lddx, void *ws, hipStream_t s) {
  return a.dtype == BSR_F32 ? backward<float>(a, GU, ldgu, dH, lddh, dGU, lddgu, dX, lddx, ws, s)
                            : backward<uint16_t>(a, GU, ldgu, dH, lddh, dGU, lddgu, dX, lddx, ws, s);
}

}  // namespace bsr
