// The matrix products of the gated feed-forward block, for the translation units of their element types.
#pragma once

// [G | U] = X W with act(G) * U made from it, or dX = dGU W^T.  Tiles of the result are computed by workgroups of 4 or 8 waves, a wave
// 32 .. 128 rows x 64 columns; the forward pass gives a wave 32 columns of the gate and the same 32 of the other projection, so that
// activation and product happen in its registers.
//
// Operands go from global memory into LDS by the texture path (buffer_load ... lds, 16 bytes a lane), in stages of 64 or 128 bytes of the
// contraction, through a ring of two to four stages: what is not being multiplied is on its way.  128 bytes are whole lines of operands
// that lie along the contraction: in stages of 64 each line would pass from the second cache to the first twice.  A stage is multiplied in
// phases of 32 bytes, whose fragments are requested while the phase before is multiplied, across the barrier between stages too; there is
// one barrier a stage.
// LDS rows along the contraction are 64 or 128 bytes, their 16-byte chunks permuted by the row (chosen by the lane that fetches them) so
// that the reads of a fragment touch every bank once; W's in the forward pass are 128 bytes of columns, read by transposing loads.
// The matrix instructions take B's fragment first: a lane then holds four consecutive columns of one row of the result, and
// exchanges between the halves of a wave make 16-byte stores of them.
//
// Bound by the matrix cores: 8192 x 2048 x [2 x 5504] bfloat16, 369 GFLOP, takes 372 us with GU written (0.99 PFLOP/s), about what a library's
// product of this size takes that stores [G | U] and nothing else (379 us, 354 with W transposed).  What is lost: the first stages of a tile and its
// results, in which the matrix cores wait (one workgroup of 256 x 256 fills a compute unit, so nothing runs beside them), and the last
// round of tiles, which is not full: they are busy for 55 % of the cycles.  Binary32 reaches 121 TFLOP/s of the 154 that a library does.
// Measured and not kept (this size): 256 x 256 and 128 x 256 tiles in one launch, the last round in the smaller ones: 360 us, but 2048 rows 96 for 93 and
// 25088 x 384 x [2 x 1024] 72 for 66; wave tiles of 128 x 128 and of 64 x 128; results stored past the caches 495; results in whole
// 64-byte rows by more exchanges 375.

#include "gated.h"

namespace bsr {

namespace {

typedef __attribute__((ext_vector_type(4))) short v4s;
typedef __attribute__((ext_vector_type(8))) short v8s;
typedef __attribute__((ext_vector_type(8))) __bf16 v8bf;
typedef __attribute__((ext_vector_type(4))) float v4f;
typedef __attribute__((ext_vector_type(16))) float v16f;

// One global -> LDS copy: lane l's BYTES land at lds_addr + BYTES * l.  Inline assembly, so that the compiler keeps no account of
// it (it would wait for all copies in front of the next LDS read); the waits are explicit.
template <int BYTES>
__device__ __forceinline__ void copy_to_lds(__amdgpu_buffer_rsrc_t rsrc, uint32_t lds_addr, uint32_t voff) {
  if constexpr (BYTES == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(lds_addr), "v"(voff), "s"(rsrc) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "buffer_load_dword %1, %2, 0 offen lds"
                 :: "s"(lds_addr), "v"(voff), "s"(rsrc) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N < 63 ? N : 63) : "memory");       // (the counter ends at 63)
}

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
// A wave's tile is TM x TN fragments of 32 x 32; WM x WN waves; RING stages of ROW bytes of the contraction in LDS.  WHOLE: the contraction
// and the rows of B end with whole vectors (what it takes where they do not costs the others 2 to 10 %).
template <typename T, bool GATED, int TM, int TN, int WM, int WN, int RING, int ROW, bool WHOLE, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN, (WM * WN == 4 && RING * 32 * (TM * WM + TN * WN) * ROW > 80 * 1024 ? 1 : 2)) void product_kernel(ProductArgs a) {
  constexpr int kWaves = WM * WN;
  constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN;            // BN: columns of B in a tile; of a gated tile half belong to G
  constexpr int kStageBytes = (BM + BN) * ROW;
  constexpr int kCopiesA = BM * ROW / 1024, kCopiesB = BN * ROW / 1024, kCopies = kCopiesA + kCopiesB;
  constexpr int kMine = (kCopies + kWaves - 1) / kWaves;         // copies of a wave per stage; the last waves have one less
  constexpr int kLess = kMine * kWaves - kCopies;
  constexpr int SK = ROW / (int)sizeof(T), VE = kVec<T>;        // contraction of a stage
  constexpr int kPhases = ROW / 32;                              // parts of a stage that are multiplied at a time
  __shared__ __attribute__((aligned(1024))) uint8_t ring[RING * kStageBytes];

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

  // 16-byte chunk c of a row is held in the place of chunk c ^ permuted(row): 16 rows of one chunk lie in 16 different places
  // of 256 bytes, which is what a read of a fragment takes at a time
  auto permuted = [](int row) { return ROW == 64 ? (row >> 2) & 3 : (row >> 1) & 7; };

  // ---- this wave's copies: 1 KB each, the first kCopiesA of a stage for A ----
  const uint8_t *const baseA = static_cast<const uint8_t *>(a.A) + (m0 * a.lda + first_stage * SK) * (int64_t)sizeof(T);
  const uint8_t *const baseB = static_cast<const uint8_t *>(a.B) +
                               (GATED ? first_stage * SK * a.ldb + n0 : n0 * a.ldb + first_stage * SK) * (int64_t)sizeof(T);
  const int64_t stepA = SK * (int64_t)sizeof(T), stepB = GATED ? SK * a.ldb * (int64_t)sizeof(T) : SK * (int64_t)sizeof(T);
  const uint32_t ring_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)ring;
  const int32_t k_all = (int32_t)(a.K - first_stage * SK);       // contraction from the first stage on
  // bytes from the tile's part of B to the end of the matrix: whole vectors of its last row may lie in part beyond it
  const int64_t endB = ((a.K - 1 - first_stage * SK) * a.ldb + a.cols - n0) * (int64_t)sizeof(T);
  // the stage in which the contraction ends inside a vector, if it does
  const int32_t tail = !WHOLE && a.K % VE != 0 ? (int32_t)(a.K / SK - first_stage) : -1;
  uint32_t voff[kMine];          // per-lane offset of a copy
  int32_t kfirst[kMine];         // first index of the contraction (within the stage) that the lane's bytes belong to
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int c = wave + i * kWaves;
    if (c < kCopiesA || !GATED) {
      // rows of ROW bytes
      const bool isA = c < kCopiesA;
      const int row = (isA ? c : c - kCopiesA) * (1024 / ROW) + lane / (ROW / 16);
      const int64_t last = (isA ? a.M - m0 : a.N - n0) - 1;
      kfirst[i] = (lane % (ROW / 16) ^ permuted(row)) * VE;
      voff[i] = (uint32_t)((min((int64_t)row, last) * (isA ? a.lda : a.ldb) + kfirst[i]) * (int64_t)sizeof(T));
      kfirst[i] += VE - 1;       // (a vector in which the contraction ends: issue_tail)
    } else {
      // rows of 128 bytes of a panel: the first half of the panels from G's columns, the others from U's
      constexpr int kPanelCols = 128 / (int)sizeof(T), kPanels = BN / kPanelCols, kPerPanel = SK / 8;
      const int p = (c - kCopiesA) / kPerPanel, r = ((c - kCopiesA) % kPerPanel) * 8 + (lane >> 3);
      const int chunk = sizeof(T) == 2 ? (lane & 7) ^ (4 * ((r >> 1) & 1)) : lane & 7;
      const int64_t col = (p % (kPanels / 2)) * kPanelCols + chunk * VE;
      voff[i] = n0 + col < a.N ? (uint32_t)((r * a.ldb + (p >= kPanels / 2 ? a.up : 0) + col) * (int64_t)sizeof(T)) : kBeyond;
      kfirst[i] = r;
    }
  }
  const bool with_last = kLess == 0 || wave + (kMine - 1) * kWaves < kCopies;
  // The range of B's part of a stage: the hardware reads words beyond it as zeros.
  auto range_of = [&](bool isA, int stage) -> uint32_t {
    if (WHOLE || !GATED || isA) return kRange;
    const int64_t left = endB - stage * stepB;
    return left < 0 ? 0u : left < (int64_t)kRange ? (uint32_t)left : kRange;
  };
  auto issue = [&](int stage, uint32_t slot, int i) {           // copy i of this wave's of a stage
    const int c = wave + i * kWaves;
    const uint32_t v = kfirst[i] < k_all - stage * SK ? voff[i] : kBeyond;
    if (kLess != 0 && i == kMine - 1 && !with_last) return;
    // (known at compile time where the waves share A's copies evenly)
    const bool isA = kCopiesA % kWaves == 0 ? i < kCopiesA / kWaves : c < kCopiesA;
    const uint8_t *const base = isA ? baseA + stage * stepA : baseB + stage * stepB;
    copy_to_lds<16>(make_rsrc(base, range_of(isA, stage)), ring_lds + slot * kStageBytes + (uint32_t)c * 1024u, v);
  };
  // The stage in which the contraction ends inside a vector: rows along it word by word, the words behind its end as zeros.  (More
  // copies than the waits below count on, which then wait for more than they need.)
  auto issue_tail = [&](int stage, uint32_t slot) {
    const int32_t left = k_all - stage * SK;
    for (int c = wave; c < kCopies; c += kWaves) {
      const bool isA = c < kCopiesA;
      const uint8_t *const base = isA ? baseA + stage * stepA : baseB + stage * stepB;
      const uint32_t to = ring_lds + slot * kStageBytes + (uint32_t)c * 1024u;
      if (GATED && !isA) continue;
      for (int part = 0; part < 4; ++part) {
        const int at = part * 256 + lane * 4, row = (isA ? c : c - kCopiesA) * (1024 / ROW) + at / ROW;
        const int64_t last = (isA ? a.M - m0 : a.N - n0) - 1;
        const int k = ((at % ROW / 16) ^ permuted(row)) * VE + at % 16 / (int)sizeof(T);
        const uint32_t v = (uint32_t)((min((int64_t)row, last) * (isA ? a.lda : a.ldb) + k) * (int64_t)sizeof(T));
        copy_to_lds<4>(make_rsrc(base, kRange), to + (uint32_t)(part * 256), k < left ? v : kBeyond);
      }
    }
  };
  auto issue_any = [&](int stage, uint32_t slot, int i) {
    if constexpr (WHOLE) return issue(stage, slot, i);
    const bool isA = kCopiesA % kWaves == 0 ? i < kCopiesA / kWaves : wave + i * kWaves < kCopiesA;
    if (stage != tail || (GATED && !isA)) issue(stage, slot, i);
    if (stage == tail && i == kMine - 1) issue_tail(stage, slot);
  };
  // the copies of all but the last `STAGES` stages that this wave issued have landed
  auto wait_for = [&](auto stages_c) {
    constexpr int N = decltype(stages_c)::value;
    if (!with_last) wait_copies<N * (kMine - 1)>();
    else wait_copies<N * kMine>();
  };

  // ---- fragments ----
  struct Frags {
    Words4 a[TM], b[TN];
  };
  const int g4 = lane >> 4, L = lane & 15, half = lane >> 5;
  // 16-byte chunk `2 * ks + half` of row lane % 32
  uint32_t offRow[kPhases];
#pragma unroll
  for (int ks = 0; ks < kPhases; ++ks) offRow[ks] = (uint32_t)((lane & 31) * ROW + (((2 * ks + half) ^ permuted(lane & 31)) * 16));
  const uint32_t offB = !GATED ? 0u
                        : sizeof(T) == 2
                            ? (uint32_t)((8 * (g4 >> 1) + (L >> 2)) * 128 + ((2 * (g4 & 1) + ((L & 3) >> 1)) ^ (4 * ((L >> 3) & 1))) * 16 + 8 * (L & 1))
                            : (uint32_t)(4 * half * 128 + (lane & 31) * 4);
  // fragment n of the TN of B and the TM of A (of part ks of a stage), in this order
  auto load_frag = [&](Frags &f, uint32_t slot, int ks, int n) {
    const uint8_t *const st = ring + slot * kStageBytes, *const sb = st + BM * ROW;
    if (n >= TN) {
      f.a[n - TN] = *reinterpret_cast<const Words4 *>(st + (wm * TM + n - TN) * 32 * ROW + offRow[ks]);
    } else if constexpr (!GATED) {
      f.b[n] = *reinterpret_cast<const Words4 *>(sb + (wn * TN + n) * 32 * ROW + offRow[ks]);
    } else {
      // strip of 32 columns: of G for the first half of the wave's fragments, of U for the others
      const int strip = wn * (TN / 2) + n % (TN / 2) + (n >= TN / 2 ? BN / 64 : 0);
      if constexpr (sizeof(T) == 2) {
        typedef v4s __attribute__((address_space(3))) * lds_v4s;
        const uint8_t *p = sb + (strip >> 1) * SK * 128 + (offB ^ ((strip & 1) * 64u)) + ks * 2048;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)p);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(p + 512));
        const v8s r = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        f.b[n] = __builtin_bit_cast(Words4, r);
      } else {
        const uint8_t *p = sb + strip * SK * 128 + offB + ks * 1024;
#pragma unroll
        for (int q = 0; q < 4; ++q) f.b[n][q] = *reinterpret_cast<const uint32_t *>(p + q * 128);
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
  // Multiplies the fragments of a phase and does `actions` other things between the matrix instructions: a wave issues them
  // while the matrix core is busy, where all of them together in front would leave it idle (both waves of a SIMD come to that
  // place at the same time).  The order is the program's: the compiler would gather them again.  Where a wave has a SIMD for itself, the last
  // fragment is requested some matrix instructions before it is waited for (997 x 411 x [2 x 1003] binary32 26.8 -> 25.8 us; in the
  // largest tile, whose other wave covers that, 1 % slower).
  constexpr bool kEarly = TM * TN <= 4;
  auto multiply = [&](const Frags &f, auto actions, auto action) {
    constexpr int kActions = decltype(actions)::value, kSteps = sizeof(T) == 2 ? 1 : 4, kAll = TM * TN * kSteps;
#pragma unroll
    for (int n = 0; n < kAll; ++n) {
      const int i = n % (TM * TN) / TN, j = n % TN, q = n / (TM * TN);
      if constexpr (sizeof(T) == 2)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, f.b[j]), __builtin_bit_cast(v8bf, f.a[i]), acc[i][j], 0, 0, 0);
      else
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(f.b[j][q]), __uint_as_float(f.a[i][q]), acc[i][j], 0, 0, 0);
#pragma unroll
      for (int k = 0; k < kActions; ++k)
        if ((kEarly ? k * kAll / kActions : ((k + 1) * kAll - 1) / kActions) == n) action(k);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Keeps the compiler from moving the loads of fragments to where they are used.
  auto held = [&](Frags &f) {
#pragma unroll
    for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(f.a[i]));
#pragma unroll
    for (int j = 0; j < TN; ++j) asm volatile("" : "+v"(f.b[j]));
  };

  // ---- stages ----
  if (stages > 0) {
    for (int s = 0; s < RING; ++s)
#pragma unroll
      for (int i = 0; i < kMine; ++i) issue_any(s, (uint32_t)s, i);
    wait_for(std::integral_constant<int, RING - 1>());
    asm volatile("s_barrier" ::: "memory");
    Frags f0, f1;
#pragma unroll
    for (int n = 0; n < TM + TN; ++n) load_frag(f0, 0, 0, n);
    uint32_t slot = 0;
    for (int s = 0; s < stages; ++s) {
#pragma unroll
      for (int ks = 0; ks + 1 < kPhases; ++ks) {
        Frags &now = ks % 2 ? f1 : f0, &then = ks % 2 ? f0 : f1;
        multiply(now, std::integral_constant<int, TM + TN>(), [&](int k) { load_frag(then, slot, ks + 1, k); });
      }
      // everybody's copies of the next stage have landed, and everybody has the fragments of this one
      wait_for(std::integral_constant<int, RING - 2>());
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      const uint32_t next = slot == RING - 1 ? 0 : slot + 1;
      multiply(f1, std::integral_constant<int, TM + TN + kMine>(), [&](int k) {
        if (k < TM + TN) load_frag(f0, next, 0, k);
        else issue_any(s + RING, slot, k - TM - TN);
      });
      slot = next;
      held(f0);
    }
    // no copy may be on its way when the workgroup gives its LDS back
    wait_copies<0>();
  }

  // ---- results ----
  const int64_t mw = m0 + wm * 32 * TM + (lane & 31);
  if constexpr (SPLIT) {
    float *out = a.partial + (int64_t)split * a.M * a.pitch;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        float v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = acc[i][j][r];
        if constexpr (GATED) {
          const int64_t n = n0 + (wn * (TN / 2) + j % (TN / 2)) * 32;
          store_tile<float>(out + (j >= TN / 2 ? a.pitch / 2 : 0), a.pitch, mw + 32 * i, a.M, n, a.N, v);
        } else {
          store_tile<float>(out, a.pitch, mw + 32 * i, a.M, n0 + (wn * TN + j) * 32, a.N, v);
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
          h[r] = activation_value(a.act, g[r]) * u[r];
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

// The parts of a split contraction added up: four columns to a group of 2^LG threads, which share the parts.
template <typename T, bool GATED, int LG>
__global__ __launch_bounds__(256) void join_kernel(int act, const float *__restrict__ partial, int splits, int64_t M, int64_t N, int64_t pitch,
                                                   T *__restrict__ out, int64_t ldo, T *__restrict__ gu, int64_t ldgu) {
  const int64_t quads = (N + 3) / 4;
  const int part = threadIdx.x & ((1 << LG) - 1);
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> LG; i < M * quads; i += (int64_t)gridDim.x * (256 >> LG)) {
    const int64_t m = i / quads, n = i % quads * 4;
    v4f g = {0.0f, 0.0f, 0.0f, 0.0f}, u = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int s = part; s < splits; s += 1 << LG) {
      const float *p = partial + ((int64_t)s * M + m) * pitch + n;
      g += *reinterpret_cast<const v4f *>(p);
      if constexpr (GATED) u += *reinterpret_cast<const v4f *>(p + pitch / 2);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      g[q] = group_sum<LG>(g[q]);
      if constexpr (GATED) u[q] = group_sum<LG>(u[q]);
    }
    if (part != 0) continue;
    const int there = N - n >= 4 ? 4 : (int)(N - n);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q >= there) continue;
      if constexpr (GATED) {
        out[m * ldo + n + q] = from_float<T>(activation_value(act, g[q]) * u[q]);
        if (gu != nullptr) {
          gu[m * ldgu + n + q] = from_float<T>(g[q]);
          gu[m * ldgu + N + n + q] = from_float<T>(u[q]);
        }
      } else out[m * ldo + n + q] = from_float<T>(g[q]);
    }
  }
}

template <typename T, bool GATED, bool WHOLE, bool SPLIT>
void launch_tile(Tile t, dim3 grid, const ProductArgs &a, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if constexpr (!SPLIT) {
      if (t == kTile256) {
        product_kernel<T, GATED, 4, 2, 2, 4, 2, 128, WHOLE, SPLIT><<<grid, 512, 0, s>>>(a);
        return;
      }
    }
    if constexpr (GATED) {
      if (t == kTileWide) {
        product_kernel<T, GATED, 2, 2, 2, 4, 3, 64, WHOLE, SPLIT><<<grid, 512, 0, s>>>(a);
        return;
      }
    }
    if constexpr (!GATED && !SPLIT) {
      if (t == kTile96Alone) {
        product_kernel<T, GATED, 3, 1, 1, 4, 4, 128, WHOLE, SPLIT><<<grid, 256, 0, s>>>(a);
        return;
      }
    }
    if (t == kTile128Alone) {
      product_kernel<T, GATED, 2, 2, 2, 2, 3, 128, WHOLE, SPLIT><<<grid, 256, 0, s>>>(a);
      return;
    }
  }
  if (t == kTile128) product_kernel<T, GATED, 2, 2, 2, 2, 2, 128, WHOLE, SPLIT><<<grid, 256, 0, s>>>(a);
  else if (t == kTile64) product_kernel<T, GATED, 1, 2, 2, 2, 3, 128, WHOLE, SPLIT><<<grid, 256, 0, s>>>(a);
  else product_kernel<T, GATED, 1, 2, 1, 4, 4, 64, WHOLE, SPLIT><<<grid, 256, 0, s>>>(a);
}

template <typename T, bool GATED>
int run_product(const Plan &p, ProductArgs a, hipStream_t s) {
  a.tiles_n = p.tiles_n;
  a.splits = p.splits;
  a.stages_per_split = p.stages_per_split;
  a.pitch = partial_pitch(a.N, GATED);
  // a launch's lanes are counted in 32 bits: more tiles than that go by parts of the rows
  constexpr int64_t kMostItems = int64_t(1) << 22;
  const int64_t height = kTiles[p.tile].rows;
  const int64_t rows_at_once = p.splits > 1 ? a.M : std::max<int64_t>(1, kMostItems / p.tiles_n) * height;
  const ProductArgs all = a;
  for (int64_t r = 0; r < all.M; r += rows_at_once) {
    a.M = std::min(all.M - r, rows_at_once);
    a.A = static_cast<const T *>(all.A) + r * all.lda;
    a.out = static_cast<T *>(all.out) + r * all.ldo;
    a.gu = all.gu != nullptr ? static_cast<T *>(all.gu) + r * all.ldgu : nullptr;
    a.tiles_m = (int32_t)ceil_div(a.M, height);
    const dim3 grid((uint32_t)(ceil_div((int64_t)a.tiles_m * a.tiles_n * a.splits, (int64_t)8) * 8));
    const bool whole = a.K % kVec<T> == 0 && (!GATED || a.cols % (2 * kVec<T>) == 0);
    if (p.splits > 1) whole ? launch_tile<T, GATED, true, true>(p.tile, grid, a, s) : launch_tile<T, GATED, false, true>(p.tile, grid, a, s);
    else whole ? launch_tile<T, GATED, true, false>(p.tile, grid, a, s) : launch_tile<T, GATED, false, false>(p.tile, grid, a, s);
    if (const int rc = check_launch(); rc != BSR_OK) return rc;
    if (p.splits > 1) {
      auto join = [&](auto lg) {
        constexpr int LG = decltype(lg)::value;
        join_kernel<T, GATED, LG><<<dim3((uint32_t)blocks_for(a.M * ceil_div(a.N, (int64_t)4) << LG)), 256, 0, s>>>(
            a.act, a.partial, p.splits, a.M, a.N, a.pitch, static_cast<T *>(a.out), a.ldo, static_cast<T *>(a.gu), a.ldgu);
      };
      if (p.splits >= 6) join(std::integral_constant<int, 3>());
      else join(std::integral_constant<int, 0>());
      if (const int rc = check_launch(); rc != BSR_OK) return rc;
    }
  }
  return BSR_OK;
}

}  // namespace

}  // namespace bsr
