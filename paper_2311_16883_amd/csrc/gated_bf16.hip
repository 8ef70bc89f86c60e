// The gated block's products of bfloat16 operands, and [G | U] of few rows.
#include "gated_product.h"

namespace bsr {

namespace {

// [G | U] and H of the M <= 32 rows of X, one workgroup to 32 columns of G and the same of U, over the whole contraction: W is read once.
// Its waves take slices of 16 rows of W in turn, of which each has eight on their way, by plain loads at any alignment; a slice goes through
// the wave's own part of LDS, from which transposing loads make the matrix instructions' operand, so that nobody waits for anybody before
// the waves' sums are added up, in their order.
constexpr int kRowsWaves = 8, kRowsThreads = 64 * kRowsWaves, kSlices = 8, kSliceBytes = 16 * 128;
__global__ __launch_bounds__(kRowsThreads) void gated_rows_kernel(int act, const uint16_t *__restrict__ X, int M, int64_t D, int64_t ldx,
                                                                  const uint16_t *__restrict__ W, int64_t F, int64_t ldw, uint16_t *__restrict__ H,
                                                                  int64_t ldh, uint16_t *__restrict__ GU, int64_t ldgu, int groups) {
  typedef RowVec<uint16_t, 8> R;
  __shared__ __attribute__((aligned(1024))) uint8_t slices[kRowsWaves][kSlices * kSliceBytes];
  const int per_xcd = (groups + 7) / 8, group = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if (group >= groups || (int)(blockIdx.x >> 3) >= per_xcd) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, g4 = lane >> 4, L = lane & 15;
  uint8_t *const mine = slices[wave];
  const int row = lane >> 2, chunk = lane & 3;                 // of a slice: this lane's row and its 8 columns of the 32
  const int64_t c = (int64_t)group * 32 + chunk * 8;
  const int there = F - c >= 8 ? 8 : F > c ? (int)(F - c) : 0;
  const uint16_t *const x = X + ((lane & 31) < M ? (lane & 31) : M - 1) * ldx;
  // rows of 128 bytes, G's chunks of 16 in front, those of every other pair of rows changed with U's: reads touch every bank once
  const uint32_t to = (uint32_t)(row * 128 + ((chunk ^ (4 * ((row >> 1) & 1))) * 16));
  const uint32_t from = (uint32_t)((8 * (g4 >> 1) + (L >> 2)) * 128 + ((2 * (g4 & 1) + ((L & 3) >> 1)) ^ (4 * ((L >> 3) & 1))) * 16 + 8 * (L & 1));
  auto part = [](const uint16_t *p, int n) {                   // the first n of 8 numbers, zeros behind them
    uint16_t e[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) e[q] = q < n ? p[q] : (uint16_t)0;
    Words4 v;
    __builtin_memcpy(&v, e, 16);
    return v;
  };
  Words4 g[kSlices], u[kSlices], a[kSlices];
  auto load = [&](int64_t k0) {
#pragma unroll
    for (int t = 0; t < kSlices; ++t) {
      const int64_t k = k0 + (t * kRowsWaves + wave) * 16, kw = k + row, kx = k + 8 * half;
      g[t] = u[t] = a[t] = R::zero();
      if (kw < D) {
        const uint16_t *p = W + kw * ldw + c;
        if (there == 8) {
          g[t] = R::load(p);
          u[t] = R::load(p + F);
        } else if (there > 0) {
          g[t] = part(p, there);
          u[t] = part(p + F, there);
        }
      }
      if (kx + 8 <= D) a[t] = R::load(x + kx);
      else if (kx < D) a[t] = part(x + kx, (int)(D - kx));
    }
  };
  v16f acc[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.0f;
  constexpr int64_t kStep = kSlices * kRowsWaves * 16;
  load(0);
  for (int64_t k0 = 0; k0 < D; k0 += kStep) {
    Words4 now[kSlices];
#pragma unroll
    for (int t = 0; t < kSlices; ++t) {
      *reinterpret_cast<Words4 *>(mine + t * kSliceBytes + to) = g[t];
      *reinterpret_cast<Words4 *>(mine + t * kSliceBytes + (to ^ 64u)) = u[t];
      now[t] = a[t];
    }
    __builtin_amdgcn_wave_barrier();
    if (k0 + kStep < D) load(k0 + kStep);
#pragma unroll
    for (int t = 0; t < kSlices; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        typedef v4s __attribute__((address_space(3))) * lds_v4s;
        const uint8_t *p = mine + t * kSliceBytes + (from ^ (j * 64u));
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(p + 512));
        const v8s b = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, b), __builtin_bit_cast(v8bf, now[t]), acc[j], 0, 0, 0);
      }
    __builtin_amdgcn_wave_barrier();
  }
  // a wave's sums take its part of LDS: number r of lane l at 64 r + l
  float *const sums = reinterpret_cast<float *>(mine);
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) sums[(j * 16 + r) * 64 + lane] = acc[j][r];
  __syncthreads();
  const int m = lane & 31;
#pragma unroll
  for (int r = wave; r < 16; r += kRowsWaves) {
    const int64_t col = (int64_t)group * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
    float gs = 0.0f, us = 0.0f;
#pragma unroll
    for (int w = 0; w < kRowsWaves; ++w) {
      const float *p = reinterpret_cast<const float *>(slices[w]);
      gs += p[r * 64 + lane];
      us += p[(16 + r) * 64 + lane];
    }
    if (m >= M || col >= F) continue;
    H[m * ldh + col] = from_float<uint16_t>(activation_value(act, gs) * us);
    if (GU != nullptr) {
      GU[m * ldgu + col] = from_float<uint16_t>(gs);
      GU[m * ldgu + F + col] = from_float<uint16_t>(us);
    }
  }
}
static_assert(kSlices * kSliceBytes >= 32 * 64 * 4, "a wave's sums fit its part of LDS");

}  // namespace

int launch_gated_rows_bf16(const GatedArgs &g, void *H, int64_t ldh, void *GU, int64_t ldgu, hipStream_t s) {
  const int64_t groups = ceil_div(g.F, (int64_t)32);
  gated_rows_kernel<<<dim3((uint32_t)(ceil_div(groups, (int64_t)8) * 8)), kRowsThreads, 0, s>>>(
      g.act, static_cast<const uint16_t *>(g.X), (int)g.M, g.D, g.ldx, static_cast<const uint16_t *>(g.W), g.F, g.ldw,
      static_cast<uint16_t *>(H), ldh, static_cast<uint16_t *>(GU), ldgu, (int)groups);
  return check_launch();
}

int launch_product_bf16(const Plan &p, const ProductArgs &a, bool gated, hipStream_t s) {
  return gated ? run_product<uint16_t, true>(p, a, s) : run_product<uint16_t, false>(p, a, s);
}

}  // namespace bsr
