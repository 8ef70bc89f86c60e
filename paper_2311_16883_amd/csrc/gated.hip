// Gated feed-forward block, forward and backward.
#include <algorithm>

#include "layer_ops.h"

namespace bsr {

namespace {

constexpr int kTile = 32;

template <int ACT>
__device__ __forceinline__ float act_of(float g) {
  if constexpr (ACT == BSR_ACT_SILU) return g / (1.0f + expf(-g));
  else if constexpr (ACT == BSR_ACT_GELU) return 0.5f * g * (1.0f + erff(g * 0.70710678118654752f));
  else if constexpr (ACT == BSR_ACT_GELU_TANH) return 0.5f * g * (1.0f + tanhf(0.79788456080286536f * (g + 0.044715f * g * g * g)));
  else return fmaxf(g, 0.0f);
}
template <int ACT>
__device__ __forceinline__ float slope_of(float g) {
  if constexpr (ACT == BSR_ACT_SILU) {
    const float p = 1.0f / (1.0f + expf(-g));
    return p * (1.0f + g * (1.0f - p));
  } else if constexpr (ACT == BSR_ACT_GELU) {
    return 0.5f * (1.0f + erff(g * 0.70710678118654752f)) + g * expf(-0.5f * g * g) * 0.39894228040143268f;
  } else if constexpr (ACT == BSR_ACT_GELU_TANH) {
    const float t = tanhf(0.79788456080286536f * (g + 0.044715f * g * g * g));
    return 0.5f * (1.0f + t) + 0.5f * g * (1.0f - t * t) * 0.79788456080286536f * (1.0f + 3.0f * 0.044715f * g * g);
  } else return g > 0.0f ? 1.0f : 0.0f;
}

template <typename T, int ACT>
__global__ __launch_bounds__(1024) void gated_simple_kernel(const T *__restrict__ X, int64_t M, int64_t D, int64_t ldx,
                                                            const T *__restrict__ W, int64_t F, int64_t ldw, T *__restrict__ H,
                                                            int64_t ldh, T *__restrict__ GU, int64_t ldgu) {
  __shared__ float sx[kTile][kTile + 1], sg[kTile][kTile + 1], su[kTile][kTile + 1];
  const int c = threadIdx.x % kTile, r = threadIdx.x / kTile;
  for (int64_t m0 = (int64_t)blockIdx.y * kTile; m0 < M; m0 += (int64_t)gridDim.y * kTile) {
    const int64_t m = m0 + r, f = (int64_t)blockIdx.x * kTile + c;
    float g = 0.0f, u = 0.0f;
    for (int64_t k0 = 0; k0 < D; k0 += kTile) {
      sx[r][c] = m < M && k0 + c < D ? elem_to_float<T>(X[m * ldx + k0 + c]) : 0.0f;
      sg[r][c] = k0 + r < D && f < F ? elem_to_float<T>(W[(k0 + r) * ldw + f]) : 0.0f;
      su[r][c] = k0 + r < D && f < F ? elem_to_float<T>(W[(k0 + r) * ldw + F + f]) : 0.0f;
      __syncthreads();
      for (int k = 0; k < kTile; ++k) {
        g += sx[r][k] * sg[k][c];
        u += sx[r][k] * su[k][c];
      }
      __syncthreads();
    }
    if (m < M && f < F) {
      H[m * ldh + f] = from_float<T>(act_of<ACT>(g) * u);
      if (GU != nullptr) {
        GU[m * ldgu + f] = from_float<T>(g);
        GU[m * ldgu + F + f] = from_float<T>(u);
      }
    }
  }
}

template <typename T, int ACT>
__global__ __launch_bounds__(256) void gated_slope_kernel(const T *GU, int64_t M, int64_t F, int64_t ldgu, const T *__restrict__ dH,
                                                          int64_t lddh, T *dGU, int64_t lddgu) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * F; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / F, f = i % F;
    const float g = elem_to_float<T>(GU[m * ldgu + f]), u = elem_to_float<T>(GU[m * ldgu + F + f]), d = elem_to_float<T>(dH[m * lddh + f]);
    dGU[m * lddgu + f] = from_float<T>(d * u * slope_of<ACT>(g));
    dGU[m * lddgu + F + f] = from_float<T>(d * act_of<ACT>(g));
  }
}

// C = A B^T
template <typename T>
__global__ __launch_bounds__(1024) void product_simple_kernel(const T *__restrict__ A, int64_t M, int64_t K, int64_t lda,
                                                              const T *__restrict__ B, int64_t N, int64_t ldb, T *__restrict__ C,
                                                              int64_t ldc) {
  __shared__ float sa[kTile][kTile + 1], sb[kTile][kTile + 1];
  const int c = threadIdx.x % kTile, r = threadIdx.x / kTile;
  for (int64_t m0 = (int64_t)blockIdx.y * kTile; m0 < M; m0 += (int64_t)gridDim.y * kTile) {
    const int64_t m = m0 + r, n0 = (int64_t)blockIdx.x * kTile;
    float sum = 0.0f;
    for (int64_t k0 = 0; k0 < K; k0 += kTile) {
      sa[r][c] = m < M && k0 + c < K ? elem_to_float<T>(A[m * lda + k0 + c]) : 0.0f;
      sb[r][c] = n0 + r < N && k0 + c < K ? elem_to_float<T>(B[(n0 + r) * ldb + k0 + c]) : 0.0f;
      __syncthreads();
      for (int k = 0; k < kTile; ++k) sum += sa[r][k] * sb[c][k];
      __syncthreads();
    }
    if (m < M && n0 + c < N) C[m * ldc + n0 + c] = from_float<T>(sum);
  }
}

template <typename F>
void with_act(int act, F f) {
  if (act == BSR_ACT_SILU) f(std::integral_constant<int, BSR_ACT_SILU>());
  else if (act == BSR_ACT_GELU) f(std::integral_constant<int, BSR_ACT_GELU>());
  else if (act == BSR_ACT_GELU_TANH) f(std::integral_constant<int, BSR_ACT_GELU_TANH>());
  else f(std::integral_constant<int, BSR_ACT_RELU>());
}

dim3 tiles(int64_t M, int64_t N) {
  return dim3((uint32_t)ceil_div(N, (int64_t)kTile), (uint32_t)std::min(ceil_div(M, (int64_t)kTile), int64_t(16)));
}

template <typename T>
int forward(const GatedArgs &a, void *H, int64_t ldh, void *GU, int64_t ldgu, hipStream_t s) {
  with_act(a.act, [&](auto act) {
    gated_simple_kernel<T, decltype(act)::value><<<tiles(a.M, a.F), 1024, 0, s>>>(
        static_cast<const T *>(a.X), a.M, a.D, a.ldx, static_cast<const T *>(a.W), a.F, a.ldw, static_cast<T *>(H), ldh,
        static_cast<T *>(GU), ldgu);
  });
  return check_launch();
}

template <typename T>
int backward(const GatedArgs &a, const void *GU, int64_t ldgu, const void *dH, int64_t lddh, void *dGU, int64_t lddgu, void *dX,
             int64_t lddx, hipStream_t s) {
  if (a.M > 0 && a.F > 0) {
    with_act(a.act, [&](auto act) {
      gated_slope_kernel<T, decltype(act)::value>
          <<<dim3((uint32_t)std::min(ceil_div(a.M * a.F, (int64_t)256), int64_t(1) << 20)), 256, 0, s>>>(
              static_cast<const T *>(GU), a.M, a.F, ldgu, static_cast<const T *>(dH), lddh, static_cast<T *>(dGU), lddgu);
    });
    if (const int rc = check_launch(); rc != BSR_OK) return rc;
  }
  if (dX == nullptr || a.D == 0) return BSR_OK;
  product_simple_kernel<T><<<tiles(a.M, a.D), 1024, 0, s>>>(static_cast<const T *>(dGU), a.M, 2 * a.F, lddgu,
                                                            static_cast<const T *>(a.W), a.D, a.ldw, static_cast<T *>(dX), lddx);
  return check_launch();
}

}  // namespace

size_t gated_ff_ws_bytes(const GatedArgs &) { return 0; }

int launch_gated_ff(const GatedArgs &a, void *H, int64_t ldh, void *GU, int64_t ldgu, void *, hipStream_t s) {
  return a.dtype == BSR_F32 ? forward<float>(a, H, ldh, GU, ldgu, s) : forward<uint16_t>(a, H, ldh, GU, ldgu, s);
}

size_t gated_ff_grad_ws_bytes(const GatedArgs &, const void *, int64_t) { return 0; }

int launch_gated_ff_grad(const GatedArgs &a, const void *GU, int64_t ldgu, const void *dH, int64_t lddh, void *dGU, int64_t lddgu,
                         void *dX, int64_t lddx, void *, hipStream_t s) {
  return a.dtype == BSR_F32 ? backward<float>(a, GU, ldgu, dH, lddh, dGU, lddgu, dX, lddx, s)
                            : backward<uint16_t>(a, GU, ldgu, dH, lddh, dGU, lddgu, dX, lddx, s);
}

}  // namespace bsr
