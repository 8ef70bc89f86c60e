// Internal declarations of the layer operators (see include/bsr_layer_ops.h): launchers and the device helpers that
// their kernels share.
#pragma once

#include "bsr_layer_ops.h"
#include "common.h"
#include "token_step.h"

namespace bsr {

// ---- launchers; all enqueue on `s` and return BSR_OK or BSR_ERR_HIP ----

// layer_norm.hip
int launch_layer_norm(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx, const void *gamma, const void *beta,
                      int param_dtype, float eps, void *Y, int64_t ldy, float *stats, hipStream_t s);
size_t layer_norm_grad_ws_bytes(int64_t M, int64_t D);
int launch_layer_norm_grad(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx, const void *gamma, int param_dtype,
                           const float *stats, const void *dY, int64_t lddy, void *dX, int64_t lddx, float *dgamma, float *dbeta,
                           int accumulate, void *ws, hipStream_t s);

// gated.hip
struct GatedArgs {
  const void *X;           // forward: [M x D]
  int dtype;
  int64_t M, D, ldx;
  const void *W;           // [D x 2F]
  int64_t F, ldw;
  int act;
};
size_t gated_ff_ws_bytes(const GatedArgs &a);
int launch_gated_ff(const GatedArgs &a, void *H, int64_t ldh, void *GU, int64_t ldgu, void *ws, hipStream_t s);
size_t gated_ff_grad_ws_bytes(const GatedArgs &a, const void *dGU, int64_t lddgu);
int launch_gated_ff_grad(const GatedArgs &a, const void *GU, int64_t ldgu, const void *dH, int64_t lddh, void *dGU, int64_t lddgu,
                         void *dX, int64_t lddx, void *ws, hipStream_t s);

// adamw.hip
constexpr int kMomentBlock = 128;
int launch_adamw(const bsr_adamw_item *items, int n, int param_dtype, int grad_dtype, int moments, const bsr_adamw_options &o,
                 hipStream_t s);
int launch_adamw_state_values(const uint8_t *codes, const uint8_t *scales, int64_t n, int which, void *out, int dtype,
                              hipStream_t s);

// ---- device helpers ----

// Sum over the aligned group of 2^LG lanes that a lane is in, the same bits in all of them: pairs, then pairs of pairs, and so on.
template <int CTRL>
__device__ __forceinline__ float dpp_of(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float other_row(float v) {           // lanes 0-15 and 16-31, 32-47 and 48-63 change places
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float((threadIdx.x & 16) ? r[0] : r[1]);
}
__device__ __forceinline__ float other_half(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
template <int LG>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (LG >= 1) v += dpp_of<0xB1>(v);      // neighbours (quad_perm 1,0,3,2)
  if constexpr (LG >= 2) v += dpp_of<0x4E>(v);      // pairs of them (2,3,0,1)
  if constexpr (LG >= 3) v += dpp_of<0x141>(v);     // quads of a half row, mirrored
  if constexpr (LG >= 4) v += dpp_of<0x140>(v);     // halves of a row of 16, mirrored
  if constexpr (LG >= 5) v += other_row(v);
  if constexpr (LG >= 6) v += other_half(v);
  return v;
}
// ... and the largest of numbers that compare as their bits do.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_of(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
template <int LG>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  v = max(v, dpp_of<0xB1>(v));
  v = max(v, dpp_of<0x4E>(v));
  v = max(v, dpp_of<0x141>(v));
  if constexpr (LG >= 4) v = max(v, dpp_of<0x140>(v));
  if constexpr (LG >= 5) v = max(v, __float_as_uint(other_row(__uint_as_float(v))));
  if constexpr (LG >= 6) v = max(v, __float_as_uint(other_half(__uint_as_float(v))));
  return v;
}

// VE consecutive numbers from element c on of an array of binary32 (bf16 false) or bfloat16; `otherwise` without an array.
template <int VE>
__device__ __forceinline__ void load_params(const void *p, bool bf16, int64_t c, float otherwise, float *out) {
  if (p == nullptr) {
#pragma unroll
    for (int q = 0; q < VE; ++q) out[q] = otherwise;
  } else if (bf16) {
    typedef uint32_t __attribute__((ext_vector_type(VE >= 2 ? VE / 2 : 2))) Words;
    struct __attribute__((packed, aligned(2))) Any { Words w; };
    const uint16_t *h = static_cast<const uint16_t *>(p) + c;
    if constexpr (VE == 1) out[0] = bf16_bits_to_float(*h);
    else {
      const Words w = reinterpret_cast<const Any *>(h)->w;
#pragma unroll
      for (int q = 0; q < VE; ++q) out[q] = __uint_as_float(q % 2 ? w[q / 2] & 0xFFFF0000u : w[q / 2] << 16);
    }
  } else {
    const float *f = static_cast<const float *>(p) + c;
    if constexpr (VE == 1) out[0] = *f;
    else {
#pragma unroll
      for (int q = 0; q < VE; q += 4) {
        const Words4 w = reinterpret_cast<const Any16 *>(f + q)->w;
#pragma unroll
        for (int i = 0; i < 4; ++i) out[q + i] = __uint_as_float(w[i]);
      }
    }
  }
}

}  // namespace bsr
