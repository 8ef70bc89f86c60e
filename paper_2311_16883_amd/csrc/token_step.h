// Internal declarations of the token operators (see include/bsr_token_step.h): launchers and the device helpers that
// their kernels share.
#pragma once

#include "bsr_token_step.h"
#include "common.h"

namespace bsr {

// ---- launchers; all enqueue on `s` and return BSR_OK or BSR_ERR_HIP ----

// token_rows.hip: whole rows copied, scaled, weighted and added up.
int launch_embedding_lookup(const void *table, int dtype, int64_t V, int64_t D, int64_t ldt, const void *tokens, int index_type,
                            int64_t T, float scale, void *out, int64_t ldo, hipStream_t s);
int launch_expert_gather(const void *X, int dtype, int64_t T, int64_t D, int64_t ldx, const int32_t *slots, int64_t k,
                         const int32_t *order, int64_t rows, void *Xs, int64_t ldxs, hipStream_t s);
int launch_expert_combine(const void *Ys, int dtype, int64_t rows, int64_t D, int64_t ldys, const int32_t *slots, int64_t T,
                          int64_t k, const float *weights, void *out, int64_t ldo, hipStream_t s);
int launch_expert_combine_grad(const void *Ys, int dtype, int64_t rows, int64_t D, int64_t ldys, const int32_t *slots,
                               const int32_t *order, int64_t T, int64_t k, const float *weights, const void *dOut, int64_t lddo,
                               void *dYs, int64_t lddys, float *dweights, hipStream_t s);

// token_sort.hip: stable sorts by key.
constexpr int kMaxExperts = BSR_MAX_EXPERTS;
size_t expert_sort_ws_bytes(int64_t n, int64_t E);
int launch_expert_sort(const void *ids, int index_type, int64_t n, int64_t E, int64_t align, int32_t *offsets, int32_t *counts,
                       int32_t *order, int64_t rows, int32_t *slots, void *ws, hipStream_t s);
// (token, position) pairs in ascending order, positions ascending among equal tokens, those with a token outside [0, V) last
// (with the key V).  The sort leaves most of the GPU idle, so its launches also clear [V x D] binary32 where `clear` is set.
size_t token_sort_ws_bytes(int64_t T, int64_t V);
struct ClearJob {
  float *p;                // null: nothing to clear
  int64_t rows, cols, ld;
  bool stream;             // past the caches; p is 16-byte aligned and ld == cols then
  int64_t per;             // elements that a workgroup clears, set by the sort
};
int launch_token_sort(const void *tokens, int index_type, int64_t T, int64_t V, const ClearJob &clear, void *ws,
                      const uint2 **sorted, hipStream_t s);

// token_grad.hip: sums of rows with equal tokens.
size_t embedding_grad_ws_bytes(int64_t T, int64_t V, int64_t D);
int launch_embedding_grad(const void *tokens, int index_type, int64_t T, const void *dY, int dtype, int64_t D, int64_t lddy,
                          float scale, int64_t V, float *dE, int64_t ldde, int accumulate, void *ws, hipStream_t s);

// distill.hip
constexpr int kMaxTeacher = 1024;
size_t distill_ws_bytes(int64_t N, int64_t V, int64_t K);
struct DistillArgs {
  const void *logits;
  int dtype;
  int64_t N, V, ldz;
  const void *ids;
  int index_type;
  const void *teacher;
  int teacher_dtype;
  int64_t K;
  float temperature;
};
int launch_distill_loss(const DistillArgs &a, float *loss, float *stats, void *ws, hipStream_t s);
int launch_distill_grad(const DistillArgs &a, const float *stats, const float *dloss, void *dlogits, int64_t ldd, hipStream_t s);
int launch_distill_loss_grad(const DistillArgs &a, const float *dloss, float *loss, void *dlogits, int64_t ldd, void *ws,
                             hipStream_t s);

// Whether rows that are read or written once pass by the caches: not where the caches can hold them (fewer than `least` bytes of them
// all), and not where they share 128-byte lines.
inline bool stream_rows(const void *p, int64_t rows, int64_t D, int64_t ld, int dtype, int64_t least) {
  const int64_t e = elem_bytes(dtype);
  return (uintptr_t)p % 128 == 0 && D * e % 128 == 0 && ld * e % 128 == 0 && rows * D * e >= least;
}

// ---- device helpers ----

// Index i of an int32 or int64 array, as int64.
template <typename I>
__device__ __forceinline__ int64_t load_index(const void *p, int64_t i) { return (int64_t)static_cast<const I *>(p)[i]; }

// 16 bytes at any element (global memory takes them at any alignment).
struct __attribute__((packed, aligned(2))) Any16 {
  uint32_t __attribute__((ext_vector_type(4))) w;
};
typedef uint32_t __attribute__((ext_vector_type(4))) Words4;

// A vector of a row: VE = 16 / sizeof(T) elements, or one where rows are shorter than that.
template <typename T, int VE>
struct RowVec;
template <typename T>
struct RowVec<T, 16 / (int)sizeof(T)> {
  typedef Words4 Raw;
  static __device__ __forceinline__ Raw load(const T *p) { return reinterpret_cast<const Any16 *>(p)->w; }
  static __device__ __forceinline__ void store(T *p, const Raw &v) { reinterpret_cast<Any16 *>(p)->w = v; }
  static __device__ __forceinline__ Raw zero() { return Raw{0, 0, 0, 0}; }
  static __device__ __forceinline__ float elem(const Raw &v, int q) { return raw_elem<T, 16 / (int)sizeof(T)>(v, q); }
};
template <typename T>
struct RowVec<T, 1> {
  typedef T Raw;
  static __device__ __forceinline__ Raw load(const T *p) { return *p; }
  static __device__ __forceinline__ void store(T *p, const Raw &v) { *p = v; }
  static __device__ __forceinline__ Raw zero() { return (T)0; }
  static __device__ __forceinline__ float elem(const Raw &v, int) { return elem_to_float<T>(v); }
};

// binary32 -> T, to nearest even.
typedef __bf16 __attribute__((ext_vector_type(2))) Bf16x2;
typedef float __attribute__((ext_vector_type(2))) Float2;
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(Float2{a, b}, Bf16x2));
}
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ uint16_t from_float<uint16_t>(float v) { return (uint16_t)bf16_pair(v, 0.0f); }

template <typename T, int VE>
__device__ __forceinline__ typename RowVec<T, VE>::Raw pack_row(const float *v) {
  if constexpr (VE == 1) return from_float<T>(v[0]);
  else if constexpr (sizeof(T) == 4)
    return Words4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  else return Words4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
}

// A vector of a row that is read once: non-temporal (STREAM) or as any other.
template <typename T, int VE, bool STREAM>
__device__ __forceinline__ typename RowVec<T, VE>::Raw load_once(const T *p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const typename RowVec<T, VE>::Raw *>(p));
  else return RowVec<T, VE>::load(p);
}

// ... and one that is written and left.
template <typename T, int VE, bool STREAM>
__device__ __forceinline__ void store_once(T *p, const typename RowVec<T, VE>::Raw &v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<typename RowVec<T, VE>::Raw *>(p));
  else RowVec<T, VE>::store(p, v);
}

// Rows are taken VE elements at a time by the lanes of a group.  The last vector of a row that is no whole number of vectors
// ends with the row: it starts earlier and holds elements of the one before again, which copies and sums may write twice
// (the same values).
__device__ __forceinline__ int64_t vector_start(int64_t v, int VE, int64_t D) {
  const int64_t c = v * VE;
  return c + VE <= D ? c : D - VE;
}

}  // namespace bsr
