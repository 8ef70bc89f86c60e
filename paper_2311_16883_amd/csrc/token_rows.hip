// Whole rows moved by index: the token table's lookup, tokens to the experts and back, and the gradients of that.
//
// All of these are bound by memory: a few operations per element, every needed row read once and every row of the result
// written once.  A row belongs to a group of `1 << sh` lanes of one wave (16 .. 64, by the row's length: row_lanes), which
// walk along it 16 bytes a lane, at any alignment; nothing is shared between groups, so there is no LDS and no barrier, and
// the loads of many rows are on their way per compute unit.
// bf16: lookup of [32768 x 1536] 22.7 us (5.8 TB/s of the rows that are read and written; a copy on this GPU 5.1, a fill 6.8), [25088 x 4] of
// 1536 to their experts 63 (6.0), weighted return of [25088 x 2] 43 (5.3), gradients of that 60 (6.3), of the odd [9947 x 3] of 805 12 (5.0).
#include "token_step.h"

namespace bsr {

namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;          // vectors that a lane has on their way, per row
// Bytes from which rows pass by the caches.  Read: [25088 x 2] choices of 1536 bf16, weighted return 48.9 -> 42.2 us, [4096 x 8] of 2048,
// gradients, 116.7 -> 109.5; of rows that share lines, [9947 x 3] of 805, 12.0 -> 14.5.  Written: lookup of [32768 x 1536] bf16 28.9 -> 23.4,
// [25088 x 4] of 1536 to their experts 87 -> 75.6, return of [30000 x 1] of 1024 23.5 -> 19.4; of rows that share lines, [8000 x 2] of
// 1537 to their experts, 22.0 -> 23.7.
constexpr int64_t kStreamRead = int64_t(64) << 20, kStreamWrite = int64_t(32) << 20;
constexpr int kChoices = 8;        // choices of a token that are handled together

// The workgroup's number in a grid of two dimensions (the lanes of the first are counted in 32 bits).
__device__ __forceinline__ int64_t block_number() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// out[t] = scale * table[tokens[t]]
template <typename T, int VE, typename I, bool OUT>
__global__ __launch_bounds__(kThreads) void embedding_lookup_kernel(const T *__restrict__ table, int64_t V, int64_t D,
                                                                    int64_t ldt, const void *__restrict__ tokens, int64_t rows,
                                                                    float scale, T *__restrict__ out, int64_t ldo, int sh) {
  typedef RowVec<T, VE> R;
  const int64_t row = (block_number() * kThreads + threadIdx.x) >> sh;
  if (row >= rows) return;
  const int li = threadIdx.x & ((1 << sh) - 1), step = 1 << sh;
  const int64_t tok = load_index<I>(tokens, row);
  const bool there = tok >= 0 && tok < V;
  const T *src = table + (there ? tok : 0) * ldt;
  T *dst = out + row * ldo;
  const int64_t vecs = ceil_div(D, (int64_t)VE);
  for (int64_t v0 = li; v0 < vecs; v0 += (int64_t)kAhead * step) {
    typename R::Raw x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t v = v0 + (int64_t)u * step;
      x[u] = R::zero();
      if (there && v < vecs) x[u] = R::load(src + vector_start(v, VE, D));
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t v = v0 + (int64_t)u * step;
      if (v >= vecs) continue;
      float f[VE];
#pragma unroll
      for (int q = 0; q < VE; ++q) f[q] = there ? R::elem(x[u], q) * scale : 0.0f;
      store_once<T, VE, OUT>(dst + vector_start(v, VE, D), pack_row<T, VE>(f));
    }
  }
}

// +0.0 in the rows of [s0, s0 + count) that hold no entry, by one wave; count <= 64.
template <typename T, int VE>
__device__ __forceinline__ void clear_padding(const int32_t *__restrict__ order, int64_t rows, int64_t s0, int count,
                                              T *__restrict__ Xs, int64_t ldxs, int64_t D, int lane) {
  typedef RowVec<T, VE> R;
  if (s0 >= rows) return;
  const int64_t s = s0 + lane;
  uint64_t pad = __ballot(lane < count && s < rows && order[s < rows ? s : s0] < 0);
  const int64_t vecs = ceil_div(D, (int64_t)VE);
  for (; pad != 0; pad &= pad - 1) {
    T *dst = Xs + (s0 + __builtin_ctzll(pad)) * ldxs;
    for (int64_t v = lane; v < vecs; v += 64) R::store(dst + vector_start(v, VE, D), R::zero());
  }
}

// Xs[slots[t][j]] = X[t] for all j: every row of X is read once.  The first `pad_blocks` workgroups clear the padding.
template <typename T, int VE, bool OUT>
__global__ __launch_bounds__(kThreads) void expert_gather_kernel(const T *__restrict__ X, int64_t tokens, int64_t D, int64_t ldx,
                                                                 const int32_t *__restrict__ slots, int64_t k,
                                                                 const int32_t *__restrict__ order, int64_t rows,
                                                                 T *__restrict__ Xs, int64_t ldxs, int sh, int64_t pad_blocks,
    int pad_rows) {
  typedef RowVec<T, VE> R;
  const int t = threadIdx.x;
  const int64_t block = block_number();
  if (block < pad_blocks) {
    clear_padding<T, VE>(order, rows, (block * (kThreads / 64) + (t >> 6)) * pad_rows, pad_rows, Xs, ldxs, D, t & 63);
    return;
  }
  const int64_t row = ((block - pad_blocks) * kThreads + t) >> sh;
  if (row >= tokens) return;
  const int li = t & ((1 << sh) - 1), step = 1 << sh;
  const T *src = X + row * ldx;
  const int32_t *mine = slots + row * k;
  const int64_t vecs = ceil_div(D, (int64_t)VE);
  for (int64_t v0 = li; v0 < vecs; v0 += (int64_t)kAhead * step) {
    typename R::Raw x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t v = v0 + (int64_t)u * step;
      if (v < vecs) x[u] = R::load(src + vector_start(v, VE, D));
    }
    for (int64_t j = 0; j < k; ++j) {
      const int64_t slot = mine[j];
      if (slot < 0 || slot >= rows) continue;
      T *dst = Xs + slot * ldxs;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int64_t v = v0 + (int64_t)u * step;
        if (v < vecs) store_once<T, VE, OUT>(dst + vector_start(v, VE, D), x[u]);
      }
    }
  }
}

// The slots (and weights) of up to kChoices choices of a token; a choice without a slot has the weight 0 and the row 0, which
// is read but not used.
struct Choices {
  int32_t slot[kChoices];
  float weight[kChoices];
  bool there[kChoices];
};
template <int KC>
__device__ __forceinline__ void load_choices(const int32_t *__restrict__ slots, const float *__restrict__ weights, int64_t first,
                                             int count, int64_t rows, Choices *c) {
#pragma unroll
  for (int j = 0; j < KC; ++j) {
    const int32_t slot = j < count ? slots[first + j] : -1;
    c->there[j] = slot >= 0 && slot < rows;
    c->slot[j] = c->there[j] ? slot : 0;
    c->weight[j] = !c->there[j] ? 0.0f : weights != nullptr ? weights[first + j] : 1.0f;
  }
}

// out[t] = sum_j weights[t][j] * Ys[slots[t][j]]; KC choices are read together.
template <typename T, int VE, int KC, bool STREAM, bool OUT>
__global__ __launch_bounds__(kThreads) void expert_combine_kernel(const T *__restrict__ Ys, int64_t rows, int64_t D, int64_t ldys,
                                                                  const int32_t *__restrict__ slots, int64_t tokens, int64_t k,
                                                                  const float *__restrict__ weights, T *__restrict__ out,
                                                                  int64_t ldo, int sh) {
  typedef RowVec<T, VE> R;
  const int64_t row = (block_number() * kThreads + threadIdx.x) >> sh;
  if (row >= tokens) return;
  const int li = threadIdx.x & ((1 << sh) - 1), step = 1 << sh;
  T *dst = out + row * ldo;
  const int64_t vecs = ceil_div(D, (int64_t)VE);
  Choices c;
  load_choices<KC>(slots, weights, row * k, (int)(k < KC ? k : KC), rows, &c);
  for (int64_t v = li; v < vecs; v += step) {
    const int64_t at = vector_start(v, VE, D);
    float sum[VE];
#pragma unroll
    for (int q = 0; q < VE; ++q) sum[q] = 0.0f;
    for (int64_t j0 = 0; j0 < k; j0 += KC) {
      if (k > KC) load_choices<KC>(slots, weights, row * k + j0, (int)(k - j0 < KC ? k - j0 : KC), rows, &c);
      typename R::Raw y[KC];
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        y[j] = R::zero();
        if (c.there[j]) y[j] = load_once<T, VE, STREAM>(Ys + (int64_t)c.slot[j] * ldys + at);
      }
#pragma unroll
      for (int j = 0; j < KC; ++j) {
#pragma unroll
        for (int q = 0; q < VE; ++q) sum[q] = fmaf(c.weight[j], R::elem(y[j], q), sum[q]);
      }
    }
    store_once<T, VE, OUT>(dst + at, pack_row<T, VE>(sum));
  }
}

// dYs[slots[t][j]] = weights[t][j] * dOut[t], dweights[t][j] = <Ys[slots[t][j]], dOut[t]>: dOut is read once per KC choices, and
// the products of a row are added up by its lanes in a fixed order.
template <typename T, int VE, int KC, bool STREAM, bool OUT>
__global__ __launch_bounds__(kThreads) void expert_combine_grad_kernel(
    const T *__restrict__ Ys, int64_t rows, int64_t D, int64_t ldys, const int32_t *__restrict__ slots,
    const int32_t *__restrict__ order, int64_t tokens, int64_t k, const float *__restrict__ weights, const T *__restrict__ dOut,
    int64_t lddo, T *__restrict__ dYs, int64_t lddys, float *__restrict__ dweights, int sh, int64_t pad_blocks,
    int pad_rows) {
  typedef RowVec<T, VE> R;
  const int t = threadIdx.x;
  const int64_t block = block_number();
  if (block < pad_blocks) {
    clear_padding<T, VE>(order, rows, (block * (kThreads / 64) + (t >> 6)) * pad_rows, pad_rows, dYs, lddys, D, t & 63);
    return;
  }
  const int64_t row = ((block - pad_blocks) * kThreads + t) >> sh;
  if (row >= tokens) return;
  const int li = t & ((1 << sh) - 1), step = 1 << sh;
  const T *src = dOut + row * lddo;
  const int64_t vecs = ceil_div(D, (int64_t)VE);
  for (int64_t j0 = 0; j0 < k; j0 += KC) {
    const int count = (int)(k - j0 < KC ? k - j0 : KC);
    Choices c;
    load_choices<KC>(slots, weights, row * k + j0, count, rows, &c);
    float dot[KC];
#pragma unroll
    for (int j = 0; j < KC; ++j) dot[j] = 0.0f;
    for (int64_t v = li; v < vecs; v += step) {
      const int64_t at = vector_start(v, VE, D);
      const int again = (int)(v * VE - at);              // elements that the vector before holds as well
      const typename R::Raw g = R::load(src + at);
      typename R::Raw y[KC];
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        y[j] = R::zero();
        if (c.there[j]) y[j] = load_once<T, VE, STREAM>(Ys + (int64_t)c.slot[j] * ldys + at);
      }
      float gf[VE];
#pragma unroll
      for (int q = 0; q < VE; ++q) gf[q] = R::elem(g, q);
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        if (!c.there[j]) continue;
        float p[VE];
#pragma unroll
        for (int q = 0; q < VE; ++q) p[q] = c.weight[j] * gf[q];
        store_once<T, VE, OUT>(dYs + (int64_t)c.slot[j] * lddys + at, pack_row<T, VE>(p));
#pragma unroll
        for (int q = 0; q < VE; ++q) dot[j] = q >= again ? fmaf(R::elem(y[j], q), gf[q], dot[j]) : dot[j];
      }
    }
#pragma unroll
    for (int j = 0; j < KC; ++j) {
      for (int d = step >> 1; d >= 1; d >>= 1) dot[j] += __shfl_xor(dot[j], d, 64);
      if (li == 0 && j < count) dweights[row * k + j0 + j] = dot[j];
    }
  }
}

// Lanes that share a row (as a power of two): 64 for rows of 64 vectors or more, fewer for short ones, down to 16.
int row_lanes(int64_t vecs) { return vecs > 32 ? 6 : vecs > 16 ? 5 : 4; }

int64_t row_blocks(int64_t rows, int sh) { return ceil_div(rows << sh, (int64_t)kThreads); }

dim3 grid_of(int64_t blocks) {
  const int64_t x = blocks < 1 ? 1 : blocks < (int64_t(1) << 22) ? blocks : int64_t(1) << 22;
  return dim3((unsigned)x, (unsigned)ceil_div(blocks, x));
}

// Rows of the sorted matrix that one wave looks over for padding, one after the other: few where there are few rows.
int padding_rows(int64_t rows) { return rows < 4096 ? 1 : rows < 32768 ? 4 : 16; }
int64_t padding_blocks(int64_t rows) { return ceil_div(rows, (int64_t)padding_rows(rows) * (kThreads / 64)); }

}  // namespace

// f32 / bf16 and whole or single-element vectors
#define BSR_BY_ROW(dtype, D, CALL)                              \
  if ((dtype) == BSR_F32) {                                     \
    if ((D) >= 4) { CALL(float, 4); } else { CALL(float, 1); }  \
  } else {                                                      \
    if ((D) >= 8) { CALL(uint16_t, 8); } else { CALL(uint16_t, 1); } \
  }

int launch_embedding_lookup(const void *table, int dtype, int64_t V, int64_t D, int64_t ldt, const void *tokens, int index_type,
                            int64_t T, float scale, void *out, int64_t ldo, hipStream_t s) {
  const bool write = stream_rows(out, T, D, ldo, dtype, kStreamWrite);
#define BSR_CALL__(TY, VE, I, OUT)                                                                                            \
  const int sh = row_lanes(ceil_div(D, (int64_t)VE));                                                                         \
  hipLaunchKernelGGL((embedding_lookup_kernel<TY, VE, I, OUT>), grid_of(row_blocks(T, sh)), dim3(kThreads), 0, s,                 \
                     static_cast<const TY *>(table), V, D, ldt, tokens, T, scale, static_cast<TY *>(out), ldo, sh)
#define BSR_CALL_(TY, VE, I)                                                \
  if (write) { BSR_CALL__(TY, VE, I, (VE != 1)); } else { BSR_CALL__(TY, VE, I, false); }
#define BSR_CALL(TY, VE)                                                    \
  if (index_type == BSR_I64) { BSR_CALL_(TY, VE, int64_t) } else { BSR_CALL_(TY, VE, int32_t) }
  BSR_BY_ROW(dtype, D, BSR_CALL)
#undef BSR_CALL
#undef BSR_CALL_
#undef BSR_CALL__
  return check_launch();
}

int launch_expert_gather(const void *X, int dtype, int64_t T, int64_t D, int64_t ldx, const int32_t *slots, int64_t k,
                         const int32_t *order, int64_t rows, void *Xs, int64_t ldxs, hipStream_t s) {
  const int64_t pad = padding_blocks(rows);
  const bool write = stream_rows(Xs, rows, D, ldxs, dtype, kStreamWrite);
#define BSR_CALL_(TY, VE, OUT)                                                                                                \
  const int sh = row_lanes(ceil_div(D, (int64_t)VE));                                                                         \
  hipLaunchKernelGGL((expert_gather_kernel<TY, VE, OUT>), grid_of(pad + row_blocks(T, sh)), dim3(kThreads), 0, s,                 \
                     static_cast<const TY *>(X), T, D, ldx, slots, k, order, rows, static_cast<TY *>(Xs), ldxs, sh, pad,       \
                     padding_rows(rows))
#define BSR_CALL(TY, VE)                                                    \
  if (write) { BSR_CALL_(TY, VE, (VE != 1)); } else { BSR_CALL_(TY, VE, false); }
  BSR_BY_ROW(dtype, D, BSR_CALL)
#undef BSR_CALL
#undef BSR_CALL_
  return check_launch();
}

// as many choices together as a token has, up to kChoices
#define BSR_CHOICES(TY, VE, READ, WRITE)                       \
  if (k <= 2) { BSR_CALL_(TY, VE, 2, READ, WRITE); }           \
  else if (k <= 4) { BSR_CALL_(TY, VE, 4, READ, WRITE); }      \
  else { BSR_CALL_(TY, VE, kChoices, READ, WRITE); }

int launch_expert_combine(const void *Ys, int dtype, int64_t rows, int64_t D, int64_t ldys, const int32_t *slots, int64_t T,
                          int64_t k, const float *weights, void *out, int64_t ldo, hipStream_t s) {
  const bool read = stream_rows(Ys, rows, D, ldys, dtype, kStreamRead), write = stream_rows(out, T, D, ldo, dtype, kStreamWrite);
#define BSR_CALL_(TY, VE, KC, READ, WRITE)                                                                                    \
  const int sh = row_lanes(ceil_div(D, (int64_t)VE));                                                                         \
  hipLaunchKernelGGL((expert_combine_kernel<TY, VE, KC, READ, WRITE>), grid_of(row_blocks(T, sh)), dim3(kThreads), 0, s,          \
                     static_cast<const TY *>(Ys), rows, D, ldys, slots, T, k, weights, static_cast<TY *>(out), ldo, sh)
#define BSR_CALL(TY, VE)                                                    \
  if (read && write) { BSR_CHOICES(TY, VE, (VE != 1), (VE != 1)) }          \
  else if (read) { BSR_CHOICES(TY, VE, (VE != 1), false) }                  \
  else if (write) { BSR_CHOICES(TY, VE, false, (VE != 1)) }                 \
  else { BSR_CHOICES(TY, VE, false, false) }
  BSR_BY_ROW(dtype, D, BSR_CALL)
#undef BSR_CALL
#undef BSR_CALL_
  return check_launch();
}

int launch_expert_combine_grad(const void *Ys, int dtype, int64_t rows, int64_t D, int64_t ldys, const int32_t *slots,
                               const int32_t *order, int64_t T, int64_t k, const float *weights, const void *dOut, int64_t lddo,
                               void *dYs, int64_t lddys, float *dweights, hipStream_t s) {
  const int64_t pad = padding_blocks(rows);
  const bool read = stream_rows(Ys, rows, D, ldys, dtype, kStreamRead), write = stream_rows(dYs, rows, D, lddys, dtype, kStreamWrite);
#define BSR_CALL_(TY, VE, KC, READ, WRITE)                                                                                    \
  const int sh = row_lanes(ceil_div(D, (int64_t)VE));                                                                         \
  hipLaunchKernelGGL((expert_combine_grad_kernel<TY, VE, KC, READ, WRITE>), grid_of(pad + row_blocks(T, sh)), dim3(kThreads), 0,  \
                     s, static_cast<const TY *>(Ys), rows, D, ldys, slots, order, T, k, weights, static_cast<const TY *>(dOut), \
                     lddo, static_cast<TY *>(dYs), lddys, dweights, sh, pad, padding_rows(rows))
#define BSR_CALL(TY, VE)                                                    \
  if (read && write) { BSR_CHOICES(TY, VE, (VE != 1), (VE != 1)) }          \
  else if (write) { BSR_CHOICES(TY, VE, false, (VE != 1)) }                 \
  else { BSR_CHOICES(TY, VE, false, false) }
  BSR_BY_ROW(dtype, D, BSR_CALL)
#undef BSR_CALL
#undef BSR_CALL_
  return check_launch();
}

}  // namespace bsr
