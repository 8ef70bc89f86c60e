// Layer norm and its gradient.
//
// Both are bound by memory: a row is read once into registers, its sums are made there, and the result is written; a row belongs
// to 8 .. 64 lanes of a wave, longer ones to the 4 .. 16 waves of a workgroup, the longest are read again for every pass over them.
// [25088 x 1536] bfloat16: 28 us, 5.5 TB/s; gradient with those of weight and bias: 46 us, 5.0 TB/s ([25088 x 384]: 16.6 us, most of it in the
// caches, and the second launch).  A large copy reaches 5.1 TB/s on this card.
// The variance is the sum of squares of the distances from a first mean, less what that mean is off: rows far from 0 lose
// nothing.  16 bytes a lane at any alignment; the last vector of a row that is no whole number of vectors ends with the row, and the
// elements that it shares with the one before count there only.
// The gradients of weight and bias are sums over all rows.  The workgroups of the backward pass walk down the matrix and keep the sums of
// their rows in registers, column by column; a second launch adds up the workgroups.  No atomics: the order is that of the rows.
// (Requesting the next row while one is summed took the registers of other waves: 25088 x 384 18 -> 20 us.)
#include <algorithm>
#include <type_traits>

#include "layer_ops.h"

namespace bsr {

namespace {

// A row of VE-element vectors in the registers of its lanes: vector li + u * lanes in x[u].
template <typename T, int VE, int NV>
struct RowRegs {
  typename RowVec<T, VE>::Raw x[NV];
};

// How the lanes of a workgroup share rows: groups of 2^LG lanes of its MANY waves, or (WAVES > 1) all of its WAVES waves.
template <int LG, int WAVES, int MANY = 4>
struct Share {
  static constexpr int kThreads = 64 * (WAVES > 1 ? WAVES : MANY);
  static constexpr int kLanes = WAVES > 1 ? 64 * WAVES : 1 << LG;
  static constexpr int kRows = kThreads / kLanes;           // rows that a workgroup has in hand
  static __device__ __forceinline__ int lane() { return threadIdx.x & (kLanes - 1); }
  static __device__ __forceinline__ int row() { return threadIdx.x / kLanes; }
  // sums over the lanes of a row; `lds`: 2 * N * WAVES numbers, `turn` 0 or 1 by turns
  template <int N>
  static __device__ __forceinline__ void sum(float (&v)[N], float *lds, int &turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = group_sum<(WAVES > 1 ? 6 : LG)>(v[i]);
    if constexpr (WAVES > 1) {
      float *mine = lds + turn * N * WAVES;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) mine[i * WAVES + (threadIdx.x >> 6)] = v[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v[i] += mine[i * WAVES + w];
      }
    }
  }
};

// Elements at the front of vector v that belong to the vector before it.
__device__ __forceinline__ int shared_front(int64_t v, int VE, int64_t D) {
  const int64_t over = v * VE + VE - D;
  return over > 0 ? (int)over : 0;
}

template <typename T, int VE, int NV, int LG, int WAVES, bool RAGGED>
__global__ __launch_bounds__((Share<LG, WAVES>::kThreads)) void layer_norm_kernel(
    const T *X, int64_t M, int64_t D, int64_t ldx, const void *__restrict__ gamma, const void *__restrict__ beta, bool bf16,
    float eps, T *Y, int64_t ldy, float *__restrict__ stats, bool in, bool out) {
  typedef RowVec<T, VE> R;
  typedef Share<LG, WAVES> S;
  __shared__ float lds[4 * WAVES];
  int turn = 0;
  const int li = S::lane();
  const int vecs = (int)((D + VE - 1) / VE);
  const float inv = 1.0f / (float)D;
  for (int64_t row = (int64_t)blockIdx.x * S::kRows + S::row(); row < M; row += (int64_t)gridDim.x * S::kRows) {
    const T *src = X + row * ldx;
    typename R::Raw x[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int v = li + u * S::kLanes;
      x[u] = R::zero();
      if (v < vecs) x[u] = in ? load_once<T, VE, VE != 1>(src + vector_start(v, VE, D)) : R::load(src + vector_start(v, VE, D));
    }
    float sums[2] = {0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int front = RAGGED ? shared_front(li + u * S::kLanes, VE, D) : 0;
#pragma unroll
      for (int q = 0; q < VE; ++q)
        if (!RAGGED || q >= front) sums[0] += R::elem(x[u], q);
    }
    S::sum(sums, lds, turn);
    float mean = sums[0] * inv;
    sums[0] = sums[1] = 0.0f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int v = li + u * S::kLanes;
      const int front = RAGGED ? shared_front(v, VE, D) : 0;
      if (v < vecs) {
#pragma unroll
        for (int q = 0; q < VE; ++q)
          if (!RAGGED || q >= front) {
            const float d = R::elem(x[u], q) - mean;
            sums[0] += d;
            sums[1] += d * d;
          }
      }
    }
    S::sum(sums, lds, turn);
    const float off = sums[0] * inv;                 // what the mean is off by its own rounding
    const float var = fmaxf(sums[1] * inv - off * off, 0.0f) + (sums[1] - sums[1]);      // (fmaxf alone would lose a NaN)
    const float rstd = 1.0f / sqrtf(var + eps);
    if (stats != nullptr && li == 0) {
      stats[2 * row] = mean + off;
      stats[2 * row + 1] = rstd;
    }
    T *dst = Y + row * ldy;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int v = li + u * S::kLanes;
      if (v >= vecs) continue;
      const int64_t c = vector_start(v, VE, D);
      float g[VE], b[VE], f[VE];
      load_params<VE>(gamma, bf16, c, 1.0f, g);
      load_params<VE>(beta, bf16, c, 0.0f, b);
#pragma unroll
      for (int q = 0; q < VE; ++q) f[q] = (R::elem(x[u], q) - mean - off) * rstd * g[q] + b[q];
      if (out) store_once<T, VE, VE != 1>(dst + c, pack_row<T, VE>(f));
      else R::store(dst + c, pack_row<T, VE>(f));
    }
  }
}

// Rows longer than registers hold: read three times.
constexpr int kLongWaves = 16;
template <typename T>
__global__ __launch_bounds__(64 * kLongWaves) void layer_norm_long_kernel(const T *X, int64_t M, int64_t D, int64_t ldx,
                                                                          const void *__restrict__ gamma, const void *__restrict__ beta,
                                                                          bool bf16, float eps, T *Y, int64_t ldy, float *__restrict__ stats) {
  constexpr int VE = 16 / sizeof(T);
  typedef RowVec<T, VE> R;
  typedef RowVec<T, 1> R1;
  typedef Share<6, kLongWaves> S;
  __shared__ float lds[4 * kLongWaves];
  int turn = 0;
  const int64_t vecs = D / VE;                       // whole vectors; the rest of the row element by element
  const float inv = 1.0f / (float)D;
  for (int64_t row = blockIdx.x; row < M; row += gridDim.x) {
    const T *src = X + row * ldx;
    auto each = [&](auto f) {
      for (int64_t v = threadIdx.x; v < vecs; v += S::kThreads) {
        const typename R::Raw x = R::load(src + v * VE);
#pragma unroll
        for (int q = 0; q < VE; ++q) f(R::elem(x, q));
      }
      const int64_t c = vecs * VE + threadIdx.x;
      if (c < D) f(R1::elem(R1::load(src + c), 0));
    };
    float sums[2] = {0.0f, 0.0f};
    each([&](float x) { sums[0] += x; });
    S::sum(sums, lds, turn);
    const float mean = sums[0] * inv;
    sums[0] = sums[1] = 0.0f;
    each([&](float x) {
      const float d = x - mean;
      sums[0] += d;
      sums[1] += d * d;
    });
    S::sum(sums, lds, turn);
    const float off = sums[0] * inv;
    const float var = fmaxf(sums[1] * inv - off * off, 0.0f) + (sums[1] - sums[1]);
    const float rstd = 1.0f / sqrtf(var + eps);
    if (stats != nullptr && threadIdx.x == 0) {
      stats[2 * row] = mean + off;
      stats[2 * row + 1] = rstd;
    }
    T *dst = Y + row * ldy;
    for (int64_t v = threadIdx.x; v < vecs; v += S::kThreads) {
      const typename R::Raw x = R::load(src + v * VE);
      float g[VE], b[VE], f[VE];
      load_params<VE>(gamma, bf16, v * VE, 1.0f, g);
      load_params<VE>(beta, bf16, v * VE, 0.0f, b);
#pragma unroll
      for (int q = 0; q < VE; ++q) f[q] = (R::elem(x, q) - mean - off) * rstd * g[q] + b[q];
      R::store(dst + v * VE, pack_row<T, VE>(f));
    }
    const int64_t c = vecs * VE + threadIdx.x;
    if (c < D) {
      float g[1], b[1];
      load_params<1>(gamma, bf16, c, 1.0f, g);
      load_params<1>(beta, bf16, c, 0.0f, b);
      const float f[1] = {(R1::elem(R1::load(src + c), 0) - mean - off) * rstd * g[0] + b[0]};
      R1::store(dst + c, pack_row<T, 1>(f));
    }
  }
}

// ---- backward ----

// Sum over the groups of 2^LG lanes of a wave, lane by lane.
template <int LG>
__device__ __forceinline__ float sum_of_groups(float v) {
  if constexpr (LG <= 3) v += dpp_of<0x128>(v);      // the other half of 16 lanes (rotation by 8)
  if constexpr (LG <= 4) v += other_row(v);
  if constexpr (LG <= 5) v += other_half(v);
  return v;
}

// dX of the rows that a workgroup walks over, and (SUMS) their sums of dY * xh and dY by column: partial[workgroup] = 2 x D, or, of one
// workgroup alone, the results themselves.
struct Sums {
  float *partial, *dgamma, *dbeta;                   // partial null: the results
  int32_t accumulate;
  __device__ __forceinline__ void put(int64_t D, int64_t c, float g, float b) const {
    if (partial != nullptr) {
      float *out = partial + (int64_t)blockIdx.x * 2 * D;
      out[c] = g;
      out[D + c] = b;
    } else {
      if (dgamma != nullptr) dgamma[c] = accumulate ? dgamma[c] + g : g;
      if (dbeta != nullptr) dbeta[c] = accumulate ? dbeta[c] + b : b;
    }
  }
};
// Waves of a workgroup whose rows are one wave's or less: as many as LDS has sums for (64 KB).
template <int VE, int NV>
constexpr int walking_waves() { return VE * NV <= 16 ? 8 : 4; }
template <typename T, int VE, int NV, int LG, int WAVES, bool RAGGED, bool SUMS>
__global__ __launch_bounds__((Share<LG, WAVES, walking_waves<VE, NV>()>::kThreads)) void layer_norm_grad_kernel(
    const T *X, int64_t M, int64_t D, int64_t ldx, const void *__restrict__ gamma, bool bf16, const float *__restrict__ stats,
    const T *dY, int64_t lddy, T *dX, int64_t lddx, Sums out, bool read_once) {
  typedef RowVec<T, VE> R;
  typedef Share<LG, WAVES, walking_waves<VE, NV>()> S;
  __shared__ float lds[4 * WAVES];
  extern __shared__ float columns[];                 // SUMS, rows of one wave or less: 2 x D for each wave
  int turn = 0;
  const int li = S::lane();
  const int vecs = (int)((D + VE - 1) / VE);
  const float inv = 1.0f / (float)D;
  float weight[NV][VE], dg[SUMS ? NV : 1][VE], db[SUMS ? NV : 1][VE];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int v = li + u * S::kLanes;
#pragma unroll
    for (int q = 0; q < VE; ++q) {
      weight[u][q] = 0.0f;
      if constexpr (SUMS) dg[u][q] = db[u][q] = 0.0f;
    }
    if (v < vecs) load_params<VE>(gamma, bf16, vector_start(v, VE, D), 1.0f, weight[u]);
  }
  for (int64_t row = (int64_t)blockIdx.x * S::kRows + S::row(); row < M; row += (int64_t)gridDim.x * S::kRows) {
    typename R::Raw x[NV], y[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int v = li + u * S::kLanes;
      x[u] = y[u] = R::zero();
      if (v < vecs) {
        const T *px = X + row * ldx + vector_start(v, VE, D), *py = dY + row * lddy + vector_start(v, VE, D);
        x[u] = read_once ? load_once<T, VE, VE != 1>(px) : R::load(px);
        y[u] = read_once ? load_once<T, VE, VE != 1>(py) : R::load(py);
      }
    }
    const float mean = stats[2 * row], rstd = stats[2 * row + 1];
    float sums[2] = {0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int front = RAGGED ? shared_front(li + u * S::kLanes, VE, D) : 0;
      if (li + u * S::kLanes < vecs) {
#pragma unroll
        for (int q = 0; q < VE; ++q) {
          const float d = R::elem(y[u], q), xh = (R::elem(x[u], q) - mean) * rstd, g = d * weight[u][q];
          if (!RAGGED || q >= front) {
            sums[0] += g;
            sums[1] += g * xh;
          }
          if constexpr (SUMS) {
            dg[u][q] += d * xh;
            db[u][q] += d;
          }
        }
      }
    }
    S::sum(sums, lds, turn);
    const float a = sums[0] * inv, b = sums[1] * inv;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int v = li + u * S::kLanes;
      if (v >= vecs) continue;
      float f[VE];
#pragma unroll
      for (int q = 0; q < VE; ++q) {
        const float xh = (R::elem(x[u], q) - mean) * rstd;
        f[q] = rstd * (R::elem(y[u], q) * weight[u][q] - a - xh * b);
      }
      R::store(dX + row * lddx + vector_start(v, VE, D), pack_row<T, VE>(f));
    }
  }
  if constexpr (SUMS) {
    if constexpr (WAVES > 1) {                       // every column is some lane's alone
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int v = li + u * S::kLanes;
        if (v >= vecs) continue;
        const int64_t c = vector_start(v, VE, D);
        if (out.partial != nullptr && VE >= 4) {     // (two vectors' shared columns: whoever writes last has the same sums)
          float *to = out.partial + (int64_t)blockIdx.x * 2 * D + c;
#pragma unroll
          for (int q = 0; q < VE; q += 4) {
            RowVec<float, 4>::store(to + q, pack_row<float, 4>(dg[u] + q));
            RowVec<float, 4>::store(to + D + q, pack_row<float, 4>(db[u] + q));
          }
        } else {
#pragma unroll
          for (int q = 0; q < VE; ++q)
            if (!RAGGED || q >= shared_front(v, VE, D)) out.put(D, c + q, dg[u][q], db[u][q]);
        }
      }
    } else {
      constexpr int kWaves = S::kThreads / 64;
      const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
      float *mine = columns + (int64_t)wave * 2 * D;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int v = li + u * S::kLanes;
#pragma unroll
        for (int q = 0; q < VE; ++q) {
          dg[u][q] = sum_of_groups<LG>(dg[u][q]);
          db[u][q] = sum_of_groups<LG>(db[u][q]);
          if (lane < S::kLanes && v < vecs && (!RAGGED || q >= shared_front(v, VE, D))) {
            const int64_t c = vector_start(v, VE, D) + q;
            mine[c] = dg[u][q];
            mine[D + c] = db[u][q];
          }
        }
      }
      __syncthreads();
      for (int64_t c = threadIdx.x; c < D; c += S::kThreads) {
        float g = 0.0f, b = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          g += columns[(int64_t)w * 2 * D + c];
          b += columns[(int64_t)w * 2 * D + D + c];
        }
        out.put(D, c, g, b);
      }
    }
  }
}

// dX of rows longer than registers hold.
template <typename T>
__global__ __launch_bounds__(64 * kLongWaves) void layer_norm_grad_long_kernel(const T *X, int64_t M, int64_t D, int64_t ldx,
                                                                               const void *__restrict__ gamma, bool bf16,
                                                                               const float *__restrict__ stats, const T *dY,
                                                                               int64_t lddy, T *dX, int64_t lddx) {
  constexpr int VE = 16 / sizeof(T);
  typedef RowVec<T, VE> R;
  typedef RowVec<T, 1> R1;
  typedef Share<6, kLongWaves> S;
  __shared__ float lds[4 * kLongWaves];
  int turn = 0;
  const int64_t vecs = D / VE;
  const float inv = 1.0f / (float)D;
  for (int64_t row = blockIdx.x; row < M; row += gridDim.x) {
    const T *src = X + row * ldx, *grad = dY + row * lddy;
    T *dst = dX + row * lddx;
    const float mean = stats[2 * row], rstd = stats[2 * row + 1];
    float sums[2] = {0.0f, 0.0f};
    for (int64_t v = threadIdx.x; v < vecs; v += S::kThreads) {
      const typename R::Raw x = R::load(src + v * VE), y = R::load(grad + v * VE);
      float w[VE];
      load_params<VE>(gamma, bf16, v * VE, 1.0f, w);
#pragma unroll
      for (int q = 0; q < VE; ++q) {
        const float g = R::elem(y, q) * w[q];
        sums[0] += g;
        sums[1] += g * ((R::elem(x, q) - mean) * rstd);
      }
    }
    const int64_t c = vecs * VE + threadIdx.x;
    float w1[1] = {0.0f}, x1 = 0.0f, y1 = 0.0f;
    if (c < D) {
      load_params<1>(gamma, bf16, c, 1.0f, w1);
      x1 = R1::elem(R1::load(src + c), 0);
      y1 = R1::elem(R1::load(grad + c), 0);
      sums[0] += y1 * w1[0];
      sums[1] += y1 * w1[0] * ((x1 - mean) * rstd);
    }
    S::sum(sums, lds, turn);
    const float a = sums[0] * inv, b = sums[1] * inv;
    for (int64_t v = threadIdx.x; v < vecs; v += S::kThreads) {
      const typename R::Raw x = R::load(src + v * VE), y = R::load(grad + v * VE);
      float w[VE], f[VE];
      load_params<VE>(gamma, bf16, v * VE, 1.0f, w);
#pragma unroll
      for (int q = 0; q < VE; ++q) f[q] = rstd * (R::elem(y, q) * w[q] - a - (R::elem(x, q) - mean) * rstd * b);
      R::store(dst + v * VE, pack_row<T, VE>(f));
    }
    if (c < D) {
      const float f[1] = {rstd * (y1 * w1[0] - a - (x1 - mean) * rstd * b)};
      R1::store(dst + c, pack_row<T, 1>(f));
    }
  }
}

// Sums of dY * xh and dY by column, apart from dX (which may be dY: this runs first): partial[slice] = 2 x D.
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_columns_kernel(const T *__restrict__ X, int64_t M, int64_t D, int64_t ldx,
                                                                 const float *__restrict__ stats, const T *__restrict__ dY,
                                                                 int64_t lddy, float *__restrict__ partial, int64_t per_slice) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= D) return;
  const int64_t r0 = (int64_t)blockIdx.y * per_slice, r1 = r0 + per_slice < M ? r0 + per_slice : M;
  float dg = 0.0f, db = 0.0f;
  for (int64_t r = r0; r < r1; ++r) {
    const float y = elem_to_float<T>(dY[r * lddy + c]);
    dg += y * ((elem_to_float<T>(X[r * ldx + c]) - stats[2 * r]) * stats[2 * r + 1]);
    db += y;
  }
  float *out = partial + (int64_t)blockIdx.y * 2 * D;
  out[c] = dg;
  out[D + c] = db;
}

// dgamma, dbeta = (accumulate ? themselves : 0) + the sum of the partial sums: 32 columns and 32 slices of them to a workgroup.
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const float *__restrict__ partial, int64_t parts, int64_t D,
                                                               float *__restrict__ dgamma, float *__restrict__ dbeta, int accumulate) {
  __shared__ float sums[32][33];
  const int col = threadIdx.x & 31, slice = threadIdx.x >> 5;
  for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < 2 * D; c0 += (int64_t)gridDim.x * 32) {
    const int64_t c = c0 + col;
    float sum = 0.0f;
    if (c < 2 * D) {
#pragma unroll 8
      for (int64_t p = slice; p < parts; p += 32) sum += partial[p * 2 * D + c];
    }
    sums[slice][col] = sum;
    __syncthreads();
    // 32 lanes to a column: two columns to a wave
    sum = group_sum<5>(sums[col][slice]);
    const int64_t mine = c0 + slice;
    if (col == 0 && mine < 2 * D) {
      float *out = mine < D ? dgamma : dbeta;
      const int64_t at = mine < D ? mine : mine - D;
      if (out != nullptr) out[at] = accumulate ? out[at] + sum : sum;
    }
    __syncthreads();
  }
}

// ---- which form ----

// Bytes from which rows of whole lines pass by the caches, read and (forward) written: [25088 x 1536] bfloat16 31.0 -> 28.0 us, the gradient of
// [16384 x 2048] binary32 75 -> 65; dX written so too 65 -> 70, and the gradient of [25088 x 1536] 46 -> 51.
constexpr int64_t kStreamRead = int64_t(64) << 20, kStreamWrite = int64_t(32) << 20;
constexpr int64_t kMostWorkgroups = int64_t(1) << 20;      // rows beyond what they have in hand are taken in turn
// Workgroups that walk over the rows of a backward pass where columns are added up: rows in hand for each where there are few, then
// as many rows for each of about 512 (of 16 waves: 256), as more of them have more sums to add up.
constexpr int64_t kWalkers = 512;
int64_t walkers(int64_t groups, int waves) {
  const int64_t most = waves == 16 ? kWalkers / 2 : kWalkers;
  return groups <= 2 * most ? groups : ceil_div(groups, ceil_div(groups, most));
}

// Calls f with the form of a row of `vecs` vectors: f(NV, LG, WAVES), false if rows are longer than registers hold.
template <int N>
using Int = std::integral_constant<int, N>;
template <bool WALK, typename F>
bool with_row_form(int64_t vecs, F f) {
  if (vecs <= 8) f(Int<1>(), Int<3>(), Int<1>());
  else if (vecs <= 16) f(Int<1>(), Int<4>(), Int<1>());
  else if (vecs <= 32) f(Int<1>(), Int<5>(), Int<1>());
  else if (vecs <= 64) f(Int<1>(), Int<6>(), Int<1>());
  else if (vecs <= 128) f(Int<2>(), Int<6>(), Int<1>());
  else if (vecs <= 192) f(Int<3>(), Int<6>(), Int<1>());
  else if (vecs <= 256) f(Int<4>(), Int<6>(), Int<1>());
  else if (!WALK && vecs <= 512) f(Int<2>(), Int<6>(), Int<4>());
  else if (!WALK && vecs <= 1024) f(Int<4>(), Int<6>(), Int<4>());
  else if (WALK && vecs <= 512) f(Int<1>(), Int<6>(), Int<8>());
  else if (WALK && vecs <= 1024) f(Int<1>(), Int<6>(), Int<16>());
  else if (vecs <= 2048) f(Int<2>(), Int<6>(), Int<16>());
  else if (vecs <= 4096) f(Int<4>(), Int<6>(), Int<16>());
  else return false;
  return true;
}

template <typename T>
int norm_of(const T *X, int64_t M, int64_t D, int64_t ldx, const void *gamma, const void *beta, bool bf16, float eps, T *Y,
            int64_t ldy, float *stats, hipStream_t s) {
  constexpr int VE = 16 / sizeof(T), kType = sizeof(T) == 4 ? BSR_F32 : BSR_BF16;
  const bool in = stream_rows(X, M, D, ldx, kType, kStreamRead), out = stream_rows(Y, M, D, ldy, kType, kStreamWrite);
  auto launch = [&](auto ve, auto nv, auto lg, auto waves, auto ragged) {
    typedef Share<decltype(lg)::value, decltype(waves)::value> S;
    const int64_t grid = std::min(ceil_div(M, (int64_t)S::kRows), kMostWorkgroups);
    layer_norm_kernel<T, decltype(ve)::value, decltype(nv)::value, decltype(lg)::value, decltype(waves)::value, decltype(ragged)::value>
        <<<dim3((uint32_t)grid), S::kThreads, 0, s>>>(X, M, D, ldx, gamma, beta, bf16, eps, Y, ldy, stats, in, out);
  };
  if (D < VE) {
    launch(Int<1>(), Int<1>(), Int<3>(), Int<1>(), std::false_type());
  } else {
    const bool found = with_row_form<false>(ceil_div(D, (int64_t)VE), [&](auto nv, auto lg, auto waves) {
      if (D % VE) launch(Int<VE>(), nv, lg, waves, std::true_type());
      else launch(Int<VE>(), nv, lg, waves, std::false_type());
    });
    if (!found)
      layer_norm_long_kernel<T><<<dim3((uint32_t)std::min(M, kMostWorkgroups)), 64 * kLongWaves, 0, s>>>(X, M, D, ldx, gamma, beta, bf16,
                                                                                                   eps, Y, ldy, stats);
  }
  return check_launch();
}

// Workgroups whose partial sums a backward pass adds up.
int64_t partial_sums(int64_t M) { return std::min<int64_t>(2 * kWalkers, std::max<int64_t>(M, 1)); }

template <typename T>
int norm_grad_of(const T *X, int64_t M, int64_t D, int64_t ldx, const void *gamma, bool bf16, const float *stats, const T *dY,
                 int64_t lddy, T *dX, int64_t lddx, float *dgamma, float *dbeta, int accumulate, float *partial, hipStream_t s) {
  constexpr int VE = 16 / sizeof(T);
  constexpr int kType = sizeof(T) == 4 ? BSR_F32 : BSR_BF16;
  const bool sums = dgamma != nullptr || dbeta != nullptr;
  const bool in = stream_rows(X, M, D, ldx, kType, kStreamRead) && stream_rows(dY, M, D, lddy, kType, 0);
  const int64_t vecs = ceil_div(D, (int64_t)VE);
  // bfloat16 rows of more vectors than this would take more registers for their sums than 16 waves have
  const bool apart = sums && vecs > (VE == 8 ? 2048 : 4096);
  int64_t parts = 0;
  if (apart) {
    const int64_t per = ceil_div(M, std::min<int64_t>(M, 64));
    parts = ceil_div(M, per);
    layer_norm_columns_kernel<T><<<dim3((uint32_t)ceil_div(D, (int64_t)256), (uint32_t)parts), 256, 0, s>>>(X, M, D, ldx, stats, dY, lddy,
                                                                                                 partial, per);
    if (const int rc = check_launch(); rc != BSR_OK) return rc;
  }
  auto launch = [&](auto ve, auto nv, auto lg, auto waves, auto ragged) {
    constexpr int WAVES = decltype(waves)::value;
    typedef Share<decltype(lg)::value, WAVES, walking_waves<decltype(ve)::value, decltype(nv)::value>()> S;
    const int64_t groups = ceil_div(M, (int64_t)S::kRows);
    auto go = [&](auto with) {
      constexpr bool SUMS = decltype(with)::value;
      // little more than a workgroup has in hand, of rows that are a wave's or less: one does it all, and nothing is left to add up (one workgroup and
      // several, in a graph; bfloat16: [25 x 1024] 7.0 us and 7.8, [32 x 1024] 7.7 and 7.6, [36 x 337] 5.7 and 5.9, [48 x 337] 6.7 and 5.9, [256 x 64] 5.2
      // and 5.9, [400 x 64] 6.2 and 5.9, [8 x 2048] 8.8 and 9.6, [12 x 2048] 10.1 and 9.5; binary32: [128 x 64] 4.3 and 5.2, [256 x 64] 5.7 and 5.3,
      // [25 x 1024] 6.7 and 6.9; rows of several waves: [8 x 1536] 7.5 and 5.1)
      const bool alone = groups <= 1 || (WAVES == 1 && groups <= S::kThreads / 128 && M * D <= 25600);
      const int64_t grid = !SUMS ? std::min(groups, kMostWorkgroups) : alone ? 1 : walkers(groups, WAVES);
      Sums out = {grid > 1 ? partial : nullptr, dgamma, dbeta, accumulate};
      if (SUMS) parts = grid;
      layer_norm_grad_kernel<T, decltype(ve)::value, decltype(nv)::value, decltype(lg)::value, WAVES, decltype(ragged)::value, SUMS>
          <<<dim3((uint32_t)grid), S::kThreads, SUMS && WAVES == 1 ? (size_t)(S::kThreads / 64 * 2 * D * 4) : 0, s>>>(
              X, M, D, ldx, gamma, bf16, stats, dY, lddy, dX, lddx, out, in);
    };
    if constexpr (decltype(ve)::value == 8 && WAVES == 16 && decltype(nv)::value == 4) go(std::false_type());
    else if (sums) go(std::true_type());
    else go(std::false_type());
  };
  if (D < VE) {
    launch(Int<1>(), Int<1>(), Int<3>(), Int<1>(), std::false_type());
  } else {
    const bool found = with_row_form<true>(vecs, [&](auto nv, auto lg, auto waves) {
      if (D % VE) launch(Int<VE>(), nv, lg, waves, std::true_type());
      else launch(Int<VE>(), nv, lg, waves, std::false_type());
    });
    if (!found)
      layer_norm_grad_long_kernel<T><<<dim3((uint32_t)std::min(M, kMostWorkgroups)), 64 * kLongWaves, 0, s>>>(
          X, M, D, ldx, gamma, bf16, stats, dY, lddy, dX, lddx);
  }
  if (const int rc = check_launch(); rc != BSR_OK || !sums || (parts == 1 && !apart)) return rc;
  const int64_t grid = std::min(ceil_div(2 * D, (int64_t)32), kMostWorkgroups);
  layer_norm_join_kernel<<<dim3((uint32_t)grid), 1024, 0, s>>>(partial, parts, D, dgamma, dbeta, accumulate);
  return check_launch();
}

__global__ __launch_bounds__(256) void clear_sums_kernel(float *dgamma, float *dbeta, int64_t D) {
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < D; c += (int64_t)gridDim.x * 256) {
    if (dgamma != nullptr) dgamma[c] = 0.0f;
    if (dbeta != nullptr) dbeta[c] = 0.0f;
  }
}

}  // namespace

int launch_layer_norm(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx, const void *gamma, const void *beta,
                      int param_dtype, float eps, void *Y, int64_t ldy, float *stats, hipStream_t s) {
  const bool bf16 = param_dtype == BSR_BF16;
  return dtype == BSR_F32 ? norm_of(static_cast<const float *>(X), M, D, ldx, gamma, beta, bf16, eps, static_cast<float *>(Y), ldy, stats, s)
                          : norm_of(static_cast<const uint16_t *>(X), M, D, ldx, gamma, beta, bf16, eps, static_cast<uint16_t *>(Y),
                                    ldy, stats, s);
}

size_t layer_norm_grad_ws_bytes(int64_t M, int64_t D) { return (size_t)partial_sums(M) * 2 * (size_t)D * 4; }

int launch_layer_norm_grad(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx, const void *gamma, int param_dtype,
                           const float *stats, const void *dY, int64_t lddy, void *dX, int64_t lddx, float *dgamma, float *dbeta,
                           int accumulate, void *ws, hipStream_t s) {
  if (M == 0) {
    if (accumulate || (dgamma == nullptr && dbeta == nullptr)) return BSR_OK;
    clear_sums_kernel<<<dim3((uint32_t)std::min(ceil_div(D, (int64_t)256), kMostWorkgroups)), 256, 0, s>>>(dgamma, dbeta, D);
    return check_launch();
  }
  const bool bf16 = param_dtype == BSR_BF16;
  float *partial = static_cast<float *>(ws);
  return dtype == BSR_F32
             ? norm_grad_of(static_cast<const float *>(X), M, D, ldx, gamma, bf16, stats, static_cast<const float *>(dY), lddy,
                            static_cast<float *>(dX), lddx, dgamma, dbeta, accumulate, partial, s)
             : norm_grad_of(static_cast<const uint16_t *>(X), M, D, ldx, gamma, bf16, stats, static_cast<const uint16_t *>(dY), lddy,
                            static_cast<uint16_t *>(dX), lddx, dgamma, dbeta, accumulate, partial, s);
}

}  // namespace bsr
