// Distillation from a teacher's top logits: loss, its gradient, or both.
//
// With e_j = exp((t_j - max t) / tau) over a row's entries, T = sum e_j, and the row's statistics m = max z, S = sum exp((z - m) / tau):
//   loss = tau^2 * (sum_j e_j * ((t_j - max t) - (z_j - m)) / (tau T) - log T + log S),
//   dz_v = g * tau * (exp((z_v - m) / tau) / S - sum over j at v of e_j / T).
// Exponentials are powers of two of (z - m) * log2(e) / tau: the difference first, so that the type's lowest value as a mask
// overflows nowhere.  Maxima, sums and differences are binary32; the running maximum and sum of a lane are corrected once per batch
// of vectors.
//
// Bound by memory: N * V logits in, as many gradients out.  A row is cut into chunks where there are few rows, so that every
// compute unit has some (row_chunks): the first kernel leaves every chunk's (maximum, sum), the second joins those of its row and
// writes its chunk of the gradient.
#include "token_step.h"

namespace bsr {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kAhead = 4;                      // vectors of a lane on their way
constexpr float kLog2E = 1.44269504088896340736f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float minus_inf() { return -__builtin_inff(); }

// What the kernels know of a call.
struct Distill {
  const void *logits, *ids, *teacher;
  int64_t N, V, ldz;
  int K, teacher_bf16, ids64;
  float tau, c;                                // c = log2(e) / tau
  int64_t chunk;                               // columns of a chunk: whole vectors
  int chunks;
};

__device__ __forceinline__ float teacher_logit(const Distill &a, int64_t i) {
  return a.teacher_bf16 ? bf16_bits_to_float(static_cast<const uint16_t *>(a.teacher)[i]) : static_cast<const float *>(a.teacher)[i];
}
// column of an entry, or -1
__device__ __forceinline__ int64_t entry_column(const Distill &a, int64_t i) {
  const int64_t v = a.ids64 ? load_index<int64_t>(a.ids, i) : load_index<int32_t>(a.ids, i);
  return v >= 0 && v < a.V ? v : -1;
}

// maximum and sum over the workgroup; `red` is shared, one float per wave, and free again after the next barrier
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}
__device__ __forceinline__ float group_max(float v, float *red) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) v = fmaxf(v, red[w]);
  return v;
}
__device__ __forceinline__ float group_sum(float v, float *red) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) v += red[w];
  return v;
}

// (z - m) with the maximum of a part without any finite or +inf value taken as 0
__device__ __forceinline__ float base_of(float m) { return m == minus_inf() ? 0.0f : m; }

// parts[n][chunk] = (maximum, sum of exp((z - maximum) / tau)) of a chunk; the first chunk's workgroup also leaves the logits at
// the row's entries in picked[n][j].
template <typename T>
__global__ __launch_bounds__(kThreads) void distill_parts_kernel(Distill a, float2 *__restrict__ parts, float *__restrict__ picked) {
  constexpr int VE = 16 / (int)sizeof(T);
  typedef RowVec<T, VE> R;
  __shared__ float red[2][kWaves];
  const int t = threadIdx.x;
  const int64_t n = blockIdx.y;
  const T *row = static_cast<const T *>(a.logits) + n * a.ldz;
  if (blockIdx.x == 0) {
    for (int j = t; j < a.K; j += kThreads) {
      const int64_t v = entry_column(a, n * a.K + j);
      picked[n * a.K + j] = v >= 0 ? elem_to_float<T>(row[v]) : 0.0f;
    }
  }
  const int64_t lo = blockIdx.x * a.chunk, hi = lo + a.chunk < a.V ? lo + a.chunk : a.V;
  const int64_t vecs = (hi - lo) / VE;
  float m = minus_inf(), s = 0.0f;
  for (int64_t v0 = t; v0 < vecs; v0 += kAhead * kThreads) {
    typename R::Raw x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (v0 + u * kThreads < vecs) x[u] = R::load(row + lo + (v0 + u * kThreads) * VE);
    float top = m;
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (v0 + u * kThreads < vecs) {
#pragma unroll
        for (int q = 0; q < VE; ++q) top = fmaxf(top, R::elem(x[u], q));
      }
    const float base = base_of(top);
    s *= exp2_of((m - base) * a.c);
    m = top;
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (v0 + u * kThreads < vecs) {
#pragma unroll
        for (int q = 0; q < VE; ++q) s += exp2_of((R::elem(x[u], q) - base) * a.c);
      }
  }
  for (int64_t v = lo + vecs * VE + t; v < hi; v += kThreads) {
    const float z = elem_to_float<T>(row[v]), top = fmaxf(m, z), base = base_of(top);
    s = s * exp2_of((m - base) * a.c) + exp2_of((z - base) * a.c);
    m = top;
  }
  const float top = group_max(m, red[0]), base = base_of(top);
  const float sum = group_sum(s * exp2_of((m - base) * a.c), red[1]);
  if (t == 0) parts[n * a.chunks + blockIdx.x] = float2{top, sum};
}

// FROM_PARTS: statistics from the chunks' parts, and the loss (by the first chunk's workgroup); else statistics as given.
// GRAD: the chunk's gradient.
template <typename T, bool FROM_PARTS, bool GRAD>
__global__ __launch_bounds__(kThreads) void distill_finish_kernel(Distill a, const float2 *__restrict__ parts, int parts_per_row,
                                                                  const float *__restrict__ picked,
                                                                  float *__restrict__ loss, float2 *stats,
                                                                  const float *__restrict__ dloss, T *dlogits, int64_t ldd) {
  constexpr int VE = 16 / (int)sizeof(T);
  typedef RowVec<T, VE> R;
  __shared__ int32_t at[kMaxTeacher];          // columns, -1: no entry
  __shared__ float share[kMaxTeacher];         // e_j
  __shared__ float zs[kMaxTeacher];            // logits there
  __shared__ float red[6][kWaves];
  const int t = threadIdx.x;
  const int64_t n = blockIdx.y;
  const T *row = static_cast<const T *>(a.logits) + n * a.ldz;
  const int64_t lo = GRAD ? blockIdx.x * a.chunk : 0;
  const int64_t hi = !GRAD || lo + a.chunk > a.V ? a.V : lo + a.chunk;
  float tm = minus_inf();
  for (int j = t; j < a.K; j += kThreads) {
    const int64_t v = entry_column(a, n * a.K + j);
    const float x = v >= 0 ? teacher_logit(a, n * a.K + j) : minus_inf();
    at[j] = (int32_t)v;
    share[j] = x;
    // (only columns of this chunk are read from the row: others may be overwritten by their own chunk's workgroup by now)
    zs[j] = FROM_PARTS ? picked[n * a.K + j] : v >= lo && v < hi ? elem_to_float<T>(row[v]) : 0.0f;
    tm = fmaxf(tm, x);
  }
  float m, log_s;
  if constexpr (FROM_PARTS) {
    float pm = minus_inf();
    for (int i = t; i < parts_per_row; i += kThreads) pm = fmaxf(pm, parts[n * parts_per_row + i].x);
    m = group_max(pm, red[0]);
    const float base = base_of(m);
    float ps = 0.0f;
    for (int i = t; i < parts_per_row; i += kThreads) {
      const float2 p = parts[n * parts_per_row + i];
      ps += p.y * exp2_of((p.x - base) * a.c);
    }
    const float s = group_sum(ps, red[1]);
    log_s = m == minus_inf() ? __builtin_nanf("") : logf(s);
  } else {
    const float2 st = stats[n];
    m = st.x;
    log_s = st.y;
  }
  const float top = group_max(tm, red[2]);
  const bool none = top == minus_inf();
  float e_sum = 0.0f, cross = 0.0f;
  for (int j = t; j < a.K; j += kThreads) {
    const float x = share[j] - top, e = none || at[j] < 0 ? 0.0f : exp2_of(x * a.c);
    share[j] = e;
    e_sum += e;
    if (e != 0.0f) cross = fmaf(e, x - (zs[j] - m), cross);
  }
  const float total = group_sum(e_sum, red[3]);
  if constexpr (FROM_PARTS) {
    if (blockIdx.x == 0) {
      const float x = group_sum(cross, red[4]);
      if (t == 0) {
        loss[n] = none ? 0.0f : a.tau * a.tau * (x / (a.tau * total) - logf(total) + log_s);
        if (stats != nullptr) stats[n] = float2{m, log_s};
      }
    }
  }
  if constexpr (GRAD) {
    T *out = dlogits + n * ldd;
    const float g = none ? 0.0f : dloss[n] * a.tau;
    const float log2_s = log_s * kLog2E;
    auto grad = [&](float z) { return none ? 0.0f : g * exp2_of(fmaf(z - m, a.c, -log2_s)); };
    const int64_t vecs = (hi - lo) / VE;
    for (int64_t v0 = t; v0 < vecs; v0 += kAhead * kThreads) {
      typename R::Raw x[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (v0 + u * kThreads < vecs) x[u] = R::load(row + lo + (v0 + u * kThreads) * VE);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (v0 + u * kThreads < vecs) {
          float f[VE];
#pragma unroll
          for (int q = 0; q < VE; ++q) f[q] = grad(R::elem(x[u], q));
          R::store(out + lo + (v0 + u * kThreads) * VE, pack_row<T, VE>(f));
        }
    }
    for (int64_t v = lo + vecs * VE + t; v < hi; v += kThreads) out[v] = from_float<T>(grad(elem_to_float<T>(row[v])));
    if (none) return;
    __syncthreads();                           // the chunk is written; now the entries' columns again, with the teacher's shares
    const float by = 1.0f / total;
    for (int j = t; j < a.K; j += kThreads) {
      const int32_t v = at[j];
      if (v < lo || v >= hi) continue;
      float q = 0.0f;
      for (int i = 0; i < a.K; ++i) q += at[i] == v ? share[i] : 0.0f;
      out[v] = from_float<T>(g * (exp2_of(fmaf(zs[j] - m, a.c, -log2_s)) - q * by));
    }
  }
}

// Chunks of a row: enough that the rows' chunks fill the compute units several times over, none shorter than 8192 columns.
constexpr int64_t kLeastChunk = 8192, kEnoughWorkgroups = 2048;
void row_chunks(int64_t N, int64_t V, int64_t *chunk, int *chunks) {
  int64_t c = ceil_div(kEnoughWorkgroups, N > 0 ? N : 1);
  if (c > ceil_div(V, kLeastChunk)) c = ceil_div(V, kLeastChunk);
  if (c < 1) c = 1;
  *chunk = ceil_div(ceil_div(V, c), (int64_t)64) * 64;
  if (*chunk < 64) *chunk = 64;
  *chunks = (int)ceil_div(V, *chunk);
  if (*chunks < 1) *chunks = 1;
}

Distill describe(const DistillArgs &d) {
  Distill a = {d.logits, d.ids, d.teacher, d.N, d.V, d.ldz, (int)d.K, d.teacher_dtype == BSR_BF16, d.index_type == BSR_I64,
               d.temperature, kLog2E / d.temperature, 0, 0};
  row_chunks(d.N, d.V, &a.chunk, &a.chunks);
  return a;
}

size_t parts_bytes(int64_t N, int64_t V) {
  int64_t chunk;
  int chunks;
  row_chunks(N, V, &chunk, &chunks);
  return align_up((size_t)N * chunks * sizeof(float2), 256);
}

// Rows per launch: the grid's second dimension ends at 65535.
constexpr int64_t kRowsPerLaunch = 65535;

Distill rows_from(const Distill &a, int64_t n, int dtype) {
  Distill b = a;
  b.logits = static_cast<const char *>(a.logits) + n * a.ldz * elem_bytes(dtype);
  b.ids = static_cast<const char *>(a.ids) + n * a.K * (a.ids64 ? 8 : 4);
  b.teacher = static_cast<const char *>(a.teacher) + n * a.K * (a.teacher_bf16 ? 2 : 4);
  b.N = a.N - n < kRowsPerLaunch ? a.N - n : kRowsPerLaunch;
  return b;
}

template <typename T, bool GRAD>
int run_both(const DistillArgs &d, const float *dloss, float *loss, float *stats, void *dlogits, int64_t ldd, void *ws,
             hipStream_t s) {
  const Distill a = describe(d);
  float2 *parts = static_cast<float2 *>(ws);
  float *picked = reinterpret_cast<float *>(static_cast<char *>(ws) + parts_bytes(d.N, d.V));
  for (int64_t n = 0; n < d.N; n += kRowsPerLaunch) {
    const Distill b = rows_from(a, n, d.dtype);
    hipLaunchKernelGGL((distill_parts_kernel<T>), dim3(a.chunks, (unsigned)b.N), dim3(kThreads), 0, s, b, parts + n * a.chunks,
                       picked + n * a.K);
    int rc = check_launch();
    if (rc != BSR_OK) return rc;
    hipLaunchKernelGGL((distill_finish_kernel<T, true, GRAD>), dim3(GRAD ? a.chunks : 1, (unsigned)b.N), dim3(kThreads), 0, s, b,
                       parts + n * a.chunks, a.chunks, picked + n * a.K, loss + n,
                       stats != nullptr ? reinterpret_cast<float2 *>(stats) + n : nullptr, dloss + (dloss != nullptr ? n : 0),
                       dlogits != nullptr ? static_cast<T *>(dlogits) + n * ldd : nullptr, ldd);
    rc = check_launch();
    if (rc != BSR_OK) return rc;
  }
  return BSR_OK;
}

template <typename T>
int run_grad(const DistillArgs &d, const float *stats, const float *dloss, void *dlogits, int64_t ldd, hipStream_t s) {
  const Distill a = describe(d);
  for (int64_t n = 0; n < d.N; n += kRowsPerLaunch) {
    const Distill b = rows_from(a, n, d.dtype);
    hipLaunchKernelGGL((distill_finish_kernel<T, false, true>), dim3(a.chunks, (unsigned)b.N), dim3(kThreads), 0, s, b,
                       nullptr, 0, nullptr, nullptr, reinterpret_cast<float2 *>(const_cast<float *>(stats)) + n, dloss + n,
                       static_cast<T *>(dlogits) + n * ldd, ldd);
    const int rc = check_launch();
    if (rc != BSR_OK) return rc;
  }
  return BSR_OK;
}

}  // namespace

size_t distill_ws_bytes(int64_t N, int64_t V, int64_t K) {
  return parts_bytes(N, V) + align_up((size_t)N * K * sizeof(float), 256);
}

int launch_distill_loss(const DistillArgs &a, float *loss, float *stats, void *ws, hipStream_t s) {
  return a.dtype == BSR_F32 ? run_both<float, false>(a, nullptr, loss, stats, nullptr, 0, ws, s)
                            : run_both<uint16_t, false>(a, nullptr, loss, stats, nullptr, 0, ws, s);
}

int launch_distill_grad(const DistillArgs &a, const float *stats, const float *dloss, void *dlogits, int64_t ldd, hipStream_t s) {
  return a.dtype == BSR_F32 ? run_grad<float>(a, stats, dloss, dlogits, ldd, s)
                            : run_grad<uint16_t>(a, stats, dloss, dlogits, ldd, s);
}

int launch_distill_loss_grad(const DistillArgs &a, const float *dloss, float *loss, void *dlogits, int64_t ldd, void *ws,
                             hipStream_t s) {
  return a.dtype == BSR_F32 ? run_both<float, true>(a, dloss, loss, nullptr, dlogits, ldd, ws, s)
                            : run_both<uint16_t, true>(a, dloss, loss, nullptr, dlogits, ldd, ws, s);
}

}  // namespace bsr
