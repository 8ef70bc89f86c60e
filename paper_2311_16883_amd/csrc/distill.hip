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
#include <type_traits>

#include "buffer_access.h"
#include "token_step.h"

namespace bsr {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kAhead = 4;                      // vectors of a lane on their way
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

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

// Maximum and sum over a workgroup of WAVES waves; `red` is shared, one float per wave, and free again after the next barrier.
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
// (The waves' values are read one per lane and combined by lane exchanges: all of them in every lane would be as many registers.)
template <int WAVES>
__device__ __forceinline__ float group_max(float v, float *red) {
  v = wave_max(v);
  if (WAVES == 1) {                            // (what the lanes wrote to LDS before is there for the others, as behind a barrier)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    return v;
  }
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[threadIdx.x & (WAVES - 1)];
#pragma unroll
  for (int d = WAVES / 2; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
  return v;
}
template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float *red) {
  v = wave_sum(v);
  if (WAVES == 1) {                            // (what the lanes wrote to LDS before is there for the others, as behind a barrier)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    return v;
  }
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[threadIdx.x & (WAVES - 1)];
#pragma unroll
  for (int d = WAVES / 2; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// Maximum as the base of differences: 0 for a part without any finite or +inf value.
__device__ __forceinline__ float base_of(float m) { return m == minus_inf() ? 0.0f : m; }

// The exponents of a row's logits, (z - m) * c, in one multiply-add each: fma(z, c, -mc).  What m * c loses by its rounding is
// the same for every logit: the true exponent is smaller by `lost`.  Where m * c might overflow (|m| above 1e30 / c: a row of nothing
// but the type's lowest value, say) logits that differ from m differ by so much that their exponential is 0 with any c that is not
// tiny, and 2^-30 takes its place: m * 2^-30 is exact.
struct Exponent {
  float c, mc, lost;
  __device__ __forceinline__ Exponent(float m, float c_) {
    c = fabsf(m * c_) <= 1e30f || m != m ? c_ : 0x1p-30f;
    mc = m * c;
    lost = fabsf(m) < __builtin_inff() ? fmaf(m, c, -mc) : 0.0f;
  }
  __device__ __forceinline__ float at(float z) const { return fmaf(z, c, -mc); }
};

// g * exp((z - m) / tau) / S in one multiply-add, exponential and product: the logarithm of S goes into the constant of the exponent,
// and what that sum's rounding loses into the factor.
struct Share {
  float c, k, g;
  // log2_s: of the sum of 2^at(z)
  __device__ __forceinline__ Share(const Exponent &ex, float log2_s, float g_) : c(ex.c) {
    k = ex.mc + log2_s;
    const float hi = k - ex.mc, lo = (ex.mc - (k - hi)) + (log2_s - hi);
    g = g_ * exp2_of(fabsf(k) < __builtin_inff() ? -lo : 0.0f);
  }
  __device__ __forceinline__ float at(float z) const { return g * exp2_of(fmaf(z, c, -k)); }
};

// Columns [lo, hi) of a row as `head` single ones up to the next 16-byte boundary, whole vectors, and single ones again.
struct Cut {
  int64_t head, vecs, singles;
  template <typename T>
  __device__ __forceinline__ Cut(const T *row, int64_t lo, int64_t hi) {
    constexpr int VE = 16 / (int)sizeof(T);
    const int64_t off = (int64_t)((16 - ((uintptr_t)(row + lo) & 15)) & 15) / (int)sizeof(T);
    head = off < hi - lo ? off : hi - lo;
    vecs = (hi - lo - head) / VE;
    singles = hi - lo - vecs * VE;
  }
  // column of single i < singles
  template <int VE>
  __device__ __forceinline__ int64_t single(int64_t lo, int64_t i) const { return lo + (i < head ? i : i + vecs * VE); }
};

// A row's entries in shared memory.
struct Entries {
  int32_t *at;                                 // columns, -1: no entry
  float *share;                                // teacher's logits, then e_j
  float *z;                                    // student's logits there
  float *q;                                    // e_j of all entries of the same column
  __device__ __forceinline__ Entries(void *lds, int K)
      : at(static_cast<int32_t *>(lds)), share(static_cast<float *>(lds) + K), z(static_cast<float *>(lds) + 2 * K),
        q(static_cast<float *>(lds) + 3 * K) {}
};
size_t entries_bytes(int64_t K) { return (size_t)K * 4 * sizeof(float); }

// Entry j of row n: its column (-1: none) and the teacher's logit (-inf: none).
__device__ __forceinline__ void load_entry(const Distill &a, int64_t n, int j, int64_t *v, float *x) {
  *v = entry_column(a, n * a.K + j);
  *x = *v >= 0 ? teacher_logit(a, n * a.K + j) : minus_inf();
}

// e_j in place of the teacher's logits; returns the lane's sum.  top: their maximum.
template <int THREADS>
__device__ __forceinline__ float weigh_entries(const Distill &a, const Entries &en, float top) {
  float sum = 0.0f;
  for (int j = threadIdx.x; j < a.K; j += THREADS) {
    const float e = top == minus_inf() || en.at[j] < 0 ? 0.0f : exp2_of((en.share[j] - top) * a.c);
    en.share[j] = e;
    sum += e;
  }
  return sum;
}

// The lane's sum of e_j * log(e_j / exp((z_j - m) / tau)), in which the teacher's part is the sum of e_j * (t_j - top) = e_j * tau * log(e_j).
template <int THREADS>
__device__ __forceinline__ float cross_entries(const Distill &a, const Entries &en, float m) {
  float sum = 0.0f;
  for (int j = threadIdx.x; j < a.K; j += THREADS) {
    const float e = en.share[j];
    if (e != 0.0f) sum = fmaf(e, a.tau * kLn2 * log2f(e) - (en.z[j] - m), sum);
  }
  return sum;
}

// e_j of all entries of a column together, for every one of them; once all e_j are there.
template <int THREADS>
__device__ __forceinline__ void merge_entries(const Distill &a, const Entries &en) {
  for (int j = threadIdx.x; j < a.K; j += THREADS) {
    const int32_t v = en.at[j];
    float q = 0.0f;
#pragma unroll 8
    for (int k = 0; k < a.K; ++k) q += en.at[k] == v ? en.share[k] : 0.0f;
    en.q[j] = q;
  }
}

// Teacher's shares subtracted from the gradient at the entries' columns in [lo, hi): every wave writes those columns once more
// whose vectors it has written itself (vector i of the cut by wave i / 64 mod WAVES, single columns by the first), so that no wave
// waits for another.  (A column that several entries share gets all of them, from every one of its entries alike.)
template <int WAVES, typename T>
__device__ __forceinline__ void subtract_entries(const Distill &a, const Entries &en, const Cut &cut, float total, float g, int64_t lo,
                                                 int64_t hi, T *out, const Share &share) {
  constexpr int VE = 16 / (int)sizeof(T);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float by = 1.0f / total;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // (the wave's stores before come first)
  __builtin_amdgcn_wave_barrier();
  for (int j = lane; j < a.K; j += 64) {
    const int32_t v = en.at[j];
    if (v < lo || v >= hi) continue;
    const uint32_t i = (uint32_t)(v - lo - cut.head);
    const bool single = v - lo < cut.head || i >= (uint32_t)(cut.vecs * VE);
    if ((single ? 0u : i / (VE * 64u) % WAVES) != (uint32_t)wave) continue;
    out[v] = from_float<T>(share.at(en.z[j]) - g * (en.q[j] * by));
  }
}

__device__ __forceinline__ float loss_of(const Distill &a, float cross, float total, float log_s) {
  return a.tau * a.tau * (cross / (a.tau * total) - logf(total) + log_s);
}

// Cache policy of buffer accesses: non-temporal.
constexpr int kStream = 2;

// ---- a row in registers: loss and gradient in one pass ----

// One workgroup per row, whose lanes keep R vectors each: the logits are read once.  alike: the rows of dlogits start as far from a
// 16-byte boundary as those of the logits.  The row has a whole vector at least.
// The longest rows keep L more vectors per lane in shared memory, which they reach without passing through registers.
template <typename T, int THREADS, int R_, int L>
__global__ __launch_bounds__(THREADS, R_ <= 8 ? 8 : 4) void distill_row_kernel(Distill a, const float *__restrict__ dloss,
                                                                               float *__restrict__ loss, T *dlogits, int64_t ldd,
                                                                               bool alike) {
  constexpr int VE = 16 / (int)sizeof(T), WAVES = THREADS / 64;
  constexpr uint32_t kNothing = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;       // -inf, for vectors behind the row
  typedef RowVec<T, VE> R;
  extern __shared__ uint32_t lds[];
  __shared__ float red[5][WAVES];
  __shared__ Words4 rest[L > 0 ? L * THREADS : 1];
  const Entries en(lds, a.K);
  const int t = threadIdx.x;
  const int64_t n = blockIdx.x;
  const T *row = static_cast<const T *>(a.logits) + n * a.ldz;
  const Cut cut(row, 0, a.V);
  // The entries are on their way before the row, and what they need of each other is computed while the row is still coming.
  // the whole vectors as a buffer: accesses behind them are neither loads nor stores
  const int vecs = (int)cut.vecs;
  const __amdgpu_buffer_rsrc_t body = make_rsrc(row + cut.head, (uint32_t)vecs * 16u);
  int64_t v0 = -1;
  float x0 = minus_inf();
  if (t < a.K) load_entry(a, n, t, &v0, &x0);
  const int first = __builtin_amdgcn_readfirstlane(t & ~63);          // vectors from here on belong to this wave
  Words4 x[R_];
#pragma unroll
  for (int r = 0; r < R_; ++r) x[r] = buffer_load<16>(body, (uint32_t)t * 16u, (uint32_t)(r * THREADS) * 16u);
  const bool one = t < cut.singles;
  const int64_t single = cut.single<VE>(0, one ? t : 0);
  const float zs = one ? elem_to_float<T>(row[single]) : minus_inf();
  float tm = x0;
  for (int j = t; j < a.K; j += THREADS) {
    if (j >= THREADS) load_entry(a, n, j, &v0, &x0);
    en.at[j] = (int32_t)v0;
    en.share[j] = x0;
    en.z[j] = v0 >= 0 ? elem_to_float<T>(row[v0]) : 0.0f;
    tm = fmaxf(tm, x0);
  }
  const float top = group_max<WAVES>(tm, red[0]);
  const bool none = top == minus_inf();
  const float total = group_sum<WAVES>(weigh_entries<THREADS>(a, en, top), red[1]);
  merge_entries<THREADS>(a, en);
  // (The copies to LDS are issued after what the entries need of it: the compiler lets reads of LDS wait for them.)
  if constexpr (L > 0) {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      if (first + (R_ + l) * THREADS >= vecs) continue;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(body, (__attribute__((address_space(3))) void *)&rest[l * THREADS + first], 16,
                                               (uint32_t)t * 16u, (uint32_t)((R_ + l) * THREADS) * 16u, 0, 0);
    }
  }
  // vector R_ + l of the lane, -inf behind the row
  auto from_lds = [&](int l) {
    Words4 w = rest[l * THREADS + t];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (R_ + l) * THREADS + t < vecs ? w[i] : kNothing;
    return w;
  };
  float m = zs;
#pragma unroll
  for (int r = 0; r < R_; ++r) {
    // (Here and below: one vector after the other, unpacked anew in each pass.  Left to itself the compiler works on all of them
    // at a time and keeps every element as binary32 from one pass to the next, several times the registers.)
    if (first + r * THREADS >= vecs) continue;
    asm volatile("" : "+v"(x[r]));
    if ((r + 1) * THREADS > vecs) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[r][i] = r * THREADS + t < vecs ? x[r][i] : kNothing;
    }
#pragma unroll
    for (int q = 0; q < VE; ++q) m = fmaxf(m, R::elem(x[r], q));
    asm volatile("" : "+v"(m));
  }
  if constexpr (L > 0) {
#pragma unroll 1
    for (int l = 0; l < L && first + (R_ + l) * THREADS < vecs; ++l) {
      const Words4 w = from_lds(l);
#pragma unroll
      for (int q = 0; q < VE; ++q) m = fmaxf(m, R::elem(w, q));
    }
  }
  m = group_max<WAVES>(m, red[2]);
  T *out = dlogits + n * ldd;
  const __amdgpu_buffer_rsrc_t out_body = make_rsrc(out + cut.head, (uint32_t)vecs * 16u);
  const Exponent ex(m, a.c);
  auto put = [&](auto policy, auto f) {
    auto put_vector = [&](int r, const Words4 &z) {
      float v[VE];
#pragma unroll
      for (int q = 0; q < VE; ++q) v[q] = f(R::elem(z, q));
      const Words4 w = pack_row<T, VE>(v);
      if (alike) __builtin_amdgcn_raw_buffer_store_b128(w, out_body, (uint32_t)t * 16u, (uint32_t)(r * THREADS) * 16u, policy.value);
      else if (r * THREADS + t < vecs) R::store(out + cut.head + (int64_t)(r * THREADS + t) * VE, w);
    };
#pragma unroll
    for (int r = 0; r < R_; ++r) {
      if (first + r * THREADS >= vecs) continue;
      asm volatile("" : "+v"(x[r]));
      put_vector(r, x[r]);
    }
    if constexpr (L > 0) {
#pragma unroll 1
      for (int l = 0; l < L && first + (R_ + l) * THREADS < vecs; ++l) put_vector(R_ + l, from_lds(l));
    }
    if (one) out[single] = from_float<T>(f(zs));
  };
  if (none) {
    if (t == 0) loss[n] = 0.0f;
    put(std::integral_constant<int, kStream>(), [](float) { return 0.0f; });
    return;
  }
  float acc[4] = {exp2_of(ex.at(zs)), 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int r = 0; r < R_; ++r) {
    if (first + r * THREADS >= vecs) continue;
    asm volatile("" : "+v"(x[r]));
#pragma unroll
    for (int q = 0; q < VE; ++q) acc[q & 3] += exp2_of(ex.at(R::elem(x[r], q)));
    asm volatile("" : "+v"(acc[0]), "+v"(acc[1]), "+v"(acc[2]), "+v"(acc[3]));
  }
  if constexpr (L > 0) {
#pragma unroll 1
    for (int l = 0; l < L && first + (R_ + l) * THREADS < vecs; ++l) {
      const Words4 w = from_lds(l);
#pragma unroll
      for (int q = 0; q < VE; ++q) acc[q & 3] += exp2_of(ex.at(R::elem(w, q)));
    }
  }
  const float cross = group_sum<WAVES>(cross_entries<THREADS>(a, en, m), red[3]);
  const float s = group_sum<WAVES>((acc[0] + acc[1]) + (acc[2] + acc[3]), red[4]);
  const float log2_s = m == minus_inf() ? __builtin_nanf("") : log2f(s);
  if (t == 0) loss[n] = loss_of(a, cross, total, (log2_s - ex.lost) * kLn2);
  const float g = dloss[n] * a.tau;
  const Share share(ex, log2_s, g);
  // Stores leave the caches to others ([2048 x 131072] bf16 225 us, 231 with plain ones, [8192 x 16384] 106 and 112, [1000 x 90000]
  // f32 147 and 158) unless many of their lines are written once more for an entry, one in 64 vectors ([4096 x 32768] with 200
  // entries 140 and 131), or in the middle of the sizes, where plain ones are as fast or faster ([8192 x 50000] 323 and 311, [4096 x
  // 32768] f32 196 and 198).
  if (a.K * 64 <= vecs && THREADS * R_ != 8192) put(std::integral_constant<int, kStream>(), [&](float z) { return share.at(z); });
  else put(std::integral_constant<int, 0>(), [&](float z) { return share.at(z); });
  subtract_entries<WAVES>(a, en, cut, total, g, 0, a.V, out, share);
}

// ---- a row in chunks: two passes over the logits ----

// Columns of chunk i: boundaries are multiples of a.chunk behind the row's first 16-byte boundary.
template <typename T>
__device__ __forceinline__ void chunk_of(const Distill &a, const T *row, int64_t i, int64_t *lo, int64_t *hi) {
  const int64_t head = (int64_t)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T);
  const int64_t l = i == 0 ? 0 : i * a.chunk + head, h = (i + 1) * a.chunk + head;
  *hi = i == a.chunks - 1 || h > a.V ? a.V : h;
  *lo = l < *hi ? l : *hi;
}

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
  int64_t lo, hi;
  chunk_of(a, row, blockIdx.x, &lo, &hi);
  const Cut cut(row, lo, hi);
  const Words4 *body = reinterpret_cast<const Words4 *>(row + lo + cut.head);
  float m = minus_inf(), s = 0.0f;
  if (t < cut.singles) {
    m = elem_to_float<T>(row[cut.single<VE>(lo, t)]);
    s = exp2_of((m - base_of(m)) * a.c);
  }
  auto take = [&](auto load) {
    Words4 x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x[u] = load(u);
    float top = m;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
#pragma unroll
      for (int q = 0; q < VE; ++q) top = fmaxf(top, R::elem(x[u], q));
    }
    const float base = base_of(top);
    float acc[4] = {s * exp2_of((m - base) * a.c), 0.0f, 0.0f, 0.0f};
    m = top;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
#pragma unroll
      for (int q = 0; q < VE; ++q) acc[q & 3] += exp2_of((R::elem(x[u], q) - base) * a.c);
    }
    s = (acc[0] + acc[1]) + (acc[2] + acc[3]);
  };
  int64_t v = t;
  for (; v + (kAhead - 1) * kThreads < cut.vecs; v += kAhead * kThreads) take([&](int u) { return body[v + u * kThreads]; });
  if (v < cut.vecs) {
    constexpr uint32_t kNothing = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;     // -inf
    take([&](int u) {
      Words4 w = {kNothing, kNothing, kNothing, kNothing};
      if (v + u * kThreads < cut.vecs) w = body[v + u * kThreads];
      return w;
    });
  }
  const float top = group_max<kWaves>(m, red[0]), base = base_of(top);
  const float sum = group_sum<kWaves>(s * exp2_of((m - base) * a.c), red[1]);
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
  extern __shared__ uint32_t lds[];
  __shared__ float red[5][kWaves];
  const Entries en(lds, a.K);
  const int t = threadIdx.x;
  const int64_t n = blockIdx.y;
  const T *row = static_cast<const T *>(a.logits) + n * a.ldz;
  int64_t lo = 0, hi = a.V;
  if (GRAD) chunk_of(a, row, blockIdx.x, &lo, &hi);
  // (only columns of this chunk are read from the row: others may be overwritten by their own chunk's workgroup by now)
  float tm = minus_inf();
  for (int j = t; j < a.K; j += kThreads) {
    int64_t v;
    float x;
    load_entry(a, n, j, &v, &x);
    en.at[j] = (int32_t)v;
    en.share[j] = x;
    en.z[j] = FROM_PARTS ? picked[n * a.K + j] : v >= lo && v < hi ? elem_to_float<T>(row[v]) : 0.0f;
    tm = fmaxf(tm, x);
  }
  float m, log_s;
  if constexpr (FROM_PARTS) {
    float pm = minus_inf();
    for (int i = t; i < parts_per_row; i += kThreads) pm = fmaxf(pm, parts[n * parts_per_row + i].x);
    m = group_max<kWaves>(pm, red[0]);
    const float base = base_of(m);
    float ps = 0.0f;
    for (int i = t; i < parts_per_row; i += kThreads) {
      const float2 p = parts[n * parts_per_row + i];
      ps += p.y * exp2_of((p.x - base) * a.c);
    }
    const float s = group_sum<kWaves>(ps, red[1]);
    log_s = m == minus_inf() ? __builtin_nanf("") : logf(s);
  } else {
    const float2 st = stats[n];
    m = st.x;
    log_s = st.y;
  }
  const float top = group_max<kWaves>(tm, red[2]);
  const bool none = top == minus_inf();
  const float total = group_sum<kWaves>(weigh_entries<kThreads>(a, en, top), red[3]);
  if constexpr (FROM_PARTS) {
    if (blockIdx.x == 0) {
      const float x = group_sum<kWaves>(cross_entries<kThreads>(a, en, m), red[4]);
      if (t == 0) {
        loss[n] = none ? 0.0f : loss_of(a, x, total, log_s);
        if (stats != nullptr) stats[n] = float2{m, log_s};
      }
    }
  }
  if constexpr (GRAD) {
    T *out = dlogits + n * ldd;
    const float g = none ? 0.0f : dloss[n] * a.tau;
    const Exponent ex(m, a.c);
    const Share share(ex, log_s * kLog2E + ex.lost, g);
    const Cut cut(row, lo, hi);
    const Words4 *body = reinterpret_cast<const Words4 *>(row + lo + cut.head);
    T *out_body = out + lo + cut.head;
    auto run = [&](auto f) {
      auto take = [&](int64_t v, auto in) {
        Words4 x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (in(u)) x[u] = body[v + u * kThreads];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (in(u)) {
            float w[VE];
#pragma unroll
            for (int q = 0; q < VE; ++q) w[q] = f(R::elem(x[u], q));
            R::store(out_body + (v + u * kThreads) * VE, pack_row<T, VE>(w));
          }
      };
      int64_t v = t;
      for (; v + (kAhead - 1) * kThreads < cut.vecs; v += kAhead * kThreads) take(v, [](int) { return true; });
      if (v < cut.vecs) take(v, [&](int u) { return v + u * kThreads < cut.vecs; });
      if (t < cut.singles) {
        const int64_t c = cut.single<VE>(lo, t);
        out[c] = from_float<T>(f(elem_to_float<T>(row[c])));
      }
    };
    if (none) {
      run([](float) { return 0.0f; });
      return;
    }
    merge_entries<kThreads>(a, en);
    run([&](float z) { return share.at(z); });
    __syncthreads();
    subtract_entries<kWaves>(a, en, cut, total, g, lo, hi, out, share);
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

// Rows from which long ones (more than 8192 vectors) have a workgroup each although they may be fewer than the compute units, against
// two passes over chunks ([100 x 262144] bf16 36.9 and 37.4 us, [64 x 262144] 34.6 and 23.0, [100 x 131072] 22.5 and 21.6, [32 x
// 131072] 19.7 and 14.4).  Up to 8192 vectors a single row is as fast so ([1 x 50000] 12.0 and 12.6, [8 x 20000] 9.8 and 12.5).
constexpr int64_t kEnoughRows = 96;

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

// One workgroup per row, at most.
template <typename T, int THREADS, int R, int L = 0>
int run_rows(const Distill &a, const float *dloss, float *loss, void *dlogits, int64_t ldd, hipStream_t s) {
  const bool alike = ((uintptr_t)dlogits - (uintptr_t)a.logits) % 16 == 0 && (ldd - a.ldz) * (int64_t)sizeof(T) % 16 == 0;
  hipLaunchKernelGGL((distill_row_kernel<T, THREADS, R, L>), dim3((unsigned)a.N), dim3(THREADS), entries_bytes(a.K), s, a, dloss, loss,
                     static_cast<T *>(dlogits), ldd, alike);
  return check_launch();
}

template <typename T, bool GRAD>
int run_both(const DistillArgs &d, const float *dloss, float *loss, float *stats, void *dlogits, int64_t ldd, void *ws,
             hipStream_t s) {
  const Distill a = describe(d);
  if constexpr (GRAD) {
    const int64_t vecs = a.V / (16 / (int64_t)sizeof(T));
    if (vecs >= 2 && (vecs <= 8192 || a.N >= kEnoughRows)) {
      if (vecs <= 512) return run_rows<T, 64, 8>(a, dloss, loss, dlogits, ldd, s);
      if (vecs <= 1024) return run_rows<T, 128, 8>(a, dloss, loss, dlogits, ldd, s);
      if (vecs <= 2048) return run_rows<T, 256, 8>(a, dloss, loss, dlogits, ldd, s);
      if (vecs <= 4096) return run_rows<T, 512, 8>(a, dloss, loss, dlogits, ldd, s);
      if (vecs <= 8192) return run_rows<T, 1024, 8>(a, dloss, loss, dlogits, ldd, s);
      if (vecs <= 16384) return run_rows<T, 1024, 16>(a, dloss, loss, dlogits, ldd, s);
      if (vecs <= 24576) return run_rows<T, 1024, 24>(a, dloss, loss, dlogits, ldd, s);
      if (vecs <= 32768) return run_rows<T, 1024, 24, 8>(a, dloss, loss, dlogits, ldd, s);
    }
  }
  float2 *parts = static_cast<float2 *>(ws);
  float *picked = reinterpret_cast<float *>(static_cast<char *>(ws) + parts_bytes(d.N, d.V));
  for (int64_t n = 0; n < d.N; n += kRowsPerLaunch) {
    const Distill b = rows_from(a, n, d.dtype);
    hipLaunchKernelGGL((distill_parts_kernel<T>), dim3(a.chunks, (unsigned)b.N), dim3(kThreads), 0, s, b, parts + n * a.chunks,
                       picked + n * a.K);
    int rc = check_launch();
    if (rc != BSR_OK) return rc;
    hipLaunchKernelGGL((distill_finish_kernel<T, true, GRAD>), dim3(GRAD ? a.chunks : 1, (unsigned)b.N), dim3(kThreads),
                       entries_bytes(a.K), s, b,
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
    hipLaunchKernelGGL((distill_finish_kernel<T, false, true>), dim3(a.chunks, (unsigned)b.N), dim3(kThreads),
                       entries_bytes(a.K), s, b, nullptr, 0, nullptr, nullptr, reinterpret_cast<float2 *>(const_cast<float *>(stats)) + n, dloss + n,
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
