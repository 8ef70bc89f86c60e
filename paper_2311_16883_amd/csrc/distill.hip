// Distillation from a teacher's top logits: loss, its gradient, or both.
//
// With e_j = exp((t_j - max t) / tau) over a row's entries, T = sum e_j, and the row's statistics m = max z, S = sum exp((z - m) / tau):
//   loss = tau * sum_j (e_j / T) * ((t_j - max t) - (z_j - m)) + tau^2 * (log S - log T),
//   dz_v = g * tau * (exp((z_v - m) / tau) / S - sum over j at v of e_j / T).
// Exponentials are powers of two of (z - m) * log2(e) / tau.  Maxima, sums and differences are binary32.
//
// Bound by memory: N * V logits in, as many gradients out.  A row whose lanes can keep it in registers is read once, whatever is asked
// for (distill_row_kernel; the longest ones keep a quarter in LDS).  Long rows that are fewer than the compute units are cut into chunks
// (row_chunks), so that every unit has some: one kernel leaves every chunk's (maximum, sum), the next joins those of its row and writes
// its chunk of the gradient.  The gradient alone needs no row as a whole and goes by chunks always.
// [8192 x 50000] bf16, 50 entries: loss 162 us (5.1 TB/s), gradient 302 (5.4), both 311 (5.3; a copy on this GPU 5.1, reading alone 6.2),
// in the logits' place 321.  Rows that take a compute unit whole pass their reads, arithmetic and writes one after the other, in rounds of
// as many rows as there are units: [600 x 250007] both 171 us (3.5 TB/s).  Two passes over chunks are slower still (205).
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

// The exponents of a row's logits, (z - m) * c.  Where m * c is no larger than 2^20 (`plain`) each takes one multiply-add,
// fma(z, c, -mc): what m * c loses by its rounding, a sixteenth at most, is the same for every logit, and the true exponent is smaller
// by that (`lost`).  Elsewhere -- a row of nothing but the type's lowest value, infinities, a tiny temperature -- the difference comes
// first, which neither loses nor overflows.
struct Exponent {
  float m, c, mc, lost;
  bool plain;
  __device__ __forceinline__ Exponent(float m_, float c_) : m(m_), c(c_) {
#pragma clang fp contract(off)
    mc = m * c;                                // (a product of its own wherever it is added to, or `lost` would not be what it lost)
    plain = fabsf(mc) <= 0x1p20f;
    lost = plain ? fmaf(m, c, -mc) : 0.0f;
  }
  template <bool PLAIN>
  __device__ __forceinline__ float at(float z) const { return PLAIN ? fmaf(z, c, -mc) : (z - m) * c; }
};

// g * exp((z - m) / tau) / S.  Plain: in one multiply-add, exponential and product; the logarithm of S goes into the constant of the
// exponent, and what that sum's rounding loses into the factor.
struct Share {
  float m, c, k, log2_s, plain_g, g;
  // log2_s: of the sum of 2^at(z)
  __device__ __forceinline__ Share(const Exponent &ex, float log2_s_, float g_) : m(ex.m), c(ex.c), log2_s(log2_s_), g(g_) {
#pragma clang fp contract(off)
    k = ex.mc + log2_s;
    const float hi = k - ex.mc, lo = (ex.mc - (k - hi)) + (log2_s - hi);
    plain_g = g * exp2_of(ex.plain ? -lo : 0.0f);
  }
  template <bool PLAIN>
  __device__ __forceinline__ float at(float z) const {
    return PLAIN ? plain_g * exp2_of(fmaf(z, c, -k)) : g * exp2_of(fmaf(z - m, c, -log2_s));
  }
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

// Columns of chunk i: boundaries are multiples of a.chunk behind the row's first 16-byte boundary.
template <typename T>
__device__ __forceinline__ void chunk_of(const Distill &a, const T *row, int64_t i, int64_t *lo, int64_t *hi) {
  const int64_t head = (int64_t)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T);
  const int64_t l = i == 0 ? 0 : i * a.chunk + head, h = (i + 1) * a.chunk + head;
  *hi = i == a.chunks - 1 || h > a.V ? a.V : h;
  *lo = l < *hi ? l : *hi;
}

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

// The first use of a loaded value: keeps the compiler from moving that, and the wait for the load, up to the load.
template <typename V>
__device__ __forceinline__ void used_here(V &v) { asm volatile("" : "+v"(v)); }

// Entry j of row n as it comes from memory (nothing waits for it here), and its column (-1: none) and the teacher's logit (-inf: none).
struct RawEntry {
  uint32_t id[2];                              // low and high word (of an int32: the same)
  uint16_t logit[2];                           // ... half
  __device__ __forceinline__ void load(const Distill &a, int64_t n, int j) {
    const int64_t i = n * a.K + j;
    const char *p = static_cast<const char *>(a.ids) + i * (a.ids64 ? 8 : 4), *x = static_cast<const char *>(a.teacher) + i * (a.teacher_bf16 ? 2 : 4);
    id[0] = *reinterpret_cast<const uint32_t *>(p);
    id[1] = *reinterpret_cast<const uint32_t *>(p + (a.ids64 ? 4 : 0));
    logit[0] = *reinterpret_cast<const uint16_t *>(x);
    logit[1] = *reinterpret_cast<const uint16_t *>(x + (a.teacher_bf16 ? 0 : 2));
  }
  __device__ __forceinline__ void take(const Distill &a, int64_t *v, float *x) {
    used_here(id[0]);
    used_here(id[1]);
    used_here(logit[0]);
    used_here(logit[1]);
    const int64_t c = a.ids64 ? (int64_t)((uint64_t)id[1] << 32 | id[0]) : (int64_t)(int32_t)id[0];
    *v = c >= 0 && c < a.V ? c : -1;
    *x = *v < 0 ? minus_inf() : __uint_as_float((uint32_t)logit[1] << 16 | (a.teacher_bf16 ? 0u : (uint32_t)logit[0]));
  }
};

// e_j in place of the teacher's logits; returns the lane's sum.  top: their maximum (without NaN).  The sum over the row is 0 where there are
// no entries, or none but -inf, and 1 or more elsewhere, or NaN: with NaN or +inf among the logits.
template <int THREADS>
__device__ __forceinline__ float weigh_entries(const Distill &a, const Entries &en, float top) {
  const float base = base_of(top);
  float sum = 0.0f;
  for (int j = threadIdx.x; j < a.K; j += THREADS) {
    const float e = exp2_of((en.share[j] - base) * a.c);       // (0 for -inf)
    en.share[j] = e;
    sum += e;
  }
  return sum;
}

// The lane's sum of tau^2 * q_j * log(e_j / exp((z_j - m) / tau)), in which the teacher's part is tau * log(e_j).
template <int THREADS>
__device__ __forceinline__ float cross_entries(const Distill &a, const Entries &en, float m, float total) {
  const float by = 2.0f * (a.tau / total);     // (of halves, whose difference does not overflow)
  float sum = 0.0f;
  for (int j = threadIdx.x; j < a.K; j += THREADS) {
    const float e = en.share[j];
    if (e == 0.0f) continue;
    const float cost = 0.5f * (a.tau * kLn2 * log2f(e)) - (0.5f * en.z[j] - 0.5f * m);
    sum = cost == __builtin_inff() ? sum + cost : fmaf(e * by, cost, sum);       // (e * by may have no bits left, which times inf is NaN)
  }
  return sum;
}

// e_j of all entries of a column in [lo, hi) together, for every one of them; once all e_j are there.  K comparisons for each: what bounds
// calls with many entries ([8192 x 50000] bf16, both: 311 us with 50, 437 with 200, 1360 with 1024).
template <int THREADS>
__device__ __forceinline__ void merge_entries(const Distill &a, const Entries &en, int64_t lo, int64_t hi) {
  for (int j = threadIdx.x; j < a.K; j += THREADS) {
    const int32_t v = en.at[j];
    if (v < lo || v >= hi) continue;
    float q = 0.0f;
#pragma unroll 4
    for (int k = 0; k < a.K; ++k) q += en.at[k] == v ? en.share[k] : 0.0f;
    en.q[j] = q;
  }
}

// Teacher's shares subtracted from the gradient at the entries' columns in [lo, hi): every wave writes those columns once more
// whose vectors it has written itself (vector i of the cut by wave i / (64 * each) mod WAVES, single columns by the first), so that no
// wave waits for another.  (A column that several entries share gets all of them, from every one of its entries alike.)
template <int WAVES, bool PLAIN, typename T>
__device__ __forceinline__ void subtract_entries(const Distill &a, const Entries &en, const Cut &cut, int each, float total, float g,
                                                 int64_t lo, int64_t hi, T *out, const Share &share) {
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
    if ((single ? 0u : i / (VE * 64u * (uint32_t)each) % WAVES) != (uint32_t)wave) continue;
    out[v] = from_float<T>(share.template at<PLAIN>(en.z[j]) - g * (en.q[j] * by));
  }
}

__device__ __forceinline__ float loss_of(const Distill &a, float cross, float total, float log_s) {
  return fmaf(a.tau * a.tau, log_s - logf(total), cross);
}

// Cache policy of buffer accesses: non-temporal.
constexpr int kStream = 2;

// ---- a row in registers: one pass over the logits ----

// 16 bytes per lane from a buffer to LDS, to `to` + 16 bytes times the lane's number.  Whoever reads them has to wait for vmcnt first.
__device__ __forceinline__ void copy_to_lds(__amdgpu_buffer_rsrc_t from, Words4 *to, uint32_t offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, offset, 0, 0, 0);
}

// What a call computes.
constexpr int kLoss = 1, kGrad = 2;

// One workgroup per row, whose lanes keep R vectors each: the logits are read once, all of them on their way at the same time.
// MODE: kLoss (loss and statistics), kGrad (the gradient from given statistics; a workgroup per chunk of a row), or both.
// The longest rows keep L more vectors per lane in shared memory, which they reach without passing through registers.
template <typename T, int THREADS, int R_, int L, int MODE>
__global__ __launch_bounds__(THREADS, R_ <= 8 ? 8 : 4) void distill_row_kernel(Distill a, const float *__restrict__ dloss,
                                                                               float *__restrict__ loss, float2 *stats, T *dlogits,
                                                                               int64_t ldd) {
  static_assert(L == 0 || MODE == (kLoss | kGrad), "the copies to LDS are waited for where the maximum is taken");
  constexpr int VE = 16 / (int)sizeof(T), WAVES = THREADS / 64;
  constexpr uint32_t kNothing = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;       // -inf, for vectors behind the row
  // Stores of the longest rows, which have a compute unit to themselves, leave the caches to others ([2048 x 131072] bf16 227 us,
  // 238 with plain ones, [1000 x 180000] 171 and 180; but [8192 x 50000] 329 and 312, [16384 x 4096] 64 and 51).
  constexpr int kPolicy = R_ >= 16 ? kStream : 0;
  typedef RowVec<T, VE> R;
  extern __shared__ uint32_t lds[];
  __shared__ float red[5][WAVES];
  __shared__ Words4 rest[L > 0 ? L * THREADS : 1];
  const Entries en(lds, a.K);
  const int t = threadIdx.x;
  const int64_t n = MODE == kGrad ? blockIdx.x / a.chunks : blockIdx.x;
  const T *row = static_cast<const T *>(a.logits) + n * a.ldz;
  int64_t lo = 0, hi = a.V;
  if constexpr (MODE == kGrad) chunk_of(a, row, blockIdx.x - n * a.chunks, &lo, &hi);
  const Cut cut(row, lo, hi);
  const int vecs = (int)cut.vecs;
  // The entries are on their way before the row, and what they need of each other is computed while the row is still coming.
  // (No load here is under a lane's condition, and no value has a default: the compiler would wait for the load at once.)
  RawEntry entry;
  if (a.K > 0) entry.load(a, n, t < a.K ? t : 0);
  const bool one = t < cut.singles;
  const int64_t single = one ? cut.single<VE>(lo, t) : lo;
  T raw_single, raw_z;
  if (hi > lo) raw_single = row[single];
  // Every wave has `each` times 64 consecutive vectors, four of these a buffer of their own: accesses beyond are neither loads nor
  // stores.  (What the range check goes by is the offset in the lane's register and that in the 12 bits of the instruction; vectors
  // THREADS apart in one buffer would take a register each.)
  const int lane = t & 63, each = (vecs + THREADS - 1) / THREADS, first = __builtin_amdgcn_readfirstlane(t >> 6) * each * 64;
  const int left = vecs - first < 0 ? 0 : vecs - first < each * 64 ? vecs - first : each * 64;
  auto buffer = [&](const T *p, int r) {
    const int skip = r / 4 * 256, rest = left - skip;
    return make_rsrc(p + lo + cut.head + (int64_t)(first + skip) * VE, rest > 0 ? (uint32_t)rest * 16u : 0u);
  };
  auto offset = [&](int r) { return (uint32_t)lane * 16u + r % 4 * 1024u; };
  Words4 x[R_];
#pragma unroll
  for (int r = 0; r < R_; ++r) x[r] = buffer_load<16>(buffer(row, r), offset(r));
  // (Loads return in order: what is used before the row is here has to be issued before it, and the logits at the entries, which are
  // not, are put away with the row's.  Only columns of this workgroup are read from the row: others may be overwritten by now.)
  float tm = minus_inf();
  auto put_entry = [&](int j) {                // returns where the entry's logit is read, at the first column where it is not needed
    int64_t v;
    float x;
    entry.take(a, &v, &x);
    en.at[j] = (int32_t)v;
    en.share[j] = x;
    tm = fmaxf(tm, x);
    return v >= lo && v < hi ? v : lo;
  };
  int64_t z_at = lo;
  if (t < a.K) z_at = put_entry(t);
  if (hi > lo) raw_z = row[z_at];
  for (int j = t + THREADS; j < a.K; j += THREADS) {
    entry.load(a, n, j);
    const int64_t v = put_entry(j);
    if (hi > lo) en.z[j] = elem_to_float<T>(row[v]);
  }
  const float top = group_max<WAVES>(tm, red[0]);
  const float total = group_sum<WAVES>(weigh_entries<THREADS>(a, en, top), red[1]);
  const bool none = total == 0.0f;
  if constexpr (MODE & kGrad) merge_entries<THREADS>(a, en, lo, hi);
  if constexpr (L > 0) {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      if ((R_ + l) * 64 >= left) continue;
      copy_to_lds(buffer(row, R_ + l), &rest[l * THREADS + (t - lane)], offset(R_ + l));
    }
  }
  // vector i of the wave from memory once more, for the rare rows whose exponents take more than one operation: a second set of loops
  // over the registers would cost the others registers
  auto again = [&](int i) { return *reinterpret_cast<const Words4 *>(row + lo + cut.head + (int64_t)(first + i) * VE); };
  // vector R_ + l of the lane, -inf behind the row
  auto from_lds = [&](int l) {
    Words4 w = rest[l * THREADS + t];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (R_ + l) * 64 + lane < left ? w[i] : kNothing;
    return w;
  };
  used_here(raw_single);
  const float zs = one ? elem_to_float<T>(raw_single) : minus_inf();
  float m = zs;
  if constexpr (MODE == kGrad) {
    m = stats[n].x;
    used_here(raw_z);
    if (t < a.K) en.z[t] = elem_to_float<T>(raw_z);
    __syncthreads();
  } else {
#pragma unroll
    for (int r = 0; r < R_; ++r) {
      // (Here and below: one vector after the other, unpacked anew in each pass.  Left to itself the compiler works on all of them
      // at a time and keeps every element as binary32 from one pass to the next, several times the registers.)
      if (r * 64 >= left) continue;
      asm volatile("" : "+v"(x[r]));
      if (r * 64 + 64 > left) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[r][i] = r * 64 + lane < left ? x[r][i] : kNothing;
      }
#pragma unroll
      for (int q = 0; q < VE; ++q) m = fmaxf(m, R::elem(x[r], q));
      asm volatile("" : "+v"(m));
    }
    if constexpr (L > 0) {
      // the copies have to be there: the compiler does not know that what is read here is what they write
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll 1
      for (int l = 0; l < L && (R_ + l) * 64 < left; ++l) {
        const Words4 w = from_lds(l);
#pragma unroll
        for (int q = 0; q < VE; ++q) m = fmaxf(m, R::elem(w, q));
      }
    }
    used_here(raw_z);
    if (t < a.K) en.z[t] = elem_to_float<T>(raw_z);
    m = group_max<WAVES>(m, red[2]);
  }
  T *out = dlogits + n * ldd;
  const Exponent ex(m, a.c);
  auto put = [&](auto f) {
    auto put_vector = [&](int r, const Words4 &z) {
      float v[VE];
#pragma unroll
      for (int q = 0; q < VE; ++q) v[q] = f(R::elem(z, q));
      const Words4 w = pack_row<T, VE>(v);
      __builtin_amdgcn_raw_buffer_store_b128(w, buffer(out, r), offset(r), 0, kPolicy);
    };
#pragma unroll
    for (int r = 0; r < R_; ++r) {
      if (r * 64 >= left) continue;
      asm volatile("" : "+v"(x[r]));
      put_vector(r, x[r]);
    }
    if constexpr (L > 0) {
#pragma unroll 1
      for (int l = 0; l < L && (R_ + l) * 64 < left; ++l) put_vector(R_ + l, from_lds(l));
    }
    if (one) out[single] = from_float<T>(f(zs));
  };
  if (none && (MODE & kGrad)) {
    if (t == 0 && (MODE & kLoss)) loss[n] = 0.0f;
    put([](float) { return 0.0f; });
    return;
  }
  // The rest, for rows of either kind of exponents as a whole: a branch inside would have the compiler copy the vectors where its ways
  // meet.
  auto finish = [&](auto plain) {
    constexpr bool PLAIN = decltype(plain)::value;
    float log2_s;                              // of the sum of 2^(the exponents)
    if constexpr (MODE == kGrad) {
      log2_s = fmaf(stats[n].y, kLog2E, ex.lost);
    } else {
      float acc[4] = {exp2_of(ex.template at<PLAIN>(zs)), 0.0f, 0.0f, 0.0f};
      auto add = [&](const Words4 &w) {
#pragma unroll
        for (int q = 0; q < VE; ++q) acc[q & 3] += exp2_of(ex.template at<PLAIN>(R::elem(w, q)));
      };
      if constexpr (PLAIN) {
#pragma unroll
        for (int r = 0; r < R_; ++r) {
          if (r * 64 >= left) continue;
          asm volatile("" : "+v"(x[r]));
          add(x[r]);
          asm volatile("" : "+v"(acc[0]), "+v"(acc[1]), "+v"(acc[2]), "+v"(acc[3]));
        }
        if constexpr (L > 0) {
#pragma unroll 1
          for (int l = 0; l < L && (R_ + l) * 64 < left; ++l) add(from_lds(l));
        }
      } else {
#pragma unroll 1
        for (int i = lane; i < left; i += 64) add(again(i));
      }
      const float cross = group_sum<WAVES>(cross_entries<THREADS>(a, en, m, total), red[3]);
      const float s = group_sum<WAVES>((acc[0] + acc[1]) + (acc[2] + acc[3]), red[4]);
      log2_s = m == minus_inf() ? __builtin_nanf("") : log2f(s);
      if (t == 0) {
        const float log_s = (log2_s - ex.lost) * kLn2;
        loss[n] = none ? 0.0f : loss_of(a, cross, total, log_s);
        if constexpr (MODE == kLoss) stats[n] = float2{m, log_s};
      }
    }
    if constexpr (MODE & kGrad) {
      const float g = dloss[n] * a.tau;
      const Share share(ex, log2_s, g);
      auto gradient = [&](float z) { return share.template at<PLAIN>(z); };
      if constexpr (PLAIN) {
        put(gradient);
      } else {
#pragma unroll 1
        for (int i = lane; i < left; i += 64) {
          const Words4 w = again(i);
          float v[VE];
#pragma unroll
          for (int q = 0; q < VE; ++q) v[q] = gradient(R::elem(w, q));
          R::store(out + lo + cut.head + (int64_t)(first + i) * VE, pack_row<T, VE>(v));
        }
        if (one) out[single] = from_float<T>(gradient(zs));
      }
      subtract_entries<WAVES, PLAIN>(a, en, cut, each, total, g, lo, hi, out, share);
    }
  };
  if (ex.plain) finish(std::true_type());
  else finish(std::false_type());
}

// ---- a row in chunks: two passes over the logits ----

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

// Statistics from the chunks' parts; the loss, by the first chunk's workgroup; GRAD: the chunk's gradient.
template <typename T, bool GRAD>
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
  float tm = minus_inf();
  for (int j = t; j < a.K; j += kThreads) {
    int64_t v;
    float x;
    RawEntry entry;
    entry.load(a, n, j);
    entry.take(a, &v, &x);
    en.at[j] = (int32_t)v;
    en.share[j] = x;
    en.z[j] = picked[n * a.K + j];             // (the row's own may be overwritten by other chunks' workgroups by now)
    tm = fmaxf(tm, x);
  }
  float pm = minus_inf();
  for (int i = t; i < parts_per_row; i += kThreads) pm = fmaxf(pm, parts[n * parts_per_row + i].x);
  const float m = group_max<kWaves>(pm, red[0]), base = base_of(m);
  float ps = 0.0f;
  for (int i = t; i < parts_per_row; i += kThreads) {
    const float2 p = parts[n * parts_per_row + i];
    ps += p.y * exp2_of((p.x - base) * a.c);
  }
  const float s = group_sum<kWaves>(ps, red[1]);
  const float log_s = m == minus_inf() ? __builtin_nanf("") : logf(s);
  const float top = group_max<kWaves>(tm, red[2]);
  const float total = group_sum<kWaves>(weigh_entries<kThreads>(a, en, top), red[3]);
  const bool none = total == 0.0f;
  if (blockIdx.x == 0) {
    const float x = group_sum<kWaves>(cross_entries<kThreads>(a, en, m, total), red[4]);
    if (t == 0) {
      loss[n] = none ? 0.0f : loss_of(a, x, total, log_s);
      if (stats != nullptr) stats[n] = float2{m, log_s};
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
    merge_entries<kThreads>(a, en, lo, hi);
    auto both = [&](auto plain) {
      constexpr bool PLAIN = decltype(plain)::value;
      run([&](float z) { return share.template at<PLAIN>(z); });
      __syncthreads();
      subtract_entries<kWaves, PLAIN>(a, en, cut, 1, total, g, lo, hi, out, share);
    };
    if (ex.plain) both(std::true_type());
    else both(std::false_type());
  }
}

// Chunks of a row: enough that the rows' chunks fill the compute units several times over, none shorter than 8192 columns ([8 x 131072]
// bf16, loss: 3.5 us and 4.5 for the two launches, 9.0 with the time between them).
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

// Room for the parts of up to N rows: ceil(kEnoughWorkgroups / n) of each, at most.
size_t parts_bytes(int64_t N) { return align_up((size_t)(kEnoughWorkgroups + N) * sizeof(float2), 256); }

// Rows from which long ones (more than 8192 vectors) have a workgroup each although they may be fewer than the compute units, against
// two passes over chunks ([100 x 262144] bf16 36.9 and 37.4 us, [64 x 262144] 34.6 and 23.0, [100 x 131072] 22.5 and 21.6, [32 x
// 131072] 19.7 and 14.4).  Up to 8192 vectors a single row is as fast so ([1 x 50000] 12.0 and 12.6, [8 x 20000] 9.8 and 12.5).
constexpr int64_t kEnoughRows = 96, kFewRows = 48, kComputeUnits = 256;

// Rows per launch of a two-dimensional grid, workgroups of a one-dimensional one: the second dimension ends at 65535, the first at
// 2^32 lanes.
constexpr int64_t kRowsPerLaunch = 65535, kWorkgroupsPerGrid = int64_t(1) << 21;

// The call's rows from n on, `most` at most.
Distill rows_from(const Distill &a, int64_t n, int dtype, int64_t most) {
  Distill b = a;
  b.logits = static_cast<const char *>(a.logits) + n * a.ldz * elem_bytes(dtype);
  b.ids = static_cast<const char *>(a.ids) + n * a.K * (a.ids64 ? 8 : 4);
  b.teacher = static_cast<const char *>(a.teacher) + n * a.K * (a.teacher_bf16 ? 2 : 4);
  b.N = a.N - n < most ? a.N - n : most;
  return b;
}

template <typename T, int THREADS, int R, int L, int MODE>
int run_rows(const Distill &whole, const float *dloss, float *loss, float2 *stats, void *dlogits, int64_t ldd, hipStream_t s) {
  const int64_t chunk = (int64_t)THREADS * (R + L) * (16 / (int64_t)sizeof(T)), chunks = MODE == kGrad ? ceil_div(whole.V, chunk) : 1;
  const int64_t most = chunks < kWorkgroupsPerGrid ? kWorkgroupsPerGrid / chunks : 1;
  for (int64_t n = 0; n < whole.N; n += most) {
    Distill a = rows_from(whole, n, sizeof(T) == 4 ? BSR_F32 : BSR_BF16, most);
    a.chunk = chunk;
    a.chunks = (int)chunks;
    hipLaunchKernelGGL((distill_row_kernel<T, THREADS, R, L, MODE>), dim3((unsigned)(a.N * chunks)), dim3(THREADS),
                       entries_bytes(a.K), s, a, dloss == nullptr ? dloss : dloss + n, loss == nullptr ? loss : loss + n,
                       stats == nullptr ? stats : stats + n, dlogits == nullptr ? nullptr : static_cast<T *>(dlogits) + n * ldd, ldd);
    const int rc = check_launch();
    if (rc != BSR_OK) return rc;
  }
  return BSR_OK;
}

// Two passes over chunks of rows.
template <typename T, bool GRAD>
int run_chunks(const DistillArgs &d, const float *dloss, float *loss, float2 *stats, void *dlogits, int64_t ldd, void *ws,
               hipStream_t s) {
  const Distill a = describe(d);
  float2 *parts = static_cast<float2 *>(ws);
  float *picked = reinterpret_cast<float *>(static_cast<char *>(ws) + parts_bytes(d.N));
  for (int64_t n = 0; n < d.N; n += kRowsPerLaunch) {
    const Distill b = rows_from(a, n, d.dtype, kRowsPerLaunch);
    hipLaunchKernelGGL((distill_parts_kernel<T>), dim3(a.chunks, (unsigned)b.N), dim3(kThreads), 0, s, b, parts + n * a.chunks,
                       picked + n * a.K);
    int rc = check_launch();
    if (rc != BSR_OK) return rc;
    hipLaunchKernelGGL((distill_finish_kernel<T, GRAD>), dim3(GRAD ? a.chunks : 1, (unsigned)b.N), dim3(kThreads),
                       entries_bytes(a.K), s, b, parts + n * a.chunks, a.chunks, picked + n * a.K, loss + n,
                       stats != nullptr ? stats + n : nullptr, dloss + (dloss != nullptr ? n : 0),
                       dlogits != nullptr ? static_cast<T *>(dlogits) + n * ldd : nullptr, ldd);
    rc = check_launch();
    if (rc != BSR_OK) return rc;
  }
  return BSR_OK;
}

template <typename T, bool GRAD>
int run_both(const DistillArgs &d, const float *dloss, float *loss, float *stats, void *dlogits, int64_t ldd, void *ws,
             hipStream_t s) {
  Distill a = describe(d);
  const int64_t vecs = a.V / (16 / (int64_t)sizeof(T));
  constexpr int MODE = GRAD ? kLoss | kGrad : kLoss;
  float2 *st = reinterpret_cast<float2 *>(stats);
  if (vecs <= 512) return run_rows<T, 64, 8, 0, MODE>(a, dloss, loss, st, dlogits, ldd, s);
  if (vecs <= 1024) return run_rows<T, 128, 8, 0, MODE>(a, dloss, loss, st, dlogits, ldd, s);
  if (vecs <= 2048) return run_rows<T, 256, 8, 0, MODE>(a, dloss, loss, st, dlogits, ldd, s);
  if (vecs <= 4096) return run_rows<T, 512, 8, 0, MODE>(a, dloss, loss, st, dlogits, ldd, s);
  if (vecs <= 8192) return run_rows<T, 1024, 8, 0, MODE>(a, dloss, loss, st, dlogits, ldd, s);
  if constexpr (GRAD) {
    // Longer rows have a compute unit to themselves: a last round of few of them goes by chunks ([270 x 262144] bf16 97 -> 78 us, [300 x
    // 131072] 48.6 -> 46.8; but [600 x 250007], 88 in the last round, 173.6 and 173.9, [1100 x 131072], 76, 139.7 and 142.7).
    const int64_t last = d.N % kComputeUnits, few = d.N < kComputeUnits ? kEnoughRows : kFewRows, whole = last < few ? d.N - last : d.N;
    if (whole > 0 && vecs <= 32768) {
      a.N = whole;
      const int rc = vecs <= 16384   ? run_rows<T, 1024, 16, 0, MODE>(a, dloss, loss, st, dlogits, ldd, s)
                     : vecs <= 24576 ? run_rows<T, 1024, 24, 0, MODE>(a, dloss, loss, st, dlogits, ldd, s)
                                     : run_rows<T, 1024, 24, 8, MODE>(a, dloss, loss, st, dlogits, ldd, s);
      if (rc != BSR_OK || whole == d.N) return rc;
      DistillArgs rest = d;
      rest.N = d.N - whole;
      rest.logits = static_cast<const T *>(d.logits) + whole * d.ldz;
      rest.ids = static_cast<const char *>(d.ids) + whole * d.K * (d.index_type == BSR_I64 ? 8 : 4);
      rest.teacher = static_cast<const char *>(d.teacher) + whole * d.K * elem_bytes(d.teacher_dtype);
      return run_chunks<T, GRAD>(rest, dloss + whole, loss + whole, st, static_cast<T *>(dlogits) + whole * ldd, ldd, ws, s);
    }
  }
  // The loss alone of such rows goes by chunks whatever their number, as its second launch reads no row again ([8 x 131072] bf16, 30 calls
  // in a row, 10.8 us, with a workgroup per row 12.1, [256 x 131072] 18.3 and 19.7, [2048 x 131072] 106.5 and 132, [1000 x 180000] 73.4 and
  // 96.4).
  return run_chunks<T, GRAD>(d, dloss, loss, st, dlogits, ldd, ws, s);
}

template <typename T>
int run_grad(const DistillArgs &d, const float *stats, const float *dloss, void *dlogits, int64_t ldd, hipStream_t s) {
  const Distill a = describe(d);
  const int64_t vecs = a.V / (16 / (int64_t)sizeof(T));
  float2 *st = reinterpret_cast<float2 *>(const_cast<float *>(stats));
  if (vecs <= 512) return run_rows<T, 64, 8, 0, kGrad>(a, dloss, nullptr, st, dlogits, ldd, s);
  if (vecs <= 1024) return run_rows<T, 128, 8, 0, kGrad>(a, dloss, nullptr, st, dlogits, ldd, s);
  return run_rows<T, 256, 4, 0, kGrad>(a, dloss, nullptr, st, dlogits, ldd, s);
}

}  // namespace

// (Of rows of any length, although none of up to 8192 vectors goes by chunks.)
size_t distill_ws_bytes(int64_t N, int64_t V, int64_t K) {
  (void)V;
  return parts_bytes(N) + align_up((size_t)N * K * sizeof(float), 256);
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
