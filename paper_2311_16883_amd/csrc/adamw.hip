// One AdamW step over many tensors, moments in binary32 or in 8 bits.
//
// Bound by memory: 28 bytes per element with binary32 weights, gradients and moments, 16 with 8-bit moments.  49 million elements of the
// first kind and bfloat16 copies of the weights: 271 us, 5.4 TB/s; 180 million of the second, bfloat16 gradients and copies: 580 us, 5.0 TB/s.
// (A large copy: 5.1.)  The tensors of a call
// are cut into chunks of whole blocks, a chunk to a workgroup; the list of tensors travels in the kernel's arguments, so
// there is nothing to copy or to keep for the device.  A lane holds four consecutive elements of a block, 32 lanes a block, whose largest magnitudes
// meet by lane exchanges.
//
// 8-bit moments: codes of 4 exponent bits in units of a power of two per block, so that scaling is exact and a value fits bfloat16.
// sqrt(v) is held in place of v: half the range in the exponent, and the update needs the root anyway.  Rounding is to one of the two
// neighbours with the probability of the distances, by bits of a counter hash: with beta2 = 0.999 a step changes sqrt(v) by 0.05 % of
// itself, its codes are 3 to 6 % apart, and to nearest it would never move.  A root does not become 0 beside others that do not, since the
// first moment beside it may be larger than its smallest code and would be divided by eps.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "layer_ops.h"

namespace bsr {

namespace {

constexpr int kThreads = 256;
// Consecutive elements of a lane: 16 bytes of the largest kind of number that is read.  (49 million bfloat16 weights and gradients, 8-bit
// moments: four a lane 149 us, eight 132; moments in binary32: 212 and 219.)
constexpr int per_lane(size_t param_bytes, bool small) { return param_bytes == 2 && small ? 8 : 4; }
constexpr int64_t kManyElements = int64_t(4) << 20;    // from here on a workgroup takes four rounds, below one
// From here on everything is read and written past the caches, which hold none of it until the next step: 49 million elements with binary32 moments
// 291 -> 271 us (5.4 TB/s), 180 million with 8-bit moments 592 -> 548 (codes from binary32, as then); stores alone 290
// and 580, loads alone 289 and 600; 4.8 million 28.8 -> 30.0.
constexpr int64_t kStreamElements = int64_t(16) << 20;
constexpr int kItems = 40;                             // tensors per launch: their list is 3.5 KB of arguments

struct Item {
  void *param;
  const void *grad;
  void *m, *v;
  uint8_t *scale_m, *scale_v;
  uint16_t *copy;
  int64_t n, first;                                    // elements; number of the first one in the whole list
  float decay;
};
struct Options {
  float lr, b1, c1, b2, c2, eps, grad_scale;           // c = 1 - b
  float first_full, root;                              // 1 / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
  uint32_t key;
  double beta1, beta2, scale64;
  const float *lr_device, *grad_scale_device;
  const int64_t *step_device;
  uint64_t seed;
};
struct List {
  Item it[kItems];
  uint32_t chunk_begin[kItems + 1];
  Options o;
};

__host__ __device__ inline uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x85A308D3u;
  x = (x ^ (x >> 15)) * 0xA4093823u;
  return x ^ (x >> 16);
}
__host__ __device__ inline uint32_t key_of(uint64_t seed, int64_t step) {
  return mix(mix((uint32_t)seed + 0x9E3779B1u * (uint32_t)step) ^ (uint32_t)(seed >> 32));
}
__host__ __device__ inline double power(double b, int64_t n) {
  double r = 1.0;
  for (; n > 0; n >>= 1, b *= b)
    if (n & 1) r *= b;
  return r;
}
__host__ __device__ inline void step_numbers(Options &o, int64_t step) {
  o.first_full = (float)(1.0 / (1.0 - power(o.beta1, step)));
  o.root = (float)(1.0 / sqrt(1.0 - power(o.beta2, step)));
  o.key = key_of(o.seed, step);
}

// N consecutive numbers, of which `left` are there (the others: 0), at any alignment.
template <int N, bool STREAM, typename T>
__device__ __forceinline__ void load_some(const T *p, int left, T *out) {
  constexpr int kBytes = N * sizeof(T), kEach = kBytes < 16 ? kBytes : 16;
  if (left >= N) {
#pragma unroll
    for (int b = 0; b < kBytes; b += kEach) {
      typedef typename RawWords<kEach>::type Loose __attribute__((aligned(1)));
      const auto *at = reinterpret_cast<const Loose *>(reinterpret_cast<const char *>(p) + b);
      const typename RawWords<kEach>::type w = STREAM ? __builtin_nontemporal_load(at) : *at;
      __builtin_memcpy(reinterpret_cast<char *>(out) + b, &w, kEach);
    }
  } else {
#pragma unroll
    for (int q = 0; q < N; ++q) out[q] = q < left ? p[q] : (T)0;
  }
}
template <int N, bool STREAM, typename T>
__device__ __forceinline__ void store_some(T *p, int left, const T *v) {
  constexpr int kBytes = N * sizeof(T), kEach = kBytes < 16 ? kBytes : 16;
  if (left >= N) {
#pragma unroll
    for (int b = 0; b < kBytes; b += kEach) {
      typename RawWords<kEach>::type w;
      __builtin_memcpy(&w, reinterpret_cast<const char *>(v) + b, kEach);
      typedef typename RawWords<kEach>::type Loose __attribute__((aligned(1)));
      auto *at = reinterpret_cast<Loose *>(reinterpret_cast<char *>(p) + b);
      if (STREAM) __builtin_nontemporal_store(w, at);
      else *at = w;
    }
  } else {
#pragma unroll
    for (int q = 0; q < N; ++q)
      if (q < left) p[q] = v[q];
  }
}

// A code's exponent and fraction are those of a binary32 number when they are moved to its place, the codes without an exponent among
// the subnormals: x = that number * 2^(scale - 15).  Scale 255: NaN.
template <int BITS>
__device__ __forceinline__ float decode(uint32_t code, uint32_t scale) {
  const uint32_t w = BITS == 3 ? (code & 127u) << 20 | (code & 128u) << 24 : code << 19;
  return __uint_as_float(__float_as_uint(ldexpf(__uint_as_float(w), (int)scale - 15)) | (scale == 255u ? 0x7FC00000u : 0u));
}

// The scale byte of a block whose largest magnitude has these bits: the exponent of the smallest power of two above which the
// largest code lies.
template <int BITS>
__device__ __forceinline__ uint32_t scale_of(uint32_t most) {
  const uint32_t b = (most + (0x7FFFFFu >> BITS)) >> 23;
  return b < 32u ? 0u : b > 255u ? 255u : b;
}

// How far a block's numbers are moved; those of a block without a scale far enough to be 0.
constexpr int kAway = -1000;
__device__ __forceinline__ int shift_of(uint32_t scale) { return scale == 0u ? kAway : 15 - (int)scale; }

// The code of a number >= 0, rounded to one of its two neighbours by u in [0, 2^16): `moved` is the number nearest to it in the codes' place,
// `above` whether that is above it, and so not what it is cut off to there.  The bits below a code's last are added to and cut off.  (The
// scale leaves room for it: the largest of a block is not above the largest code.)
template <int BITS>
__device__ __forceinline__ uint32_t encode(float moved, bool above, uint32_t u) {
  return (__float_as_uint(moved) - (above ? 1u : 0u) + (u << (7 - BITS))) >> (23 - BITS);
}

// The root of v cut off to binary32, as bits; `root`: one of the two numbers beside it.  What a code's border decides hangs on the last bit: of 49
// million elements 40 .. 60 have another code where m and v are made in binary32.  Binary64, whose multiplies and adds are as fast, costs 4 %.
__device__ __forceinline__ uint32_t root_cut_off(double v, float root) {
  return __float_as_uint(root) - (__builtin_fma((double)root, (double)root, -v) > 0.0 ? 1u : 0u);
}

// The root of v >= 0 to one unit in its last place.  The square of a binary32 number need not be one, so half of the (even part of the)
// exponent goes round the root, and the rest of v through it; infinities and NaN become infinities.
__device__ __forceinline__ float root_of(double v) {
  const uint64_t bits = (uint64_t)__double_as_longlong(v);
  const double rest = __longlong_as_double((long long)((bits & 0x001FFFFFFFFFFFFFu) | 0x3FE0000000000000u));       // in [1/2, 2)
  return ldexpf(__builtin_amdgcn_sqrtf((float)rest), (int)(bits >> 53) - 511);
}
// ... of a binary32 v, whose subnormals the root instruction would lose.
__device__ __forceinline__ float root_of(float v) {
  const bool small = v < 0x1p-96f;
  return __builtin_amdgcn_sqrtf(v * (small ? 0x1p64f : 1.0f)) * (small ? 0x1p-32f : 1.0f);
}

template <typename P, typename G, bool SMALL, bool COPY, bool STREAM>
__global__ __launch_bounds__(kThreads) void adamw_kernel(List list, int n, int rounds) {
  constexpr int PL = per_lane(sizeof(P), SMALL), kGroup = PL == 8 ? 4 : 5;      // lanes of a block: 2^kGroup
  // this workgroup's tensor
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (blockIdx.x >= list.chunk_begin[mid]) lo = mid;
    else hi = mid;
  }
  const Item &it = list.it[lo];
  const int64_t chunk0 = (int64_t)(blockIdx.x - list.chunk_begin[lo]) * rounds * (kThreads * PL);
  Options o = list.o;
  if (o.step_device != nullptr) step_numbers(o, *o.step_device);
  if (o.lr_device != nullptr) o.lr = *o.lr_device;
  if (o.grad_scale_device != nullptr) o.grad_scale = *o.grad_scale_device;
  const double c1 = 1.0 - o.beta1, c2 = 1.0 - o.beta2;
  const double grad_scale = o.grad_scale_device != nullptr ? (double)o.grad_scale : o.scale64;
  P *const param = static_cast<P *>(it.param);
  const G *const grad = static_cast<const G *>(it.grad);
  const float keep = 1.0f - o.lr * it.decay, rate = o.lr * o.first_full;
  for (int r = 0; r < rounds; ++r) {
    const int64_t i = chunk0 + (int64_t)r * (kThreads * PL) + threadIdx.x * PL;
    if (chunk0 + (int64_t)r * (kThreads * PL) >= it.n) break;
    const int left = it.n - i >= PL ? PL : it.n > i ? (int)(it.n - i) : 0;
    P p0[PL];
    G g0[PL];
    float m[PL], root[PL], p[PL];
    double m64[SMALL ? PL : 1];
    uint32_t cut_r[SMALL ? PL : 1];
    load_some<PL, STREAM>(param + i, left, p0);
    load_some<PL, STREAM>(grad + i, left, g0);
    const int64_t block = i / kMomentBlock;
    float eps = o.eps;
    if constexpr (SMALL) {
      uint8_t cm[PL], cv[PL];
      load_some<PL, STREAM>(static_cast<const uint8_t *>(it.m) + i, left, cm);
      load_some<PL, STREAM>(static_cast<const uint8_t *>(it.v) + i, left, cv);
      const uint32_t sm = left > 0 ? it.scale_m[block] : 0u, sv = left > 0 ? it.scale_v[block] : 0u;
#pragma unroll
      for (int q = 0; q < PL; ++q) {
        m[q] = decode<3>(cm[q], sm);
        root[q] = decode<4>(cv[q], sv);
      }
      if (sv == 255u) eps = __uint_as_float(0x7FC00000u);      // (root_of does not pass on a NaN)
    } else {
      load_some<PL, STREAM>(static_cast<const float *>(it.m) + i, left, m);
      load_some<PL, STREAM>(static_cast<const float *>(it.v) + i, left, root);
    }
#pragma unroll
    for (int q = 0; q < PL; ++q) {
      float rt;
      if constexpr (SMALL) {
        const double g = (double)elem_to_float<G>(g0[q]) * grad_scale, old = root[q];
        m64[q] = __builtin_fma(o.beta1, (double)m[q], c1 * g);
        const double v = __builtin_fma(o.beta2 * old, old, c2 * g * g);
        m[q] = (float)m64[q];
        rt = root_of(v);
        cut_r[q] = root_cut_off(v, rt);
      } else {
        const float g = elem_to_float<G>(g0[q]) * o.grad_scale;
        m[q] = o.b1 * m[q] + o.c1 * g;
        root[q] = o.b2 * root[q] + o.c2 * g * g;
        rt = root_of(root[q]);
      }
      p[q] = elem_to_float<P>(p0[q]) * keep - rate * m[q] * __builtin_amdgcn_rcpf(rt * o.root + eps);
    }
#pragma unroll
    for (int q = 0; q < PL; ++q) p0[q] = from_float<P>(p[q]);
    store_some<PL, STREAM>(param + i, left, p0);
    if constexpr (COPY) {
      uint16_t c[PL];
#pragma unroll
      for (int q = 0; q < PL; ++q) c[q] = from_float<uint16_t>(p[q]);
      store_some<PL, STREAM>(it.copy + i, left, c);
    }
    if constexpr (SMALL) {
      uint32_t most_m = 0u, most_v = 0u;
#pragma unroll
      for (int q = 0; q < PL; ++q) {
        most_m = max(most_m, q < left ? __float_as_uint(m[q]) & 0x7FFFFFFFu : 0u);
        most_v = max(most_v, q < left ? cut_r[q] : 0u);
      }
      const uint32_t sm = scale_of<3>(group_max<kGroup>(most_m)), sv = scale_of<4>(group_max<kGroup>(most_v));
      const int by_m = shift_of(sm), by_r = shift_of(sv);
      const uint32_t least = sv == 0u ? 0u : 1u;
      uint8_t cm[PL], cv[PL];
      const uint64_t number = (uint64_t)(it.first + i);       // (its high half is that of all)
      const uint32_t base = (uint32_t)number * 0x9E3779B1u + (uint32_t)(number >> 32) * 0x7F4A7C15u + o.key;
#pragma unroll
      for (int q = 0; q < PL; ++q) {
        const uint32_t h = mix(base + (uint32_t)q * 0x9E3779B1u);
        const float near = ldexpf(fabsf(m[q]), by_m), cut = __uint_as_float(cut_r[q]), near_r = ldexpf(cut, by_r);
        const uint32_t c = encode<3>(near, (double)ldexpf(near, -by_m) > fabs(m64[q]), h & 0xFFFFu);
        cm[q] = (uint8_t)(c | (c != 0u && m[q] < 0.0f ? 128u : 0u));
        cv[q] = (uint8_t)max(encode<4>(near_r, ldexpf(near_r, -by_r) > cut, h >> 16), min(cut_r[q], least));
      }
      if (sm == 255u)
#pragma unroll
        for (int q = 0; q < PL; ++q) cm[q] = 0;
      if (sv == 255u)
#pragma unroll
        for (int q = 0; q < PL; ++q) cv[q] = 0;
      store_some<PL, STREAM>(static_cast<uint8_t *>(it.m) + i, left, cm);
      store_some<PL, STREAM>(static_cast<uint8_t *>(it.v) + i, left, cv);
      if (threadIdx.x % (kMomentBlock / PL) == 0 && left > 0) {
        it.scale_m[block] = (uint8_t)sm;
        it.scale_v[block] = (uint8_t)sv;
      }
    } else {
      store_some<PL, STREAM>(static_cast<float *>(it.m) + i, left, m);
      store_some<PL, STREAM>(static_cast<float *>(it.v) + i, left, root);
    }
  }
}

// Sixteen codes to a lane.
template <typename T, int BITS, bool STREAM>
__global__ __launch_bounds__(kThreads) void state_values_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                                int64_t n, T *__restrict__ out) {
  for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 16; i < n; i += (int64_t)gridDim.x * kThreads * 16) {
    const uint32_t scale = scales[i / kMomentBlock];
    if (n - i >= 16) {
      uint8_t c[16];
      load_some<16, STREAM>(codes + i, 16, c);
      T v[16];
#pragma unroll
      for (int q = 0; q < 16; ++q) v[q] = from_float<T>(decode<BITS>(c[q], scale));
      store_some<16, STREAM>(out + i, 16, v);
    } else {
      for (int64_t j = i; j < n; ++j) out[j] = from_float<T>(decode<BITS>(codes[j], scale));
    }
  }
}

template <typename P, typename G, bool SMALL, bool COPY>
void launch_list(const List &list, int n, uint32_t chunks, int rounds, bool stream, hipStream_t s) {
  if (stream) adamw_kernel<P, G, SMALL, COPY, true><<<dim3(chunks), kThreads, 0, s>>>(list, n, rounds);
  else adamw_kernel<P, G, SMALL, COPY, false><<<dim3(chunks), kThreads, 0, s>>>(list, n, rounds);
}

}  // namespace

int launch_adamw(const bsr_adamw_item *items, int n, int param_dtype, int grad_dtype, int moments, const bsr_adamw_options &opt,
                 hipStream_t s) {
  List list;
  Options &o = list.o;
  o.b1 = (float)opt.beta1;
  o.c1 = (float)(1.0 - opt.beta1);
  o.b2 = (float)opt.beta2;
  o.c2 = (float)(1.0 - opt.beta2);
  o.eps = (float)opt.eps;
  o.grad_scale = (float)opt.grad_scale;
  o.beta1 = opt.beta1;
  o.beta2 = opt.beta2;
  o.scale64 = opt.grad_scale;
  o.seed = opt.seed;
  o.lr_device = opt.lr_device;
  o.grad_scale_device = opt.grad_scale_device;
  o.step_device = opt.step_device;
  o.lr = (float)opt.lr;
  step_numbers(o, opt.step);
  const bool small = moments == BSR_MOMENTS_8BIT;
  int64_t first = 0;
  int held = 0;
  bool copies = false;
  uint32_t chunks = 0;
  int64_t all = 0;
  for (int i = 0; i < n; ++i) all += items[i].n;
  const int rounds = all >= kManyElements ? 4 : 1;
  const bool stream = all >= kStreamElements;
  const int64_t chunk = (int64_t)kThreads * rounds * per_lane((size_t)elem_bytes(param_dtype), small);
  auto flush = [&]() {
    if (held == 0) return (int)BSR_OK;
    list.chunk_begin[held] = chunks;
    auto go = [&](auto p, auto g) {
      typedef decltype(p) P;
      typedef decltype(g) G;
      if (small) copies ? launch_list<P, G, true, true>(list, held, chunks, rounds, stream, s) : launch_list<P, G, true, false>(list, held, chunks, rounds, stream, s);
      else copies ? launch_list<P, G, false, true>(list, held, chunks, rounds, stream, s) : launch_list<P, G, false, false>(list, held, chunks, rounds, stream, s);
    };
    if (param_dtype == BSR_F32) grad_dtype == BSR_F32 ? go(float(), float()) : go(float(), uint16_t());
    else grad_dtype == BSR_F32 ? go(uint16_t(), float()) : go(uint16_t(), uint16_t());
    held = 0;
    chunks = 0;
    return check_launch();
  };
  for (int i = 0; i < n; ++i) {
    const bsr_adamw_item &x = items[i];
    if (x.n > 0) {
      // chunks of a launch: its lanes are counted in 32 bits; a tensor beyond that goes in parts of whole blocks
      constexpr int64_t kMostChunks = int64_t(1) << 23;
      for (int64_t at = 0; at < x.n; at += kMostChunks * chunk) {
        const int64_t part = std::min(x.n - at, kMostChunks * chunk), needs = ceil_div(part, chunk);
        const bool copy = x.copy != nullptr;
        if (held == kItems || (held > 0 && (copy != copies || chunks + needs > kMostChunks)))
          if (const int rc = flush(); rc != BSR_OK) return rc;
        copies = copy;
        const int64_t pe = elem_bytes(param_dtype) * at, ge = elem_bytes(grad_dtype) * at, me = (small ? 1 : 4) * at;
        Item &it = list.it[held];
        it.param = static_cast<char *>(x.param) + pe;
        it.grad = static_cast<const char *>(x.grad) + ge;
        it.m = static_cast<char *>(x.m) + me;
        it.v = static_cast<char *>(x.v) + me;
        it.scale_m = small ? x.scales + at / kMomentBlock : nullptr;
        it.scale_v = small ? x.scales + x.scales_stride + at / kMomentBlock : nullptr;
        it.copy = copy ? static_cast<uint16_t *>(x.copy) + at : nullptr;
        it.n = part;
        it.first = first + at;
        it.decay = x.weight_decay;
        list.chunk_begin[held++] = chunks;
        chunks += (uint32_t)needs;
      }
    }
    first += ceil_div(x.n, (int64_t)kMomentBlock) * kMomentBlock;
  }
  return flush();
}

int launch_adamw_state_values(const uint8_t *codes, const uint8_t *scales, int64_t n, int which, void *out, int dtype, hipStream_t s) {
  const dim3 grid((uint32_t)std::min(ceil_div(n, (int64_t)kThreads * 16), int64_t(1) << 23));
  auto go = [&](auto type, auto bits) {
    typedef decltype(type) T;
    if (n >= kStreamElements) state_values_kernel<T, decltype(bits)::value, true><<<grid, kThreads, 0, s>>>(codes, scales, n, static_cast<T *>(out));
    else state_values_kernel<T, decltype(bits)::value, false><<<grid, kThreads, 0, s>>>(codes, scales, n, static_cast<T *>(out));
  };
  typedef std::integral_constant<int, 3> M;
  typedef std::integral_constant<int, 4> R;
  if (dtype == BSR_F32) which == 0 ? go(float(), M()) : go(float(), R());
  else which == 0 ? go(uint16_t(), M()) : go(uint16_t(), R());
  return check_launch();
}

}  // namespace bsr
