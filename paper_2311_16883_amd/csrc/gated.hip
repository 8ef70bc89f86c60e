// Gated feed-forward block, forward and backward: two matrix products with what surrounds them fused in.
//
//   forward   [G | U] = X W,  H = act(G) * U         (W as it is stored, [D x 2F]: the contraction is its slow axis)
//   backward  dGU from GU and dH, then dX = dGU W^T  (both operands contiguous along the contraction)
//
// bfloat16 operands whose rows are not whole words are copied into the workspace first, rows padded; then so is the contraction,
// with zeros.  Where there are few tiles the contraction is split and a second kernel adds the parts up, in order.  Few rows read W once, at the
// rate of memory: 1 x 2048 x [2 x 5504] bfloat16 11.0 us (4.1 TB/s).  Large products are bound by the matrix cores (8192 rows of the same: 372 us, 0.99
// PFLOP/s), the slopes by memory (25088 x [2 x 1024]: 257 MB in 41 us, 6.3 TB/s).
#include "gated.h"

namespace bsr {

namespace {

// ---- few rows ----

// Sum over the lanes of a wave whose numbers are equal modulo V.
template <int V>
__device__ __forceinline__ float sum_strided(float v) {
  static_assert(V == 4 || V == 8, "");
  v += dpp_of<0x128>(v);                             // rotations within 16 lanes
  if constexpr (V <= 4) v += dpp_of<0x124>(v);
  v += other_row(v);
  return v + other_half(v);
}

// [G | U] and H of the M <= MR rows of X, one workgroup to V 16-byte vectors of columns of G and the same of U, over the whole
// contraction: W is read once, by plain loads of whole vectors at any alignment, those of a lane on their way together.
// Consecutive workgroups of an XCD have neighbouring columns, whose 128-byte lines they share.
constexpr int kFewThreads = 1024, kFewWaves = kFewThreads / 64, kFewK = 2048;
template <typename T, int MR, int V>
__global__ __launch_bounds__(kFewThreads) void gated_few_kernel(int act, const T *__restrict__ X, int M, int64_t D, int64_t ldx,
                                                                const T *__restrict__ W, int64_t F, int64_t ldw, T *__restrict__ H,
                                                                int64_t ldh, T *__restrict__ GU, int64_t ldgu, int groups) {
  constexpr int VE = kVec<T>, kSums = 2 * VE * MR, kRows = 64 / V, kStep = kRows * kFewWaves, kTogether = 4;
  typedef RowVec<T, VE> R;
  __shared__ float xs[MR][kFewK];
  __shared__ float sums[kFewWaves][V][kSums];
  const int per_xcd = (groups + 7) / 8, group = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if (group >= groups || (int)(blockIdx.x >> 3) >= per_xcd) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane / V, vec = lane % V;
  const int64_t c = ((int64_t)group * V + vec) * VE;
  const bool there = c < F;
  const int64_t at = !there ? 0 : c + VE <= F ? c : F - VE;       // (the last vector ends with G's columns; F >= VE)
  float acc[kSums];
#pragma unroll
  for (int i = 0; i < kSums; ++i) acc[i] = 0.0f;
  typename R::Raw g[kTogether], u[kTogether];
  auto load = [&](int64_t k0, int k1, int here) {
#pragma unroll
    for (int t = 0; t < kTogether; ++t) {
      const int k = k1 + t * kStep;
      g[t] = u[t] = R::zero();
      if (there && k < here) {
        const T *p = W + (k0 + k) * ldw + at;
        g[t] = R::load(p);
        u[t] = R::load(p + F);
      }
    }
  };
  for (int64_t k0 = 0; k0 < D; k0 += kFewK) {
    const int here = D - k0 < kFewK ? (int)(D - k0) : kFewK, first = wave * kRows + row;
    load(k0, first, here);                           // on their way while X is copied
    if (k0 > 0) __syncthreads();
    for (int i = threadIdx.x; i < MR * kFewK; i += kFewThreads) {
      const int m = i / kFewK, k = i % kFewK;
      xs[m][k] = m < M && k < here ? elem_to_float<T>(X[m * ldx + k0 + k]) : 0.0f;
    }
    __syncthreads();
    for (int k1 = first; k1 < here; k1 += kTogether * kStep) {
      if (k1 != first) load(k0, k1, here);
#pragma unroll
      for (int t = 0; t < kTogether; ++t) {
        const int k = k1 + t * kStep;
        if (k >= here) continue;
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          const float x = xs[m][k];
#pragma unroll
          for (int q = 0; q < VE; ++q) {
            acc[m * 2 * VE + q] += x * R::elem(g[t], q);
            acc[m * 2 * VE + VE + q] += x * R::elem(u[t], q);
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kSums; ++i) acc[i] = sum_strided<V>(acc[i]);
  if (row == 0) {
#pragma unroll
    for (int i = 0; i < kSums; ++i) sums[wave][vec][i] = acc[i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < V * VE * MR; i += kFewThreads) {
    const int m = i / (V * VE), v = i / VE % V, q = i % VE;
    const int64_t c0 = ((int64_t)group * V + v) * VE;
    if (m >= M || c0 >= F) continue;
    float g = 0.0f, u = 0.0f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      g += sums[w][v][m * 2 * VE + q];
      u += sums[w][v][m * 2 * VE + VE + q];
    }
    const int64_t col = (c0 + VE <= F ? c0 : F - VE) + q;          // (columns that two vectors share are written twice, the same)
    H[m * ldh + col] = from_float<T>(activation_value(act, g) * u);
    if (GU != nullptr) {
      GU[m * ldgu + col] = from_float<T>(g);
      GU[m * ldgu + F + col] = from_float<T>(u);
    }
  }
}

// ---- operands in whole words ----

// Columns [from, from + cols) of a matrix into rows of `pitch` elements from column `to` on, zeros up to column `to + padded`.
struct PackJob {
  const void *src;
  int64_t rows, ld, from, cols;
  void *dst;
  int64_t pitch, to, padded;
};
template <typename T>
__device__ __forceinline__ void pack(const PackJob &j, int64_t block, int64_t blocks) {
  constexpr int VE = kVec<T>;
  const int64_t vecs = j.padded / VE;
  for (int64_t i = block * 256 + threadIdx.x; i < j.rows * vecs; i += blocks * 256) {
    const int64_t r = i / vecs, c = i % vecs * VE;
    const T *p = static_cast<const T *>(j.src) + r * j.ld + j.from + c;
    Words4 v = {0, 0, 0, 0};
    if (c + VE <= j.cols) v = RowVec<T, VE>::load(p);
    else {
      T e[VE];
#pragma unroll
      for (int q = 0; q < VE; ++q) e[q] = c + q < j.cols ? p[q] : (T)0;
      __builtin_memcpy(&v, e, 16);
    }
    *reinterpret_cast<Words4 *>(static_cast<T *>(j.dst) + r * j.pitch + j.to + c) = v;
  }
}
constexpr int kPackJobs = 3;
struct PackList {
  PackJob it[kPackJobs];
  int32_t begin[kPackJobs + 1];                      // first workgroup of each
};
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(PackList l) {
  const int b = (int)blockIdx.x, i = b >= l.begin[2] ? 2 : b >= l.begin[1] ? 1 : 0;
  pack<T>(l.it[i], b - l.begin[i], l.begin[i + 1] - l.begin[i]);
}

// dGU from GU and dH, a vector of columns to a thread; `also`: a second copy with rows of `pitch` elements, or null.  The workgroups from
// `blocks` on pack W.
template <typename T, int VE, int ACT, bool STREAM>
__global__ __launch_bounds__(256) void gated_slope_kernel(const T *GU, int64_t M, int64_t F, int64_t ldgu, const T *__restrict__ dH,
                                                          int64_t lddh, T *dGU, int64_t lddgu, T *__restrict__ also, int64_t pitch,
                                                          int32_t blocks, PackJob job) {
  typedef RowVec<T, VE> R;
  if ((int)blockIdx.x >= blocks) {
    pack<T>(job, (int)blockIdx.x - blocks, (int)gridDim.x - blocks);
    return;
  }
  const int64_t vecs = F / VE;                       // whole vectors
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * vecs; i += (int64_t)blocks * 256) {
    const int64_t m = i / vecs, f = i % vecs * VE;
    const typename R::Raw g = load_once<T, VE, STREAM>(GU + m * ldgu + f), u = load_once<T, VE, STREAM>(GU + m * ldgu + F + f),
                          d = load_once<T, VE, STREAM>(dH + m * lddh + f);
    float a[VE], b[VE];
#pragma unroll
    for (int q = 0; q < VE; ++q) {
      const Activation x = activation<ACT>(R::elem(g, q));
      const float dh = R::elem(d, q);
      a[q] = dh * R::elem(u, q) * x.slope;
      b[q] = dh * x.value;
    }
    const typename R::Raw pa = pack_row<T, VE>(a), pb = pack_row<T, VE>(b);
    R::store(dGU + m * lddgu + f, pa);
    R::store(dGU + m * lddgu + F + f, pb);
    if (also != nullptr) {
      R::store(also + m * pitch + f, pa);
      R::store(also + m * pitch + F + f, pb);
    }
  }
  if (also != nullptr) {                             // zeros behind the last column
    const int64_t pad = pitch - 2 * F;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * pad; i += (int64_t)blocks * 256)
      also[i / pad * pitch + 2 * F + i % pad] = (T)0;
  }
  if constexpr (VE > 1) {
    const int64_t rest = F - vecs * VE;
    if (rest == 0) return;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * rest; i += (int64_t)blocks * 256) {
      const int64_t m = i / rest, f = vecs * VE + i % rest;
      const Activation x = activation<ACT>(elem_to_float<T>(GU[m * ldgu + f]));
      const float u = elem_to_float<T>(GU[m * ldgu + F + f]), dh = elem_to_float<T>(dH[m * lddh + f]);
      const T a = from_float<T>(dh * u * x.slope), b = from_float<T>(dh * x.value);
      dGU[m * lddgu + f] = a;
      dGU[m * lddgu + F + f] = b;
      if (also != nullptr) {
        also[m * pitch + f] = a;
        also[m * pitch + F + f] = b;
      }
    }
  }
}

// ---- host ----

template <typename F>
void with_act(int act, F f) {
  if (act == BSR_ACT_SILU) f(std::integral_constant<int, BSR_ACT_SILU>());
  else if (act == BSR_ACT_GELU) f(std::integral_constant<int, BSR_ACT_GELU>());
  else if (act == BSR_ACT_GELU_TANH) f(std::integral_constant<int, BSR_ACT_GELU_TANH>());
  else f(std::integral_constant<int, BSR_ACT_RELU>());
}

constexpr int kCus = 256;
// Bytes of GU from which it and dH pass by the caches, which then keep more of dGU for the product (25088 x 384 x [2 x 1024]: 97.3 us, 90.7 so).
constexpr int64_t kStream = int64_t(64) << 20;

int64_t padded(int64_t n, int dtype) {
  const int64_t ve = 16 / elem_bytes(dtype);
  return ceil_div(n, ve) * ve;
}

// Whether a product takes an operand as it is: rows of whole words at whole words (binary32 always), offsets of a tile within its range.
bool in_place(const void *p, int dtype, int64_t ld, int64_t inner) {
  const int64_t e = elem_bytes(dtype);
  return (uintptr_t)p % 4 == 0 && ld * e % 4 == 0 && inner * e % 4 == 0 && ld * e * 256 < (int64_t)kRange;
}

// Tiles that are never the best of their kind are not there: binary32 is bound by the matrix cores in any of them (8192 rows: 125
// TFLOP/s in 128 x 256, 121 in 128 x 128, 95 in 256 x 256), and rows of 64 bytes of both operands are half of every line.
bool has_tile(Tile t, int dtype, bool gated) {
  if (dtype == BSR_F32) return t == kTile128 || t == kTile64 || t == kTile32;
  return t == kTileWide ? gated : t == kTile96Alone ? !gated : true;
}

// Estimated microseconds, from what the kernels were measured to do: TFLOP/s of a compute unit with one workgroup in it and with two
// (bfloat16: 8192 x 2048 x [2 x 5504] in 256 x 256 tiles 326 us, in 128 x 256 349, in 128 x 128 390; 2048 rows 97, 85, 93; 512 rows 42, 27, 29;
// 2999 x 3080 x 808 in 96 x 128 tiles, 224 of them, 24, in 128 x 128, 168 of them, alone in their unit 26, otherwise 45).  A tile's beginning
// and end cost as much as some more of the contraction, most where nothing runs beside it (16384 x 128 x [2 x 2048] in 256 x 256 tiles 46 us, in 128 x 256 35,
// in 128 x 128 51; 8192 x 512 x [2 x 2816] 64, 53, 68).  Tiles of 32 rows, in 16 and in up to 64 parts: one row of 16384 x [2 x 512] 14.9 and
// 12.4 us, of 40000 x [2 x 64] 26.1 and 13.7, binary32 47 and 20, 103 and 33.  (Whether GU is written has no part in it: H would have other bits
// with GU than without.)  Tiles of 32 rows are for up to 32: bfloat16 of 33 to 96 rows is no faster in them (48 x 2048 x [2 x 5504] 15.2 us and 20.3,
// 33 x 8192 x [2 x 1024] 13.6 and 13.8); binary32 takes a tenth more or less (64 x 4096 x [2 x 4096] 49.4 and 50.5, 33 x 2048 x [2 x 5504] 40.5 and 38.8), but
// small products and gradients of few columns, which more than 16 parts would share, up to half (48 x 411 x [2 x 1003] 14.9 and 11.7, gradient of
// 48 x 512 x [2 x 8192] 46 and 23).
double estimate_us(Tile t, int64_t M, int64_t N, int64_t K, int dtype, bool gated, int64_t splits) {
  const double rates[2][7][2] = {{{4.9, 4.9}, {4.6, 4.4}, {2.4, 3.6}, {3.4, 3.4}, {3.0, 3.0}, {2.9, 2.8}, {1.0, 1.8}},
                                 {{0, 0}, {0, 0}, {0.46, 0.53}, {0, 0}, {0, 0}, {0.45, 0.47}, {0.43, 0.45}}};
  const TileSize &s = kTiles[t];
  const bool f32 = dtype == BSR_F32;
  const int64_t tiles = ceil_div(M, (int64_t)s.rows) * ceil_div(N, (int64_t)(gated ? s.cols / 2 : s.cols)) * splits;
  const int64_t each = ceil_div(tiles, (int64_t)kCus);
  const bool whole = t == kTile32 && !f32 && splits == 1;
  const bool results = gated && splits == 1;         // activations and two or three results
  const double rate = whole ? 1.9 : results && t == kTile256 ? 5.4 : rates[f32][t][each > 1];
  const double with_results[] = {365.0, 140.0, 200.0, 256.0, 0.0, 256.0, 170.0};
  const double more = f32 ? (results ? 48.0 : 24.0) : whole || results ? with_results[t] : 128.0;
  double us = 3.0 + (double)each * s.rows * s.cols * 2.0 * (ceil_div(K, splits) + more) / (rate * 1e6);
  if (splits > 1) us += 4.0 + (double)splits * (M * N * (gated ? 2 : 1) * 8.0 / 4e6 + 0.025);
  return us;
}

Plan plan_product(int64_t M, int64_t N, int64_t K, int dtype, bool gated) {
  Plan p = {kTile32, 0, 1, 0, 0.0};
  double best = 0.0;
  int64_t splits = 1;
  for (int t = kTile256; t <= kTile32; ++t) {
    if ((t == kTile32) != (M <= 32) || !has_tile((Tile)t, dtype, gated)) continue;
    const TileSize &s = kTiles[t];
    const int64_t stages = std::max<int64_t>(1, ceil_div(K, (int64_t)(s.row_bytes / elem_bytes(dtype))));
    // (more than 16 parts of long contractions only where they have a compute unit each, of bfloat16 two: more of them at a time are slower)
    const int64_t across = std::max<int64_t>(1, ceil_div(N, (int64_t)(gated ? s.cols / 2 : s.cols)));
    const int64_t each = kCus / (dtype == BSR_F32 ? 1 : 2) / across;
    const int64_t most = t == kTile256 || t == kTile96Alone ? 1 : t != kTile32 ? 16 : std::min<int64_t>(64, std::max<int64_t>(16, each));
    for (int64_t n = 1; n <= most && n * 4 <= std::max<int64_t>(stages, 4); n = t == kTile32 && n < 16 ? n + 1 : 2 * n) {
      const double us = estimate_us((Tile)t, M, N, K, dtype, gated, n);
      if (best == 0.0 || us < best) {
        best = us;
        p.tile = (Tile)t;
        splits = n;
      }
    }
  }
  p.us = best;
  const TileSize &s = kTiles[p.tile];
  const int64_t stages = std::max<int64_t>(1, ceil_div(K, (int64_t)(s.row_bytes / elem_bytes(dtype))));
  p.tiles_n = (int32_t)ceil_div(N, (int64_t)(gated ? s.cols / 2 : s.cols));
  p.stages_per_split = (int32_t)ceil_div(stages, splits);
  p.splits = (int32_t)ceil_div(stages, (int64_t)p.stages_per_split);
  return p;
}

size_t partial_bytes(const Plan &p, int64_t M, int64_t N, bool gated) {
  return p.splits > 1 ? align_up((size_t)p.splits * (size_t)M * (size_t)partial_pitch(N, gated) * 4, 256) : 0;
}

template <typename T>
int product_of(const Plan &p, const ProductArgs &a, bool gated, hipStream_t s) {
  if constexpr (sizeof(T) == 2) return launch_product_bf16(p, a, gated, s);
  else return launch_product_f32(p, a, gated, s);
}

// What goes into the workspace, in this order.
struct Layout {
  Plan plan;
  size_t a = 0, b = 0, partial = 0, all = 0;         // bytes of the packed operands (0: taken in place), of the parts, together
  enum { kTiles, kFew, kRows } by = kTiles;          // forward: by product_kernel, gated_few_kernel or gated_rows_kernel
};

// Rows that gated_few_kernel takes (with four, its sums leave registers for half as many waves: 19 us, the matrix cores 16), and the vectors of
// columns of its workgroups: whole lines as soon as half of the compute units have some (2048 x [2 x 5504] in 172 workgroups of 64 bytes 11.0 us, in
// 86 of 128 bytes 12.1, in 344 of 32 bytes 19.4; 4096 x [2 x 11008] in 172 of 128 bytes 38.6 (4.7 TB/s), in 344 of 64 bytes 54).
constexpr int64_t kFewRows = 2;
int few_vectors(const GatedArgs &g) { return ceil_div(g.F, 16 / (int64_t)elem_bytes(g.dtype)) >= 4 * kCus ? 8 : 4; }

Layout forward_layout(const GatedArgs &g) {
  Layout l;
  l.plan = plan_product(g.M, g.F, g.D, g.dtype, true);
  const size_t e = (size_t)elem_bytes(g.dtype);
  if (g.D > 0 && !in_place(g.X, g.dtype, g.ldx, g.D)) l.a = align_up((size_t)g.M * (size_t)padded(g.D, g.dtype) * e, 256);
  if (g.D > 0 && !in_place(g.W, g.dtype, g.ldw, g.F)) l.b = align_up((size_t)g.D * 2 * (size_t)padded(g.F, g.dtype) * e, 256);
  // Few rows by one launch that reads W once and copies nothing, where a compute unit's share of W, which it reads at 36 GB/s, is not so long
  // that more of them sharing the contraction are faster.  Microseconds by tiles, of gated_few_kernel with one row and two, of gated_rows_kernel:
  // 2048 x [2 x 5504] 15.4, 10.9, 13.2, 10.7; 1024 x [2 x 1024] 8.8, 5.9, 8.2, 5.8; 4096 x [2 x 11008] 41, 38.6, 41, 51; 4096 x [2 x 4096] 18.8, 21.7, 24, 22;
  // 8192 x [2 x 1024] 12, 34, 37, 32; rows that are no whole vectors, 2048 x [2 x 5503] 31, 12.8, 14.6, 21.3; 4000 x [2 x 1500] 11, 18.7, 21.6, 29; binary32,
  // 2048 x [2 x 5504] 24.6, 20.5, 21.3, 11008 x [2 x 2048] 39, 84, 89.
  const double bytes = 2.0 * (double)g.D * (double)g.F * (double)e;
  double best = std::max(l.plan.us, 4.0 + bytes / 4.7e6) + (l.b != 0 ? 3.0 + 2.0 * (double)l.b / 5e6 : 0.0);
  auto consider = [&](decltype(l.by) by, int64_t columns, double per_mb) {       // columns of G of a workgroup
    const double share = (double)ceil_div(ceil_div(g.F, columns), (int64_t)kCus) * (double)g.D * (double)(2 * columns) * (double)e;
    const double us = 4.9 + std::max(share / 1e6 * per_mb, bytes / 4.7e6 - 4.9) + (by == Layout::kFew && g.M > 1 ? 2.4 : 0.0);
    if (us > best) return;
    best = us;
    l.by = by;
  };
  if (g.D > 0 && g.M <= kFewRows && g.F >= 16 / (int64_t)e) consider(Layout::kFew, few_vectors(g) * 16 / (int64_t)e, 28.0);
  const bool vectors = (uintptr_t)g.W % 16 == 0 && g.ldw % 8 == 0 && g.F % 8 == 0;
  if (g.dtype == BSR_BF16 && g.M <= 32 && (g.D >= 128 || l.b != 0) && ceil_div(g.F, (int64_t)32) <= kCus)
    consider(Layout::kRows, 32, (vectors ? 26.0 : 54.0) * (1.0 + (double)g.M / 64.0));
  if (l.by != Layout::kTiles) {
    l.a = l.b = 0;
    return l;
  }
  l.partial = partial_bytes(l.plan, g.M, g.F, true);
  l.all = l.a + l.b + l.partial;
  return l;
}

// Elements between packed rows of `n`: whole lines.
int64_t lines(int64_t n, int dtype) {
  const int64_t le = 128 / elem_bytes(dtype);
  return ceil_div(n, le) * le;
}

Layout backward_layout(const GatedArgs &g, const void *dGU, int64_t lddgu) {
  Layout l;
  l.plan = plan_product(g.M, g.D, 2 * g.F, g.dtype, false);
  const size_t e = (size_t)elem_bytes(g.dtype);
  const int64_t pitch = lines(2 * g.F, g.dtype);
  const size_t a = align_up((size_t)g.M * (size_t)pitch * e, 256), b = align_up((size_t)g.D * (size_t)pitch * e, 256);
  // Both operands' rows lie along the contraction and are read a line at a time.  Rows that are no whole lines make that two lines, which costs
  // about a fifth of the product for each operand (4096 x 2048 x [2 x 4096]: 134 us, 159 with such a dGU, 179 with such a W too): there a
  // copy in whole lines pays, written beside dGU, or read and written beside the slopes.  (Not in small products, which wait for other
  // things: 1000 x 1000 x [2 x 1000] 20 us, copied 23.)
  auto crooked = [&](const void *p, int64_t ld) { return g.dtype == BSR_BF16 && ((uintptr_t)p % 128 != 0 || ld * (int64_t)e % 128 != 0); };
  auto pays = [&](double bytes) { return 0.2 * (l.plan.us - 12.0) > bytes / 5e6; };
  if (g.F == 0) return l;                            // (zeros: nothing is read or added up)
  if (!in_place(dGU, g.dtype, lddgu, 2 * g.F) || (crooked(dGU, lddgu) && pays((double)a))) l.a = a;
  if (!in_place(g.W, g.dtype, g.ldw, 2 * g.F) || (crooked(g.W, g.ldw) && pays(2.0 * (double)b))) l.b = b;
  l.partial = partial_bytes(l.plan, g.M, g.D, false);
  l.all = l.a + l.b + l.partial;
  return l;
}

template <typename T>
void run_few(const GatedArgs &g, void *H, int64_t ldh, void *GU, int64_t ldgu, hipStream_t s) {
  const int64_t vecs = ceil_div(g.F, (int64_t)kVec<T>);
  auto go = [&](auto mr, auto v) {
    constexpr int MR = decltype(mr)::value, V = decltype(v)::value;
    const int64_t groups = ceil_div(vecs, (int64_t)V);
    gated_few_kernel<T, MR, V><<<dim3((uint32_t)(ceil_div(groups, (int64_t)8) * 8)), kFewThreads, 0, s>>>(
        g.act, static_cast<const T *>(g.X), (int)g.M, g.D, g.ldx, static_cast<const T *>(g.W), g.F, g.ldw, static_cast<T *>(H), ldh,
        static_cast<T *>(GU), ldgu, (int)groups);
  };
  auto rows = [&](auto v) {
    if (g.M == 1) go(std::integral_constant<int, 1>(), v);
    else go(std::integral_constant<int, 2>(), v);
  };
  if (few_vectors(g) == 8) rows(std::integral_constant<int, 8>());
  else rows(std::integral_constant<int, 4>());
}

template <typename T>
int forward(const GatedArgs &g, void *H, int64_t ldh, void *GU, int64_t ldgu, void *ws, hipStream_t s) {
  const Layout l = forward_layout(g);
  if (l.by == Layout::kFew) {
    run_few<T>(g, H, ldh, GU, ldgu, s);
    return check_launch();
  }
  if (l.by == Layout::kRows) return launch_gated_rows_bf16(g, H, ldh, GU, ldgu, s);
  uint8_t *const at = static_cast<uint8_t *>(ws);
  ProductArgs a = {};
  a.A = g.X;
  a.lda = g.ldx;
  a.B = g.W;
  a.ldb = g.ldw;
  a.up = g.F;
  a.cols = 2 * g.F;
  a.M = g.M;
  a.N = g.F;
  a.K = g.D;
  PackList jobs = {};
  int n = 0;
  auto add = [&](const void *src, int64_t rows, int64_t ld, int64_t from, int64_t cols, void *dst, int64_t pitch, int64_t to, int64_t pad) {
    jobs.it[n] = {src, rows, ld, from, cols, dst, pitch, to, pad};
    jobs.begin[n + 1] = jobs.begin[n] + blocks_for(rows * pad / kVec<T>);
    ++n;
  };
  if (l.a != 0) {
    a.A = at;
    a.lda = padded(g.D, g.dtype);
    add(g.X, g.M, g.ldx, 0, g.D, at, a.lda, 0, a.lda);
  }
  if (l.b != 0) {
    a.B = at + l.a;
    a.up = padded(g.F, g.dtype);
    a.ldb = a.cols = 2 * a.up;
    for (int i = 0; i < 2; ++i) add(g.W, g.D, g.ldw, i * g.F, g.F, at + l.a, a.ldb, i * a.up, a.up);
  }
  if (n > 0) {
    const int32_t blocks = jobs.begin[n];
    for (int i = n; i < kPackJobs; ++i) jobs.begin[i] = jobs.begin[i + 1] = blocks;
    pack_kernel<T><<<dim3((uint32_t)blocks), 256, 0, s>>>(jobs);
    if (const int rc = check_launch(); rc != BSR_OK) return rc;
  }
  a.out = H;
  a.ldo = ldh;
  a.gu = GU;
  a.ldgu = ldgu;
  a.partial = reinterpret_cast<float *>(at + l.a + l.b);
  a.act = g.act;
  return product_of<T>(l.plan, a, true, s);
}

template <typename T>
int backward(const GatedArgs &g, const void *GU, int64_t ldgu, const void *dH, int64_t lddh, void *dGU, int64_t lddgu, void *dX,
             int64_t lddx, void *ws, hipStream_t s) {
  const bool product = dX != nullptr && g.D > 0;
  const Layout l = product ? backward_layout(g, dGU, lddgu) : Layout();
  uint8_t *const at = static_cast<uint8_t *>(ws);
  const int64_t pitch = lines(2 * g.F, g.dtype);
  T *const also = l.a != 0 ? reinterpret_cast<T *>(at) : nullptr;
  PackJob job = {};
  int32_t packers = 0;
  if (l.b != 0) {
    job = {g.W, g.D, g.ldw, 0, 2 * g.F, at + l.a, pitch, 0, pitch};
    packers = std::min(blocks_for(g.D * pitch / kVec<T>), 4096);
  }
  if (g.F > 0) {
    const int32_t blocks = blocks_for(g.M * ceil_div(g.F, (int64_t)kVec<T>));
    auto go = [&](auto act, auto stream) {
      gated_slope_kernel<T, kVec<T>, decltype(act)::value, decltype(stream)::value><<<dim3((uint32_t)(blocks + packers)), 256, 0, s>>>(
          static_cast<const T *>(GU), g.M, g.F, ldgu, static_cast<const T *>(dH), lddh, static_cast<T *>(dGU), lddgu, also, pitch, blocks, job);
    };
    const bool stream = g.F * (int64_t)sizeof(T) % 128 == 0 && stream_rows(GU, g.M, 2 * g.F, ldgu, g.dtype, kStream) &&
                        stream_rows(dH, g.M, g.F, lddh, g.dtype, 0);
    with_act(g.act, [&](auto act) { stream ? go(act, std::true_type()) : go(act, std::false_type()); });
    if (const int rc = check_launch(); rc != BSR_OK) return rc;
  }
  if (!product) return BSR_OK;
  // The operand is the dGU that was stored, in bfloat16 rounded: the matrix instructions take no wider one, and the weights' gradient takes the same.
  // (Against binary64 dX is off by 0.235 % of its norm, of which its own rounding makes 0.166 %; both halves of unrounded slopes would be twice the product.)
  ProductArgs a = {};
  a.A = also != nullptr ? also : dGU;
  a.lda = also != nullptr ? pitch : lddgu;
  a.B = l.b != 0 ? job.dst : g.W;
  a.ldb = l.b != 0 ? pitch : g.ldw;
  a.M = g.M;
  a.N = g.D;
  a.K = l.a != 0 && l.b != 0 ? padded(2 * g.F, g.dtype) : 2 * g.F;      // (both are zeros behind their last column)
  a.out = dX;
  a.ldo = lddx;
  a.partial = reinterpret_cast<float *>(at + l.a + l.b);
  return product_of<T>(l.plan, a, false, s);
}

}  // namespace

size_t gated_ff_ws_bytes(const GatedArgs &a) { return forward_layout(a).all; }

int launch_gated_ff(const GatedArgs &a, void *H, int64_t ldh, void *GU, int64_t ldgu, void *ws, hipStream_t s) {
  return a.dtype == BSR_F32 ? forward<float>(a, H, ldh, GU, ldgu, ws, s) : forward<uint16_t>(a, H, ldh, GU, ldgu, ws, s);
}

size_t gated_ff_grad_ws_bytes(const GatedArgs &a, const void *dGU, int64_t lddgu) { return backward_layout(a, dGU, lddgu).all; }

int launch_gated_ff_grad(const GatedArgs &a, const void *GU, int64_t ldgu, const void *dH, int64_t lddh, void *dGU, int64_t lddgu,
                         void *dX, int64_t lddx, void *ws, hipStream_t s) {
  return a.dtype == BSR_F32 ? backward<float>(a, GU, ldgu, dH, lddh, dGU, lddgu, dX, lddx, ws, s)
                            : backward<uint16_t>(a, GU, ldgu, dH, lddh, dGU, lddgu, dX, lddx, ws, s);
}

}  // namespace bsr
