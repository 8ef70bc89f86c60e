// Gradient of the token table: dE[v] (+)= scale * sum of the rows of dY whose token is v, positions ascending.
//
// The positions are sorted by token first (token_sort.hip; its launches also clear dE).  The sorted order is cut into windows of
// 4 to 32 positions (62 of billions), whatever tokens they hold: a wave takes 64 vectors of columns of one window, walks its positions
// with kAhead rows on their way, and keeps the sum of the current token's rows in registers.  A token whose positions all lie in one
// window is written to dE straight away; of one that reaches into others every window leaves a partial sum, and a
// second kernel adds these up window by window.  So the work per wave is the same however often a token occurs, and the order of
// every sum follows from the tokens alone.  Bound by memory: dY once, dE once, and the rows of dE that occur a second time, as these
// were cleared before it is known which do.
// [65536 x 1024] bf16 into 65536 rows 92 us: the sort's four launches clear 268 MB in 46 of them (5.8 TB/s), the windows read 134 MB and write
// the rows in 41, joining takes 7.  [2999 x 411] binary32 into 10007 15.8 us: three launches, each after the last, 7 + 5 + 5.
#include "token_step.h"

namespace bsr {

namespace {

constexpr int kAhead = 8;
// dY read past the caches, which then hold more of the dE that was just cleared ([65536 x 1024] bf16 into 65536 rows 96.5 -> 92.1 us,
// into 1000 54.2 -> 51.0, [30000 x 2048] into 100000 185 -> 182, into 32768 95.0 -> 91.5; but [65536 x 512] into 1000 rows 36 -> 38).
constexpr int64_t kStreamBytes = int64_t(96) << 20;
constexpr int kGroup = 4;                      // windows whose runs a workgroup of the second kernel joins
constexpr int kLong = 15;                      // windows of a run from which the waves share it
constexpr int kLeastWindow = 4, kMostWindow = 62;
// (waves for each window size: window_size)
constexpr int64_t kEnoughWaves = 2048, kEnoughLongRuns = 256, kOften = 32;
constexpr int kThreads = 256;

// The sum of a run of equal tokens, positions [first, last) of the sorted order (inside one window, [lo, hi)): to its row of dE,
// or to partial[2 * window] where the run goes on from the window before, to partial[2 * window + 1] where it only goes on
// into the next.
template <int VE>
__device__ __forceinline__ void put_sum(const float *sum, bool goes_on_before, bool goes_on_behind, float scale, float *row,
                                        float *partial, int64_t at, int skip, bool accumulate) {
  const bool whole = !goes_on_before && !goes_on_behind;
  float *dst = (whole ? row : partial) + at;
  const float by = whole ? scale : 1.0f;
  const bool add = whole && accumulate;
  if constexpr (VE % 4 == 0) {
    if (skip == 0) {
#pragma unroll
      for (int q = 0; q < VE; q += 4) {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = sum[q + i] * by;
        if (add) {
          const Words4 old = RowVec<float, 4>::load(dst + q);
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] += __uint_as_float(old[i]);
        }
        RowVec<float, 4>::store(dst + q, pack_row<float, 4>(f));
      }
      return;
    }
  }
#pragma unroll
  for (int q = 0; q < VE; ++q) {
    if (q < skip) continue;
    const float v = sum[q] * by;
    dst[q] = add ? dst[q] + v : v;
  }
}

template <typename T, int VE, bool STREAM>
__global__ __launch_bounds__(kThreads) void window_sum_kernel(const uint2 *__restrict__ sorted, int64_t n, uint32_t V,
                                                              const T *__restrict__ dY, int64_t D, int64_t lddy, float scale,
                                                              float *__restrict__ dE, int64_t ldde, int accumulate,
                                                              float *__restrict__ partial, int64_t slices, int size) {
  typedef RowVec<T, VE> R;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int64_t window = unit / slices, slice = unit - window * slices;
  const int64_t lo = window * size;
  if (lo >= n) return;
  const int count = (int)(n - lo < size ? n - lo : size);
  // lane l holds position lo - 1 + l of the sorted order: its neighbours tell where runs go on
  uint2 e = uint2{0xFFFFFFFFu, 0};
  if (lane <= count + 1 && lo - 1 + lane >= 0 && lo - 1 + lane < n) e = sorted[lo - 1 + lane];
  const uint32_t before = __builtin_amdgcn_readlane(e.x, 0), behind = __builtin_amdgcn_readlane(e.x, count + 1);
  const int64_t v = slice * 64 + lane, vecs = ceil_div(D, (int64_t)VE);
  const bool in = v < vecs;
  const int64_t at = vector_start(in ? v : 0, VE, D);
  const int skip = in ? (int)(v * VE - at) : VE;       // elements that belong to the vector before; all for a lane without columns
  float sum[VE];
#pragma unroll
  for (int q = 0; q < VE; ++q) sum[q] = 0.0f;
  float *head = partial + (2 * window) * D, *tail = head + D;
  uint32_t token = __builtin_amdgcn_readlane(e.x, 1);
  int first = 0;
  for (int i0 = 0; i0 < count && token < V; i0 += kAhead) {
    typename R::Raw x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + u < count ? i0 + u : count - 1;
      const uint32_t pos = __builtin_amdgcn_readlane(e.y, 1 + i);
      x[u] = load_once<T, VE, STREAM>(dY + (int64_t)pos * lddy + at);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + u;
      if (i >= count || token >= V) continue;
      const uint32_t next = __builtin_amdgcn_readlane(e.x, 2 + i);
#pragma unroll
      for (int q = 0; q < VE; ++q) sum[q] += R::elem(x[u], q);
      if (next != token || i == count - 1) {
        const bool b = first == 0 && before == token, f = i == count - 1 && behind == token;
        put_sum<VE>(sum, b, f, scale, dE + (int64_t)token * ldde, b ? head : tail, at, skip, accumulate != 0);
#pragma unroll
        for (int q = 0; q < VE; ++q) sum[q] = 0.0f;
        first = i + 1;
        token = next;
      }
    }
  }
}

// sum += the first sums (`partial`, 2 D apart) of `count` windows, in order.
template <int VE>
__device__ __forceinline__ void add_windows(const float *partial, int64_t count, int64_t D, float *sum) {
  typedef RowVec<float, VE> R;
  for (int64_t i0 = 0; i0 < count; i0 += kAhead) {
    typename R::Raw x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x[u] = R::load(partial + 2 * (i0 + u < count ? i0 + u : count - 1) * D);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int q = 0; q < VE; ++q) sum[q] = i0 + u < count ? sum[q] + R::elem(x[u], q) : sum[q];
  }
}

// dE[token] for the tokens that reach over several windows: one workgroup per kGroup windows and 64 vectors of columns takes the
// runs that start in them.  Its waves take the short runs in turn; the windows of a long one are shared out among them in four parts,
// whose sums are added in order.
template <int VE>
__global__ __launch_bounds__(kThreads) void join_kernel(const uint2 *__restrict__ sorted, int64_t n, uint32_t V, int64_t D,
                                                        float scale, float *__restrict__ dE, int64_t ldde, int accumulate,
                                                        const float *__restrict__ partial, int64_t windows, int64_t slices, int size) {
  constexpr int kWaves = kThreads / 64;
  typedef RowVec<float, VE> R;
  __shared__ float parts[kWaves][64 * VE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t group = blockIdx.x / slices, slice = blockIdx.x - group * slices;
  // lane l: whether a run starts in window l of the group and goes on behind it, and whose it is
  const int64_t mine = group * kGroup + lane, lo = mine * size, behind = lo + size;
  uint32_t token = V;
  if (lane < kGroup && behind < n) {
    const uint32_t last = sorted[behind - 1].x, next = sorted[behind].x, start = sorted[lo].x, before = lo > 0 ? sorted[lo - 1].x : V;
    if (last == next && !(start == last && before == last)) token = last;
  }
  uint64_t runs = __ballot(token < V);
  if (runs == 0) return;
  const int64_t v = slice * 64 + lane, vecs = ceil_div(D, (int64_t)VE);
  const bool in = v < vecs;
  const int64_t at = vector_start(in ? v : 0, VE, D);
  const int skip = in ? (int)(v * VE - at) : VE;
  // windows behind window w that a run of `tok` goes on into, up to `most` of them or a few more
  auto reach_of = [&](int64_t w, uint32_t tok, int64_t most) {
    int64_t reach = 0;
    while (reach < most) {
      const int64_t x = w + 1 + reach + lane;
      const uint64_t more = __ballot(x < windows && sorted[x < windows ? x * size : 0].x == tok);
      reach += more == ~uint64_t(0) ? 64 : __builtin_ctzll(~more);
      if (more != ~uint64_t(0)) break;
    }
    return reach;
  };
  uint64_t late = 0;
  for (int turn = 0; runs != 0; runs &= runs - 1, ++turn) {
    const int l = __builtin_ctzll(runs);
    const int64_t w = group * kGroup + l;
    const uint32_t tok = __builtin_amdgcn_readlane(token, l);
    // (a run is long for all waves or for none: whether the window kLong behind still begins with its token)
    if (w + 1 + kLong < windows && sorted[(w + 1 + kLong) * size].x == tok) {
      late |= uint64_t(1) << l;
      continue;
    }
    if (turn % kWaves != wave) continue;
    const int64_t reach = reach_of(w, tok, 64);
    float sum[VE];
    const typename R::Raw own = R::load(partial + (2 * w + 1) * D + at);
#pragma unroll
    for (int q = 0; q < VE; ++q) sum[q] = R::elem(own, q);
    add_windows<VE>(partial + 2 * (w + 1) * D + at, reach, D, sum);
    put_sum<VE>(sum, false, false, scale, dE + (int64_t)tok * ldde, nullptr, at, skip, accumulate != 0);
  }
  for (; late != 0; late &= late - 1) {
    const int l = __builtin_ctzll(late);
    const int64_t w = group * kGroup + l;
    const uint32_t tok = __builtin_amdgcn_readlane(token, l);
    const int64_t reach = reach_of(w, tok, windows), share = (reach + kWaves - 1) / kWaves;
    const int64_t from = wave * share < reach ? wave * share : reach, count = reach - from < share ? reach - from : share;
    float sum[VE];
#pragma unroll
    for (int q = 0; q < VE; ++q) sum[q] = 0.0f;
    if (wave == 0) {
      const typename R::Raw own = R::load(partial + (2 * w + 1) * D + at);
#pragma unroll
      for (int q = 0; q < VE; ++q) sum[q] = R::elem(own, q);
    }
    add_windows<VE>(partial + 2 * (w + 1 + from) * D + at, count, D, sum);
#pragma unroll
    for (int q = 0; q < VE; ++q) parts[wave][q * 64 + lane] = sum[q];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int q = 0; q < VE; ++q) {
        for (int o = 1; o < kWaves; ++o) sum[q] += parts[o][q * 64 + lane];
      }
      put_sum<VE>(sum, false, false, scale, dE + (int64_t)tok * ldde, nullptr, at, skip, accumulate != 0);
    }
    __syncthreads();
  }
}

// Positions of a window: 32, or fewer where that leaves too few waves (512 columns of a window each) to hide the loads' latency
// ([16384 x 768] bf16 into 32768 rows 43 us, 48 with 1024 waves; but [65536 x 512] into 1000 rows 36 and, with 8192 waves, 52).
// Where rows occur kOften times on the average, most windows leave partial sums, and fewer waves do ([8192 x 384] into 2 rows 50 -> 24,
// [16384 x 64] binary32 into 50 25 -> 21).  Where windows of 32 would be more than 2^31 lanes (a launch takes fewer than 2^32: 2^31 positions of
// up to 256 columns) they are as long as a wave's lanes hold beside the two neighbours.
int window_size(int64_t T, int64_t V, int64_t D) {
  if (ceil_div(T, (int64_t)32) * ceil_div(D, (int64_t)256) * 64 > (int64_t(1) << 31)) return kMostWindow;
  const int64_t enough = T / kOften >= V ? kEnoughLongRuns : kEnoughWaves;
  int size = 32;
  while (size > kLeastWindow && T > size / 2 && ceil_div(T, (int64_t)size) * ceil_div(D, (int64_t)512) < enough) size /= 2;
  return size;
}

size_t partial_bytes(int64_t T, int64_t V, int64_t D) {
  const int64_t windows = ceil_div(T, (int64_t)window_size(T, V, D));
  return windows > 1 ? align_up((size_t)windows * 2 * D * sizeof(float), 256) : 0;
}

}  // namespace

size_t embedding_grad_ws_bytes(int64_t T, int64_t V, int64_t D) { return token_sort_ws_bytes(T, V) + partial_bytes(T, V, D); }

int launch_embedding_grad(const void *tokens, int index_type, int64_t T, const void *dY, int dtype, int64_t D, int64_t lddy,
                          float scale, int64_t V, float *dE, int64_t ldde, int accumulate, void *ws, hipStream_t s) {
  // Cleared past the caches where many of the rows will be written again, and the caches are for those ([8192 x 1024] bf16 into 32768
  // rows 48.8 -> 38.7 us, [65536 x 1024] into 65536 105 -> 98; but [2048 x 1024] into 32768 28 -> 33, which the caches absorb).
  const bool stream = 8 * T >= V && (uintptr_t)dE % 16 == 0 && ldde == D;
  const ClearJob clear = {accumulate ? nullptr : dE, V, D, ldde, stream, 0};
  float *partial = static_cast<float *>(ws);
  const uint2 *sorted = nullptr;
  int rc = launch_token_sort(tokens, index_type, T, V, clear, static_cast<char *>(ws) + partial_bytes(T, V, D), &sorted, s);
  if (rc != BSR_OK || T == 0) return rc;
  const int size = window_size(T, V, D);
  const int64_t windows = ceil_div(T, (int64_t)size);
  const bool read = stream_rows(dY, T, D, lddy, dtype, kStreamBytes);
#define BSR_CALL_(TY, VE, STREAM)                                                                                              \
  const int64_t slices = ceil_div(ceil_div(D, (int64_t)VE), (int64_t)64);                                                      \
  hipLaunchKernelGGL((window_sum_kernel<TY, VE, STREAM>), dim3((unsigned)ceil_div(windows * slices, (int64_t)(kThreads / 64))),         \
                     dim3(kThreads), 0, s, sorted, T, (uint32_t)V, static_cast<const TY *>(dY), D, lddy, scale, dE, ldde,      \
                     accumulate, partial, slices, size)
#define BSR_CALL(TY, VE) \
  if (read) { BSR_CALL_(TY, VE, true); } else { BSR_CALL_(TY, VE, false); }
  if (dtype == BSR_F32) {
    if (D >= 4) { BSR_CALL(float, 4) } else { BSR_CALL_(float, 1, false); }
  } else {
    if (D >= 8) { BSR_CALL(uint16_t, 8) } else { BSR_CALL_(uint16_t, 1, false); }
  }
#undef BSR_CALL
#undef BSR_CALL_
  rc = check_launch();
  if (rc != BSR_OK || windows == 1) return rc;
#define BSR_JOIN(VE)                                                                                                           \
  const int64_t slices = ceil_div(ceil_div(D, (int64_t)VE), (int64_t)64);                                                      \
  hipLaunchKernelGGL((join_kernel<VE>), dim3((unsigned)(ceil_div(windows, (int64_t)kGroup) * slices)), dim3(kThreads),         \
                     0, s, sorted, T, (uint32_t)V, D, scale, dE, ldde, accumulate, partial, windows, slices, size)
  if (D >= 4) { BSR_JOIN(4); } else { BSR_JOIN(1); }
#undef BSR_JOIN
  return check_launch();
}

}  // namespace bsr
