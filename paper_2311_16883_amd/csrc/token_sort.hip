// Stable sorts by key: entries by expert, positions by token.
//
// A counting sort of up to kMaxBins values, in two launches: every workgroup counts the values of its stretch of entries
// (count_kernel); then every workgroup adds up the counts of all, which says where the entries of a value start in the whole
// and where its own among them, and moves its entries there in order (place_kernel).  Tokens, which have too many values for one such
// pass, take one per digit, lowest first.  One stretch of entries needs no counts of others, and one launch per pass.  Up to kOneSort
// tokens take one launch in which every entry is compared with all others.
//
// Latency bound: a few bytes per entry.  [25088 x 4] choices of 64 experts 4.8 + 7.4 us, 33 x 2 3.7 (one launch), 2999 tokens of 10007 6.8
// (one launch, with 16 MB of dE cleared beside it).  Order within a workgroup: its waves own consecutive parts of the stretch, a wave takes 64
// entries at a time and finds, for every lane, the lanes before it with the same value from one ballot per bit of the value.
// No atomic decides an order (they only count), so the result is the stable one whatever the timing.
#include "token_step.h"

namespace bsr {

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxBins = 1025;                 // kMaxExperts and the dropped entries; digits of up to 10 bits
constexpr int kDigitBits = 10;
constexpr int kFewSteps = 4, kManySteps = 16;  // times 64 entries that a wave takes
// Workgroups from which each takes kManySteps, as each reads the counts of all ([1048576 x 4] choices of 256 experts, 32 columns, 216 us,
// 444 with kFewSteps; but [25088 x 4] of 64 17 with kFewSteps and 27.5 with kManySteps).  That reading grows with the square of the entries,
// and from millions of them on it is most of the time.
constexpr int kManyBlocks = 256;
// Elements that a workgroup clears, or more where that takes more than kClearBlocks workgroups.  Past the caches one store per lane:
// [65536 x 1024] bf16 into 65536 rows 98.8 us with kClear, 91.9 so, [30000 x 2048] into 100000 198 and 180, [8000 x 1024] into 32768 42.8
// and 35.7; through the caches [500 x 512] into 32768 18.4 and 19.1.
constexpr int64_t kClear = 32768, kClearBlocks = int64_t(1) << 21;

enum Source { kFromI32, kFromI64, kFromPairs };

// What a pass sorts: entry i has a key, of which the pass goes by (key >> shift) & mask.
struct Keys {
  const void *p;
  int64_t n;
  uint32_t limit;            // the key of indices outside [0, limit)
  int shift;
  uint32_t mask;
  int bins, bits;            // values that (key >> shift) & mask can have, and their bits
};

template <Source S>
__device__ __forceinline__ uint2 load_entry(const Keys &k, int64_t i) {
  if constexpr (S == kFromPairs) return static_cast<const uint2 *>(k.p)[i];
  const int64_t v = S == kFromI64 ? load_index<int64_t>(k.p, i) : load_index<int32_t>(k.p, i);
  return uint2{v >= 0 && v < (int64_t)k.limit ? (uint32_t)v : k.limit, (uint32_t)i};
}
__device__ __forceinline__ uint32_t digit_of(const Keys &k, uint32_t key) { return (key >> k.shift) & k.mask; }

// +0.0 over one workgroup's part of a matrix.
__device__ __forceinline__ void clear_part(const ClearJob &c, int64_t part) {
  if (c.ld == c.cols || c.rows == 1) {
    const int64_t total = c.rows * c.cols, lo = part * c.per;
    const int64_t hi = lo + c.per < total ? lo + c.per : total;
    for (int64_t i = lo + 4 * threadIdx.x; i < hi; i += 4 * (int)blockDim.x) {
      if (i + 4 <= hi) {
        if (c.stream) __builtin_nontemporal_store(Words4{0, 0, 0, 0}, reinterpret_cast<Words4 *>(c.p + i));
        else reinterpret_cast<Any16 *>(c.p + i)->w = Words4{0, 0, 0, 0};
      } else {
        for (int64_t j = i; j < hi; ++j) c.p[j] = 0.0f;
      }
    }
    return;
  }
  const int64_t per = c.per / c.cols > 0 ? c.per / c.cols : 1;
  for (int64_t r = part * per; r < (part + 1) * per && r < c.rows; ++r)
    for (int64_t j = threadIdx.x; j < c.cols; j += blockDim.x) c.p[r * c.ld + j] = 0.0f;
}

// counts[block][bin]
template <Source S, int STEPS>
__global__ __launch_bounds__(kThreads) void count_kernel(Keys k, uint32_t *__restrict__ counts, int blocks, ClearJob clear,
                                                         unsigned part) {
  __shared__ uint32_t bin[kMaxBins];
  const int t = threadIdx.x;
  if ((int)blockIdx.x >= blocks) {
    clear_part(clear, (int64_t)part + blockIdx.x - blocks);
    return;
  }
  for (int b = t; b < k.bins; b += kThreads) bin[b] = 0;
  __syncthreads();
  const int64_t per = (int64_t)STEPS * kThreads, lo = blockIdx.x * per;
  const int64_t hi = lo + per < k.n ? lo + per : k.n;
  for (int64_t i = lo + t; i < hi; i += kThreads) atomicAdd(&bin[digit_of(k, load_entry<S>(k, i).x)], 1u);
  __syncthreads();
  for (int b = t; b < k.bins; b += kThreads) counts[(int64_t)blockIdx.x * k.bins + b] = bin[b];
}

// Where a pass puts its entries.
struct Places {
  uint2 *pairs;                                // (key, position) in order; or, for experts:
  int32_t *offsets, *counts, *order, *slots;
  int64_t rows, align, experts;
};

// a[i] -> sum of a[0 .. i) over the whole workgroup of WAVES waves; `sums` is shared, one number per wave.
template <int WAVES>
__device__ __forceinline__ void scan_bins(uint32_t *a, int n, uint32_t *sums) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, threads = WAVES * 64;
  const int per = (n + threads - 1) / threads, lo = t * per, hi = lo + per < n ? lo + per : n;
  uint32_t sum = 0;
  for (int i = lo; i < hi; ++i) sum += a[i];
  uint32_t before = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(before, d, 64);
    if (lane >= d) before += o;
  }
  if (lane == 63) sums[w] = before;
  __syncthreads();
  before -= sum;
  for (int o = 0; o < w; ++o) before += sums[o];
  for (int i = lo; i < hi; ++i) {
    const uint32_t v = a[i];
    a[i] = before;
    before += v;
  }
  __syncthreads();
}

// The entry's number among its wave's entries of the same value so far (`count`: how many there were of every value), by the wave as
// a whole; lanes with in == false have no entry.  count goes on.
__device__ __forceinline__ uint32_t rank_entry(uint32_t *count, uint32_t d, int bits, bool in, int lane) {
  uint64_t same = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const bool one = (d >> b) & 1u;
    const uint64_t ones = __ballot(one);
    same &= one ? ones : ~ones;
  }
  uint32_t rank = 0;
  if (in) rank = count[d] + (uint32_t)__builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
  // (the wave's reads above come before the write, and the write before the next round's reads: one wave's LDS accesses are
  // executed in order; the fences keep the compiler to that)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (in && (same >> lane) >> 1 == 0) count[d] += (uint32_t)__builtin_popcountll(same);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  return rank;
}

// STEPS times 64 entries per wave.
template <Source S, bool EXPERTS, int STEPS>
__global__ __launch_bounds__(kThreads) void place_kernel(Keys k, const uint32_t *__restrict__ counts, int blocks, Places out,
                                                         ClearJob clear, unsigned part) {
  __shared__ uint32_t next[kWaves][kMaxBins];  // a wave's entries of a value, then where they start among the workgroup's and all before it
  __shared__ uint32_t start[kMaxBins];         // of a value's entries in the whole
  __shared__ uint32_t total[EXPERTS ? kMaxBins : 1];
  __shared__ uint32_t sums[kWaves];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  if ((int)blockIdx.x >= blocks) {
    clear_part(clear, (int64_t)part + blockIdx.x - blocks);
    return;
  }
  const int64_t lo = ((int64_t)blockIdx.x * kWaves + w) * STEPS * 64;
  uint2 e[STEPS];
  if (k.n > 0) {
#pragma unroll
    for (int q = 0; q < STEPS; ++q) e[q] = load_entry<S>(k, lo + q * 64 + lane < k.n ? lo + q * 64 + lane : 0);
  }
  for (int b = lane; b < k.bins; b += 64) next[w][b] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  uint32_t rank[STEPS];
#pragma unroll
  for (int q = 0; q < STEPS; ++q) {
    rank[q] = 0;
    if (lo + q * 64 < k.n) rank[q] = rank_entry(next[w], digit_of(k, e[q].x), k.bits, lo + q * 64 + lane < k.n, lane);
  }
  __syncthreads();
  // a value's entries in all workgroups, and in those before this one
  for (int b = t; b < k.bins; b += kThreads) {
    uint32_t all = 0, before = 0;
    if (blocks > 1) {
#pragma unroll 8
      for (int c = 0; c < blocks; ++c) {
        const uint32_t n = counts[(int64_t)c * k.bins + b];
        before += c < (int)blockIdx.x ? n : 0;
        all += n;
      }
    }
    uint32_t here = before;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const uint32_t n = next[v][b];
      next[v][b] = here;
      here += n;
    }
    if (blocks == 1) all = here;
    if constexpr (EXPERTS) {
      total[b] = all;
      all = (uint32_t)((all + out.align - 1) / out.align * out.align);
    }
    start[b] = all;
  }
  __syncthreads();
  scan_bins<kWaves>(start, k.bins, sums);
#pragma unroll
  for (int q = 0; q < STEPS; ++q) {
    const int64_t i = lo + q * 64 + lane;
    if (i >= k.n) continue;
    const uint32_t d = digit_of(k, e[q].x), place = start[d] + next[w][d] + rank[q];
    if constexpr (EXPERTS) {
      const bool kept = (int64_t)d < out.experts;
      out.slots[i] = kept ? (int32_t)place : -1;
      if (kept && (int64_t)place < out.rows) out.order[place] = (int32_t)i;
    } else {
      out.pairs[place] = e[q];
    }
  }
  if constexpr (EXPERTS) {
    // the last value stands for dropped entries: its start is the end of the last segment
    if (blockIdx.x == 0) {
      for (int x = t; x <= out.experts; x += kThreads) {
        out.offsets[x] = (int32_t)start[x];
        if (x < out.experts) out.counts[x] = (int32_t)total[x];
      }
    }
    for (int64_t x = blockIdx.x * kWaves + w; x < out.experts; x += (int64_t)blocks * kWaves)
      for (int64_t s = (int64_t)start[x] + total[x] + lane; s < start[x + 1]; s += 64) out.order[s] = -1;
    for (int64_t s = (int64_t)start[out.experts] + blockIdx.x * kThreads + t; s < out.rows; s += (int64_t)blocks * kThreads)
      out.order[s] = -1;
  }
}

// Up to kOneSort positions sorted in one launch: the place of an entry is the number of those before it in the order, with smaller
// keys or with its own and smaller positions, so each workgroup finds kOneEntries places by comparing with all keys, which it has in
// LDS.  Further workgroups clear.  Bound by the comparisons, T * T of two operations: [2999 x 411] binary32 into 10007 rows 16.5 us in all, 20
// with all digits sorted by one workgroup, [8000 x 64] bf16 into 2000 22.7 and 27.9; 12000 positions 34.5, with two launches per digit 34.4.
// 64 entries to a workgroup 18.5 and 28.2, 16 of them 15.8 and 22.0, but these leave less room to clear ([8000 x 1024] into 32768 40
// instead of 35.7).
constexpr int kOneSort = 8192, kOneEntries = 32, kOneParts = kThreads / kOneEntries, kOneLoads = 4;
template <Source S>
__global__ __launch_bounds__(kThreads) void sort_one_kernel(Keys k, uint2 *__restrict__ sorted, ClearJob clear, int blocks) {
  __shared__ alignas(16) uint32_t keys[kOneSort];
  __shared__ uint32_t before[kOneParts][kOneEntries];
  const int t = threadIdx.x, n = (int)k.n;
  if ((int)blockIdx.x >= blocks) {
    clear_part(clear, (int64_t)blockIdx.x - blocks);
    return;
  }
  // whole entries of kOneEntries, those behind the last greater than any key
  const int all = (n + kOneEntries - 1) / kOneEntries * kOneEntries;
  for (int i0 = t; i0 < all; i0 += kOneLoads * kThreads) {
    uint32_t key[kOneLoads];
#pragma unroll
    for (int u = 0; u < kOneLoads; ++u) {
      const int i = i0 + u * kThreads;
      key[u] = i < n ? load_entry<S>(k, i).x : 0xFFFFFFFFu;
    }
#pragma unroll
    for (int u = 0; u < kOneLoads; ++u)
      if (i0 + u * kThreads < all) keys[i0 + u * kThreads] = key[u];
  }
  __syncthreads();
  // Every lane compares one entry with its part of the keys, four at a time: keys before the workgroup's entries count up to equal
  // ones, those behind only if they are smaller, its own by their positions.
  const int first = blockIdx.x * kOneEntries, i = first + (t & (kOneEntries - 1)), part = t / kOneEntries;
  const uint32_t mine = keys[i];
  const Words4 *fours = reinterpret_cast<const Words4 *>(keys);
  uint32_t count = 0;
#pragma unroll 4
  for (int g = part; g < first / 4; g += kOneParts) {
    const Words4 w = fours[g];
#pragma unroll
    for (int q = 0; q < 4; ++q) count += w[q] < mine + 1;
  }
#pragma unroll 4
  for (int g = (first + kOneEntries) / 4 + part; g < all / 4; g += kOneParts) {
    const Words4 w = fours[g];
#pragma unroll
    for (int q = 0; q < 4; ++q) count += w[q] < mine;
  }
  for (int g = first / 4 + part; g < (first + kOneEntries) / 4; g += kOneParts) {
    const Words4 w = fours[g];
#pragma unroll
    for (int q = 0; q < 4; ++q) count += w[q] < mine || (w[q] == mine && g * 4 + q < i);
  }
  before[part][t & (kOneEntries - 1)] = count;
  __syncthreads();
  if (t < kOneEntries && i < n) {
    uint32_t place = 0;
#pragma unroll
    for (int s = 0; s < kOneParts; ++s) place += before[s][t];
    sorted[place] = uint2{mine, (uint32_t)i};
  }
}

int bit_length(uint32_t v) { return v == 0 ? 0 : 32 - __builtin_clz(v); }

// Stretches of n entries.
int steps_of(int64_t n) { return n > (int64_t)kManyBlocks * kFewSteps * kThreads ? kManySteps : kFewSteps; }
int blocks_of(int64_t n) { return n > 0 ? (int)ceil_div(n, (int64_t)steps_of(n) * kThreads) : 1; }

size_t counts_bytes(int64_t n, int bins) {
  const int blocks = blocks_of(n);
  return blocks > 1 ? align_up((size_t)blocks * bins * sizeof(uint32_t), 256) : 0;
}

int64_t clear_blocks(const ClearJob &c) {
  if (c.p == nullptr) return 0;
  if (c.ld == c.cols || c.rows == 1) return ceil_div(c.rows * c.cols, c.per);
  const int64_t per = c.per / c.cols > 0 ? c.per / c.cols : 1;
  return ceil_div(c.rows, per);
}

// The job with its workgroups' shares.
ClearJob shared(ClearJob c) {
  c.per = c.stream ? 4 * kThreads : kClear;
  while (clear_blocks(c) > kClearBlocks) c.per *= 2;
  return c;
}

// What is to be cleared, handed out to the launches of a sort: each takes its share of the parts that are left.
struct Clearing {
  ClearJob job;
  unsigned parts, next = 0;
  explicit Clearing(const ClearJob &j) : job(shared(j)), parts((unsigned)clear_blocks(job)) {}
  // the share of a launch with `launches` more to come, in workgroups; *first: its first part
  unsigned share(int launches, unsigned *first) {
    *first = next;
    const unsigned n = (parts - next) / (unsigned)(launches + 1);
    const unsigned mine = launches == 0 ? parts - next : n;
    next += mine;
    return mine;
  }
};

// One pass, with `later` launches of the sort behind it.
template <Source S, bool EXPERTS, int STEPS>
int launch_pass_(const Keys &k, int blocks, uint32_t *counts, const Places &out, Clearing *clear, int later, hipStream_t s) {
  unsigned first, extra;
  if (blocks > 1) {
    extra = clear->share(later + 1, &first);
    hipLaunchKernelGGL((count_kernel<S, STEPS>), dim3(blocks + extra), dim3(kThreads), 0, s, k, counts, blocks, clear->job, first);
    const int rc = check_launch();
    if (rc != BSR_OK) return rc;
  }
  extra = clear->share(later, &first);
  hipLaunchKernelGGL((place_kernel<S, EXPERTS, STEPS>), dim3(blocks + extra), dim3(kThreads), 0, s, k, counts, blocks, out,
                     clear->job, first);
  return check_launch();
}

template <Source S, bool EXPERTS>
int launch_pass(const Keys &k, int blocks, uint32_t *counts, const Places &out, Clearing *clear, int later, hipStream_t s) {
  return steps_of(k.n) == kFewSteps ? launch_pass_<S, EXPERTS, kFewSteps>(k, blocks, counts, out, clear, later, s)
                                    : launch_pass_<S, EXPERTS, kManySteps>(k, blocks, counts, out, clear, later, s);
}

int digit_passes(int64_t V) { return V < 1 ? 1 : (bit_length((uint32_t)V) + kDigitBits - 1) / kDigitBits; }
int digit_bits(int64_t V) { return V < 1 ? 1 : (bit_length((uint32_t)V) + digit_passes(V) - 1) / digit_passes(V); }

}  // namespace

size_t expert_sort_ws_bytes(int64_t n, int64_t E) { return counts_bytes(n, (int)E + 1); }

int launch_expert_sort(const void *ids, int index_type, int64_t n, int64_t E, int64_t align, int32_t *offsets, int32_t *counts,
                       int32_t *order, int64_t rows, int32_t *slots, void *ws, hipStream_t s) {
  const Keys k = {ids, n, (uint32_t)E, 0, 0xFFFFFFFFu, (int)E + 1, bit_length((uint32_t)E)};
  const int blocks = blocks_of(n);
  const Places out = {nullptr, offsets, counts, order, slots, rows, align, E};
  Clearing none(ClearJob{nullptr, 0, 0, 0, false, 0});
  return index_type == BSR_I64 ? launch_pass<kFromI64, true>(k, blocks, static_cast<uint32_t *>(ws), out, &none, 0, s)
                               : launch_pass<kFromI32, true>(k, blocks, static_cast<uint32_t *>(ws), out, &none, 0, s);
}

size_t token_sort_ws_bytes(int64_t T, int64_t V) {
  const int buffers = digit_passes(V) > 1 ? 2 : 1;
  return buffers * align_up((size_t)T * sizeof(uint2), 256) + counts_bytes(T, 1 << digit_bits(V));
}

int launch_token_sort(const void *tokens, int index_type, int64_t T, int64_t V, const ClearJob &clear, void *ws,
                      const uint2 **sorted, hipStream_t s) {
  const int passes = digit_passes(V), bits = digit_bits(V);
  const size_t pairs_bytes = align_up((size_t)T * sizeof(uint2), 256);
  char *base = static_cast<char *>(ws);
  uint2 *buffer[2] = {reinterpret_cast<uint2 *>(base), reinterpret_cast<uint2 *>(base + (passes > 1 ? pairs_bytes : 0))};
  uint32_t *counts = reinterpret_cast<uint32_t *>(base + (passes > 1 ? 2 : 1) * pairs_bytes);
  if (T <= kOneSort) {
    const ClearJob job = shared(clear);
    const int blocks = (int)ceil_div(T, (int64_t)kOneEntries);
    const dim3 grid(blocks + (unsigned)clear_blocks(job));
    const Keys k = {tokens, T, (uint32_t)V, 0, 0, 0, 0};
    if (index_type == BSR_I64) hipLaunchKernelGGL((sort_one_kernel<kFromI64>), grid, dim3(kThreads), 0, s, k, buffer[0], job, blocks);
    else hipLaunchKernelGGL((sort_one_kernel<kFromI32>), grid, dim3(kThreads), 0, s, k, buffer[0], job, blocks);
    *sorted = buffer[0];
    return check_launch();
  }
  Clearing clearing(clear);
  for (int p = 0; p < passes; ++p) {
    const Keys k = {p == 0 ? tokens : buffer[(p - 1) & 1], T, (uint32_t)V, p * bits, (1u << bits) - 1u, 1 << bits, bits};
    const int blocks = blocks_of(T);
    Places out = {};
    out.pairs = buffer[p & 1];
    const int later = (passes - 1 - p) * 2;
    const int rc = p > 0 ? launch_pass<kFromPairs, false>(k, blocks, counts, out, &clearing, later, s)
                   : index_type == BSR_I64 ? launch_pass<kFromI64, false>(k, blocks, counts, out, &clearing, later, s)
                                           : launch_pass<kFromI32, false>(k, blocks, counts, out, &clearing, later, s);
    if (rc != BSR_OK) return rc;
  }
  *sorted = buffer[(passes - 1) & 1];
  return BSR_OK;
}

}  // namespace bsr
