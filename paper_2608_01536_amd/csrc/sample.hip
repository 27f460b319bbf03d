// celty_sample (include/celty_decode.h) for gfx950: one token per row of
// logits under temperature, top-k, top-p and min-p, from given noise.
//
// The kept tokens are a prefix of the order (logit falling, index rising), cut
// by top-k and top-p, less those that min-p drops; the result is the best of
// them by z - log(noise), a maximum, so what has to be found is where the cuts
// lie, not the order.  Three launches share a row out to slices of it:
//
//   top     the largest (logit, lowest index) of each slice; clears the row's
//           words for the other two;
//   bins    counts and weights of the row by bins of the distance from the
//           largest logit, 64 to a factor of two, as integers: weights are
//           multiples of 2^-38 of the largest, so sums are exact in 64 bits and do
//           not depend on their order;
//   finish  every slice finds the bins that the cuts fall into from the row's
//           sums; tokens above them race at once, those within are listed, and
//           the slice that arrives last orders the list (some dozens of
//           tokens), cuts it exactly and lets the rest race.
//
// A row whose cut bins hold more tokens than the list does (4096) is cut by the
// last slice alone, with bins of the logits' bits over the row: 0.2 ms at 32000
// logits, 0.6 at 100000.  Those are rows with thousands of equal logits at a cut,
// as 16-bit ones of large magnitude have, or whose top-k (of thousands) cuts a
// dense part far below the largest.
// A row of 150000 logits of one normal distribution, of any mean and any spread
// from 2^-6 to 100, has fewer than 4096 in every bin.
//
// Bound for one row by the three launches and the round trips within them (the
// last: bins, listing, ticket, list), 21 us at 32000 logits and 25 at 131072; for
// many by the weights' arithmetic and the bins' atomics, 55 us for 64 rows of
// 100277 (12.8 MB).  Greedy rows take 5 us, 9 for those 64; rows without top-k
// and top-p 12 and 47.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "celty_decode.h"
#include "common.h"
#include "tensor.h"

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 8 * kThreads;    // logits a workgroup takes at once
constexpr int kMaxSlices = 64;
constexpr int kList = 4096;             // tokens of the cut bins that a cut is found among
constexpr int kBins = 16 * 64;          // distances from the largest logit, from 2^-6 (below: one bin) to 2^10 (above: one bin)
constexpr int kRowsAtOnce = 1024;       // rows that the workspace has room for
constexpr int kWeightBits = 38;         // the largest logit's weight is 2^38; 2^24 of them fit in 64 bits

// A row's words in the workspace.
struct alignas(256) RowWork {
  uint64_t list[kList];       // key, complement of the index
  uint64_t mass[kBins];
  uint32_t count[kBins];
  uint64_t top[kMaxSlices];   // per slice: key, then the complement of the index
  uint64_t best;              // of the race: score key, complement of the index
  uint64_t total;             // weight of the row
  uint32_t listed, arrived;
};

struct SampleArgs {
  const void* logits;
  const float* noise;
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* tokens;
  RowWork* work;
  int64_t ldl, ldn;
  int V, slices, per;   // per: logits of a slice of the first two launches, a multiple of kChunk
  int finish_per;       // and of the third
};

// Unsigned integers in the order of the logits; 0 for NaN and -infinity, which
// are never chosen.
__device__ __forceinline__ uint32_t key_of(float l) {
  if (!(l > -INFINITY)) return 0u;
  const uint32_t b = __float_as_uint(l + 0.0f);   // -0 and +0 are equal
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key);
}

__device__ __forceinline__ uint64_t token_word(uint32_t key, int i) {
  return static_cast<uint64_t>(key) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(i));
}
__device__ __forceinline__ int index_of(uint64_t word) {
  return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(word));
}

// The slices of a row run on dies whose L2 caches are not shared: words that
// they pass to each other within a launch go past them.
__device__ __forceinline__ void put(uint64_t* p, uint64_t v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename V>
__device__ __forceinline__ V get(const V* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <typename V>
__device__ __forceinline__ V wave_max(V v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const V w = __shfl_xor(v, o, kWave);
    v = w > v ? w : v;
  }
  return v;
}

// A thread's eight logits from p[at], as keys; 0 past n.
template <typename T>
__device__ __forceinline__ void load_keys8(const T* p, int at, int n, uint32_t (&key)[8]) {
  float x[8];
  load8(p + at, n - at, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) key[i] = at + i < n ? key_of(x[i]) : 0u;
}

// What a row's filters come to, and its weights.
struct Row {
  uint32_t top;   // largest key
  int top_index;
  float L, twice_inv, p, min_p;   // twice_inv: 2 / T
  int k;          // 0: off
  bool greedy;
  __device__ __forceinline__ float z(uint32_t key) const {
    if (key == top) return 0.0f;
    if (key == 0 || L == INFINITY) return -INFINITY;
    return (0.5f * logit_of(key) - 0.5f * L) * twice_inv;   // halves: a difference of finite logits stays finite
  }
  __device__ __forceinline__ float relative(uint32_t key) const {   // exp(z) <= 1
    return __builtin_amdgcn_exp2f(z(key) * 1.44269504088896341f);
  }
  __device__ __forceinline__ uint64_t weight(uint32_t key) const {
    const uint32_t w = __float_as_uint(relative(key));
    return (static_cast<uint64_t>((w & 0x7FFFFFu) | 0x800000u) << (kWeightBits - 23)) >> min(127u - (w >> 23), 63u);
  }
  // Bin of a key other than 0: does not fall as the key rises.  How far the logit
  // lies below the largest is all that the result depends on.
  __device__ __forceinline__ int bin(uint32_t key) const {
    const float d = fmaxf(L - logit_of(key), 0.0f);   // of two infinities: 0
    return kBins - 1 - min(max(static_cast<int>(__float_as_uint(d) >> 17) - ((127 - 6) << 6), 0), kBins - 1);
  }
  // The race's score of a kept token as a key; 0: not in the race.
  __device__ __forceinline__ uint32_t score(uint32_t key, float noise) const {
    const float e = noise != noise ? INFINITY : fmaxf(noise, 0x1p-126f);
    return key_of(fmaxf(z(key) - logf(e), -3.402823466e38f));
  }
  __device__ __forceinline__ bool races(uint32_t key) const {
    const float v = z(key);
    return v > -INFINITY && (!(min_p > 0.0f) || relative(key) >= min_p);
  }
};

__device__ __forceinline__ Row row_of(const SampleArgs& a, const RowWork& w, int64_t row) {
  Row r;
  const int lane = threadIdx.x & (kWave - 1);
  const uint64_t top = wave_max<unsigned long long>(lane < a.slices ? w.top[lane] : 0ull);   // written by the launch before
  r.top = static_cast<uint32_t>(top >> 32);
  r.top_index = index_of(top);
  r.L = logit_of(r.top);
  const float T = a.temperature ? a.temperature[row] : 1.0f;
  r.twice_inv = fminf(__fdiv_rn(2.0f, T), 3.402823466e38f);
  r.greedy = !a.noise || !(T > 0.0f);
  const int k = a.top_k ? a.top_k[row] : 0;
  r.k = k >= 1 && k < a.V ? k : 0;
  r.p = a.top_p ? a.top_p[row] : 1.0f;
  r.p = r.p < 1.0f ? fmaxf(r.p, 0.0f) : 1.0f;   // a share below zero keeps the first token, as zero does
  const float m = a.min_p ? a.min_p[row] : 0.0f;
  r.min_p = m > 0.0f ? fminf(m, 1.0f) : 0.0f;   // fminf alone would make 1 of NaN
  return r;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void top_kernel(SampleArgs a) {
  __shared__ uint64_t lds[kThreads / kWave];
  const int tid = threadIdx.x, slice = blockIdx.x;
  const int64_t row = blockIdx.y;
  RowWork& w = a.work[row];
  const T* x = static_cast<const T*>(a.logits) + row * a.ldl;
  uint64_t best = 0;
  const int end = min(a.V, (slice + 1) * a.per);
  for (int at = slice * a.per + 8 * tid; at < end; at += kChunk) {
    uint32_t key[8];
    load_keys8(x, at, end, key);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint64_t t = key[i] ? token_word(key[i], at + i) : 0;
      best = t > best ? t : best;
    }
  }
  for (int i = slice * kThreads + tid; i < kBins; i += a.slices * kThreads) w.mass[i] = 0, w.count[i] = 0;
  if (slice == 0 && tid == 0) w.best = 0, w.total = 0, w.listed = 0, w.arrived = 0;
  best = wave_max<unsigned long long>(best);
  if ((tid & (kWave - 1)) == 0) lds[tid / kWave] = best;
  __syncthreads();
  if (tid == 0) {
    for (int i = 0; i < kThreads / kWave; ++i) best = lds[i] > best ? lds[i] : best;
    w.top[slice] = best;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void bins_kernel(SampleArgs a) {
  __shared__ unsigned long long mass[kBins];
  __shared__ uint32_t count[kBins];
  const int tid = threadIdx.x, slice = blockIdx.x;
  const int64_t row = blockIdx.y;
  RowWork& w = a.work[row];
  const Row r = row_of(a, w, row);
  if (r.greedy || r.top == 0 || (r.k == 0 && r.p >= 1.0f)) return;   // nothing to cut
  for (int i = tid; i < kBins; i += kThreads) mass[i] = 0, count[i] = 0;
  __syncthreads();
  // With top-p alone, tokens of weights below (1 - p) / V together hold less than
  // 1 - p of the row (its largest weighs 1), so the cut lies above them: they
  // count in the total only, not in the bins, which saves most of the atomics.
  // The margin covers the integers' rounding.
  const float least = r.k == 0 && r.p < 0.999f ? 0.99f * (1.0f - r.p) / static_cast<float>(a.V) : 0.0f;
  const uint64_t floor = static_cast<uint64_t>(least * 0x1p38f);
  const T* x = static_cast<const T*>(a.logits) + row * a.ldl;
  const int end = min(a.V, (slice + 1) * a.per);
  uint64_t sum = 0;
  for (int at = slice * a.per + 8 * tid; at < end; at += kChunk) {
    uint32_t key[8];
    load_keys8(x, at, end, key);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (key[i]) {
        const uint64_t m = r.weight(key[i]);
        sum += m;
        if (m >= floor) {
          const int b = r.bin(key[i]);
          atomicAdd(&count[b], 1u);
          atomicAdd(&mass[b], static_cast<unsigned long long>(m));
        }
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < kBins; i += kThreads) {
    if (count[i]) {
      __hip_atomic_fetch_add(&w.count[i], count[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_fetch_add(&w.mass[i], static_cast<uint64_t>(mass[i]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  sum = wave_sum<unsigned long long>(sum);
  if ((tid & (kWave - 1)) == 0 && sum) __hip_atomic_fetch_add(&w.total, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// wave_inclusive_scan's steps on two words.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t moved64(uint64_t v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(v >> 32), CTRL, ROWS, 0xF, false);
  return static_cast<uint64_t>(hi) << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_inclusive_scan64(uint64_t v) {
  v += moved64<0x111, 0xF>(v);   // row_shr:1
  v += moved64<0x112, 0xF>(v);
  v += moved64<0x114, 0xF>(v);
  v += moved64<0x118, 0xF>(v);
  v += moved64<0x142, 0xA>(v);   // row_bcast:15 -> rows 1, 3
  v += moved64<0x143, 0xC>(v);   // row_bcast:31 -> rows 2, 3
  return v;
}

// Sums before and up to this thread's values over the workgroup, in the order
// of the threads; every thread calls it.
struct Scan {
  uint32_t count[kThreads / kWave];
  unsigned long long mass[kThreads / kWave];
};
__device__ __forceinline__ void inclusive(uint32_t& c, uint64_t& m, Scan& s) {
  const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
  c = static_cast<uint32_t>(wave_inclusive_scan(static_cast<int>(c)));
  m = wave_inclusive_scan64(m);
  __syncthreads();   // the words' last readers are done
  if (lane == kWave - 1) s.count[wv] = c, s.mass[wv] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / kWave; ++i)
    if (i < wv) c += s.count[i], m += s.mass[i];
}

// The first bin, from `from` down, whose inclusive sums reach a target: a count
// (need > 0) or else a weight.  With it the sums before it and of it.
struct Cut {
  int bin;
  uint32_t count_above, count;
  uint64_t mass_above, mass;
};
// A thread's PER bins, from - PER t and those below it, and the sums before and
// through them on top of count0 and mass0.  The threads hold all bins: from < PER
// kThreads.
template <int PER>
struct Page {
  uint32_t above, through, count[PER];
  uint64_t mass_above, mass_through, mass[PER];
};
template <int PER, typename Count, typename Mass>
__device__ __forceinline__ Page<PER> page_of_bins(int from, Count count_at, Mass mass_at, uint32_t count0, uint64_t mass0, Scan& scan) {
  Page<PER> g;
  uint32_t own = 0;
  uint64_t own_mass = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int bin = from - PER * static_cast<int>(threadIdx.x) - i;
    g.count[i] = bin >= 0 ? count_at(bin) : 0u;
    g.mass[i] = bin >= 0 ? mass_at(bin) : 0u;
    own += g.count[i], own_mass += g.mass[i];
  }
  g.through = own, g.mass_through = own_mass;
  inclusive(g.through, g.mass_through, scan);
  g.through += count0, g.mass_through += mass0;
  g.above = g.through - own, g.mass_above = g.mass_through - own_mass;
  return g;
}
template <int PER>
__device__ __forceinline__ Cut find_cut(int from, const Page<PER>& g, uint32_t need, double want, Cut& out) {
  const int first = from - PER * static_cast<int>(threadIdx.x);
  auto reaches = [&](uint32_t c, uint64_t m) { return need ? c >= need : static_cast<double>(m) >= want; };
  // the one thread whose sums go past the target; nothing is before the first bin
  const bool mine = first >= 0 && reaches(g.through, g.mass_through) && (threadIdx.x == 0 || !reaches(g.above, g.mass_above));
  if (mine) {
    uint32_t c = g.above;
    uint64_t m = g.mass_above;
    bool found = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (!found && reaches(c + g.count[i], m + g.mass[i])) {
        out = Cut{first - i, c, g.count[i], m, g.mass[i]};
        found = true;
      }
      c += g.count[i], m += g.mass[i];
    }
  }
  const bool any = __syncthreads_or(mine);
  const Cut cut = any ? out : Cut{-1, 0, 0, 0, 0};   // not reached
  __syncthreads();   // `out` may be written again
  return cut;
}

// What the finish needs of LDS.
struct FinishLds {
  Scan scan;
  Cut cut;
  uint64_t best[kThreads / kWave], word;
  uint64_t lo[kThreads / kWave], hi[kThreads / kWave];
  uint32_t base, listed, found;
  union {
    struct {
      uint64_t list[kList], few[kWave];
      unsigned long long mass[kThreads];
      uint32_t count[kThreads];
    };
    struct {
      unsigned long long mass[2048];
      uint32_t count[2048];
    } bins;
  };
};

// Finds the cut of a whole row by its keys' bits, 11 + 11 + 10: the key it
// falls on and the sums above that key.
template <typename T, typename Keep>
__device__ Cut cut_by_bits(const SampleArgs& a, const T* x, const Row& r, Keep keep, uint32_t need, double want, FinishLds& s,
                           uint32_t& key_out) {
  uint32_t prefix = 0, ca = 0;
  uint64_t ma = 0;
  Cut c = {};
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
    __syncthreads();
    for (int i = threadIdx.x; i < 2048; i += kThreads) s.bins.mass[i] = 0, s.bins.count[i] = 0;
    __syncthreads();
    for (int at = 8 * static_cast<int>(threadIdx.x); at < a.V; at += kChunk) {
      uint32_t key[8];
      load_keys8(x, at, a.V, key);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (key[i] && (level == 0 || key[i] >> (shift + bits) == prefix) && keep(key[i], at + i)) {
          const uint32_t b = key[i] >> shift & ((1u << bits) - 1);
          atomicAdd(&s.bins.count[b], 1u);
          atomicAdd(&s.bins.mass[b], static_cast<unsigned long long>(r.weight(key[i])));
        }
      }
    }
    __syncthreads();
    // the largest key's bin is where the sums begin
    const uint32_t top = r.top >> shift;
    const int from = level == 0 || top >> bits == prefix ? static_cast<int>(top & ((1u << bits) - 1)) : (1 << bits) - 1;
    auto count_at = [&](int b) { return s.bins.count[b]; };
    auto mass_at = [&](int b) { return static_cast<uint64_t>(s.bins.mass[b]); };
    c = find_cut(from, page_of_bins<2048 / kThreads>(from, count_at, mass_at, ca, ma, s.scan), need, want, s.cut);
    if (c.bin < 0) break;
    prefix = prefix << bits | static_cast<uint32_t>(c.bin);
    ca = c.count_above, ma = c.mass_above;
  }
  key_out = prefix;
  return c;
}

// The index below which the row holds exactly r (>= 1) kept tokens of a key.
template <typename T, typename Keep>
__device__ int index_after(const SampleArgs& a, const T* x, uint32_t key, uint32_t r, Keep keep, FinishLds& s) {
  // thread t looks at the t-th stretch of the row
  const int stretch = (a.V + kThreads - 1) / kThreads, lo = static_cast<int>(threadIdx.x) * stretch;
  const int hi = min(a.V, lo + stretch);
  uint32_t n = 0;
  for (int i = lo; i < hi; ++i) n += key_of(static_cast<float>(x[i])) == key && keep(key, i) ? 1u : 0u;
  uint32_t c = n;
  uint64_t m = 0;
  inclusive(c, m, s.scan);
  if (threadIdx.x == 0) s.base = static_cast<uint32_t>(a.V);
  __syncthreads();
  if (c >= r && c - n < r) {
    uint32_t seen = c - n;
    for (int i = lo; i < hi; ++i)
      if (key_of(static_cast<float>(x[i])) == key && keep(key, i) && ++seen == r) {
        s.base = static_cast<uint32_t>(i) + 1;
        break;
      }
  }
  __syncthreads();
  const int index = static_cast<int>(s.base);
  __syncthreads();
  return index;
}

// Places for the lanes that append to a counter in LDS: one atomic a wavefront.
__device__ __forceinline__ uint32_t place(uint32_t* counter, bool on) {
  const uint64_t mask = __ballot(on);
  if (!mask) return 0;
  uint32_t base = 0;
  const int leader = __builtin_ctzll(mask);
  if ((threadIdx.x & (kWave - 1)) == static_cast<unsigned>(leader)) base = atomicAdd(counter, static_cast<uint32_t>(__popcll(mask)));
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(base), leader)) + lanes_below(mask);
}

// The best of the workgroup's words, in thread 0.
__device__ __forceinline__ uint64_t block_best(uint64_t best, FinishLds& s) {
  __syncthreads();
  best = wave_max<unsigned long long>(best);
  if ((threadIdx.x & (kWave - 1)) == 0) s.best[threadIdx.x / kWave] = best;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int i = 0; i < kThreads / kWave; ++i) best = s.best[i] > best ? s.best[i] : best;
  return best;
}

// The whole row by one workgroup.
template <typename T>
__device__ uint64_t finish_row(const SampleArgs& a, const T* x, const float* noise, const Row& r, FinishLds& s) {
  uint32_t cut = 0;   // kept: key > cut, or key == cut and index < cut_index
  int cut_index = a.V;
  auto keep = [&](uint32_t key, int i) { return key > cut || (key == cut && i < cut_index); };
  if (r.k) {
    uint32_t key;
    const Cut c = cut_by_bits(a, x, r, keep, static_cast<uint32_t>(r.k), 0.0, s, key);
    if (c.bin >= 0) {   // else the row holds fewer
      const int index = index_after(a, x, key, static_cast<uint32_t>(r.k) - c.count_above, keep, s);
      cut = key, cut_index = index;
    }
  }
  if (r.p < 1.0f) {
    uint64_t sum = 0;
    for (int at = 8 * static_cast<int>(threadIdx.x); at < a.V; at += kChunk) {
      uint32_t key[8];
      load_keys8(x, at, a.V, key);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (key[i] && keep(key[i], at + i)) sum += r.weight(key[i]);
    }
    uint32_t none = 0;
    inclusive(none, sum, s.scan);
    __syncthreads();
    if (threadIdx.x == kThreads - 1) s.scan.mass[0] = sum;
    __syncthreads();
    const double want = static_cast<double>(r.p) * static_cast<double>(s.scan.mass[0]);
    uint32_t key;
    const Cut c = cut_by_bits(a, x, r, keep, 0u, want, s, key);
    if (c.bin >= 0) {
      const double w = static_cast<double>(r.weight(key)), over = want - static_cast<double>(c.mass_above);
      const double n = w > 0.0 ? ceil(over / w) : 1.0;   // equal tokens kept: the sum before each is below `want`
      const int index = index_after(a, x, key, n >= 1.0 ? static_cast<uint32_t>(fmin(n, 16777216.0)) : 1u, keep, s);
      cut = key, cut_index = index;
    }
  }
  uint64_t best = 0;
  for (int at = 8 * static_cast<int>(threadIdx.x); at < a.V; at += kChunk) {
    uint32_t key[8];
    load_keys8(x, at, a.V, key);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (key[i] && keep(key[i], at + i) && r.races(key[i])) {
        const uint64_t t = token_word(r.score(key[i], noise[at + i]), at + i);
        best = t > best ? t : best;
      }
    }
  }
  return best;
}

// The cut among the listed tokens of one bin, whose tokens come after the
// sums count0 and mass0: the word of the last kept token (need > 0: the one that
// makes the count, else the one that makes the weight), and the weight up to it.
// The bin's sums reach the target, so there is one.
__device__ uint64_t cut_list(const Row& r, uint32_t listed, int bin, uint32_t count0, uint64_t mass0, uint32_t need, double want,
                             uint64_t& upto, FinishLds& s) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
  uint64_t from = 0, to = ~0ull;   // the bin's tokens that may be the last kept
  uint32_t n;
  for (;;) {
    __syncthreads();
    if (tid == 0) s.found = 0;
    s.mass[tid] = 0, s.count[tid] = 0;
    __syncthreads();
    uint64_t lo = ~0ull, hi = 0;
    for (uint32_t i0 = 0; i0 < listed; i0 += kThreads) {
      const uint64_t own = i0 + tid < listed ? s.list[i0 + tid] : 0;
      const bool on = own && own >= from && own <= to && r.bin(static_cast<uint32_t>(own >> 32)) == bin;
      const uint32_t at = place(&s.found, on);
      if (on) {
        if (at < kWave) s.few[at] = own;
        lo = own < lo ? own : lo, hi = own > hi ? own : hi;
      }
    }
    lo = ~wave_max<unsigned long long>(~lo), hi = wave_max<unsigned long long>(hi);
    if (lane == 0) s.lo[wv] = lo, s.hi[wv] = hi;
    __syncthreads();
    n = s.found;
    if (n <= kWave) break;
    // 256 bins of the words' own range, whose low half orders equal logits, leave
    // few; no two words are equal, so that at last each has a bin of its own
#pragma unroll
    for (int i = 0; i < kThreads / kWave; ++i) lo = s.lo[i] < lo ? s.lo[i] : lo, hi = s.hi[i] > hi ? s.hi[i] : hi;
    const int shift = max(56 - __builtin_clzll((hi - lo) | 1u), 0);
    for (uint32_t i = tid; i < listed; i += kThreads) {
      const uint64_t own = s.list[i];
      if (own >= lo && own <= hi) {
        const int b = static_cast<int>((own - lo) >> shift);
        atomicAdd(&s.count[b], 1u);
        atomicAdd(&s.mass[b], static_cast<unsigned long long>(r.weight(static_cast<uint32_t>(own >> 32))));
      }
    }
    __syncthreads();
    const int top = static_cast<int>((hi - lo) >> shift);
    const Cut c = find_cut(top, page_of_bins<1>(top, [&](int b) { return s.count[b]; },
                                                [&](int b) { return static_cast<uint64_t>(s.mass[b]); }, count0, mass0, s.scan),
                           need, want, s.cut);
    from = lo + (static_cast<uint64_t>(c.bin) << shift), to = from + ((1ull << shift) - 1);
    count0 = c.count_above, mass0 = c.mass_above;
  }
  // what comes before a token, by looking at all
  if (tid < static_cast<int>(n)) {
    const uint64_t own = s.few[tid];
    uint32_t rank = count0;
    uint64_t before = mass0;
    for (uint32_t i = 0; i < n; ++i)
      if (s.few[i] > own) ++rank, before += r.weight(static_cast<uint32_t>(s.few[i] >> 32));
    const uint64_t after = before + r.weight(static_cast<uint32_t>(own >> 32));
    // of the weight's cut: the last token with less than `want` before it, at least the first
    const bool last = need ? rank == need - 1
                           : static_cast<double>(after) >= want && (static_cast<double>(before) < want || rank == 0);
    if (last) s.word = own, s.scan.mass[0] = after;
  }
  __syncthreads();
  upto = s.scan.mass[0];
  return s.word;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void finish_kernel(SampleArgs a) {
  __shared__ FinishLds s;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave, slice = blockIdx.x;
  const int64_t row = blockIdx.y;
  RowWork& w = a.work[row];
  const Row r = row_of(a, w, row);
  if (r.greedy || r.top == 0) {   // the same for the whole row
    if (slice == 0 && tid == 0) a.tokens[row] = r.top == 0 ? -1 : r.top_index;
    return;
  }
  const T* x = static_cast<const T*>(a.logits) + row * a.ldl;
  const float* noise = a.noise + row * a.ldn;
  // Bins that the cuts fall into.  Where top-k cuts, the weight that top-p takes
  // its share of lies between the sums above and through its bin, and top-p's cut
  // between the bins of those.
  Cut by_k{-1, 0, 0, 0, 0}, by_p{-1, 0, 0, 0, 0};
  const bool cuts = r.k || r.p < 1.0f, all = !cuts && !(r.min_p > 0.0f);   // the same for the whole row
  const uint64_t total = r.p < 1.0f ? w.total : 0;
  Page<kBins / kThreads> bins = {};
  if (cuts)   // written by the launch before
    bins = page_of_bins<kBins / kThreads>(
        kBins - 1, [&](int b) { return w.count[b]; }, [&](int b) { return w.mass[b]; }, 0u, 0u, s.scan);
  auto cut_at = [&](uint32_t need, double of) { return find_cut(kBins - 1, bins, need, static_cast<double>(r.p) * of, s.cut); };
  if (r.k) by_k = cut_at(static_cast<uint32_t>(r.k), 0.0);
  int p_low = -1, high = by_k.bin;
  if (r.p < 1.0f) {
    by_p = cut_at(0u, static_cast<double>(by_k.bin >= 0 ? by_k.mass_above + by_k.mass : total));
    p_low = by_p.bin;
    if (by_k.bin >= 0) by_p = cut_at(0u, static_cast<double>(by_k.mass_above));
    high = by_p.bin;
  }
  if (tid == 0) s.listed = 0;
  __syncthreads();
  uint64_t best = 0;
  auto race = [&](uint32_t key, int i, auto noise_at) {
    if (r.races(key)) {
      const uint64_t t = token_word(r.score(key, noise_at()), i);
      best = t > best ? t : best;
    }
  };
  const int end = min(a.V, (slice + 1) * a.finish_per);
  uint32_t next[8];
  int at = slice * a.finish_per + 8 * tid;
  load_keys8(x, min(at, end), end, next);
  for (int at0 = slice * a.finish_per; at0 < end; at0 += kChunk, at += kChunk) {   // the same trips for every thread
    uint32_t key[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) key[i] = next[i];
    float e[8];
    if (all) load8(noise + min(at, end), end - at, e);   // every number races
    if (at0 + kChunk < end) load_keys8(x, min(at + kChunk, end), end, next);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int b = key[i] ? r.bin(key[i]) : -2;
      if (b > high) {   // passes both
        if (key[i]) race(key[i], at + i, [&] { return all ? e[i] : noise[at + i]; });
      }
      const bool on = b <= high && b >= 0 && (b == by_k.bin || (p_low >= 0 && b >= p_low));
      const uint32_t to = place(&s.listed, on);   // in any order: the list is ordered below
      if (on && to < kList) s.list[to] = token_word(key[i], at + i);
    }
  }
  __syncthreads();
  uint32_t listed = s.listed;
  if (gridDim.x > 1) {
    if (listed) {
      if (tid == 0) s.base = __hip_atomic_fetch_add(&w.listed, listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      for (uint32_t i = tid; i < min(listed, static_cast<uint32_t>(kList)) && s.base + i < kList; i += kThreads)
        put(&w.list[s.base + i], s.list[i]);
    }
    best = block_best(best, s);
    if (tid == 0 && best) __hip_atomic_fetch_max(&w.best, best, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wavefront's words are out
    __syncthreads();
    if (tid == 0) s.base = __hip_atomic_fetch_add(&w.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (s.base != gridDim.x - 1) return;
    best = tid == 0 ? get(&w.best) : 0;
    listed = get(&w.listed);
    if (listed <= kList) {
      uint64_t word[kList / kThreads];   // all loads in flight
#pragma unroll
      for (int u = 0; u < kList / kThreads; ++u) {
        const uint32_t i = tid + u * kThreads;
        if (i < listed) word[u] = get(&w.list[i]);
      }
#pragma unroll
      for (int u = 0; u < kList / kThreads; ++u) s.list[tid + u * kThreads] = word[u];
    }
    __syncthreads();
  }
  if (listed > kList) {
    best = finish_row(a, x, noise, r, s);
  } else if (listed) {
    uint64_t cut = 0, upto = total;   // listed tokens from this word up are kept
    if (by_k.bin >= 0)
      cut = cut_list(r, listed, by_k.bin, by_k.count_above, by_k.mass_above, static_cast<uint32_t>(r.k), 0.0, upto, s);
    if (r.p < 1.0f) {
      const double of = static_cast<double>(upto);
      if (by_k.bin >= 0) {
        __syncthreads();
        by_p = cut_at(0u, of);
      }
      const uint64_t c = cut_list(r, listed, by_p.bin, by_p.count_above, by_p.mass_above, 0u, static_cast<double>(r.p) * of, upto, s);
      cut = c > cut ? c : cut;
    }
    for (uint32_t i = tid; i < listed; i += kThreads)
      if (s.list[i] >= cut) race(static_cast<uint32_t>(s.list[i] >> 32), index_of(s.list[i]), [&] { return noise[index_of(s.list[i])]; });
  }
  best = block_best(best, s);
  if (tid == 0) a.tokens[row] = index_of(best);
}

struct SamplePlan {
  int slices, per, finish_slices, finish_per, rows;
};

// One chunk a slice where the rows alone do not fill the compute units, four
// where they do; kMaxSlices of a row at most.  The finish keeps two workgroups a
// unit busy for one round.
SamplePlan make_plan(int32_t rows, int32_t V) {
  const int chunks = (V + kChunk - 1) / kChunk, n = std::min(rows, kRowsAtOnce);
  int per = static_cast<int64_t>(n) * chunks > 2048 ? 4 : 1;
  per = std::max(per, (chunks + kMaxSlices - 1) / kMaxSlices);
  const int fit = std::max(1, 512 / n);
  const int finish = std::max(per, (chunks + fit - 1) / fit);
  return {(chunks + per - 1) / per, per * kChunk, (chunks + finish - 1) / finish, finish * kChunk, n};
}

}  // namespace

extern "C" size_t celty_sample_workspace_bytes(int32_t rows, int32_t V) {
  return rows < 0 || V < 1 || V > (1 << 24) ? 0 : std::max<size_t>(256, sizeof(RowWork) * std::min(rows, kRowsAtOnce));
}

extern "C" celty_status celty_sample(int32_t rows, int32_t V, int32_t dtype, const void* logits, int64_t ldl,
                                     const float* noise, int64_t ldn, const celty_filters* filters, int32_t* tokens,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  if (rows < 0 || V < 1 || V > (1 << 24)) return CELTY_EINVAL;
  if (dtype != CELTY_F16 && dtype != CELTY_BF16 && dtype != CELTY_F32) return CELTY_EINVAL;
  if (rows == 0) return CELTY_OK;   // empty tensors may have no address
  if (!logits || !tokens || !workspace || ldl < V || (noise && ldn < V)) return CELTY_EINVAL;
  if (ldl > (int64_t{1} << 31) || (noise && ldn > (int64_t{1} << 31))) return CELTY_EINVAL;
  const int size = dtype == CELTY_F32 ? 4 : 2;
  if (misaligned(logits, size) || misaligned(noise, 4) || misaligned(tokens, 4) || misaligned(workspace, 256) ||
      workspace_bytes < celty_sample_workspace_bytes(rows, V))
    return CELTY_EINVAL;
  SampleArgs a{};
  if (filters) {
    a.temperature = filters->temperature;
    a.top_k = filters->top_k;
    a.top_p = filters->top_p;
    a.min_p = filters->min_p;
    if (misaligned(a.temperature, 4) || misaligned(a.top_k, 4) || misaligned(a.top_p, 4) || misaligned(a.min_p, 4))
      return CELTY_EINVAL;
  }
  const SamplePlan plan = make_plan(rows, V);
  const bool cuts = noise && (a.top_k || a.top_p);
  a.work = static_cast<RowWork*>(workspace);
  a.ldl = ldl, a.ldn = ldn, a.V = V, a.slices = plan.slices, a.per = plan.per, a.finish_per = plan.finish_per;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  // as many rows at a time as the workspace holds
  for (int32_t at = 0; at < rows; at += plan.rows) {
    const int32_t n = std::min(plan.rows, rows - at);
    SampleArgs b = a;
    b.logits = static_cast<const char*>(logits) + at * ldl * size;
    b.noise = noise ? noise + at * ldn : nullptr;
    b.tokens = tokens + at;
    if (b.temperature) b.temperature += at;
    if (b.top_k) b.top_k += at;
    if (b.top_p) b.top_p += at;
    if (b.min_p) b.min_p += at;
    auto go = [&](auto kernel, int slices) {
      hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(slices), static_cast<unsigned>(n)), dim3(kThreads), 0, st, b);
    };
    auto typed = [&](auto t) {
      using T = decltype(t);
      go(top_kernel<T>, plan.slices);
      if (cuts) go(bins_kernel<T>, plan.slices);
      go(finish_kernel<T>, plan.finish_slices);
    };
    if (dtype == CELTY_F16) typed(half_t{});
    else if (dtype == CELTY_BF16) typed(bf16_t{});
    else typed(0.0f);
  }
  return hipGetLastError() == hipSuccess ? CELTY_OK : CELTY_EHIP;
}
