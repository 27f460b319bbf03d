// celty_kv4_attention (include/celty_decode.h) for gfx950: causal attention
// over the 4-bit cache.
//
// With keys k_j = m_j + s_j c_j and values in the same form, a score is
// s_j (q . c_j) + m_j sum(q) and the output sum_j p_j s_j (c_j - 8) + sum_j p_j
// (m_j + 8 s_j), so both products run on the matrix instructions with the codes
// as one operand; scales and minima meet the scores and the probabilities, one
// each per position, never the D channels.  A key's code needs no conversion:
// the bits of a nibble in the low bits of a half are that number times 2^-24
// (or, four bits up, 2^-20) as an fp16 subnormal, which the matrix instructions
// take exactly, so a word of eight codes becomes an operand by one shift and
// four ands, and the query carries the difference of 2^4.  Value codes are made
// numbers about zero (centred_of), nine instructions a word.
//
// Two kernels.  decode_kernel: 16 queries of a key head (a group's heads of one
// token, or of a few), the positions shared out to eight wavefronts and, where
// units are few, to several workgroups; bound by reading the cache where those
// fill the chip evenly: 64 heads over 8, 128 channels, 16 sequences of 16000
// positions 50 us, 5.6 TB/s, 32 of them 105 us, 5.3 TB/s; one of 131001 33 us, 4.3
// TB/s, the launch, the first loads' round trips and the join of 32 workgroups
// among them.  Between, units are left idle: 17 sequences take 83 us (3.6 TB/s).
// At 128 channels it takes 136 registers, three wavefronts a SIMD, so that a
// compute unit holds one workgroup of eight; up to 128 registers it held two.
// chunk_kernel: 32 queries a wavefront; vector and matrix instructions in turn
// (below).
//
// Layout of a tile of 32 positions (16x16x32 instructions; lane = 16 g + r):
//   scores  S^T = K Q^T, twice 16 positions: lane row r of tile h holds the
//           codes of position 8 (r / 4) + 4 h + r % 4, channels g D/4 ..; the
//           result has column r (a query) and positions 8 g + 4 h + 0..3, so a
//           lane's eight scores are those of positions 8 g .. 8 g + 7;
//   values  O^T = V^T P^T: a word of value codes is one channel at positions
//           8 g .. 8 g + 7, and the lane's own eight probabilities are the
//           other operand as they stand: nothing is exchanged between lanes.
//
// The softmax keeps a reference M per query for exp2(score - M) that is raised
// only when a probability times its value scale would leave fp16's range
// (2^15, against 2^9 when it is set), so most tiles need no exchange for the
// maximum and no scaling of the output.  M includes the largest value scale
// that the query has seen: what is rounded to fp16 is p s, at its best
// resolution whatever the values' magnitude, and one that is 2^-23 of the largest
// is still kept to a part in 2^11 (2^-33 to one bit).  The sums of p and of
// p (m + 8 s) take the unrounded p, in fp32.  M is kept in two parts, the largest
// score and the rest: scores are taken as differences from the former (the
// addend of a product that is made anyway), so that their size does not matter.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "celty_decode.h"
#include "common.h"
#include "kv4.h"
#include "tensor.h"

namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint2_t __attribute__((ext_vector_type(2)));

struct AttnArgs {
  const void* q;
  void* out;
  int64_t q_token, q_head, o_token, o_head;
  int group;              // query heads of a key head
  float scale;            // log2(e) included
  int window;
  int n_splits;           // workgroups that may share a unit
  int tiles_per_seq;      // column tiles of a sequence when q_start is NULL
  int tiles;              // column tiles that the grid holds
  uint32_t* tickets;      // per unit, zero between calls
  float* partial;         // per unit and split: 16 x D sums, then 16 x (L, M)
};

constexpr float kLow = -3e38f;       // a reference below every score
// log2 of p s when the reference is set: a score may then rise by 2^3 and a scale
// by 2^3.  (With 11, 2^2 each, queries that raise theirs alone do so more often:
// sixteen sequences of five tokens under a window 16.7 us against 16.0.)
constexpr float kHeadroom = 9.0f;
constexpr float kLimit = 15.0f;      // and when it must be raised
constexpr float kSlack = (kLimit - kHeadroom) / 2;
constexpr float kScaleMargin = 1 << static_cast<int>(kSlack);
constexpr int kMaxSplits = 128;      // of a unit: (L, M) of all fit the join's LDS
constexpr int kMinBlocks = 16;       // least tiles of 32 positions a split takes

// Eight codes of a word as an operand: nibbles 0 4 1 5 2 6 3 7, the odd
// pairs (1 5, 3 7) 2^4 larger.
__device__ __forceinline__ half8_t operand_of(uint32_t w) {
  const uint32_t h = w >> 8;
  const uint4_t u = {w & 0x000F000Fu, w & 0x00F000F0u, h & 0x000F000Fu, h & 0x00F000F0u};
  return __builtin_bit_cast(half8_t, u);
}

// The same of value codes less 8: over the bits of 1024 (or 64) a nibble adds
// its number, exactly, and 1032 (72) is taken off again.  The output is a mean of
// values about zero; of codes from 0 up it would be the small difference of two
// large sums (131001 positions: 5.3e-4 off against 2.4e-4, of which fp16's own
// rounding is 2.1e-4).
// The two constants are held in vector registers: an instruction that masks and
// sets bits reads one scalar or literal only.
struct Bits {
  uint32_t low, high;
};
__device__ __forceinline__ Bits number_bits() {
  Bits k = {0x64006400u, 0x54005400u};   // 1024 and 64, twice
  asm volatile("" : "+v"(k.low), "+v"(k.high));
  return k;
}
__device__ __forceinline__ half8_t centred_of(uint32_t w, const Bits& k) {
  const uint32_t h = w >> 8;
  const half2_t low = {-1032.0f16, -1032.0f16}, high = {-72.0f16, -72.0f16};
  auto pair = [](uint32_t bits, half2_t less) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, bits) + less); };
  const uint4_t u = {pair((w & 0x000F000Fu) | k.low, low), pair((w & 0x00F000F0u) | k.high, high),
                     pair((h & 0x000F000Fu) | k.low, low), pair((h & 0x00F000F0u) | k.high, high)};
  return __builtin_bit_cast(half8_t, u);
}

__device__ __forceinline__ float4_t mfma16(half8_t a, half8_t b, float4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float scale_of(uint32_t p) { return static_cast<float>(__builtin_bit_cast(half2_t, p)[0]); }
__device__ __forceinline__ float minimum_of(uint32_t p) { return static_cast<float>(__builtin_bit_cast(half2_t, p)[1]); }

// Over the four lanes that share a column (lane bits 4 and 5): the two swaps
// pair a row of 16 lanes, then a half of the wavefront, with the other.
template <typename F>
__device__ __forceinline__ float over_column(float v, F f) {
  const auto h = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(h[0]), __uint_as_float(h[1]));
  const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float column_max(float v) {
  return over_column(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float column_sum(float v) {
  return over_column(v, [](float a, float b) { return a + b; });
}
// Over the two lanes that share a column of 32 (lane bit 5).
template <typename F>
__device__ __forceinline__ float over_halves(float v, F f) {
  const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float halves_max(float v) {
  return over_halves(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float halves_sum(float v) {
  return over_halves(v, [](float a, float b) { return a + b; });
}

// Over the 16 lanes of a row.
template <int ROR>
__device__ __forceinline__ float max_rotated(float v) {
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + ROR, 0xF, 0xF, false)));
}
__device__ __forceinline__ float row_max(float v) {
  return max_rotated<1>(max_rotated<2>(max_rotated<4>(max_rotated<8>(v))));
}

// The largest of N scores; written as the instruction, for fmaxf would first
// quiet its operands' NaN, an instruction each.
template <int N>
__device__ __forceinline__ float largest(const float (&x)[N]) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i + 1 < N; i += 2) asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(m), "v"(x[i]), "v"(x[i + 1]));
  if (N % 2 == 0) m = fmaxf(m, x[N - 1]);
  return m;
}

// One lane's share of the keys and of the values of 32 positions.
template <int D>
struct Keys {
  uint32_t c[2][D / 32];   // rows of the two score tiles
  uint32_t p[8];           // parameters of positions 8 g ..
};
template <int D>
struct Values {
  uint32_t c[D / 16];      // channels 64 n + 4 r + 0..3 at positions 8 g ..
  uint32_t p[8];
  uint32_t own;            // parameters of position lane % 32, for the largest scale of a tile seen whole
};

// Loads go through a buffer descriptor of the 32 positions: a scalar base,
// one 32-bit offset a lane and constant offsets.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), static_cast<short>(0), bytes, 0x00020000);
}

__device__ __forceinline__ int own_offset() { return 4 * (threadIdx.x & 31); }

__device__ __forceinline__ void load_params(const __amdgpu_buffer_rsrc_t rs, int p_lane, uint32_t (&out)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto w = __builtin_amdgcn_raw_buffer_load_b128(rs, p_lane, 16 * h, 0);
    out[4 * h] = w[0], out[4 * h + 1] = w[1], out[4 * h + 2] = w[2], out[4 * h + 3] = w[3];
  }
}

// slot: of the first of the 32 positions, the same for the whole wavefront
template <int D>
__device__ __forceinline__ void load_keys(const Kv4Args& a, int64_t slot, int k_lane, int p_lane, Keys<D>& t) {
  const __amdgpu_buffer_rsrc_t rs = rsrc_of(a.k_codes + slot * (D / 2), 16 * D);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (D == 128) {
      const auto w = __builtin_amdgcn_raw_buffer_load_b128(rs, k_lane, h * 4 * (D / 2), 0);
      t.c[h][0] = w[0], t.c[h][1] = w[1], t.c[h][2] = w[2], t.c[h][3] = w[3];
    } else {
      const auto w = __builtin_amdgcn_raw_buffer_load_b64(rs, k_lane, h * 4 * (D / 2), 0);
      t.c[h][0] = w[0], t.c[h][1] = w[1];
    }
  }
  load_params(rsrc_of(a.k_params + slot, 32 * 4), p_lane, t.p);
}

template <int D>
__device__ __forceinline__ void load_values(const Kv4Args& a, int64_t slot, int v_lane, int p_lane, Values<D>& t) {
  const __amdgpu_buffer_rsrc_t rs = rsrc_of(reinterpret_cast<const uint8_t*>(a.v_codes) + slot * (D / 2), 16 * D);
#pragma unroll
  for (int n = 0; n < D / 64; ++n) {
    const auto w = __builtin_amdgcn_raw_buffer_load_b128(rs, v_lane, 256 * n, 0);
    t.c[4 * n] = w[0], t.c[4 * n + 1] = w[1], t.c[4 * n + 2] = w[2], t.c[4 * n + 3] = w[3];
  }
  const __amdgpu_buffer_rsrc_t ps = rsrc_of(a.v_params + slot, 32 * 4);
  load_params(ps, p_lane, t.p);
  t.own = __builtin_amdgcn_raw_buffer_load_b32(ps, own_offset(), 0, 0);
}

// A wavefront's running softmax and output for 16 queries.
template <int D>
struct Running {
  float4_t o[D / 16];   // channels 64 (t / 4) + 16 g + 4 i + t % 4
  float l, pm;          // this lane's part of sum p and sum p m
  float top;            // the largest score the reference was set from; scores are taken from it on
  float limit;          // the score above it that raises it, kLow until something is seen
  float vmax;           // the largest value scale the reference was set from
  float shift;          // cs top less the reference M
  float scale_limit;    // the value scale of a tile seen whole that raises every query's
};

// Sets a query's reference from scores up to xc above its present one and value
// scales up to sc, takes the scores x from it on and returns the factor of the
// sums so far, of which those of p are brought along.  Scores are compared as
// differences from the largest: however large they are, its exponent is exact.
template <int N, typename S>
__device__ __forceinline__ float raise_reference(float xc, float sc, float cs, S& s, float (&x)[N]) {
  const bool before = s.limit > kLow, seen = before || xc > kLow;   // nothing seen: all sums are zero, or NaN
  const float rise = before ? fmaxf(xc, 0.0f) : seen ? xc : 0.0f;
  s.vmax = fmaxf(s.vmax, fminf(sc, 65504.0f));   // infinity shows in the product
  const float shift = kHeadroom - __builtin_amdgcn_logf(s.vmax);   // to base 2; what it rounds to is kept in s.shift
  const float r = before ? __builtin_amdgcn_exp2f(fmaf(-cs, rise, shift - s.shift)) : 1.0f;
  s.top += rise, s.shift = shift;
  s.limit = seen ? kSlack * __builtin_amdgcn_rcpf(cs) : kLow;
  s.l *= r;
  s.pm *= r;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] -= rise;
  return r;
}
// Sums that were taken apart are joined as multiples of exp2 of their largest
// score: the shift, which a large score would swallow, is taken off them first.
template <typename S>
__device__ __forceinline__ float top_score(float cs, const S& s) {
  return s.limit > kLow ? cs * s.top : kLow;
}

// The largest value scale of those given; NaN counts for nothing.
template <int N>
__device__ __forceinline__ float largest_scale(const half2_t (&p)[N]) {
  half2_t m = p[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = __builtin_elementwise_max(m, p[i]);
  return static_cast<float>(m[0]);
}

template <int D>
__device__ __forceinline__ void attend_tile(const Keys<D>& k, const Values<D>& v, const half8_t (&q)[D / 32], float cs, float qm, bool masked,
                                            int from, int to, const Bits& bits, Running<D>& s) {
  __builtin_amdgcn_sched_barrier(0);
  float4_t acc[2] = {};
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    acc[0] = mfma16(operand_of(k.c[0][j]), q[j], acc[0]);
    acc[1] = mfma16(operand_of(k.c[1][j]), q[j], acc[1]);
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_sched_barrier(0);   // the phases one after another: hoisted operands would cost registers
  float x[8];   // positions 8 g + i, above the reference's score, in units of 1 / cs
  half2_t vp[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = fmaf(scale_of(k.p[i]), acc[i / 4][i % 4], fmaf(minimum_of(k.p[i]), qm, -s.top));
    vp[i] = __builtin_bit_cast(half2_t, v.p[i]);
  }
  float sm = scale_of(v.own), scale_limit = s.scale_limit;
  if (masked) {   // the same for the whole wavefront
    // neither what a hidden position's score is nor its value's parameters may matter
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool hidden = i < from || i > to;
      x[i] = hidden ? -INFINITY : x[i];
      vp[i] = hidden ? half2_t{} : vp[i];
    }
    sm = largest_scale(vp);
    scale_limit = s.vmax * kScaleMargin;
  }
  const float xm = largest(x);
  // p s <= 2^limit holds while the score's and the scale's excess over what the
  // reference was set from are within half the margin each.  A tile that all
  // queries see whole raises all of them for its scales, another each query for
  // those it sees: no result depends on what another query's window holds.
  if (__any(xm > s.limit || sm > scale_limit)) {
    const float xc = column_max(xm), sc = masked ? column_max(sm) : row_max(column_max(sm));
    if (xc > s.limit || sc > scale_limit) {   // this query's own
      const float r = raise_reference(xc, sc, cs, s, x);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) s.o[c] *= r;
    }
    if (!masked && sc > scale_limit) s.scale_limit = sc * kScaleMargin;
  }
  half8_t b;   // probabilities times the values' scales
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float e = __builtin_amdgcn_exp2f(fmaf(cs, x[i], s.shift)), scale = static_cast<float>(vp[i][0]);
    s.l += e;
    s.pm = fmaf(e, fmaf(scale, 8.0f, static_cast<float>(vp[i][1])), s.pm);
    b[2 * (i % 4) + i / 4] = static_cast<half_t>(fmaf(e, scale, 0.0f));   // one instruction, product and rounding
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    s.o[c] = mfma16(centred_of(v.c[c], bits), b, s.o[c]);
    if (c & 1) __builtin_amdgcn_sched_barrier(0);
  }
}

// One column's query as an operand: scaled by a power of two to at most 2^15,
// the pairs that meet the larger codes by 2^-4 more, the sign of the call's
// scale taken in (zero makes every score zero).  Returns the factor of a score and sum(q) in its units.
// A lane holds N channels: a quarter of them (16 columns) or half (32).
template <typename T, int D, int N>
__device__ __forceinline__ void load_query(const T* q, float scale, half8_t (&out)[N / 8], float& cs, float& qm) {
  constexpr bool kQuarter = N == D / 4;
  float v[N];
  float big = 0.0f, sum = 0.0f;
#pragma unroll
  for (int j = 0; j < N / 8; ++j) {
    float y[8];
    load8(q + 8 * j, 8, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[8 * j + i] = y[i];
      big = fmaxf(big, fabsf(y[i]));
    }
  }
  big = kQuarter ? column_max(big) : halves_max(big);
  int e = 0;
  if (big > 0.0f && big < INFINITY) {
    frexpf(big, &e);
    e -= 15;
  }
  const float sign = scale < 0.0f ? -1.0f : scale > 0.0f ? 1.0f : 0.0f;
#pragma unroll
  for (int j = 0; j < N / 8; ++j) {
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const float x = sign * ldexpf(v[8 * j + n], -e);
      sum += x;
      // nibble n is slot 2 (n % 4) + n / 4
      out[j][2 * (n % 4) + n / 4] = static_cast<half_t>((n & 1) ? x * 0.0625f : x);
    }
  }
  // above 0, for hidden scores are -infinity: scores are below 2^16 (with codes
  // below 16, scales and minima in fp16), so under 2^-100 every one is as good as
  // zero, and over 2^100 no two that differ share the weight
  cs = scale == 0.0f || big == 0.0f ? 1.0f : fminf(fmaxf(ldexpf(fabsf(scale), 24 + e), 0x1p-100f), 0x1p100f);
  qm = ldexpf(kQuarter ? column_sum(sum) : halves_sum(sum), -24);
  if (big == INFINITY) qm = NAN;   // every score: those of -infinity alone would look like nothing seen
}

// A split's sums go past the L2 caches, which the chip's dies do not share, as
// agent-scope stores; once they are done (wait_for_stores in every wavefront,
// then the barrier) the split takes its ticket.  A release fence instead would
// write back a whole L2 for every split, and an acquire fence drop it: 60 us
// against 41 for one sequence of 131001 positions in 64 splits.
__device__ __forceinline__ void store_through(float* p, float a, float b) {
  const uint64_t v = static_cast<uint64_t>(__float_as_uint(b)) << 32 | __float_as_uint(a);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_through(const float* p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return {__uint_as_float(static_cast<uint32_t>(v)), __uint_as_float(static_cast<uint32_t>(v >> 32))};
}
__device__ __forceinline__ void wait_for_stores() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

constexpr int kDecodeWaves = 8;
template <int D>
constexpr int kPartFloats = 16 * (D + 2);   // a split's sums: 16 columns of D, then (L, M) of each

template <typename T, int D>
__global__ __launch_bounds__(kDecodeWaves* kWave, 2) void decode_kernel(Kv4Args a, AttnArgs f) {
  constexpr int NW = kDecodeWaves, ROW = D + 4;   // padded against bank conflicts
  __shared__ float lds_o[NW][16][ROW];
  __shared__ float lds_l[NW][16], lds_m[NW][16], lds_shift[NW][16], lds_pm[NW][16];
  __shared__ uint32_t lds_ticket;
  static_assert(sizeof(lds_o) >= 32 * kMaxSplits * sizeof(float), "(L, M) of every split");
  const int lane = threadIdx.x & (kWave - 1), r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int split = blockIdx.x % f.n_splits, unit = blockIdx.x / f.n_splits;
  const int head = unit % a.heads, tile = unit / a.heads;
  int seq, within;
  if (a.q_start) {
    seq = find_unit(a, tile, [&](const Span& s) { return static_cast<int>((static_cast<int64_t>(s.n) * f.group + 15) >> 4); }, within);
    if (seq < 0) return;
  } else {
    seq = tile / f.tiles_per_seq;
    within = tile - seq * f.tiles_per_seq;
  }
  const Span sp = span_of(a, seq);
  const int cols = min(16, sp.n * f.group - within * 16);   // of this tile
  // this lane's query; columns past the last repeat it
  const int col = within * 16 + min(r, cols - 1);
  const int qi = col / f.group, qh = head * f.group + (col - qi * f.group);
  // positions fit in 32 bits: a table names at most 2^30
  const int p0 = static_cast<int>(sp.len) - sp.n;
  const int pos_lo = p0 + within * 16 / f.group, pos_hi = p0 + (within * 16 + cols - 1) / f.group;
  auto earliest = [&](int pos) { return f.window ? max(max(pos, -1) - f.window, -1) + 1 : 0; };   // that a query there sees
  const int lane_to = max(p0 + qi, -1), lane_from = earliest(lane_to), whole_from = earliest(pos_hi);
  const int hi = min(pos_hi, static_cast<int>(a.capacity) - 1), lo = earliest(pos_lo);
  // tiles of 32 positions, shared out to the splits and their wavefronts
  const int b_lo = lo >> 5;
  const int n_blocks = hi < lo ? 0 : (hi >> 5) - b_lo + 1;
  const int per = max((n_blocks + f.n_splits - 1) / f.n_splits, kMinBlocks);
  const int n_act = max((n_blocks + per - 1) / per, 1);
  if (split >= n_act) return;
  const int first = b_lo + split * per, last = min(first + per, b_lo + n_blocks);

  half8_t q[D / 32];
  float cs, qm;
  load_query<T, D, D / 4>(static_cast<const T*>(f.q) + (sp.first + qi) * f.q_token + qh * f.q_head + g * (D / 4), f.scale, q, cs, qm);
  const Bits bits = number_bits();
  Running<D> s = {};
  s.limit = kLow, s.vmax = s.scale_limit = 0x1p-30f;
  const int k_lane = (8 * (r >> 2) + (r & 3)) * (D / 2) + g * (D / 8), v_lane = (g * D + 4 * r) * 4, p_lane = 32 * g;
  const int32_t* table = a.table + static_cast<int64_t>(seq) * a.table_stride;
  const int shift = a.page_log2 - 5;   // tiles of a page, log2
  auto slot_at = [&](int page, int b) {
    return ((static_cast<int64_t>(page) * a.heads + head) << a.page_log2) + ((b & ((1 << shift) - 1)) << 5);
  };
  // page of a tile, -1 where there is none; loads then go to page 0, unused
  auto page_at = [&](int b) {
    const int p = __builtin_amdgcn_readfirstlane(table[min(b, last - 1) >> shift]);
    return p >= 0 && p < a.n_pages ? p : -1;
  };
  // a tile is loaded while the one before it is worked on, its page's number a
  // tile earlier; past the last tile the last one is loaded again
  int b = first + wave;
  if (b < last) {
    int page0 = page_at(b), page1 = page_at(b + NW);
    Keys<D> keys[2];
    load_keys<D>(a, slot_at(max(page0, 0), b), k_lane, p_lane, keys[0]);
    auto step = [&](int now, int next) {
      const int page2 = page_at(b + 2 * NW);
      Values<D> values;
      load_values<D>(a, slot_at(max(page0, 0), b), v_lane, p_lane, values);
      load_keys<D>(a, slot_at(max(page1, 0), min(b + NW, last - 1)), k_lane, p_lane, keys[next]);
      const int t0 = b << 5;
      // this lane's positions t0 + 8 g + from .. to; most tiles are seen whole
      const bool whole = page0 >= 0 && t0 + 31 <= pos_lo && t0 >= whole_from;
      const int from = lane_from - t0 - 8 * g, to = page0 < 0 ? -1 : lane_to - t0 - 8 * g;
      attend_tile<D>(keys[now], values, q, cs, qm, !whole, from, to, bits, s);
      page0 = page1;
      page1 = page2;
      b += NW;
    };
    while (true) {
      step(0, 1);
      if (b >= last) break;
      step(1, 0);
      if (b >= last) break;
    }
  }

  // join the wavefronts: the largest score, then sums in their order
  s.l = column_sum(s.l);
  s.pm = column_sum(s.pm);
  if (g == 0) lds_l[wave][r] = s.l, lds_m[wave][r] = top_score(cs, s), lds_shift[wave][r] = s.shift, lds_pm[wave][r] = s.pm;
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<float4_t*>(&lds_o[wave][r][64 * c + 16 * g + 4 * i]) =
          float4_t{s.o[4 * c][i], s.o[4 * c + 1][i], s.o[4 * c + 2][i], s.o[4 * c + 3][i]};
  __syncthreads();
  const int tid = threadIdx.x, oc = tid / (D / 4), od = 4 * (tid % (D / 4));   // this thread's column and channels
  const bool mine = oc < cols;   // for D = 64 the upper half of the threads has none
  float m = kLow, l = 0.0f;
  float4_t o = {};
  if (mine) {
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, lds_m[w][oc]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float e = __builtin_amdgcn_exp2f(lds_m[w][oc] - m - lds_shift[w][oc]);
      l += e * lds_l[w][oc];
      o += e * (*reinterpret_cast<const float4_t*>(&lds_o[w][oc][od]) + lds_pm[w][oc]);
    }
  }
  if (n_act > 1) {
    // leave the split's sums; the last split to arrive adds them all
    float* part = f.partial + (static_cast<int64_t>(unit) * f.n_splits + split) * kPartFloats<D>;
    if (mine) {
      store_through(part + oc * D + od, o[0], o[1]);
      store_through(part + oc * D + od + 2, o[2], o[3]);
      if (od == 0) store_through(part + 16 * D + 2 * oc, l, m);
    }
    wait_for_stores();
    __syncthreads();
    if (tid == 0) lds_ticket = __hip_atomic_fetch_add(f.tickets + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (lds_ticket != static_cast<uint32_t>(n_act - 1)) return;
    if (tid == 0) __hip_atomic_store(f.tickets + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const float* all = f.partial + static_cast<int64_t>(unit) * f.n_splits * kPartFloats<D>;
    // (L, M) of every split and column into LDS at once, then the outputs, eight
    // loads in flight.  (Sharing them out among all threads and weighing them
    // beforehand took 1 us longer: code that runs once waits for its own fetch.)
    float* pairs = &lds_o[0][0][0];
    for (int i = tid; i < 16 * n_act; i += NW * kWave)
      *reinterpret_cast<float2*>(pairs + 2 * i) = load_through(all + (i / 16) * kPartFloats<D> + 16 * D + 2 * (i % 16));
    __syncthreads();
    if (!mine) return;
    m = kLow, l = 0.0f;
    o = float4_t{};
    for (int i = 0; i < n_act; ++i) m = fmaxf(m, pairs[2 * (16 * i + oc) + 1]);
    for (int i0 = 0; i0 < n_act; i0 += 8) {
      float4_t got[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float* p = all + min(i0 + u, n_act - 1) * kPartFloats<D> + oc * D + od;
        const float2 v = load_through(p), w = load_through(p + 2);
        got[u] = float4_t{v.x, v.y, w.x, w.y};
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u < n_act) {
          const float e = __builtin_amdgcn_exp2f(pairs[2 * (16 * (i0 + u) + oc) + 1] - m);
          l += e * pairs[2 * (16 * (i0 + u) + oc)];
          o += e * got[u];
        }
    }
  }
  if (mine) {
    const int c = within * 16 + oc, i = c / f.group, h = head * f.group + (c - i * f.group);
    T* out = static_cast<T*>(f.out) + (sp.first + i) * f.o_token + h * f.o_head + od;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // nothing visible: zeros (and a NaN stays one)
    struct alignas(8) Four {
      T v[4];
    } y;
#pragma unroll
    for (int k = 0; k < 4; ++k) y.v[k] = static_cast<T>(o[k] * inv);
    *reinterpret_cast<Four*>(out) = y;
  }
}

// ---------------------------------------------------------------------------
// Chunks: many queries of a sequence.  A wavefront takes 32 columns (queries of
// one key head's group: G heads of token i, then of token i + 1) on 32x32x16
// instructions, the four wavefronts of a workgroup neighbouring columns, all
// walking the same positions, so that a tile comes once from L2 and is unpacked
// for 32 columns.  A tile takes 269 vector instructions, 1200 cycles (16 scores a
// lane at nine each, one of them an exponential, and 112 for the unpacking), and
// 16 matrix instructions, 512 cycles.  By the counters the former take 75 % of
// the SIMDs' time and the latter 32 %: a SIMD's two wavefronts overlap them
// little, and the time is nearly their sum.  2048 tokens over 8192 positions, 64
// heads over 8, 615 to 650 us by the card, 740 to 780 TFLOP/s; a library product
// of 8192^3 reaches 1130 to 1290.
//
// Layout (lane = 32 h + r): score row 16 u + 8 b + 4 h + j is position
// 8 (2 u + h) + 4 b + j, so that a lane's scores 8 u .. 8 u + 7 are the eight
// positions of octet 2 u + h, the one its words of value codes hold.
typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr int kChunkWaves = 4;
constexpr int kChunkCols = 32 * kChunkWaves;
constexpr int kChunkSplits = 8;       // most workgroups that share a unit of a chunk
constexpr int kChunkMinBlocks = 256;  // least tiles of 32 positions each of them takes
template <int D>
constexpr int kChunkPart = kChunkCols * (D + 2);   // a split's sums, then (L, M) of each column

__device__ __forceinline__ float16_t mfma32(half8_t a, half8_t b, float16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

template <int D>
struct ChunkKeys {
  uint32_t c[D / 16];   // half a row: channels h D/2 ..
  uint32_t p[16];       // parameters of octets h and 2 + h
};
template <int D>
struct ChunkValues {
  uint32_t c[2][D / 32];   // octets h and 2 + h, channels (D / 32) r ..
  uint32_t p[16];
  uint32_t own;            // parameters of position lane % 32, for the largest scale of a tile seen whole
};

__device__ __forceinline__ void load_params16(const __amdgpu_buffer_rsrc_t rs, int p_lane, uint32_t (&out)[16]) {
#pragma unroll
  for (int n = 0; n < 4; ++n) {   // octet h, then 64 bytes on octet 2 + h
    const auto w = __builtin_amdgcn_raw_buffer_load_b128(rs, p_lane, 16 * (n & 1) + 64 * (n >> 1), 0);
    out[4 * n] = w[0], out[4 * n + 1] = w[1], out[4 * n + 2] = w[2], out[4 * n + 3] = w[3];
  }
}

template <int D>
__device__ __forceinline__ void load_chunk_keys(const Kv4Args& a, int64_t slot, int k_lane, int p_lane, ChunkKeys<D>& t) {
  const __amdgpu_buffer_rsrc_t rs = rsrc_of(a.k_codes + slot * (D / 2), 16 * D);
#pragma unroll
  for (int n = 0; n < D / 64; ++n) {
    const auto w = __builtin_amdgcn_raw_buffer_load_b128(rs, k_lane, 16 * n, 0);
    t.c[4 * n] = w[0], t.c[4 * n + 1] = w[1], t.c[4 * n + 2] = w[2], t.c[4 * n + 3] = w[3];
  }
  load_params16(rsrc_of(a.k_params + slot, 32 * 4), p_lane, t.p);
}

template <int D>
__device__ __forceinline__ void load_chunk_values(const Kv4Args& a, int64_t slot, int v_lane, int p_lane, ChunkValues<D>& t) {
  const __amdgpu_buffer_rsrc_t rs = rsrc_of(reinterpret_cast<const uint8_t*>(a.v_codes) + slot * (D / 2), 16 * D);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if constexpr (D == 128) {
      const auto w = __builtin_amdgcn_raw_buffer_load_b128(rs, v_lane, u * 8 * D, 0);
      t.c[u][0] = w[0], t.c[u][1] = w[1], t.c[u][2] = w[2], t.c[u][3] = w[3];
    } else {
      const auto w = __builtin_amdgcn_raw_buffer_load_b64(rs, v_lane, u * 8 * D, 0);
      t.c[u][0] = w[0], t.c[u][1] = w[1];
    }
  }
  const __amdgpu_buffer_rsrc_t ps = rsrc_of(a.v_params + slot, 32 * 4);
  load_params16(ps, p_lane, t.p);
  t.own = __builtin_amdgcn_raw_buffer_load_b32(ps, own_offset(), 0, 0);
}

template <int D>
struct ChunkRunning {
  float16_t o[D / 32];   // channel (D / 32) row + tile
  float l, pm, top, limit, vmax, shift, scale_limit;
};

template <int D>
__device__ __forceinline__ void attend_chunk(const ChunkKeys<D>& k, const ChunkValues<D>& v, const half8_t (&q)[D / 16], float cs,
                                             float qm, bool masked, int from, int to, const Bits& bits, ChunkRunning<D>& s) {
  float16_t acc = {};
#pragma unroll
  for (int j = 0; j < D / 16; ++j) acc = mfma32(operand_of(k.c[j]), q[j], acc);
  float x[16];
  half2_t vp[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    x[i] = fmaf(scale_of(k.p[i]), acc[i], fmaf(minimum_of(k.p[i]), qm, -s.top));
    vp[i] = __builtin_bit_cast(half2_t, v.p[i]);
  }
  float sm = scale_of(v.own), scale_limit = s.scale_limit;
  if (masked) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int at = 16 * (i / 8) + i % 8;
      const bool hidden = at < from || at > to;
      x[i] = hidden ? -INFINITY : x[i];
      vp[i] = hidden ? half2_t{} : vp[i];
    }
    sm = largest_scale(vp);
    scale_limit = s.vmax * kScaleMargin;
  }
  const float xm = largest(x);
  if (__any(xm > s.limit || sm > scale_limit)) {
    const float xc = halves_max(xm), sc = masked ? halves_max(sm) : row_max(column_max(sm));   // unmasked: over the 32 positions
    if (xc > s.limit || sc > scale_limit) {
      const float r = raise_reference(xc, sc, cs, s, x);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) s.o[c] *= r;
    }
    if (!masked && sc > scale_limit) s.scale_limit = sc * kScaleMargin;
  }
  half8_t b[2];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float e = __builtin_amdgcn_exp2f(fmaf(cs, x[i], s.shift)), scale = static_cast<float>(vp[i][0]);
    s.l += e;
    s.pm = fmaf(e, fmaf(scale, 8.0f, static_cast<float>(vp[i][1])), s.pm);
    b[i / 8][2 * (i % 4) + (i % 8) / 4] = static_cast<half_t>(fmaf(e, scale, 0.0f));
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int c = 0; c < D / 32; ++c) s.o[c] = mfma32(centred_of(v.c[u][c], bits), b[u], s.o[c]);
}

template <typename T, int D>
__global__ __launch_bounds__(kChunkWaves* kWave, 2) void chunk_kernel(Kv4Args a, AttnArgs f) {
  __shared__ uint32_t lds_ticket;
  const int lane = threadIdx.x & (kWave - 1), r = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int split = blockIdx.x % f.n_splits, unit = blockIdx.x / f.n_splits;
  const int head = unit % a.heads;
  const int tile = f.tiles - 1 - unit / a.heads;   // a sequence's last queries see the most: they go first
  int within;
  const int seq = find_unit(a, tile, [&](const Span& s) {
    return static_cast<int>((static_cast<int64_t>(s.n) * f.group + kChunkCols - 1) / kChunkCols); }, within);
  if (seq < 0) return;
  const Span sp = span_of(a, seq);
  const int all_cols = min(kChunkCols, sp.n * f.group - within * kChunkCols);   // of this unit
  const int cols = min(32, all_cols - 32 * wave);                               // of this wavefront, may be none
  const int col0 = within * kChunkCols + 32 * wave;
  const int col = col0 + max(min(r, cols - 1), 0);
  const int qi = min(col / f.group, sp.n - 1), qh = head * f.group + (col - col / f.group * f.group);
  const int p0 = static_cast<int>(sp.len) - sp.n;
  auto earliest = [&](int pos) { return f.window ? max(max(pos, -1) - f.window, -1) + 1 : 0; };
  // positions of the unit, which fix the splits, and of this wavefront
  const int unit_lo = p0 + within * kChunkCols / f.group, unit_hi = p0 + (within * kChunkCols + all_cols - 1) / f.group;
  const int hi = min(unit_hi, static_cast<int>(a.capacity) - 1), lo = earliest(unit_lo);
  const int b_lo = lo >> 5;
  const int n_blocks = hi < lo ? 0 : (hi >> 5) - b_lo + 1;
  const int per = max((n_blocks + f.n_splits - 1) / f.n_splits, kChunkMinBlocks);
  const int n_act = max((n_blocks + per - 1) / per, 1);
  if (split >= n_act) return;
  const int first = b_lo + split * per, last = min(first + per, b_lo + n_blocks);

  const int pos_lo = p0 + col0 / f.group, pos_hi = p0 + (col0 + max(cols, 1) - 1) / f.group;
  const int lane_to = max(p0 + qi, -1), lane_from = earliest(lane_to), whole_from = earliest(pos_hi);
  const Bits bits = number_bits();
  ChunkRunning<D> s = {};
  float cs = 1.0f;
  s.limit = kLow, s.vmax = s.scale_limit = 0x1p-30f;
  // tiles this wavefront's columns see
  int b = max(first, earliest(pos_lo) >> 5);
  const int end = cols > 0 && pos_hi >= 0 ? min(last, (pos_hi >> 5) + 1) : 0;
  if (b < end) {
    half8_t q[D / 16];
    float qm;
    load_query<T, D, D / 2>(static_cast<const T*>(f.q) + (sp.first + qi) * f.q_token + qh * f.q_head + h * (D / 2), f.scale, q, cs,
                            qm);
    const int token = 8 * (2 * (r >> 4) + ((r >> 2) & 1)) + 4 * ((r >> 3) & 1) + (r & 3);
    const int k_lane = token * (D / 2) + h * (D / 4), v_lane = h * 4 * D + r * (D / 8), p_lane = 32 * h;
    const int32_t* table = a.table + static_cast<int64_t>(seq) * a.table_stride;
    const int shift = a.page_log2 - 5;
    auto slot_at = [&](int page, int b) {
      return ((static_cast<int64_t>(page) * a.heads + head) << a.page_log2) + ((b & ((1 << shift) - 1)) << 5);
    };
    auto page_at = [&](int b) {
      const int p = __builtin_amdgcn_readfirstlane(table[min(b, end - 1) >> shift]);
      return p >= 0 && p < a.n_pages ? p : -1;
    };
    int page0 = page_at(b), page1 = page_at(b + 1);
    ChunkKeys<D> keys[2];
    load_chunk_keys<D>(a, slot_at(max(page0, 0), b), k_lane, p_lane, keys[0]);
    auto step = [&](int now, int next) {
      const int page2 = page_at(b + 2);
      ChunkValues<D> values;
      load_chunk_values<D>(a, slot_at(max(page0, 0), b), v_lane, p_lane, values);
      load_chunk_keys<D>(a, slot_at(max(page1, 0), min(b + 1, end - 1)), k_lane, p_lane, keys[next]);
      const int t0 = b << 5;
      const bool whole = page0 >= 0 && t0 + 31 <= pos_lo && t0 >= whole_from;
      const int from = lane_from - t0 - 8 * h, to = page0 < 0 ? -1 : lane_to - t0 - 8 * h;
      attend_chunk<D>(keys[now], values, q, cs, qm, !whole, from, to, bits, s);
      page0 = page1;
      page1 = page2;
      ++b;
    };
    while (true) {
      step(0, 1);
      if (b >= end) break;
      step(1, 0);
      if (b >= end) break;
    }
  }
  s.l = halves_sum(s.l);
  s.pm = halves_sum(s.pm);
  constexpr int NT = D / 32;   // channel tiles: a lane's channels come in runs of 4 NT
  const int qi_out = col / f.group;
  T* out = static_cast<T*>(f.out) + (sp.first + qi_out) * f.o_token + qh * f.o_head;
  if (n_act == 1) {
    if (r >= cols) return;
    const float inv = s.l == 0.0f ? 0.0f : 1.0f / s.l;
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 4 * NT; e += 8) {
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = (s.o[(e + k) % NT][4 * n + (e + k) / NT] + s.pm) * inv;
        store8(out + NT * (8 * n + 4 * h) + e, 8, y);
      }
    return;
  }
  float* mine = f.partial + (static_cast<int64_t>(unit) * f.n_splits + split) * kChunkPart<D>;
  if (r < cols) {
    const float unshift = __builtin_amdgcn_exp2f(-s.shift);
    // pairs of channels of the wavefront's 32 columns next to each other, so that
    // a store covers whole lines
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 4 * NT; e += 2)
        store_through(mine + 32 * D * wave + 32 * (NT * (8 * n + 4 * h) + e) + 2 * r,
                      (s.o[e % NT][4 * n + e / NT] + s.pm) * unshift, (s.o[(e + 1) % NT][4 * n + (e + 1) / NT] + s.pm) * unshift);
    if (h == 0) store_through(mine + kChunkCols * D + 2 * (32 * wave + r), s.l * unshift, top_score(cs, s));
  }
  wait_for_stores();
  __syncthreads();
  if (threadIdx.x == 0)
    lds_ticket = __hip_atomic_fetch_add(f.tickets + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (lds_ticket != static_cast<uint32_t>(n_act - 1)) return;
  if (threadIdx.x == 0) __hip_atomic_store(f.tickets + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const float* all = f.partial + static_cast<int64_t>(unit) * f.n_splits * kChunkPart<D>;
  // a thread takes four channels of a column; 32 of them, the columns of a wavefront
  for (int t = threadIdx.x; t < (all_cols + 31) / 32 * 32 * (D / 4); t += kChunkWaves * kWave) {
    const int w = t / (8 * D), c = 32 * w + t % 32, d = 4 * (t / 32 % (D / 4));
    if (c >= all_cols) continue;
    float m = kLow, l = 0.0f;
    float2 lm[kChunkSplits];
    float4_t got[kChunkSplits], o = {};
#pragma unroll
    for (int i = 0; i < kChunkSplits; ++i) {
      const float* p = all + min(i, n_act - 1) * kChunkPart<D>;
      lm[i] = load_through(p + kChunkCols * D + 2 * c);
      const float* pair = p + 32 * D * w + 32 * d + 2 * (t % 32);
      const float2 u = load_through(pair), v = load_through(pair + 64);
      got[i] = float4_t{u.x, u.y, v.x, v.y};
    }
#pragma unroll
    for (int i = 0; i < kChunkSplits; ++i) m = fmaxf(m, lm[i].y);
#pragma unroll
    for (int i = 0; i < kChunkSplits; ++i)
      if (i < n_act) {
        const float e = __builtin_amdgcn_exp2f(lm[i].y - m);
        l += e * lm[i].x;
        o += e * got[i];
      }
    const int at = within * kChunkCols + c, i = at / f.group, hd = head * f.group + (at - i * f.group);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    struct alignas(8) Four {
      T v[4];
    } y;
#pragma unroll
    for (int k = 0; k < 4; ++k) y.v[k] = static_cast<T>(o[k] * inv);
    *reinterpret_cast<Four*>(static_cast<T*>(f.out) + (sp.first + i) * f.o_token + hd * f.o_head + d) = y;
  }
}

// How a call is cut: units are (column tile, key head), every unit shared by up
// to n_splits workgroups; the single-token kernel's column tiles are 16 wide,
// the chunk kernel's kChunkCols.
// Tickets lie at the front of the workspace and take the same room in every call,
// so that one workspace serves calls of any shapes: at most 256 units are shared
// as the shapes suggest, and a call's grid holds at most twice as many.
constexpr size_t kTicketBytes = 2048;

struct Plan {
  bool chunk;
  int64_t tiles, units;
  int tiles_per_seq, n_splits;
  size_t bytes;
};

Plan make_plan(const celty_kv4_cache* c, const celty_kv4_seqs* s, int heads) {
  Plan p;
  const int64_t group = heads / c->kv_heads, all = s->n_tokens * group;
  const int64_t blocks = static_cast<int64_t>(s->max_pages) * (c->page_tokens / 32);
  // Column tiles of a width: at most the first, about the second where only the
  // kernel knows how the tokens are shared out.
  auto tiles_of = [&](int64_t width) { return all / width + s->n_seqs; };
  auto about_of = [&](int64_t width) { return std::max<int64_t>(1, c->kv_heads * std::max<int64_t>(all / width, s->n_seqs)); };
  auto shares = [&](int64_t least) { return std::max<int64_t>(1, (blocks + least - 1) / least); };
  // The chunk kernel takes calls that fill its columns and give it enough
  // workgroups, which a long table helps with: 64 heads over 8, 8192 positions,
  // 128, 256, 512 new tokens (64, 128, 256 units) 88, 133, 212 us against 69, 133,
  // 264 for the other kernel; 65000 positions, 64 and 256 tokens 271 and 719
  // against 246 and 896; 16 sequences of 8 tokens 135 against 81.
  const int64_t chunk_units = about_of(kChunkCols);
  p.chunk = s->q_start && all >= kChunkCols * static_cast<int64_t>(s->n_seqs) && chunk_units >= 64 &&
            chunk_units * shares(kChunkMinBlocks) >= 192;
  p.tiles_per_seq = static_cast<int>((group + 15) / 16);
  p.tiles = p.chunk ? tiles_of(kChunkCols) : s->q_start ? tiles_of(16) : static_cast<int64_t>(s->n_seqs) * p.tiles_per_seq;
  p.units = p.tiles * c->kv_heads;
  // One workgroup for each of 256 compute units (two of the chunk kernel's, which
  // pays from 8192 positions each on: 512 tokens over 20000 449 us against 480,
  // over 8192 224 against 212), as far as the table's length gives them their least tiles.
  const int64_t n = p.chunk ? std::min<int64_t>({kChunkSplits, 512 / chunk_units, shares(kChunkMinBlocks)})
                            : std::min<int64_t>({kMaxSplits, 256 / (s->q_start ? about_of(16) : std::max<int64_t>(1, p.units)),
                                                 shares(kMinBlocks)});
  p.n_splits = static_cast<int>(std::max<int64_t>(n, 1));
  p.bytes = 256;
  if (p.n_splits > 1 && p.units * 4 > static_cast<int64_t>(kTicketBytes)) p.n_splits = 1;
  if (p.n_splits > 1) {
    const size_t floats = p.chunk ? (c->head_dim == 128 ? kChunkPart<128> : kChunkPart<64>)
                                  : (c->head_dim == 128 ? kPartFloats<128> : kPartFloats<64>);
    p.bytes = kTicketBytes + static_cast<size_t>(p.units) * p.n_splits * floats * 4;
  }
  return p;
}

bool attention_sizes_ok(const celty_kv4_cache* c, const celty_kv4_seqs* s, int32_t heads) {
  if (check_cache(c, s) != CELTY_OK || heads < 1 || heads > 65535 || heads % c->kv_heads) return false;
  const Plan p = make_plan(c, s, heads);
  return p.units * p.n_splits <= (1 << 22);   // workgroups of 512 threads in one grid
}

}  // namespace

extern "C" size_t celty_kv4_attention_workspace_bytes(const celty_kv4_cache* cache, const celty_kv4_seqs* seqs,
                                                      int32_t heads) {
  return attention_sizes_ok(cache, seqs, heads) ? make_plan(cache, seqs, heads).bytes : 0;
}

extern "C" celty_status celty_kv4_attention(const celty_kv4_cache* cache, const celty_kv4_seqs* seqs, int32_t dtype,
                                            int32_t heads, const celty_heads* q, const celty_heads* out, float scale,
                                            int32_t window, void* workspace, size_t workspace_bytes, void* stream) {
  if (!attention_sizes_ok(cache, seqs, heads) || check_cache_pointers(cache, seqs) != CELTY_OK) return CELTY_EINVAL;
  if (dtype != CELTY_F16 && dtype != CELTY_BF16) return CELTY_EINVAL;
  if (window < 0 || !std::isfinite(scale)) return CELTY_EINVAL;
  if (check_heads(q, seqs->n_tokens, heads, 0) != CELTY_OK || check_heads(out, seqs->n_tokens, heads, cache->head_dim) != CELTY_OK)
    return CELTY_EINVAL;
  const Plan plan = make_plan(cache, seqs, heads);
  if (!workspace || misaligned(workspace, 256) || workspace_bytes < plan.bytes) return CELTY_EINVAL;
  if (seqs->n_tokens == 0 || seqs->n_seqs == 0) return CELTY_OK;
  const Rows qr = rows_of(q, seqs->n_tokens, heads, cache->head_dim), outr = rows_of(out, seqs->n_tokens, heads, cache->head_dim);
  if (!rows_apart(outr) || rows_overlap(qr, outr)) return CELTY_EINVAL;
  const Kv4Args a = make_args(cache, seqs);
  const AttnArgs f{q->data, out->data, q->token_stride, q->head_stride, out->token_stride, out->head_stride,
                   heads / cache->kv_heads, scale * 1.44269504088896341f, window, plan.n_splits, plan.tiles_per_seq, static_cast<int>(plan.tiles),
                   static_cast<uint32_t*>(workspace), reinterpret_cast<float*>(static_cast<char*>(workspace) + kTicketBytes)};
  const dim3 grid(static_cast<unsigned>(plan.units * plan.n_splits));
  const hipStream_t st = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, grid, dim3(waves * kWave), 0, st, a, f); };
  auto typed = [&](auto t) {
    using T = decltype(t);
    if (plan.chunk)
      cache->head_dim == 128 ? go(chunk_kernel<T, 128>, kChunkWaves) : go(chunk_kernel<T, 64>, kChunkWaves);
    else
      cache->head_dim == 128 ? go(decode_kernel<T, 128>, kDecodeWaves) : go(decode_kernel<T, 64>, kDecodeWaves);
  };
  dtype == CELTY_F16 ? typed(half_t{}) : typed(bf16_t{});
  return hipGetLastError() == hipSuccess ? CELTY_OK : CELTY_EHIP;
}
