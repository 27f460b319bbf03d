// The 4-bit key/value cache (include/celty_decode.h) for gfx950: writing new
// tokens into it and reading tokens back.
//
// The gather is bound by memory (2 x 2 D bytes of fp16 and D + 8 of cache a
// token and head), the append mostly by its vector instructions, 23 a channel;
// one token is bound by the launch.  3486 tokens of 32 heads x 128: append 23 us
// (3.1 TB/s), 19 of them vector instructions on all SIMDs, gather 16 us (4.4
// TB/s).  The unit of work is an octet:
// eight neighbouring positions of one head, which share their words of value
// codes.  A wavefront takes an octet, lane 8 t + s holding channels
// s D/8 .. of token t: a row's minimum and maximum are three exchanges, its
// key codes one store of D/16 bytes a lane, and the value codes become words
// of eight tokens by an exchange between the eight lanes of equal s that
// halves the channels a lane holds at each of three steps.  No exchange goes
// through LDS.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "celty_decode.h"
#include "common.h"
#include "kv4.h"
#include "tensor.h"

namespace {

struct HeadsPair {
  void *k, *v;
  int64_t k_token, k_head, v_token, v_head;
};

// Octets that a span's positions touch.
__device__ __forceinline__ int octets_of(const Span& s) {
  if (s.n == 0) return 0;
  return static_cast<int>(((s.len - 1) >> 3) - ((s.len - s.n) >> 3)) + 1;
}

// This lane's token of octet `index`: its position and its number in the call
// (-1: not one of the call's).
struct Octet {
  int seq, token;
  int64_t pos;   // of this lane's token
};

__device__ __forceinline__ Octet octet_of(const Kv4Args& a, int index) {
  Octet o;
  int within;
  if (a.q_start) {
    o.seq = find_unit(a, index, octets_of, within);
  } else {
    o.seq = index < a.n_seqs ? index : -1;
    within = 0;
  }
  o.token = -1;
  o.pos = -1;
  if (o.seq < 0) return o;
  const Span s = span_of(a, o.seq);
  const int t = (threadIdx.x & (kWave - 1)) >> 3;
  o.pos = ((((s.len - s.n) >> 3) + within) << 3) + t;
  const int64_t i = o.pos - (s.len - s.n);
  if (i >= 0 && i < s.n) o.token = s.first + static_cast<int>(i);
  return o;
}

constexpr int kQuantWaves = 4;
constexpr int64_t kMaxUnits = 1 << 25;   // wavefronts of a grid

// With lane l's value and those of the other seven lanes of its token: the
// exchanges are permutations within rows of lanes (quads of neighbours, then
// the eight mirrored, where the quads agree).
template <typename F>
__device__ __forceinline__ float over_token(float v, F f) {
  auto moved = [](float x, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, false));
  };
  v = f(v, moved(v, std::integral_constant<int, 0xB1>{}));   // quad_perm 1 0 3 2
  v = f(v, moved(v, std::integral_constant<int, 0x4E>{}));   // quad_perm 2 3 0 1
  return f(v, moved(v, std::integral_constant<int, 0x141>{}));   // row_half_mirror
}

// Codes and parameters of a token whose eight lanes hold N channels each.  A
// quotient is taken as a product with the reciprocal, which rounds to another
// code only within 2^-18 of a half (two roundings of a number below 16): where
// any channel of the wavefront comes within 2^-16, the divisions are made.
// Channels beyond fp16's range need no clamp of their own: their quotients are
// beyond the codes'.
template <int N>
__device__ __forceinline__ void quantise(const float (&x)[N], uint32_t (&code)[N], uint32_t& params) {
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) {   // NaN stays
    lo = __builtin_elementwise_minimum(lo, x[i]);
    hi = __builtin_elementwise_maximum(hi, x[i]);
  }
  lo = over_token(lo, [](float a, float b) { return __builtin_elementwise_minimum(a, b); });
  hi = over_token(hi, [](float a, float b) { return __builtin_elementwise_maximum(a, b); });
  const bool bad = lo != lo;
  lo = fminf(fmaxf(lo, -65504.0f), 65504.0f), hi = fminf(fmaxf(hi, -65504.0f), 65504.0f);
  const half_t m = bad ? static_cast<half_t>(NAN) : static_cast<half_t>(lo);
  const half_t s = static_cast<half_t>(__fdiv_rn(hi - static_cast<float>(m), 15.0f));
  const float mf = static_cast<float>(m), sf = static_cast<float>(s);
  const bool steps = sf > 0.0f;   // no: one value, or NaN
  const float inv = steps ? 1.0f / sf : 0.0f;
  // adding 1.5 2^23 rounds to a whole number, to even at a half, and leaves it in the low bits
  constexpr float kRound = 0x1.8p23f;
  bool close = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float q = __builtin_amdgcn_fmed3f((x[i] - mf) * inv, 0.0f, 15.0f), c = q + kRound;
    close |= fabsf(q - (c - kRound)) > 0.5f - 0x1p-16f;
    code[i] = __float_as_uint(c) & 15u;
  }
  if (__any(steps && close)) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      code[i] = __float_as_uint(__builtin_amdgcn_fmed3f(__fdiv_rn(x[i] - mf, steps ? sf : 1.0f), 0.0f, 15.0f) + kRound) & 15u;
  }
  if (__any(!steps)) {
#pragma unroll
    for (int i = 0; i < N; ++i) code[i] = steps ? code[i] : 0u;
  }
  params = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, s)) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, m)) << 16;
}

// N channels of a token, zeros where it is not stored.
template <typename T, int N>
__device__ __forceinline__ void load_row(const void* base, int64_t at, bool on, float (&x)[N]) {
  Vec8<T> q[N / 8] = {};
  if (on) {
#pragma unroll
    for (int j = 0; j < N / 8; ++j) q[j] = *reinterpret_cast<const Vec8<T>*>(static_cast<const T*>(base) + at + 8 * j);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = static_cast<float>(q[i / 8][i % 8]);
}

template <typename T, int D>
__global__ __launch_bounds__(kQuantWaves* kWave) void append_kernel(Kv4Args a, HeadsPair p) {
  constexpr int N = D / 8;   // channels a lane
  const int lane = threadIdx.x & (kWave - 1), t = lane >> 3, sub = lane & 7;
  // heads follow each other: a token's are neighbours in memory
  const int unit = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x) * kQuantWaves + static_cast<int>(threadIdx.x) / kWave);
  const int head = unit % a.heads;
  const Octet o = octet_of(a, unit / a.heads);
  const int page = o.token >= 0 ? page_of(a, o.seq, o.pos) : -1;
  // every token of an octet is in one page: a page holds whole octets
  const bool on = page >= 0;
  const uint64_t stored = __ballot(on);
  if (!stored) return;
  float x[N], y[N];
  uint32_t code[N], params;
  load_row<T>(p.k, o.token * p.k_token + head * p.k_head + sub * N, on, x);
  load_row<T>(p.v, o.token * p.v_token + head * p.v_head + sub * N, on, y);
  quantise(x, code, params);
  if (on) {
    const int64_t slot = slot_of(a, page, head, o.pos);
    uint32_t w[N / 8];
#pragma unroll
    for (int j = 0; j < N / 8; ++j) {
      w[j] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) w[j] |= code[8 * j + i] << (4 * i);
      *reinterpret_cast<uint32_t*>(a.k_codes + slot * (D / 2) + sub * (N / 2) + 4 * j) = w[j];
    }
    if (sub == 0) a.k_params[slot] = params;
  }
  quantise(y, code, params);
  if (on && sub == 0) a.v_params[slot_of(a, page, head, o.pos)] = params;
  // words of eight tokens: at each step a lane keeps half of its channels and
  // hands the other half to the lane whose token differs in one bit, from 4 down
#pragma unroll
  for (int i = 0; i < N; ++i) code[i] = on ? code[i] << (4 * t) : 0u;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const auto w = __builtin_amdgcn_permlane32_swap(code[i], code[N / 2 + i], false, false);
    code[i] = w[0] | w[1];
  }
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const auto w = __builtin_amdgcn_permlane16_swap(code[i], code[N / 4 + i], false, false);
    code[i] = w[0] | w[1];
  }
#pragma unroll
  for (int i = 0; i < N / 8; ++i) {
    const uint32_t keep = t & 1 ? code[N / 8 + i] : code[i], give = t & 1 ? code[i] : code[N / 8 + i];
    code[i] = keep | static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(give), 0x128, 0xF, 0xF, false));   // row_ror:8
  }
  // which page: any stored lane's; which tokens of the octet are new
  const int src = __builtin_ctzll(stored);
  const int pg = __builtin_amdgcn_readlane(page, src);
  uint32_t mask = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) mask |= ((stored >> (8 * i)) & 1u) ? 0xFu << (4 * i) : 0u;
  const int64_t octet = slot_of(a, pg, head, o.pos) >> 3;   // the same for the eight tokens
  const int channel = sub * N + t * (N / 8);
#pragma unroll
  for (int i = 0; i < N / 8; ++i) {
    uint32_t* w = a.v_codes + octet * D + channel + i;
    *w = mask == 0xFFFFFFFFu ? code[i] : (*w & ~mask) | code[i];
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kQuantWaves* kWave) void gather_kernel(Kv4Args a, HeadsPair p) {
  constexpr int N = D / 8;
  const int lane = threadIdx.x & (kWave - 1), t = lane >> 3, sub = lane & 7;
  // heads follow each other: a token's are neighbours in memory
  const int unit = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x) * kQuantWaves + static_cast<int>(threadIdx.x) / kWave);
  const int head = unit % a.heads;
  const Octet o = octet_of(a, unit / a.heads);
  if (o.token < 0) return;
  const int page = page_of(a, o.seq, o.pos);
  float k[N], v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) k[i] = v[i] = 0.0f;
  if (page >= 0) {
    const int64_t slot = slot_of(a, page, head, o.pos);
    const uint32_t kp = a.k_params[slot], vp = a.v_params[slot];
    const float ks = half_bits_to_float(kp & 0xFFFFu), km = half_bits_to_float(kp >> 16);
    const float vs = half_bits_to_float(vp & 0xFFFFu), vm = half_bits_to_float(vp >> 16);
#pragma unroll
    for (int j = 0; j < N / 8; ++j) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(a.k_codes + slot * (D / 2) + sub * (N / 2) + 4 * j);
#pragma unroll
      for (int i = 0; i < 8; ++i) k[8 * j + i] = fmaf(ks, static_cast<float>((w >> (4 * i)) & 15u), km);
    }
    const uint32_t* w = a.v_codes + (slot >> 3) * D + sub * N;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = fmaf(vs, static_cast<float>((w[i] >> (4 * t)) & 15u), vm);
  }
  T* ko = static_cast<T*>(p.k) + o.token * p.k_token + head * p.k_head + sub * N;
  T* vo = static_cast<T*>(p.v) + o.token * p.v_token + head * p.v_head + sub * N;
#pragma unroll
  for (int j = 0; j < N / 8; ++j) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = k[8 * j + i];
    store8(ko + 8 * j, 8, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = v[8 * j + i];
    store8(vo + 8 * j, 8, y);
  }
}

celty_status move_tokens(bool append, const celty_kv4_cache* c, const celty_kv4_seqs* s, int32_t dtype, const celty_heads* k,
                         const celty_heads* v, void* stream) {
  if (check_cache(c, s) != CELTY_OK || check_cache_pointers(c, s) != CELTY_OK) return CELTY_EINVAL;
  if (dtype != CELTY_F16 && dtype != CELTY_BF16) return CELTY_EINVAL;
  const int32_t out = append ? 0 : c->head_dim;   // gather's tensors are written
  if (check_heads(k, s->n_tokens, c->kv_heads, out) != CELTY_OK || check_heads(v, s->n_tokens, c->kv_heads, out) != CELTY_OK)
    return CELTY_EINVAL;
  if (s->n_tokens == 0 || s->n_seqs == 0) return CELTY_OK;
  if (!append) {
    const Rows kr = rows_of(k, s->n_tokens, c->kv_heads, c->head_dim), vr = rows_of(v, s->n_tokens, c->kv_heads, c->head_dim);
    if (!rows_apart(kr) || !rows_apart(vr) || rows_overlap(kr, vr)) return CELTY_EINVAL;
  }
  // at most n / 8 + 2 octets for a sequence's n tokens
  const int64_t octets = s->q_start ? s->n_tokens / 8 + 2 * static_cast<int64_t>(s->n_seqs) : s->n_seqs;
  const int64_t units = octets * c->kv_heads;
  if (units > kMaxUnits) return CELTY_EINVAL;
  const dim3 grid(static_cast<unsigned>((units + kQuantWaves - 1) / kQuantWaves));
  const Kv4Args a = make_args(c, s);
  const HeadsPair p{k->data, v->data, k->token_stride, k->head_stride, v->token_stride, v->head_stride};
  const hipStream_t st = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kQuantWaves * kWave), 0, st, a, p); };
  const bool wide = c->head_dim == 128;
  if (append) {
    if (dtype == CELTY_F16)
      wide ? go(append_kernel<half_t, 128>) : go(append_kernel<half_t, 64>);
    else
      wide ? go(append_kernel<bf16_t, 128>) : go(append_kernel<bf16_t, 64>);
  } else {
    if (dtype == CELTY_F16)
      wide ? go(gather_kernel<half_t, 128>) : go(gather_kernel<half_t, 64>);
    else
      wide ? go(gather_kernel<bf16_t, 128>) : go(gather_kernel<bf16_t, 64>);
  }
  return hipGetLastError() == hipSuccess ? CELTY_OK : CELTY_EHIP;
}

}  // namespace

extern "C" celty_status celty_kv4_append(const celty_kv4_cache* cache, const celty_kv4_seqs* seqs, int32_t dtype,
                                         const celty_heads* k, const celty_heads* v, void* stream) {
  return move_tokens(true, cache, seqs, dtype, k, v, stream);
}

extern "C" celty_status celty_kv4_gather(const celty_kv4_cache* cache, const celty_kv4_seqs* seqs, int32_t dtype,
                                         const celty_heads* k, const celty_heads* v, void* stream) {
  return move_tokens(false, cache, seqs, dtype, k, v, stream);
}
