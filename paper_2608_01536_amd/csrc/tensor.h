// Element types, vector loads and workgroup reductions of the decoding
// operators (norm.hip, kv4.hip, sample.hip).
#ifndef CELTY_CSRC_TENSOR_H
#define CELTY_CSRC_TENSOR_H

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "common.h"

namespace {

using half_t = _Float16;
using bf16_t = __bf16;

// Eight elements as they are in memory.
template <typename T>
struct Raw {
  typedef T type __attribute__((ext_vector_type(8)));
};
template <typename T>
using Vec8 = typename Raw<T>::type;

// Eight elements at any element-aligned address: gfx950 takes wide loads and
// stores there, so odd row strides need no path of their own.
template <typename T>
__device__ __forceinline__ Vec8<T> load_whole8(const T* p) {
  Vec8<T> q;
  __builtin_memcpy(&q, p, sizeof(q));
  return q;
}

// The first n of them, zeros after; n may be any number.  TAIL false: n is 8 or
// more, or 0 or less.
template <bool TAIL, typename T>
__device__ __forceinline__ Vec8<T> load_raw8(const T* p, int n) {
  if (n >= 8) return load_whole8(p);
  Vec8<T> q = {};
  if constexpr (TAIL) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) q[i] = p[i];
  }
  return q;
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float (&out)[8]) {
  const Vec8<T> q = load_raw8<true>(p, n);
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = static_cast<float>(q[i]);
}

template <bool TAIL = true, typename T>
__device__ __forceinline__ void store8(T* p, int n, const float (&in)[8]) {
  if (n >= 8) {
    Vec8<T> q;
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = static_cast<T>(in[i]);
    __builtin_memcpy(p, &q, sizeof(q));
  } else if constexpr (TAIL) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = static_cast<T>(in[i]);
  }
}

// All lanes receive the sum (or maximum) over the wavefront, in a fixed order.
template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// All threads receive the sum over a workgroup of NT threads, in a fixed
// order; `lds` holds NT / 64 values that no other reduction uses before the
// next barrier.
template <int NT, typename V>
__device__ __forceinline__ V block_sum(V v, V* lds) {
  v = wave_sum(v);
  if constexpr (NT == kWave) return v;
  if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = v;
  __syncthreads();
  V s = lds[0];
#pragma unroll
  for (int w = 1; w < NT / kWave; ++w) s += lds[w];
  return s;
}

// Address ranges [a, a + n) and [b, b + m) share a byte (host).
inline bool ranges_overlap(const void* a, uint64_t n, const void* b, uint64_t m) {
  const uint64_t x = reinterpret_cast<uint64_t>(a), y = reinterpret_cast<uint64_t>(b);
  return a && b && n && m && x < y + m && y < x + n;
}

// A grid of n x m rows of `width` bytes, `outer` and `inner` bytes apart (host).
struct Rows {
  const void* data;
  int64_t n, outer, m, inner, width;
  uint64_t span() const { return static_cast<uint64_t>((n - 1) * outer + (m - 1) * inner + width); }
};

// Rows of a grid and of another of the same counts and strides, or a single row,
// share a byte; `self`: other than each row with itself.  For each step between
// the m, the least step between the n that is not wholly below.
inline bool rows_meet(const Rows& a, const Rows& b, bool self) {
  const int64_t offset = static_cast<int64_t>(reinterpret_cast<uint64_t>(b.data) - reinterpret_cast<uint64_t>(a.data));
  const int64_t most = a.outer ? a.n - 1 : 0;   // rows on top of each other differ in no step
  if (self && a.n > 1 && !a.outer) return true;
  for (int64_t j = 1 - a.m; j < a.m; ++j) {
    const int64_t base = offset + j * a.inner;
    int64_t i = -most;
    if (most) {
      const int64_t gap = -b.width - base;   // base + i outer must be above -width
      const int64_t least = (gap >= 0 ? gap / a.outer : -((-gap + a.outer - 1) / a.outer)) + 1;
      i = std::max(i, least);
    }
    for (; i <= most; ++i) {
      const int64_t at = base + i * a.outer;
      if (at >= a.width) break;
      if (at > -b.width && !(self && i == 0 && j == 0)) return true;
    }
  }
  return false;
}

// Rows of two tensors share a byte.  Grids of different strides count as sharing
// where their whole ranges do.
inline bool rows_overlap(const Rows& a, const Rows& b) {
  if (!a.data || !b.data || !ranges_overlap(a.data, a.span(), b.data, b.span())) return false;
  const bool same = a.n == b.n && a.m == b.m && (a.n == 1 || a.outer == b.outer) && (a.m == 1 || a.inner == b.inner);
  return !(same || (b.n == 1 && b.m == 1)) || rows_meet(a, b, false);
}

// A tensor's own rows are apart.
inline bool rows_apart(const Rows& a) {
  const auto nested = [&](int64_t small, int64_t count, int64_t large) { return small >= a.width && large >= (count - 1) * small + a.width; };
  if (a.n == 1 && a.m == 1) return true;
  if (a.n == 1) return a.inner >= a.width;
  if (a.m == 1) return a.outer >= a.width;
  return nested(a.inner, a.m, a.outer) || nested(a.outer, a.n, a.inner) || !rows_meet(a, a, true);
}

}  // namespace

#endif  // CELTY_CSRC_TENSOR_H
