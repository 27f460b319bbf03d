// celty_block_norm (include/celty_decode.h): the residual update after a block
// and the norm before the next one, for gfx950.
//
//   u = post ? norm(b) w_post + b_post : b,  h' = h + alpha gate u,
//   x = norm(h') w_pre + b_pre
//
// Bound by memory where there are many rows (each operand is read once, each
// output written once, nothing in between leaves the registers) and by the
// launch, the loads' round trip and the reductions' barriers where there is
// one row.  4096 x 8192 bf16, post norm and gate: 52 us, 5.2 TB/s (copies of its size
// and more reach 5.2 to 5.3); 1 x 4096: 3.8 us in a graph with the post norm.  A workgroup takes
// one row and keeps it in registers as fp32; a reduction is one wavefront tree and
// one barrier.  Layer norms take the
// variance about the mean, not from the sum of squares, which would cancel.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "celty_decode.h"
#include "common.h"
#include "tensor.h"

namespace {

struct NormArgs {
  int n, layer, post;
  float eps, alpha;
  const void *w_pre, *b_pre, *w_post, *b_post, *gate;
  int64_t ld_gate;
  const void *h, *b;
  void *h_out, *x;
  int64_t ldh, ldb, ldho, ldx;
  int64_t row0;   // of the grid's first workgroup
};

// Mean (0 for RMS) and 1 / sqrt(mean square about it + eps) of a row held as
// CH x 8 values a thread, zeros past the row's end (n_here[c] or fewer of a
// chunk's eight are in it).
template <bool TAIL, int NT, int CH>
__device__ __forceinline__ void moments(const float (&v)[CH][8], const int (&n_here)[CH], int n, bool layer, float eps,
                                        float (*lds)[NT / kWave], float& mean, float& rstd) {
  mean = 0.0f;
  if (layer) {
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[c][i];
    mean = block_sum<NT>(s, lds[0]) / static_cast<float>(n);
  }
  float q = 0.0f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if (TAIL || n_here[c] > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = v[c][i] - mean;
        q += !TAIL || i < n_here[c] ? d * d : 0.0f;
      }
    }
  rstd = 1.0f / sqrtf(block_sum<NT>(q, lds[1]) / static_cast<float>(n) + eps);
}

template <typename V>
__device__ __forceinline__ void affine(float (&v)[8], float mean, float rstd, bool weighted, const V& w, bool biased, const V& b) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = (v[i] - mean) * rstd;
    if (weighted) v[i] *= static_cast<float>(w[i]);
    if (biased) v[i] += static_cast<float>(b[i]);
  }
}

// One row per workgroup of NT threads, n <= 8 NT CH.  TAIL: n is no multiple of
// 8, and a row's last chunk is loaded an element at a time.  Without it every
// operand is loaded before the first reduction (1 x 4096 3.34 us against 3.57
// when weights are loaded as they are used, 4096 x 4096 25.9 against 27.6);
// with it that costs registers that it does not repay (333 x 5003 13.2 against
// 10.4).
template <typename T, typename R, int NT, int CH, bool TAIL>
__global__ __launch_bounds__(NT) void norm_kernel(NormArgs a) {
  __shared__ float lds[4][NT / kWave];
  const int64_t row = a.row0 + blockIdx.x;
  int at[CH], n_here[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    at[c] = (c * NT + static_cast<int>(threadIdx.x)) * 8;
    n_here[c] = a.n - at[c];
  }
  const R* hp = static_cast<const R*>(a.h) + row * a.ldh;
  const T* bp = static_cast<const T*>(a.b) + row * a.ldb;
  Vec8<T> gate[CH], w_post[CH], b_post[CH], w_pre[CH], b_pre[CH];
  auto fetch = [&](Vec8<T> (&to)[CH], const void* p, int64_t offset = 0) {
    if (p) {
#pragma unroll
      for (int c = 0; c < CH; ++c) to[c] = load_raw8<TAIL>(static_cast<const T*>(p) + offset + at[c], n_here[c]);
    }
  };
  auto fetch_post = [&] {
    fetch(w_post, a.w_post);
    fetch(b_post, a.b_post);
    fetch(gate, a.gate, row * a.ld_gate);
  };
  auto fetch_pre = [&] {
    if (a.x) {
      fetch(w_pre, a.w_pre);
      fetch(b_pre, a.b_pre);
    }
  };
  float h[CH][8], u[CH][8];
  {
    Vec8<R> h_raw[CH];
    Vec8<T> b_raw[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) h_raw[c] = load_raw8<TAIL>(hp + at[c], n_here[c]);
    if (a.b) {
#pragma unroll
      for (int c = 0; c < CH; ++c) b_raw[c] = load_raw8<TAIL>(bp + at[c], n_here[c]);
    }
    if constexpr (!TAIL) {
      fetch_post();
      fetch_pre();
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[c][i] = static_cast<float>(h_raw[c][i]);
        if (a.b) u[c][i] = static_cast<float>(b_raw[c][i]);
      }
  }
  if (a.b) {
    if constexpr (TAIL) fetch_post();
    if (a.post) {
      float mean, rstd;
      moments<TAIL, NT, CH>(u, n_here, a.n, a.layer, a.eps, &lds[0], mean, rstd);
#pragma unroll
      for (int c = 0; c < CH; ++c) affine(u[c], mean, rstd, a.w_post, w_post[c], a.b_post, b_post[c]);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (TAIL || n_here[c] > 0) {   // past the row's end h stays zero
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float t = a.gate ? u[c][i] * static_cast<float>(gate[c][i]) : u[c][i];
          h[c][i] = !TAIL || i < n_here[c] ? h[c][i] + a.alpha * t : 0.0f;
        }
      }
  }
  if constexpr (TAIL) fetch_pre();
  if (a.h_out) {
    R* op = static_cast<R*>(a.h_out) + row * a.ldho;
#pragma unroll
    for (int c = 0; c < CH; ++c) store8<TAIL>(op + at[c], n_here[c], h[c]);
  }
  if (a.x) {
    float mean, rstd;
    moments<TAIL, NT, CH>(h, n_here, a.n, a.layer, a.eps, &lds[2], mean, rstd);
    T* xp = static_cast<T*>(a.x) + row * a.ldx;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      affine(h[c], mean, rstd, a.w_pre, w_pre[c], a.b_pre, b_pre[c]);
      store8<TAIL>(xp + at[c], n_here[c], h[c]);
    }
  }
}

// Rows too long for the registers (n > 32768): every sum is a pass over the
// row, and the last pass forms h' again and writes both outputs.
template <typename T, typename R>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  constexpr int NT = 1024;
  __shared__ float lds[4][NT / kWave];
  const int64_t row = a.row0 + blockIdx.x;
  const R* hp = static_cast<const R*>(a.h) + row * a.ldh;
  const T* bp = a.b ? static_cast<const T*>(a.b) + row * a.ldb : nullptr;
  const T* gp = a.gate ? static_cast<const T*>(a.gate) + row * a.ld_gate : nullptr;
  const T *wq = static_cast<const T*>(a.w_post), *bq = static_cast<const T*>(a.b_post);
  const T *wp = static_cast<const T*>(a.w_pre), *bb = static_cast<const T*>(a.b_pre);
  float mean_b = 0.0f, rstd_b = 1.0f, mean_h = 0.0f, rstd_h = 1.0f;
  auto block_value = [&](int i) { return static_cast<float>(bp[i]); };
  auto residual = [&](int i) {
    float v = static_cast<float>(hp[i]);
    if (bp) {
      float u = block_value(i);
      if (a.post) {
        u = (u - mean_b) * rstd_b;
        if (wq) u *= static_cast<float>(wq[i]);
        if (bq) u += static_cast<float>(bq[i]);
      }
      if (gp) u *= static_cast<float>(gp[i]);
      v += a.alpha * u;
    }
    return v;
  };
  auto row_moments = [&](auto value, float (*l)[NT / kWave], float& mean, float& rstd) {
    if (a.layer) {
      float s = 0.0f;
      for (int64_t i = threadIdx.x; i < a.n; i += NT) s += value(static_cast<int>(i));
      mean = block_sum<NT>(s, l[0]) / static_cast<float>(a.n);
    }
    float q = 0.0f;
    for (int64_t i = threadIdx.x; i < a.n; i += NT) {
      const float d = value(static_cast<int>(i)) - mean;
      q += d * d;
    }
    rstd = 1.0f / sqrtf(block_sum<NT>(q, l[1]) / static_cast<float>(a.n) + a.eps);
  };
  if (bp && a.post) row_moments(block_value, &lds[0], mean_b, rstd_b);
  if (a.x) row_moments(residual, &lds[2], mean_h, rstd_h);
  for (int64_t j = threadIdx.x; j < a.n; j += NT) {
    const int i = static_cast<int>(j);
    const float v = residual(i);   // h and b are read before the same elements are written
    if (a.h_out) (static_cast<R*>(a.h_out) + row * a.ldho)[i] = static_cast<R>(v);
    if (a.x) {
      float y = (v - mean_h) * rstd_h;
      if (wp) y *= static_cast<float>(wp[i]);
      if (bb) y += static_cast<float>(bb[i]);
      (static_cast<T*>(a.x) + row * a.ldx)[i] = static_cast<T>(y);
    }
  }
}

constexpr int kGridRows = 1 << 21;   // workgroups of up to 1024 threads in one grid

template <typename T, typename R>
void launch_norm(NormArgs a, int rows, hipStream_t st) {
  auto go = [&](auto kernel, int threads) {
    for (a.row0 = 0; a.row0 < rows; a.row0 += kGridRows)
      hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(std::min<int64_t>(kGridRows, rows - a.row0))), dim3(threads), 0, st, a);
  };
  // 8 elements a thread where that fills the workgroup, 16 from 4096 on: two
  // workgroups of 512 on a unit hide each other's reductions (4096 x 8192 in a
  // graph 49 us against 56 for one of 1024).
  auto shaped = [&](auto tail) {
    constexpr bool TAIL = decltype(tail)::value;
    if (a.n <= 512) go(norm_kernel<T, R, 64, 1, TAIL>, 64);
    else if (a.n <= 1024) go(norm_kernel<T, R, 128, 1, TAIL>, 128);
    else if (a.n <= 2048) go(norm_kernel<T, R, 256, 1, TAIL>, 256);
    else if (a.n <= 4096) go(norm_kernel<T, R, 512, 1, TAIL>, 512);
    else if (a.n <= 8192) go(norm_kernel<T, R, 512, 2, TAIL>, 512);
    else if (a.n <= 16384) go(norm_kernel<T, R, 1024, 2, TAIL>, 1024);
    else if (a.n <= 32768) go(norm_kernel<T, R, 1024, 4, TAIL>, 1024);
    else go(norm_long_kernel<T, R>, 1024);
  };
  a.n % 8 ? shaped(std::true_type{}) : shaped(std::false_type{});
}

Rows rows_of(const void* p, int rows, int n, int64_t ld, int size) { return {p, ld ? rows : 1, ld * size, 1, 0, int64_t{1} * n * size}; }

}  // namespace

extern "C" celty_status celty_block_norm(int32_t rows, int32_t n, const celty_norm* norm, int32_t dtype,
                                         int32_t res_dtype, const void* h, int64_t ldh, const void* b, int64_t ldb,
                                         void* h_out, int64_t ldho, void* x, int64_t ldx, void* stream) {
  if (!norm || rows < 0 || n < 1) return CELTY_EINVAL;
  if (dtype != CELTY_F16 && dtype != CELTY_BF16) return CELTY_EINVAL;
  if (res_dtype != dtype && res_dtype != CELTY_F32) return CELTY_EINVAL;
  if (norm->kind != CELTY_NORM_RMS && norm->kind != CELTY_NORM_LAYER) return CELTY_EINVAL;
  if (norm->post != 0 && norm->post != 1) return CELTY_EINVAL;
  if (!(norm->eps > 0.0f) || !std::isfinite(norm->eps) || std::isnan(norm->alpha)) return CELTY_EINVAL;
  if (rows == 0) return CELTY_OK;   // empty tensors may have no address
  if (!h || (!h_out && !x)) return CELTY_EINVAL;
  if ((norm->w_post || norm->b_post) && !norm->post) return CELTY_EINVAL;
  if ((norm->post || norm->gate) && !b) return CELTY_EINVAL;
  const int rs = res_dtype == CELTY_F32 ? 4 : 2;
  if (ldh < n || (b && ldb < n) || (h_out && ldho < n) || (x && ldx < n)) return CELTY_EINVAL;
  if (norm->gate && norm->ld_gate != 0 && norm->ld_gate < n) return CELTY_EINVAL;
  // a row's byte offset stays far within 64 bits
  const int64_t most = int64_t{1} << 31;
  if (ldh > most || (b && ldb > most) || (h_out && ldho > most) || (x && ldx > most) ||
      (norm->gate && norm->ld_gate > most))
    return CELTY_EINVAL;
  for (const void* p : {b, static_cast<const void*>(x), norm->w_pre, norm->b_pre, norm->w_post, norm->b_post, norm->gate})
    if (misaligned(p, 2)) return CELTY_EINVAL;
  if (misaligned(h, rs) || misaligned(h_out, rs)) return CELTY_EINVAL;
  // an output may only be the operand it replaces, row for row
  const Rows hr = rows_of(h, rows, n, ldh, rs), br = rows_of(b, rows, n, ldb, 2);
  const Rows outr = rows_of(h_out, rows, n, ldho, rs), xr = rows_of(x, rows, n, ldx, 2);
  const bool h_in_place = h_out == h && (ldho == ldh || rows == 1), b_in_place = x == b && (ldx == ldb || rows == 1);
  if (rows_overlap(outr, xr)) return CELTY_EINVAL;
  if ((!h_in_place && rows_overlap(outr, hr)) || rows_overlap(outr, br)) return CELTY_EINVAL;
  if ((!b_in_place && rows_overlap(xr, br)) || rows_overlap(xr, hr)) return CELTY_EINVAL;
  for (const void* p : {norm->w_pre, norm->b_pre, norm->w_post, norm->b_post}) {
    const Rows vector = rows_of(p, 1, n, n, 2);
    if (rows_overlap(outr, vector) || rows_overlap(xr, vector)) return CELTY_EINVAL;
  }
  const Rows gr = rows_of(norm->gate, rows, n, norm->ld_gate, 2);
  if (rows_overlap(outr, gr) || rows_overlap(xr, gr)) return CELTY_EINVAL;

  const NormArgs a{n,          norm->kind == CELTY_NORM_LAYER, norm->post, norm->eps,     norm->alpha, norm->w_pre,
                   norm->b_pre, norm->w_post, norm->b_post, norm->gate, norm->ld_gate, h, b, h_out, x, ldh, ldb, ldho, ldx, 0};
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == CELTY_F16)
    res_dtype == CELTY_F32 ? launch_norm<half_t, float>(a, rows, st) : launch_norm<half_t, half_t>(a, rows, st);
  else
    res_dtype == CELTY_F32 ? launch_norm<bf16_t, float>(a, rows, st) : launch_norm<bf16_t, bf16_t>(a, rows, st);
  return hipGetLastError() == hipSuccess ? CELTY_OK : CELTY_EHIP;
}
