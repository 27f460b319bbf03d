// What the kernels of the 4-bit key/value cache share (kv4.hip,
// kv4_attention.hip): the cache's addressing, the sequences of a call and the
// host's checks of both.
#ifndef CELTY_CSRC_KV4_H
#define CELTY_CSRC_KV4_H

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "celty_decode.h"
#include "common.h"
#include "tensor.h"

namespace {

// Cache and sequences as the kernels take them.
struct Kv4Args {
  uint8_t* k_codes;
  uint32_t* v_codes;
  uint32_t* k_params;   // fp16 scale in the low half, minimum in the high half
  uint32_t* v_params;
  const int32_t *table, *kv_len, *q_start;
  int heads, n_pages, page_log2, table_stride, n_seqs, n_tokens;
  int64_t capacity;     // positions a sequence's row of the table can name
};

// The call's tokens of one sequence.
struct Span {
  int first, n;      // tokens first .. first + n - 1 of the call
  int64_t len;       // positions of the sequence, the new ones included
};

__device__ __forceinline__ Span span_of(const Kv4Args& a, int seq) {
  Span s;
  s.len = max(a.kv_len[seq], 0);   // no positions; from here on a position's arithmetic fits in 32 bits
  if (a.q_start) {
    const int lo = min(max(a.q_start[seq], 0), a.n_tokens), hi = min(max(a.q_start[seq + 1], 0), a.n_tokens);
    s.first = lo;
    s.n = max(hi - lo, 0);
  } else {
    s.first = seq;
    s.n = 1;
  }
  return s;
}

// Unit `index` of the units that the sequences hold in order, count(span)
// each: its sequence and its number within it; sequence -1 past the last.
// Every lane of the wavefront calls this with the same index.
template <typename Count>
__device__ __forceinline__ int find_unit(const Kv4Args& a, int index, Count count, int& within) {
  const int lane = threadIdx.x & (kWave - 1);
  int base = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
    const int seq = s0 + lane;
    const int c = seq < a.n_seqs ? count(span_of(a, seq)) : 0;
    const int incl = wave_inclusive_scan(c);
    const uint64_t past = __ballot(base + incl > index);
    if (past) {
      const int l = __builtin_ctzll(past);
      within = index - base - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(c, l));
      return s0 + l;
    }
    base += __builtin_amdgcn_readlane(incl, kWave - 1);
  }
  within = 0;
  return -1;
}

// Page of a position, or -1 where it has no storage.
__device__ __forceinline__ int page_of(const Kv4Args& a, int seq, int64_t pos) {
  if (pos < 0 || pos >= a.capacity) return -1;
  const int p = a.table[static_cast<int64_t>(seq) * a.table_stride + (pos >> a.page_log2)];
  return p >= 0 && p < a.n_pages ? p : -1;
}

// Index of (page, head, token within the page) among all tokens and heads.
__device__ __forceinline__ int64_t slot_of(const Kv4Args& a, int page, int head, int64_t pos) {
  return ((static_cast<int64_t>(page) * a.heads + head) << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
}

inline celty_status check_cache(const celty_kv4_cache* c, const celty_kv4_seqs* s) {
  if (!c || !s) return CELTY_EINVAL;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->kv_heads < 1 || c->kv_heads > 65535 || c->n_pages < 1) return CELTY_EINVAL;
  if (c->page_tokens < 32 || (c->page_tokens & (c->page_tokens - 1))) return CELTY_EINVAL;
  // tokens x heads x bytes of a token stay within 62 bits
  const double bytes = 1.0 * c->n_pages * c->kv_heads * c->page_tokens * c->head_dim;
  if (bytes > 4e18) return CELTY_EINVAL;
  if (s->n_seqs < 0 || s->n_tokens < 0 || s->max_pages < 0 || s->table_stride < s->max_pages) return CELTY_EINVAL;
  if (static_cast<int64_t>(s->max_pages) * c->page_tokens > (int64_t{1} << 30)) return CELTY_EINVAL;
  if (s->n_seqs > (1 << 24) || s->n_tokens > (1 << 28)) return CELTY_EINVAL;
  if (!s->q_start && s->n_tokens != s->n_seqs) return CELTY_EINVAL;
  return CELTY_OK;
}

inline celty_status check_cache_pointers(const celty_kv4_cache* c, const celty_kv4_seqs* s) {
  if (!c->k_codes || !c->v_codes || !c->k_params || !c->v_params) return CELTY_EINVAL;
  if (misaligned(c->k_codes, 16) || misaligned(c->v_codes, 16) || misaligned(c->k_params, 16) || misaligned(c->v_params, 16))
    return CELTY_EINVAL;
  if ((s->n_seqs && !s->kv_len) || (s->n_seqs && s->max_pages && !s->block_table)) return CELTY_EINVAL;
  if (misaligned(s->block_table, 4) || misaligned(s->kv_len, 4) || misaligned(s->q_start, 4)) return CELTY_EINVAL;
  return CELTY_OK;
}

// least: the smallest stride that keeps a tensor's rows apart, for one that is written; else 0.
inline celty_status check_heads(const celty_heads* t, int32_t n_tokens, int32_t heads, int32_t least) {
  if (!t || (n_tokens && !t->data) || misaligned(t->data, 16)) return CELTY_EINVAL;
  auto stride_ok = [&](int64_t stride, int32_t count) {   // one along a single element is not looked at
    return count <= 1 || (stride >= least && stride >= 0 && stride % 8 == 0 && stride <= int64_t{1} << 31);
  };
  return stride_ok(t->token_stride, n_tokens) && stride_ok(t->head_stride, heads) ? CELTY_OK : CELTY_EINVAL;
}

// The rows of D channels of a tensor that the checks above let pass.
inline Rows rows_of(const celty_heads* t, int32_t n_tokens, int32_t heads, int32_t D) {
  return {t->data, n_tokens, n_tokens > 1 ? 2 * t->token_stride : 0, heads, heads > 1 ? 2 * t->head_stride : 0, 2 * int64_t{D}};
}

inline Kv4Args make_args(const celty_kv4_cache* c, const celty_kv4_seqs* s) {
  Kv4Args a;
  a.k_codes = c->k_codes;
  a.v_codes = c->v_codes;
  a.k_params = reinterpret_cast<uint32_t*>(c->k_params);
  a.v_params = reinterpret_cast<uint32_t*>(c->v_params);
  a.table = s->block_table;
  a.kv_len = s->kv_len;
  a.q_start = s->q_start;
  a.heads = c->kv_heads;
  a.n_pages = c->n_pages;
  a.page_log2 = __builtin_ctz(static_cast<unsigned>(c->page_tokens));
  a.table_stride = s->table_stride;
  a.n_seqs = s->n_seqs;
  a.n_tokens = s->n_tokens;
  a.capacity = static_cast<int64_t>(s->max_pages) << a.page_log2;
  return a;
}

}  // namespace

#endif  // CELTY_CSRC_KV4_H
