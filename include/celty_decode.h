/*
 * celty_decode.h -- C ABI of libcelty's operators around the sparse products
 * of a decoding step (single-user LLM decoding, Section 1): the norms with
 * the residual update between two products, the key/value cache in 4 bits
 * with the attention that reads it, and the choice of the next token.  The
 * products themselves are in celty.h, whose status codes and general rules
 * hold here too: caller-owned buffers, no exception across the interface,
 * every argument checked on the host before any launch, work enqueued on the
 * given HIP stream (NULL = the default stream) without synchronising.  Every
 * call may be recorded in a HIP graph.
 *
 * Device arrays of integers (block tables, lengths, starts, top_k) are read by
 * the kernels, not by the host: values out of range are defined below and
 * never lead to an access outside the buffers.
 */
#ifndef CELTY_DECODE_H
#define CELTY_DECODE_H

#include "celty.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of tensors. */
#define CELTY_F16 0
#define CELTY_BF16 1
#define CELTY_F32 2

/* ------------------------------------------------------------------------
 * Block norm
 * ------------------------------------------------------------------------ */
#define CELTY_NORM_RMS 0   /* v / sqrt(mean(v^2) + eps) */
#define CELTY_NORM_LAYER 1 /* (v - mean v) / sqrt(mean((v - mean v)^2) + eps) */

/* What celty_block_norm applies.  Every pointer is device memory or NULL
 * (absent) and holds n elements of the call's dtype; gate holds n, or rows x n
 * with row stride ld_gate (0 = the same n for every row). */
typedef struct celty_norm {
  int32_t kind;        /* CELTY_NORM_RMS or CELTY_NORM_LAYER, for both norms */
  int32_t post;        /* 1: the block's output is normalised before it is added */
  float eps;           /* > 0 */
  float alpha;         /* residual scale */
  const void* w_pre;   /* weight and bias of the norm before the next block */
  const void* b_pre;
  const void* w_post;  /* weight and bias of the norm after this block (post = 1) */
  const void* b_post;
  const void* gate;
  int64_t ld_gate;
} celty_norm;

/*
 * The residual update after a block and the norm before the next one, in one
 * launch.  For each of `rows` rows of n elements:
 *
 *     u     = post ? norm(b) * w_post + b_post : b
 *     h_out = h + alpha * gate * u
 *     x     = norm(h_out) * w_pre + b_pre
 *
 * in fp32, x from the fp32 h_out; each output is rounded once (to nearest
 * even).  x in fp16 is the activation celty_spmspv takes.
 *   dtype      CELTY_F16 or CELTY_BF16: b, x, gate, weights and biases.
 *   res_dtype  h and h_out: the same, or CELTY_F32.
 *   h, b, h_out, x   device, row strides ldh, ldb, ldho, ldx (elements, >= n),
 *              aligned to their element.  b NULL: no update (u = 0).  h_out
 *              NULL: not written; x NULL: not written (one of them is
 *              needed).  h_out may be h, and x may be b; any other element
 *              that an output shares with another operand is refused (rows
 *              beside each other in one larger matrix share none).
 * rows = 0 does nothing.
 * Errors: EINVAL (null h or norm, both outputs null, rows < 0, n < 1, bad kind
 *         or dtype, eps not positive and finite, NaN alpha, short stride,
 *         misalignment, overlapping outputs, post weights without post or
 *         without b), EHIP.
 */
celty_status celty_block_norm(int32_t rows, int32_t n, const celty_norm* norm, int32_t dtype, int32_t res_dtype,
                              const void* h, int64_t ldh, const void* b, int64_t ldb, void* h_out, int64_t ldho,
                              void* x, int64_t ldx, void* stream);

/* ------------------------------------------------------------------------
 * The key/value cache in 4 bits
 * ------------------------------------------------------------------------
 * A cache holds n_pages pages of page_tokens tokens for kv_heads heads of
 * head_dim channels D.  A token's D channels of one head, keys and values
 * alike, are kept as D codes c of 4 bits and two fp16 numbers:
 *
 *     m = fp16(min x),  s = fp16((max x - m) / 15),
 *     c = min(max(rint((x - m) / s), 0), 15)  (0 where s = 0),
 *
 * and stand for m + s c.  The quotients are IEEE fp32 divisions; x beyond
 * +-65504 counts as +-65504; a NaN among the channels makes m, and with it all
 * D values, NaN.  D + 8 bytes a token and head, keys and values together.
 */
typedef struct celty_kv4_cache {
  int32_t head_dim;    /* 64 or 128 */
  int32_t kv_heads;
  int32_t page_tokens; /* a power of two, at least 32 */
  int32_t n_pages;
  uint8_t* k_codes;    /* [n_pages][kv_heads][page_tokens][D/2]; channel 2i in the low half of byte i */
  uint32_t* v_codes;   /* [n_pages][kv_heads][page_tokens/8][D]; token t of the page in bits 4(t%8) of word t/8 */
  uint16_t* k_params;  /* [n_pages][kv_heads][page_tokens][2] fp16: s, m */
  uint16_t* v_params;  /* as k_params; all four arrays device, 16-byte aligned */
} celty_kv4_cache;

/* The sequences of a call.  Sequence b's token at position t is in page
 * block_table[b * table_stride + t / page_tokens], at token t % page_tokens.
 * The call's n_tokens tokens belong to the sequences in order: those of b are
 * q_start[b] .. q_start[b+1]-1, the last ones of its kv_len[b] positions
 * (token i of its n is at position kv_len[b] - n + i).  q_start NULL: one
 * token a sequence, n_tokens = n_seqs.
 * A position outside 0 .. max_pages * page_tokens - 1, or whose page number is
 * outside 0 .. n_pages - 1, has no storage: it is not written, reads as zero
 * and is hidden from attention.  q_start is clamped to 0 .. n_tokens; a token
 * that no sequence covers is skipped. */
typedef struct celty_kv4_seqs {
  int32_t n_seqs;
  int32_t n_tokens;
  int32_t max_pages;           /* columns of block_table; max_pages * page_tokens <= 2^30 */
  int32_t table_stride;        /* >= max_pages */
  const int32_t* block_table;  /* device [n_seqs][table_stride] */
  const int32_t* kv_len;       /* device [n_seqs] */
  const int32_t* q_start;      /* device [n_seqs + 1], or NULL */
} celty_kv4_seqs;

/* A [n_tokens][heads][D] tensor in device memory: strides in elements, the
 * channels contiguous, the pointer aligned to 16 bytes and the strides multiples
 * of 8; at least D in a tensor that is written, whose rows of D channels may not
 * share elements with each other or with another operand (a stride along one
 * element is of no matter). */
typedef struct celty_heads {
  void* data;
  int64_t token_stride;
  int64_t head_stride;
} celty_heads;

/*
 * Quantise the call's tokens into the cache.  k, v: [n_tokens][kv_heads][D] of
 * dtype (CELTY_F16 or CELTY_BF16).  Tokens of the cache other than the call's
 * keep their codes.  Two sequences of a call must not write to one page.
 * Errors: EINVAL (null or misaligned pointers, bad sizes, strides or dtype,
 *         more than 2^25 octets of positions, summed over the heads), EHIP.
 */
celty_status celty_kv4_append(const celty_kv4_cache* cache, const celty_kv4_seqs* seqs, int32_t dtype,
                              const celty_heads* k, const celty_heads* v, void* stream);

/* The reverse: the values that the call's tokens stand for, rounded to dtype
 * (CELTY_F16 or CELTY_BF16).  Errors: as celty_kv4_append. */
celty_status celty_kv4_gather(const celty_kv4_cache* cache, const celty_kv4_seqs* seqs, int32_t dtype,
                              const celty_heads* k, const celty_heads* v, void* stream);

/*
 * Causal attention of the call's tokens over the cache (the tokens' own keys
 * and values are appended first):
 *
 *     out_i = sum_j softmax_j(scale * q_i . k_j) v_j
 *
 * over the positions j of the sequence's storage with j <= p_i and, when
 * window > 0, j > p_i - window (p_i the token's position).  A token that sees
 * no position gets zeros; one that sees any gets NaN for a query that is not
 * finite or for a NaN key or value among them.  Query head h reads key head
 * h / (heads / kv_heads).
 *   dtype      CELTY_F16 or CELTY_BF16: q and out, [n_tokens][heads][D].
 *   heads      a multiple of kv_heads.
 *   scale      finite.
 *   workspace  device, at least celty_kv4_attention_workspace_bytes bytes,
 *              zero-filled before first use (celty_spmspv_workspace_init)
 *              and left ready by every completed call, for calls of any
 *              sizes that it is long enough for; calls that may overlap need
 *              workspaces of their own.
 * Sums, maxima and the softmax are in fp32.  What goes into the matrix
 * instructions is in fp16: a query's channels, scaled by a power of two (exact
 * for those above 2^-25 of the token and head's largest, else to 2^-35 of it), and
 * probabilities times the value scales, scaled so that small ones keep their
 * bits.  The latter rounding adds about as much to an fp16 result's error as the
 * result's own (2.1e-4 -> 2.9e-4 in norm).  The result does not depend on timing.
 * Errors: EINVAL (as celty_kv4_append, heads not a multiple of kv_heads,
 *         window < 0, scale not finite, short workspace, out overlapping q,
 *         more than 2^22 workgroups: about a token and key head each for single
 *         tokens, 128 / group tokens for chunks), EHIP.
 */
celty_status celty_kv4_attention(const celty_kv4_cache* cache, const celty_kv4_seqs* seqs, int32_t dtype, int32_t heads,
                                 const celty_heads* q, const celty_heads* out, float scale, int32_t window,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of device workspace for celty_kv4_attention with these sizes (host only, the arrays
 * are not looked at; 0 for sizes that the call refuses). */
size_t celty_kv4_attention_workspace_bytes(const celty_kv4_cache* cache, const celty_kv4_seqs* seqs, int32_t heads);

/* ------------------------------------------------------------------------
 * Sampling
 * ------------------------------------------------------------------------ */
/* Filters of celty_sample: device arrays of `rows` values, or NULL. */
typedef struct celty_filters {
  const float* temperature; /* NULL: 1.  T > 0; T <= 0 or NaN takes the largest logit */
  const int32_t* top_k;     /* NULL or a value < 1: off */
  const float* top_p;       /* NULL or a value >= 1 or NaN: off */
  const float* min_p;       /* NULL or a value <= 0 or NaN: off; above 1: 1 */
} celty_filters;

/*
 * One token per row of logits.  With L the row's largest logit and z = (l - L) / T,
 * w = exp(z), the tokens ordered by falling logit, equal ones by rising index:
 *
 *   top_k   keeps the first top_k tokens;
 *   top_p   of these, keeps a token iff the weights before it sum to less than
 *           top_p times the sum over the top_k tokens;
 *   min_p   of these, keeps a token iff w >= min_p;
 *
 * the first token is always kept, one of weight zero never.  The result is the kept token with the
 * largest z - log(noise) (the lowest index of equal ones): for noise drawn
 * independently from the exponential distribution of rate 1, a draw from the
 * kept weights.
 *   logits  device, rows x V of dtype (CELTY_F16, _BF16 or _F32), row stride
 *           ldl >= V.  NaN and -infinity are never chosen; where +infinity
 *           occurs, only those tokens have weight.
 *   noise   device fp32, rows x V, row stride ldn >= V; read only where a
 *           token is kept, in a row without top_k, top_p and min_p everywhere.  Values below 2^-126 count as 2^-126, NaN as
 *           +infinity.  May be NULL: every row takes its largest logit.
 *   tokens  device int32[rows]; -1 for a row with no number to choose.
 * z, w and z - log(noise) are taken in fp32; weights are summed as multiples of
 * 2^-38 of the largest, rounded down, in 64-bit integers: the result does not
 * depend on timing.  A row whose cut by top_k or top_p falls
 * among more than 4096 tokens of nearly one logit takes about 6 us per thousand
 * logits, for one workgroup finishes it.
 *   workspace  device, at least celty_sample_workspace_bytes(rows, V) bytes (45
 *           KB a row, for 1024 rows at most), any contents; calls that may
 *           overlap need workspaces of their own.
 * Errors: EINVAL (null pointers, rows < 0, V < 1 or V > 2^24, bad dtype, short
 *         stride or workspace, misalignment), EHIP.
 */
celty_status celty_sample(int32_t rows, int32_t V, int32_t dtype, const void* logits, int64_t ldl, const float* noise,
                          int64_t ldn, const celty_filters* filters, int32_t* tokens, void* workspace,
                          size_t workspace_bytes, void* stream);

/* Bytes of device workspace for celty_sample (host only; 0 for sizes that the call refuses). */
size_t celty_sample_workspace_bytes(int32_t rows, int32_t V);

#ifdef __cplusplus
}
#endif

#endif /* CELTY_DECODE_H */
