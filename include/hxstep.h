/*
 * hxstep.h -- C ABI of the operators on either side of a serving step's cache
 * (hxkv.h) on GB300.
 *
 * Before the cache: queries and keys are turned by their positions (rotary
 * positions, Su et al. 2021).  Behind it: the step's logits are adjusted by what each
 * request has said, may say and is asked to say, and the next token is drawn
 * from them.
 *
 * Pointers, streams and errors are as in hxkv.h: device memory of the current device, structs in
 * host memory, every call enqueues its kernel on `stream` and returns, nothing is allocated,
 * and calls can be captured into a graph.  Values in device memory are checked by the
 * kernels, which treat what is out of range as each call says and never read or write outside
 * the arrays described.
 */
#ifndef HXSTEP_H
#define HXSTEP_H

#include "hxkv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Queries and keys of a step, [n_tokens][heads][head_dim], to be turned.  A head's first rotary_dim
 * values are rotary_dim / 2 pairs: values i and i + rotary_dim / 2, or 2i and 2i + 1 if
 * interleaved.  Pair i of a token at position p is turned by p * turns[i] * 2^-64 full turns and multiplied by
 * `scale`; the values behind rotary_dim are copied.  p is positions[token], or follows from the step's
 * rows: row r's tokens are row_start[r] to row_start[r + 1], the last of the kv_len[r] that it holds.
 * Tokens that no row owns are left as they are: nothing is written for them.  (A row that was refused, whose kv_len
 * is 0, has positions below zero.)  An output is its input (the same address and strides) or shares no value
 * with either input, and the outputs none with one another. */
typedef struct hx_rotate_args {
  const void* q;
  const void* k;              /* NULL: queries alone, n_kv_heads is 0 */
  void* q_out;                /* aligned to the type, as q and k */
  void* k_out;
  int64_t q_token_stride, q_head_stride;          /* elements, 0..2^38, and times their number at most 2^44 */
  int64_t k_token_stride, k_head_stride;
  int64_t q_out_token_stride, q_out_head_stride;  /* elements, 0..2^38; no two values at one place */
  int64_t k_out_token_stride, k_out_head_stride;
  int32_t n_tokens;           /* 0..HX_KV_MAX_TOKENS */
  int32_t n_heads;            /* 1..2048 */
  int32_t n_kv_heads;         /* 0..2048 */
  int32_t head_dim;           /* 2..1024 */
  int32_t rotary_dim;         /* even, 2..head_dim */
  int32_t dtype;              /* HX_BF16, HX_F16 or HX_F32 */
  int32_t interleaved;        /* 0 or 1 */
  int32_t inverse;            /* 1: turned the other way and multiplied by scale all the same: the gradient's way, and the way back
                                 where scale is 1 or -1 */
  float scale;                /* finite */
  int32_t n_rows;             /* 1..HX_KV_MAX_ROWS; 0 with positions */
  const uint64_t* turns;      /* [rotary_dim / 2] turns a position, in units of 2^-64 */
  const int32_t* positions;   /* [n_tokens], or NULL */
  const int32_t* row_start;   /* [n_rows + 1]; NULL with positions */
  const int32_t* kv_len;      /* [n_rows] */
} hx_rotate_args;

/* The angles are exact to 2^-32 of a turn at every position, their sines and cosines and the
 * products are in 32 bits, rounded once to dtype. */
int hx_rotate(const hx_rotate_args* a, void* stream);

#define HX_MAX_VOCAB 393216
#define HX_MAX_HISTORY 524287  /* entries of a row */
#define HX_MAX_BIAS 4095       /* entries of a row that count */

/* What holds for the rows of a step's logits.  Every array may be NULL where it says so. */
typedef struct hx_rules {
  int32_t n_rows;             /* 1..HX_KV_MAX_ROWS */
  int32_t history_width;      /* entries of a row of history, 0..HX_MAX_HISTORY */
  const int32_t* history;     /* [n_rows][history_stride] a request's tokens, or NULL; what is no token of the vocabulary is passed over */
  int64_t history_stride;     /* >= history_width */
  const int32_t* length;      /* [n_rows] tokens in history (at most history_width count; below 0: 0) */
  const int32_t* prompt_len;  /* [n_rows] of them the first so many are the prompt, the others were written; NULL: all were written */
  const float* repetition;    /* [n_rows] factor for tokens in history, > 0; NULL: 1 */
  const float* presence;      /* [n_rows] taken off once for tokens that were written; NULL: 0 */
  const float* frequency;     /* [n_rows] taken off as often as they were written; NULL: 0 */
  const int32_t* bias_start;  /* [n_rows + 1] row r's entries are bias_start[r] to bias_start[r + 1] (within 0..n_bias), or NULL */
  const int32_t* bias_token;  /* [n_bias] */
  const float* bias_value;    /* [n_bias] */
  const uint32_t* mask;       /* [n_masks][mask_stride] one bit a token, 1: allowed; or NULL */
  const int32_t* mask_row;    /* [n_rows] which mask holds (out of range: none); NULL: row r's is mask r */
  int64_t mask_stride;        /* words, >= mask_width */
  int32_t n_bias;             /* 0.. */
  int32_t n_masks;            /* >= 1 with a mask; >= n_rows if mask_row is NULL */
  int32_t mask_width;         /* words of a mask: at least ceil(n_vocab / 32) of every call */
} hx_rules;

/* Logits of a step, a row for each request. */
typedef struct hx_logits {
  const void* x;              /* [n_rows][stride], aligned to the type */
  int64_t stride;             /* elements, n_vocab..2^38 */
  int32_t n_rows;             /* 0..HX_KV_MAX_ROWS */
  int32_t n_vocab;            /* 1..HX_MAX_VOCAB */
  int32_t dtype;              /* HX_BF16, HX_F16 or HX_F32 */
} hx_logits;

/* out = adjusted logits, in 32 bits until they are rounded to out's type:
 *   a token in history:  x > 0 ? x / repetition : x * repetition
 *   less  frequency * times written + presence * (written at all)
 *   plus  its bias (the last of the row's entries for it)
 *   a token that the row's mask does not allow: -infinity, whatever x is.
 * out is x itself (the same address, stride and type) or does not overlap it. */
int hx_adjust(const hx_logits* x, const hx_rules* r, void* out, int64_t out_stride, int32_t out_dtype, void* stream);

/* How a row's token is picked from its adjusted logits x.  For each parameter an array by row, or NULL
 * and one value for all rows. */
typedef struct hx_pick {
  const float* noise;         /* [n_rows][noise_stride] random numbers > 0 of the exponential distribution; NULL: the likeliest token, T holds for its logprob */
  int64_t noise_stride;       /* >= n_vocab */
  const float* temperature;   /* T; not above 0: the likeliest token is picked */
  const int32_t* top_k;       /* above 0: only the k likeliest */
  const float* top_p;         /* below 1: only the likeliest, as few as have that share of the top_k's weight */
  const float* min_p;         /* above 0: only those with at least that share of the likeliest's weight */
  float all_temperature, all_top_p, all_min_p;
  int32_t all_top_k;
  int32_t* token;             /* [n_rows] out */
  float* logprob;             /* [n_rows] out, or NULL */
  void* workspace;            /* 16-byte aligned, hx_sample_workspace() bytes; used until the kernels end, by one call at a time */
  int64_t workspace_bytes;
} hx_pick;

/* Bytes of workspace that hx_sample needs for these logits. */
int64_t hx_sample_workspace(const hx_logits* x, const hx_rules* r, const hx_pick* p);

/* Tokens are ordered by x, the larger first, equal ones by their number; weights are exp((x - largest x) / T).
 * What the filters leave is a beginning of that order, of one token at least.  Of it the token with the largest
 * x / T - log(noise) is picked (the lowest of equals), which is one by their weights; logprob is the logarithm of its
 * share of all tokens' weights, before the filters (of exp(x) where T is not above 0).  Tokens with x = -infinity or NaN take no
 * part; a NaN makes the row's logprob NaN.  Where none is left, token is -1 and logprob -infinity.  A noise that is
 * not a finite number of at least 2^-126 never wins; if no token's does, the first of the order is picked.
 * Differences of logits are formed in 32 bits and may become infinite, and T below 1.5e-30 weighs as that.
 * Weights are in 32 bits (their shares within a filter, in 2^-18 of a weight); what decides where the order ends is added up in whole
 * numbers, and scores near the largest are compared in 64 bits: the same inputs give the same token and logprob. */
int hx_sample(const hx_logits* x, const hx_rules* r, const hx_pick* p, void* stream);

#ifdef __cplusplus
}
#endif
#endif
