/*
 * hxkv.h -- C ABI of the serving step's cache operators on GB300.
 *
 * The scheduler simulation (hxsim.h) describes an LLM instance by three
 * numbers: prompt tokens per second, microseconds per output token and
 * concurrent slots (Sec. 3.3's empirical performance profiles).  What an
 * instance does in one step of its running batch is here: it maps the step's
 * tokens to blocks of its cache, writes their keys and values in 8 bits, and
 * attends to everything that each request holds.
 *
 * The cache is paged.  A block holds `block_tokens` tokens of one request;
 * a request's blocks are listed in its row of a block table, position p of the
 * request being place p % block_tokens of entry p / block_tokens.  Keys and values
 * are e4m3 (8-bit floating point, at most 448 in size, no infinities), with
 * one float scale for each block and head, for K and for V: a value is
 * e4m3 * scale.
 *
 * All pointers in the structs are device memory of the current device, the
 * structs themselves host memory that may be freed when the call returns.
 * Every call enqueues its kernels on `stream` (a cudaStream_t, NULL = legacy
 * default) and returns without waiting; nothing is allocated, so the calls
 * can be captured into a graph.  Errors: HX_ERR_INVALID for arguments outside
 * the domains below (with a message, hx_last_error), HX_ERR_CUDA.  Values in
 * device memory cannot be checked before a launch: the kernels check every
 * length, block number and offset that they use, and treat what is out of range as
 * each call says; they never read or write outside the arrays described.
 */
#ifndef HXKV_H
#define HXKV_H

#include "hxsim.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { HX_BF16 = 0, HX_F16 = 1, HX_F32 = 2 };

#define HX_KV_MAX_ROWS 65536
#define HX_KV_MAX_TOKENS (1 << 30) /* tokens of one step */

/* One step's lengths and the tables that they give.  Row r is a request that
 * holds held[r] tokens; add[r] > 0: the step gives it so many more; 0: it
 * does nothing; -1: it has ended and gives its blocks back.
 *
 * Free blocks are a ring of n_blocks entries: ring_state = {first free entry,
 * free blocks}.  In row order each row takes what it needs,
 * ceil((held + add) / block_tokens) - ceil(held / block_tokens), from the ring's
 * front; ended rows' blocks go to its end, in row order, and can be taken from the next step on.
 * A row is refused when the blocks that it and the rows before it need
 * are more than are free, when its table row is too short, when its tokens end past
 * n_tokens, or when a length is malformed (held < 0, add < -1): it takes
 * nothing, its kv_len is 0 and its slots are -1. */
typedef struct hx_kv_map_args {
  int32_t n_rows;             /* 1..HX_KV_MAX_ROWS */
  int32_t n_tokens;           /* length of slots: the step's tokens, 0..HX_KV_MAX_TOKENS */
  int32_t block_tokens;       /* 16, 32, 64 or 128 */
  int32_t n_blocks;           /* blocks of the cache = entries of the ring, >= 1 */
  int32_t table_width;        /* entries of a row of the block table, >= 1 */
  int32_t n_runs;             /* length of runs, >= hx_kv_max_runs() */
  int64_t table_stride;       /* entries from one row to the next, >= table_width */
  const int32_t* held;        /* [n_rows] */
  const int32_t* add;         /* [n_rows] */
  int32_t* block_table;       /* [n_rows][table_stride]: new blocks are entered */
  int32_t* ring;              /* [n_blocks]: ended rows' blocks are entered */
  const int64_t* ring_state;  /* [2] before the step */
  int32_t* row_start;         /* [n_rows + 1] out: first token of each row among the step's (at most n_tokens) */
  int32_t* kv_len;            /* [n_rows] out: tokens held once the step's are in (0: refused or ended) */
  int64_t* slots;             /* [n_tokens] out: block * block_tokens + place of each token, -1: none */
  int32_t* runs;              /* [n_runs][4] out, 16-byte aligned: for each block that the step writes, in token
                                 order: first token, tokens, block, first place; zeros behind them */
  int32_t* counts;            /* [4] out, 16-byte aligned: tokens, runs, refused rows, blocks taken */
  int64_t* ring_state_out;    /* [2] out, not ring_state itself */
} hx_kv_map_args;

/* The runs that n_tokens of n_rows requests can give at most. */
int64_t hx_kv_max_runs(int32_t n_rows, int32_t n_tokens, int32_t block_tokens);

/* Build the tables of one step.  Outputs may not overlap what is read (held may not be this step's kv_len).  The same inputs give the same tables, also when the
 * call is repeated on the table and ring that it has changed. */
int hx_kv_map(const hx_kv_map_args* a, void* stream);

/* A cache: k and v [n_blocks][n_kv_heads][block_tokens][head_dim] e4m3, with
 * block_stride bytes from one block to the next; k_scale and v_scale
 * [n_blocks][n_kv_heads], with scale_stride floats from one block to the next.  A scale under which
 * a token sees something is zero or 2^-110 to 2^100; one that is infinite or no number makes what such tokens get
 * infinite or no number, and that of no other token. */
typedef struct hx_kv_cache {
  void* k;                    /* 16-byte aligned */
  void* v;                    /* 16-byte aligned */
  float* k_scale;
  float* v_scale;
  int64_t block_stride;       /* multiple of 16, >= n_kv_heads * block_tokens * head_dim */
  int64_t scale_stride;       /* >= n_kv_heads */
  int32_t n_blocks;           /* >= 1 */
  int32_t n_kv_heads;         /* 1..1024 */
  int32_t block_tokens;       /* 16, 32, 64 or 128 */
  int32_t head_dim;           /* 64 or 128 */
} hx_kv_cache;

/* A step's keys and values, [n_tokens][n_kv_heads][head_dim] with strides in
 * elements (multiples of 16 bytes) and 16-byte aligned bases. */
typedef struct hx_kv_new {
  const void* k;
  const void* v;
  int64_t k_token_stride, k_head_stride;
  int64_t v_token_stride, v_head_stride;
  int32_t n_tokens;
  int32_t dtype;              /* HX_BF16, HX_F16 or HX_F32 */
  const int32_t* runs;        /* [n_runs][4], as hx_kv_map gives them; every block at most once */
  int32_t n_runs;             /* 0.., n_runs * n_kv_heads below 2^30 */
} hx_kv_new;

/* Write the step's tokens into the cache.  A block's scale is the smallest power of two, 2^-100 at
 * least, that keeps every finite value of the run within 448; a run that does
 * not start its block keeps the block's scale unless it needs a larger one, and then the
 * block's older tokens are rounded to the new scale (a power of two apart: exact but
 * for what falls below e4m3's smallest normal number).  Infinities become +-448 * scale, NaN
 * stays NaN.  Runs that do not lie within the step's tokens, a block and the cache are left out. */
int hx_kv_append(const hx_kv_cache* c, const hx_kv_new* a, void* stream);

/* Queries of a step, [n_tokens][n_heads][head_dim]; heads h * (n_heads / n_kv_heads)
 * and on share kv head h.  Row r's tokens are row_start[r] to row_start[r + 1], the last of
 * the kv_len[r] that it holds. */
typedef struct hx_kv_query {
  const void* q;              /* 16-byte aligned */
  void* out;                  /* 16-byte aligned, same type as q; may not overlap it */
  float* lse;                 /* [n_tokens][n_heads] log of the sum of exponentials (-inf: nothing visible), or NULL */
  int64_t q_token_stride, q_head_stride;      /* elements, multiples of 8, 0..2^38 */
  int64_t out_token_stride, out_head_stride;  /* elements, multiples of 8 */
  int32_t n_tokens;           /* 0.., and n_tokens * n_heads / n_kv_heads at most HX_KV_MAX_TOKENS */
  int32_t n_heads;            /* a multiple of n_kv_heads, at most 128 * n_kv_heads */
  int32_t dtype;              /* HX_BF16 or HX_F16 */
  int32_t n_rows;             /* 1..HX_KV_MAX_ROWS */
  const int32_t* row_start;   /* [n_rows + 1] */
  const int32_t* kv_len;      /* [n_rows] */
  const int32_t* block_table; /* [n_rows][table_stride] */
  int64_t table_stride;
  int32_t table_width;
  int32_t max_q;              /* no row has more tokens in the step (0: not known) */
  int32_t causal;             /* 1: a token sees what is before it and itself; 0: all that its row holds */
  int32_t window;             /* > 0: and of those only positions above its own - window */
  float sm_scale;             /* factor of q.k */
  void* workspace;            /* 32-byte aligned, hx_kv_attend_workspace() bytes; used until the kernels end: a call hands partial
                                 results on through it, so another call may use it only behind all of this one's launches, on the same stream */
  int64_t workspace_bytes;
  int32_t* status;            /* one int in memory that the device can write (host memory mapped for it, or its own), or
                                 NULL: set to 1 if a wait inside a kernel ran out, and never to 0 */
} hx_kv_query;

/* Bytes of workspace that hx_kv_attend needs for these queries. */
int hx_kv_attend_workspace(const hx_kv_cache* c, const hx_kv_query* a, int64_t* bytes);

/* out = softmax(sm_scale * q k^T) v over the positions that each token sees.  A token that sees
 * nothing gets zeros and lse = -inf; so do tokens that no row owns.  Positions past kv_len, in blocks
 * whose number is out of range, or masked take no part, whatever the cache holds there.  A row with more than
 * max_q > 0 tokens gets zeros.  The kernels' waits on their own copies and products are bounded, by about two
 * seconds: a block whose wait runs out leaves NaN in what it had left to compute, and *status says so.  Scores, sums and
 * outputs are in 32 bits until they are rounded to q's type; weights are rounded to 16 bits before they multiply
 * the values (2^-11 of a weight; a weight times its block's value scale that is below 2^-25 of the token's largest may count as
 * zero there, and counts in full in the softmax's sum). */
int hx_kv_attend(const hx_kv_cache* c, const hx_kv_query* a, void* stream);

#ifdef __cplusplus
}
#endif
#endif
