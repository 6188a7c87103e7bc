// hx_kv_api.cu -- the C ABI of the cache operators (include/hxkv.h): argument
// checks, then the launches on the caller's stream.
#include <cmath>
#include <cstdio>

#include "hx_kv.cuh"

namespace {

int bad(const char* msg) { return hx::report(HX_ERR_INVALID, msg); }

int launched(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return HX_OK;
  char msg[256];
  snprintf(msg, sizeof msg, "%s: %s", what, cudaGetErrorString(e));
  return hx::report(HX_ERR_CUDA, msg);
}

bool aligned(const void* p, uintptr_t n = 16) { return ((uintptr_t)p & (n - 1)) == 0; }
struct Range {
  const void* p;
  int64_t bytes;
};
bool overlap(const Range& x, const Range& y) {
  const uintptr_t a = (uintptr_t)x.p, b = (uintptr_t)y.p;
  return x.bytes > 0 && y.bytes > 0 && (a < b ? b - a < (uint64_t)x.bytes : a - b < (uint64_t)y.bytes);
}
bool block_size(int b) { return b == 16 || b == 32 || b == 64 || b == 128; }

int check_cache(const hx_kv_cache* c) {
  if (!c) return bad("cache is NULL");
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return bad("cache: NULL pointer");
  if (c->n_blocks < 1) return bad("cache: n_blocks must be at least 1");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return bad("cache: n_kv_heads must be 1..1024");
  if (!block_size(c->block_tokens)) return bad("cache: block_tokens must be 16, 32, 64 or 128");
  if (c->head_dim != 64 && c->head_dim != 128) return bad("cache: head_dim must be 64 or 128");
  if (!aligned(c->k) || !aligned(c->v)) return bad("cache: k and v must be 16-byte aligned");
  if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return bad("cache: the scales must be 4-byte aligned");
  if (c->block_stride % 16 || c->block_stride < (int64_t)c->n_kv_heads * c->block_tokens * c->head_dim)
    return bad("cache: block_stride must be a multiple of 16 and at least one block");
  if (c->scale_stride < c->n_kv_heads) return bad("cache: scale_stride is less than n_kv_heads");
  return HX_OK;
}

int check_query(const hx_kv_cache* c, const hx_kv_query* a) {
  if (int rc = check_cache(c)) return rc;
  if (!a) return bad("queries are NULL");
  if (a->n_tokens < 0 || a->n_tokens > HX_KV_MAX_TOKENS) return bad("queries: n_tokens must be 0..2^30");
  if (a->n_rows < 1 || a->n_rows > HX_KV_MAX_ROWS) return bad("queries: n_rows must be 1..65536");
  if (a->n_heads < 1 || a->n_heads % c->n_kv_heads || a->n_heads / c->n_kv_heads > 128)
    return bad("queries: n_heads must be a multiple of n_kv_heads, at most 128 times it");
  if ((int64_t)a->n_tokens * (a->n_heads / c->n_kv_heads) > HX_KV_MAX_TOKENS)
    return bad("queries: n_tokens * (n_heads / n_kv_heads) must be at most 2^30");
  if (a->dtype != HX_BF16 && a->dtype != HX_F16) return bad("queries: dtype must be bf16 or f16");
  if (a->max_q < 0) return bad("queries: max_q is negative");
  if (a->causal != 0 && a->causal != 1) return bad("queries: causal must be 0 or 1");
  if (a->window < 0) return bad("queries: window is negative");
  if (!std::isfinite(a->sm_scale)) return bad("queries: sm_scale is not finite");
  if (!aligned(a->status, 4)) return bad("queries: status must be 4-byte aligned");
  return HX_OK;
}

}  // namespace

extern "C" {

int64_t hx_kv_max_runs(int32_t n_rows, int32_t n_tokens, int32_t block_tokens) {
  if (n_rows < 0 || n_tokens < 0 || block_tokens < 1) return 0;
  const int64_t by_block = (int64_t)n_tokens / block_tokens + 2 * (int64_t)n_rows;
  return by_block < n_tokens ? by_block : n_tokens;
}

int hx_kv_map(const hx_kv_map_args* a, void* stream) {
  if (!a) return bad("map: NULL argument");
  if (a->n_rows < 1 || a->n_rows > HX_KV_MAX_ROWS) return bad("map: n_rows must be 1..65536");
  if (a->n_tokens < 0 || a->n_tokens > HX_KV_MAX_TOKENS) return bad("map: n_tokens must be 0..2^30");
  if (!block_size(a->block_tokens)) return bad("map: block_tokens must be 16, 32, 64 or 128");
  if (a->n_blocks < 1) return bad("map: n_blocks must be at least 1");
  if (a->table_width < 1 || a->table_width > (1 << 23)) return bad("map: table_width must be 1..2^23");
  if (a->table_stride < a->table_width) return bad("map: table_stride is less than table_width");
  if (a->n_runs < hx_kv_max_runs(a->n_rows, a->n_tokens, a->block_tokens)) return bad("map: n_runs is too small");
  if (!a->held || !a->add || !a->block_table || !a->ring || !a->ring_state || !a->row_start || !a->kv_len ||
      !a->counts || !a->ring_state_out || (a->n_tokens && !a->slots) || (a->n_runs && !a->runs))
    return bad("map: NULL pointer");
  if (a->ring_state == a->ring_state_out) return bad("map: ring_state_out must not be ring_state");
  if (!aligned(a->runs) || !aligned(a->counts)) return bad("map: runs and counts must be 16-byte aligned");
  if (!aligned(a->held, 4) || !aligned(a->add, 4) || !aligned(a->block_table, 4) || !aligned(a->ring, 4) ||
      !aligned(a->row_start, 4) || !aligned(a->kv_len, 4) || !aligned(a->ring_state, 8) || !aligned(a->ring_state_out, 8) ||
      !aligned(a->slots, 8))
    return bad("map: an array is not aligned to its type");
  const int64_t n = a->n_rows;
  const Range lengths[] = {{a->held, 4 * n}, {a->add, 4 * n}, {a->ring_state, 16}, {a->ring, 4 * (int64_t)a->n_blocks}};
  const Range out[] = {{a->row_start, 4 * (n + 1)}, {a->kv_len, 4 * n}, {a->slots, 8 * (int64_t)a->n_tokens},
                       {a->runs, 16 * (int64_t)a->n_runs}, {a->counts, 16}, {a->ring_state_out, 16}};
  const Range table = {a->block_table, 4 * ((n - 1) * a->table_stride + a->table_width)};
  for (const Range& y : out) {
    for (const Range& x : lengths)
      if (overlap(x, y)) return bad("map: an output overlaps held, add, ring or ring_state");
    if (!overlap(table, y)) continue;
    for (int64_t r = 0; r < n; ++r)  // its rows; what lies between them may be anything
      if (overlap({a->block_table + r * a->table_stride, 4 * (int64_t)a->table_width}, y))
        return bad("map: an output overlaps block_table");
  }
  return launched(hx::launch_kv_map(*a, (cudaStream_t)stream), "map");
}

int hx_kv_append(const hx_kv_cache* c, const hx_kv_new* a, void* stream) {
  if (int rc = check_cache(c)) return rc;
  if (!a) return bad("append: NULL argument");
  if (a->n_tokens < 0 || a->n_tokens > HX_KV_MAX_TOKENS) return bad("append: n_tokens must be 0..2^30");
  if (a->n_runs < 0 || a->n_runs > HX_KV_MAX_TOKENS) return bad("append: n_runs must be 0..2^30");
  if (a->dtype < HX_BF16 || a->dtype > HX_F32) return bad("append: dtype must be bf16, f16 or f32");
  if (a->n_tokens == 0 || a->n_runs == 0) return HX_OK;
  if (2 * (int64_t)a->n_runs * c->n_kv_heads > 0x7fffffff) return bad("append: n_runs * n_kv_heads must be below 2^30");
  if (!a->k || !a->v || !a->runs) return bad("append: NULL pointer");
  if (!aligned(a->k) || !aligned(a->v) || !aligned(a->runs)) return bad("append: k, v and runs must be 16-byte aligned");
  const int64_t unit = a->dtype == HX_F32 ? 4 : 8;
  if (a->k_token_stride % unit || a->k_head_stride % unit || a->v_token_stride % unit || a->v_head_stride % unit)
    return bad("append: strides must be multiples of 16 bytes");
  return launched(hx::launch_kv_append(*c, *a, (cudaStream_t)stream), "append");
}

int hx_kv_attend_workspace(const hx_kv_cache* c, const hx_kv_query* a, int64_t* bytes) {
  if (int rc = check_query(c, a)) return rc;
  if (!bytes) return bad("workspace: NULL argument");
  *bytes = hx::kv_attend_workspace(*c, *a);
  return HX_OK;
}

int hx_kv_attend(const hx_kv_cache* c, const hx_kv_query* a, void* stream) {
  if (int rc = check_query(c, a)) return rc;
  if (a->n_tokens == 0) return HX_OK;
  if (!a->q || !a->out || !a->row_start || !a->kv_len || !a->block_table) return bad("queries: NULL pointer");
  if (a->table_width < 1 || a->table_width > (1 << 23)) return bad("queries: table_width must be 1..2^23");
  if (a->table_stride < a->table_width) return bad("queries: table_stride is less than table_width");
  if (!aligned(a->q) || !aligned(a->out)) return bad("queries: q and out must be 16-byte aligned");
  if (!aligned(a->lse, 4) || !aligned(a->row_start, 4) || !aligned(a->kv_len, 4) || !aligned(a->block_table, 4))
    return bad("queries: lse, row_start, kv_len and block_table must be 4-byte aligned");
  if (a->q_token_stride % 8 || a->q_head_stride % 8 || a->out_token_stride % 8 || a->out_head_stride % 8)
    return bad("queries: strides must be multiples of 8 elements");
  if (a->q_token_stride < 0 || a->q_head_stride < 0 || a->q_token_stride >= (int64_t)1 << 38 || a->q_head_stride >= (int64_t)1 << 38)
    return bad("queries: q's strides must be 0..2^38");
  const int64_t need = hx::kv_attend_workspace(*c, *a);
  if (a->workspace_bytes < need || (need && !a->workspace)) return bad("queries: workspace is too small");
  if (need && !aligned(a->workspace, 32)) return bad("queries: workspace must be 32-byte aligned");
  return launched(hx::launch_kv_attend(*c, *a, (cudaStream_t)stream), "attend");
}

}  // extern "C"
