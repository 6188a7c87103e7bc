// hx_step_api.cu -- the C ABI of the operators on either side of the cache
// (include/hxstep.h): argument checks, then the launches on the caller's stream.
#include <cmath>
#include <cstdio>
#include <utility>

#include "hx_step.cuh"

namespace {

int bad(const char* msg) { return hx::report(HX_ERR_INVALID, msg); }

int launched(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return HX_OK;
  char msg[256];
  snprintf(msg, sizeof msg, "%s: %s", what, cudaGetErrorString(e));
  return hx::report(HX_ERR_CUDA, msg);
}

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int size_of(int dtype) { return dtype == HX_F32 ? 4 : 2; }

struct Range {
  const void* p;
  int64_t bytes;
};
bool overlap(const Range& x, const Range& y) {
  const uintptr_t a = (uintptr_t)x.p, b = (uintptr_t)y.p;
  return x.bytes > 0 && y.bytes > 0 && (a < b ? b - a < (uint64_t)x.bytes : a - b < (uint64_t)y.bytes);
}

// Values in rows of `dim`, `rows` of them `row_stride` apart, `outer` times `outer_stride` apart, in bytes; the
// inner stride is the smaller one.
struct Places {
  uintptr_t p;
  int64_t outer, outer_stride, rows, row_stride, dim;
  int64_t inner() const { return (rows - 1) * row_stride + dim; }
  Range range() const { return {(const void*)p, (outer - 1) * outer_stride + inner()}; }
  bool apart() const { return (rows == 1 || row_stride >= dim) && (outer == 1 || outer_stride >= inner()); }
};
Places places(const void* p, int64_t tokens, int64_t token_stride, int64_t heads, int64_t head_stride, int64_t dim, int size) {
  Places a = {(uintptr_t)p, tokens, token_stride * size, heads, head_stride * size, dim * size};
  if (tokens == 1) a.outer_stride = 0;
  if (heads == 1) a.row_stride = 0;
  if (tokens > 1 && heads > 1 && token_stride < head_stride) {
    std::swap(a.outer, a.rows);
    std::swap(a.outer_stride, a.row_stride);
  }
  return a;
}
// Whether two arrays may share a byte.  They do not where one lies behind the other, or in the gaps of the other's heads or
// tokens, which repeat at the same distance in both: q, k and v of a token side by side.
bool meet(const Places& a, const Places& b) {
  if (!overlap(a.range(), b.range())) return false;
  auto gap = [&](int64_t period, int64_t mine, int64_t its) {
    if (period <= 0 || mine > period || its > period) return false;
    int64_t d = (int64_t)(b.p - a.p) % period;
    if (d < 0) d += period;
    return d >= mine && d + its <= period;
  };
  auto one = [](int64_t n, int64_t stride, int64_t other) { return n == 1 ? other : stride; };  // a stride of one is of no matter
  const int64_t ao = one(a.outer, a.outer_stride, b.outer_stride), bo = one(b.outer, b.outer_stride, a.outer_stride);
  if (ao == bo && gap(ao, a.inner(), b.inner())) return false;
  const int64_t ar = one(a.rows, a.row_stride, b.row_stride), br = one(b.rows, b.row_stride, a.row_stride);
  if (ar == br && ar > 0 && (a.outer == 1 || a.outer_stride % ar == 0) && (b.outer == 1 || b.outer_stride % ar == 0) &&
      gap(ar, a.dim, b.dim))
    return false;
  return true;
}

int check_rules(const hx_logits* x, const hx_rules* r) {
  if (r->n_rows != x->n_rows) return bad("rules: n_rows is not the logits'");
  if (r->history) {
    if (r->history_width < 0 || r->history_width > HX_MAX_HISTORY) return bad("rules: history_width must be 0..524287");
    if (r->history_stride < r->history_width) return bad("rules: history_stride is less than history_width");
    if (!r->length) return bad("rules: a history needs length");
  }
  if (r->bias_start) {
    if (r->n_bias < 0) return bad("rules: n_bias is negative");
    if (r->n_bias && (!r->bias_token || !r->bias_value)) return bad("rules: NULL pointer of biases");
  }
  if (r->mask) {
    if (r->n_masks < 1) return bad("rules: n_masks must be at least 1");
    if (!r->mask_row && r->n_masks < r->n_rows) return bad("rules: without mask_row there must be a mask for each row");
    if (r->mask_width < (x->n_vocab + 31) / 32) return bad("rules: a mask has fewer bits than the vocabulary has tokens");
    if (r->mask_stride < r->mask_width) return bad("rules: mask_stride is less than mask_width");
  }
  const void* words[] = {r->history, r->length, r->prompt_len, r->repetition, r->presence, r->frequency,
                         r->bias_start, r->bias_token, r->bias_value, r->mask, r->mask_row};
  for (const void* p : words)
    if (!aligned(p, 4)) return bad("rules: arrays must be 4-byte aligned");
  return HX_OK;
}

int check_logits(const hx_logits* x) {
  if (!x) return bad("logits are NULL");
  if (x->n_rows < 0 || x->n_rows > HX_KV_MAX_ROWS) return bad("logits: n_rows must be 0..65536");
  if (x->n_vocab < 1 || x->n_vocab > HX_MAX_VOCAB) return bad("logits: n_vocab must be 1..393216");
  if (x->dtype < HX_BF16 || x->dtype > HX_F32) return bad("logits: dtype must be bf16, f16 or f32");
  if (x->stride < x->n_vocab || x->stride >= (int64_t)1 << 38) return bad("logits: stride must be n_vocab..2^38");
  if (x->n_rows && !x->x) return bad("logits: NULL pointer");
  if (!aligned(x->x, size_of(x->dtype))) return bad("logits: not aligned to their type");
  return HX_OK;
}

Range of_rows(const void* p, int64_t rows, int64_t stride, int64_t width, int size) {
  return {p, p && rows ? ((rows - 1) * stride + width) * size : 0};
}

// Whether an output shares a byte with what the rules are read from.
bool over_rules(const hx_rules& r, const Range& out) {
  const int64_t n = r.n_rows;
  const Range in[] = {of_rows(r.history, n, r.history_stride, r.history_width, 4),
                      of_rows(r.length, 1, 0, n, 4), of_rows(r.prompt_len, 1, 0, n, 4), of_rows(r.repetition, 1, 0, n, 4),
                      of_rows(r.presence, 1, 0, n, 4), of_rows(r.frequency, 1, 0, n, 4), of_rows(r.bias_start, 1, 0, n + 1, 4),
                      of_rows(r.bias_token, 1, 0, r.n_bias, 4), of_rows(r.bias_value, 1, 0, r.n_bias, 4),
                      of_rows(r.mask, r.n_masks, r.mask_stride, r.mask_width, 4), of_rows(r.mask_row, 1, 0, n, 4)};
  for (const Range& x : in)
    if (overlap(x, out)) return true;
  return false;
}

}  // namespace

extern "C" {

int hx_rotate(const hx_rotate_args* a, void* stream) {
  if (!a) return bad("rotate: NULL argument");
  if (a->n_tokens < 0 || a->n_tokens > HX_KV_MAX_TOKENS) return bad("rotate: n_tokens must be 0..2^30");
  if (a->n_heads < 1 || a->n_heads > 2048) return bad("rotate: n_heads must be 1..2048");
  if (a->n_kv_heads < 0 || a->n_kv_heads > 2048) return bad("rotate: n_kv_heads must be 0..2048");
  if (a->n_tokens && (a->n_kv_heads == 0) != (a->k == nullptr)) return bad("rotate: k must be NULL where n_kv_heads is 0, and only there");
  if (a->head_dim < 2 || a->head_dim > 1024) return bad("rotate: head_dim must be 2..1024");
  if (a->rotary_dim < 2 || a->rotary_dim > a->head_dim || a->rotary_dim % 2) return bad("rotate: rotary_dim must be even, 2..head_dim");
  if (a->dtype < HX_BF16 || a->dtype > HX_F32) return bad("rotate: dtype must be bf16, f16 or f32");
  if ((a->interleaved | a->inverse) & ~1) return bad("rotate: interleaved and inverse must be 0 or 1");
  if (!std::isfinite(a->scale)) return bad("rotate: scale is not finite");
  if (a->n_tokens == 0) return HX_OK;
  if (a->positions ? a->n_rows != 0 || a->row_start || a->kv_len : a->n_rows < 1 || a->n_rows > HX_KV_MAX_ROWS)
    return bad("rotate: either positions or n_rows of 1..65536 with row_start and kv_len");
  if (!a->q || !a->q_out || (a->k && !a->k_out) || !a->turns || (!a->positions && (!a->row_start || !a->kv_len)))
    return bad("rotate: NULL pointer");
  const int size = size_of(a->dtype);
  if (!aligned(a->q, size) || !aligned(a->q_out, size) || !aligned(a->k, size) || !aligned(a->k_out, size))
    return bad("rotate: q, k and their outputs must be aligned to their type");
  if (!aligned(a->turns, 8) || !aligned(a->positions, 4) || !aligned(a->row_start, 4) || !aligned(a->kv_len, 4))
    return bad("rotate: an array is not aligned to its type");
  const int64_t strides[] = {a->q_token_stride, a->q_head_stride, a->q_out_token_stride, a->q_out_head_stride,
                             a->k_token_stride, a->k_head_stride, a->k_out_token_stride, a->k_out_head_stride};
  for (int i = 0; i < (a->k ? 8 : 4); ++i)
    if (strides[i] < 0 || strides[i] >= (int64_t)1 << 38) return bad("rotate: strides must be 0..2^38");
  const int64_t T = a->n_tokens, D = a->head_dim;
  for (int i = 0; i < (a->k ? 8 : 4); ++i)  // so that no place below overflows
    if (strides[i] > ((int64_t)1 << 44) / (i % 2 == 0 ? T : i < 4 ? a->n_heads : a->n_kv_heads))
      return bad("rotate: an array spans more than 2^44 values");
  const Places q = places(a->q, T, a->q_token_stride, a->n_heads, a->q_head_stride, D, size);
  const Places qo = places(a->q_out, T, a->q_out_token_stride, a->n_heads, a->q_out_head_stride, D, size);
  if (!qo.apart()) return bad("rotate: two values of q_out are at one place");
  const bool q_here = a->q == a->q_out;
  if (q_here && (q.outer_stride != qo.outer_stride || q.row_stride != qo.row_stride || q.outer != qo.outer))
    return bad("rotate: q_out is q with other strides");
  if (!q_here && meet(q, qo)) return bad("rotate: q_out overlaps q");
  const int64_t angles = a->rotary_dim / 2;
  const Range in[] = {{a->turns, 8 * angles}, {a->positions, a->positions ? 4 * T : 0},
                      {a->row_start, a->row_start ? 4 * ((int64_t)a->n_rows + 1) : 0}, {a->kv_len, a->kv_len ? 4 * (int64_t)a->n_rows : 0}};
  for (const Range& x : in)
    if (overlap(x, qo.range())) return bad("rotate: q_out overlaps turns, positions, row_start or kv_len");
  if (a->k) {
    const Places k = places(a->k, T, a->k_token_stride, a->n_kv_heads, a->k_head_stride, D, size);
    const Places ko = places(a->k_out, T, a->k_out_token_stride, a->n_kv_heads, a->k_out_head_stride, D, size);
    if (!ko.apart()) return bad("rotate: two values of k_out are at one place");
    const bool k_here = a->k == a->k_out;
    if (k_here && (k.outer_stride != ko.outer_stride || k.row_stride != ko.row_stride || k.outer != ko.outer))
      return bad("rotate: k_out is k with other strides");
    if (!k_here && meet(k, ko)) return bad("rotate: k_out overlaps k");
    if (meet(q, ko) || meet(k, qo) || meet(qo, ko)) return bad("rotate: an output overlaps the other's values");
    for (const Range& x : in)
      if (overlap(x, ko.range())) return bad("rotate: k_out overlaps turns, positions, row_start or kv_len");
  }
  return launched(hx::launch_rotate(*a, (cudaStream_t)stream), "rotate");
}

int hx_adjust(const hx_logits* x, const hx_rules* r, void* out, int64_t out_stride, int32_t out_dtype, void* stream) {
  if (int rc = check_logits(x)) return rc;
  if (!r) return bad("rules are NULL");
  if (int rc = check_rules(x, r)) return rc;
  if (out_dtype != x->dtype && out_dtype != HX_F32) return bad("adjust: out's type must be the logits' or f32");
  if (out_stride < x->n_vocab || out_stride >= (int64_t)1 << 38) return bad("adjust: out_stride must be n_vocab..2^38");
  if (x->n_rows == 0) return HX_OK;
  if (!out) return bad("adjust: NULL pointer");
  if (!aligned(out, size_of(out_dtype))) return bad("adjust: out is not aligned to its type");
  const Range to = of_rows(out, x->n_rows, out_stride, x->n_vocab, size_of(out_dtype));
  const bool here = out == x->x && out_dtype == x->dtype && (out_stride == x->stride || x->n_rows == 1);
  if (!here && overlap(to, of_rows(x->x, x->n_rows, x->stride, x->n_vocab, size_of(x->dtype))))
    return bad("adjust: out overlaps the logits");
  if (over_rules(*r, to)) return bad("adjust: out overlaps the rules");
  return launched(hx::launch_adjust(*x, *r, out, out_stride, out_dtype, (cudaStream_t)stream), "adjust");
}

int64_t hx_sample_workspace(const hx_logits* x, const hx_rules* r, const hx_pick* p) {
  if (check_logits(x) || !p || (r && check_rules(x, r))) return 0;
  return hx::sample_workspace(*x, *p);
}

int hx_sample(const hx_logits* x, const hx_rules* r, const hx_pick* p, void* stream) {
  if (int rc = check_logits(x)) return rc;
  if (!p) return bad("sample: NULL argument");
  if (r)
    if (int rc = check_rules(x, r)) return rc;
  if (p->noise && (p->noise_stride < x->n_vocab || p->noise_stride >= (int64_t)1 << 38))
    return bad("sample: noise_stride must be n_vocab..2^38");
  if (x->n_rows == 0) return HX_OK;
  if (!p->token) return bad("sample: NULL pointer");
  const void* words[] = {p->noise, p->temperature, p->top_k, p->top_p, p->min_p, p->token, p->logprob};
  for (const void* w : words)
    if (!aligned(w, 4)) return bad("sample: arrays must be 4-byte aligned");
  const int64_t n = x->n_rows;
  const hx_rules rules = r ? *r : hx_rules{};
  const Range out[] = {of_rows(p->token, 1, 0, n, 4), of_rows(p->logprob, 1, 0, n, 4)};
  const Range in[] = {of_rows(x->x, n, x->stride, x->n_vocab, size_of(x->dtype)), of_rows(p->noise, n, p->noise_stride, x->n_vocab, 4),
                      of_rows(p->temperature, 1, 0, n, 4), of_rows(p->top_k, 1, 0, n, 4), of_rows(p->top_p, 1, 0, n, 4),
                      of_rows(p->min_p, 1, 0, n, 4)};
  for (const Range& o : out) {
    for (const Range& i : in)
      if (overlap(i, o)) return bad("sample: an output overlaps what is read");
    if (over_rules(rules, o)) return bad("sample: an output overlaps the rules");
  }
  if (overlap(out[0], out[1])) return bad("sample: token and logprob overlap");
  const int64_t need = hx::sample_workspace(*x, *p);
  if (p->workspace_bytes < need || !p->workspace) return bad("sample: workspace is too small");
  if (!aligned(p->workspace, 16)) return bad("sample: workspace must be 16-byte aligned");
  const Range work = {p->workspace, need};
  for (const Range& i : in)
    if (overlap(i, work)) return bad("sample: workspace overlaps what is read");
  if (overlap(out[0], work) || overlap(out[1], work) || over_rules(rules, work)) return bad("sample: workspace overlaps an array");
  return launched(hx::launch_sample(*x, rules, *p, (cudaStream_t)stream), "sample");
}

}  // extern "C"
