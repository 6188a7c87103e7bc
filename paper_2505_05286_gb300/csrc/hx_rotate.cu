// hx_rotate.cu -- rotary positions of a step's queries and keys (hx_rotate).
//
// Pair (a, b) of a head becomes (a cos phi - b sin phi, a sin phi + b cos phi),
// phi = 2 pi * position * turns.  Turns a position are 64-bit fractions, so position * turns
// modulo 2^64 is the angle without loss, at any position; its upper 32 bits, less the nearest
// quarter turn, convert to 32-bit floating point within 2^-25 of a radian.
//
// Bound by memory: every value is read once and written once.  A block has a tile of tokens; their angles' cosines and sines are formed
// once for all heads, in shared memory.  Eight prompts of 5600 tokens, 32 and 8 heads of 128 in bf16: 149 us, 6.35 TB/s, 94 %
// of a copy; 28 and 4 heads of 64, half of them turned: 66 us, 85 %; 16 single tokens: 3.1 us, a launch and two chains of loads.
#include <algorithm>

#include "hx_step.cuh"

namespace hx {

namespace {

constexpr int kThreads = 256;

constexpr int kTile = 16;      // tokens of a block at most
// Loads of a thread on their way at a time: 16-byte ones one by one, as then more threads run (eight prompts of 5600, 32 and 8
// heads of 128 in bf16: 147 us, four at a time 277), narrow ones four (12 and 12 heads of 90 in f32, 30 of them turned: 61 -> 37 us).
__host__ __device__ constexpr int at_once(int bytes) { return bytes < 16 ? 4 : 1; }

struct Plan {
  int vec;         // values of a load that are turned
  int wide;        // bytes of a load that are copied, 0: nothing is
  int tile;        // tokens of a block
  int smem;
};

// The last row that begins at token t or before it, or -1: every step asks for 32 rows at once, so that the
// rows of 65536 requests take four.
__device__ int row_of(const int32_t* row_start, int n_rows, int t, int lane) {
  int lo = -1, hi = n_rows + 1;  // row_start[lo] <= t < row_start[hi]
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const int at = lo + (lane + 1) * step;
    const bool below = at < hi && row_start[at] <= t;
    const int n = __popc(__ballot_sync(~0u, below));
    const int next = lo + n * step;
    hi = min(hi, next + step);
    lo = next;
  }
  return lo;
}

// All tokens and heads of a tile, `units` loads to a head, kAtOnce of a thread on their way at a time: load(q, token, head, unit) for q in
// order, then store(q, ...).  (q indexes registers.)
template <int kAtOnce, class Load, class Store>
__device__ void walk(int n, int heads, int units, const int* on, Load load, Store store) {
  const bool whole = units <= kThreads;  // a head by fewer threads than there are
  const int lanes = whole ? kThreads / units : 1, first = whole ? threadIdx.x / units : 0;
  if (first >= lanes) return;
  const int step_tok = lanes / heads, step_h = lanes - step_tok * heads;
  for (int u = whole ? threadIdx.x % units : threadIdx.x; u < units; u += whole ? units : kThreads) {
    int tok = first / heads, h = first - tok * heads;
    while (tok < n) {
      int toks[kAtOnce], hs[kAtOnce];
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        toks[q] = tok < n && on[tok] ? tok : -1, hs[q] = h;
        if (toks[q] >= 0) load(q, tok, h, u);
        tok += step_tok, h += step_h;
        if (h >= heads) h -= heads, ++tok;
      }
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q)
        if (toks[q] >= 0) store(q, toks[q], hs[q], u);
    }
  }
}

template <class W>
__device__ void copy_rest(const hx_rotate_args& a, int64_t t0, int n, const int* on, int size) {
  const int units = (a.head_dim - a.rotary_dim) * size / (int)sizeof(W);
  constexpr int kAtOnce = at_once(sizeof(W));
  W x[kAtOnce];
  auto place = [&](int tok, int h, int u, bool out) {
    const bool key = h >= a.n_heads;
    const int64_t ts = key ? (out ? a.k_out_token_stride : a.k_token_stride) : out ? a.q_out_token_stride : a.q_token_stride;
    const int64_t hs = key ? (out ? a.k_out_head_stride : a.k_head_stride) : out ? a.q_out_head_stride : a.q_head_stride;
    const char* base = (const char*)(key ? (out ? a.k_out : a.k) : out ? a.q_out : a.q);
    return (W*)(base + ((t0 + tok) * ts + (key ? h - a.n_heads : h) * hs + a.rotary_dim) * size) + u;
  };
  walk<kAtOnce>(n, a.n_heads + a.n_kv_heads, units, on, [&](int q, int tok, int h, int u) { x[q] = *place(tok, h, u, false); },
       [&](int q, int tok, int h, int u) { *place(tok, h, u, true) = x[q]; });
}

template <class T, int V, bool kInterleaved>
__global__ void __launch_bounds__(kThreads, sizeof(T) * V == 16 ? 8 : 4) hx_rotate_kernel(const hx_rotate_args a, int tile, int wide) {
  extern __shared__ float2 s_turn[];  // cos and sin, [tile][rotary_dim / 2]: two neighbours of every unit side by side
  __shared__ int64_t s_pos[kTile];
  __shared__ int s_on[kTile];
  const int half = a.rotary_dim / 2;
  const int64_t t0 = (int64_t)blockIdx.x * tile;
  const int n = (int)min((int64_t)tile, a.n_tokens - t0);
  for (int i = threadIdx.x / 32; i < n; i += kThreads / 32) {
    const int t = (int)(t0 + i), lane = threadIdx.x & 31;
    int64_t pos = 0;
    int on = 1;
    if (a.positions) {
      pos = a.positions[t];
    } else {
      const int r = row_of(a.row_start, a.n_rows, t, lane);
      on = r >= 0 && r < a.n_rows;
      if (on) pos = (int64_t)a.kv_len[r] - a.row_start[r + 1] + t;
    }
    if (lane == 0) s_pos[i] = a.inverse ? -pos : pos, s_on[i] = on;
  }
  __syncthreads();
  constexpr int kSide = V > 1 ? 2 : 1;
  for (int i = threadIdx.x; i < n * half; i += kThreads) {
    const int tok = i / half, j = i - tok * half;
    const uint32_t turn = (uint32_t)(((uint64_t)s_pos[tok] * a.turns[j]) >> 32);
    const uint32_t quarter = (turn + (1u << 29)) >> 30;
    float c, s;
    sincospif((float)(int32_t)(turn - (quarter << 30)) * 0x1p-31f, &s, &c);
    if (quarter & 1) {
      const float x = c;
      c = -s, s = x;
    }
    if (quarter & 2) c = -c, s = -s;
    const int u = j / V, w = j - u * V;  // pair w of unit u
    s_turn[tok * half + ((w / kSide) * (half / V) + u) * kSide + w % kSide] = float2{c * a.scale, s * a.scale};
  }
  __syncthreads();
  using P = Pack<T, V>;
  const int apart = kInterleaved ? V : half, H = a.n_heads + a.n_kv_heads;
  auto turn = [&](P& x, P& y, int tok, int u) {
    const float2* cs = s_turn + tok * half;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      T& c = kInterleaved ? (2 * i < V ? x.v[2 * i % V] : y.v[2 * i % V]) : x.v[i];
      T& d = kInterleaved ? (2 * i + 1 < V ? x.v[(2 * i + 1) % V] : y.v[(2 * i + 1) % V]) : y.v[i];
      const float2 w = cs[((i / kSide) * (half / V) + u) * kSide + i % kSide];
      const float f = to_float(c), g = to_float(d);
      c = from_float<T>(f * w.x - g * w.y);
      d = from_float<T>(f * w.y + g * w.x);
    }
  };
  if constexpr (at_once(sizeof(P)) == 1) {
    const int units = half / V, lanes = kThreads / units, u = threadIdx.x % units, first = threadIdx.x / units;  // half / V <= 128
    const int at = kInterleaved ? 2 * u * V : u * V;
    for (int r = first < lanes ? first : n * H; r < n * H; r += lanes) {
      const int tok = r / H, h = r - tok * H;
      if (!s_on[tok]) continue;
      const int64_t t = t0 + tok;
      const bool key = h >= a.n_heads;
      const int hh = key ? h - a.n_heads : h;
      const T* from = (const T*)(key ? a.k : a.q) + t * (key ? a.k_token_stride : a.q_token_stride) +
                      hh * (key ? a.k_head_stride : a.q_head_stride) + at;
      T* to = (T*)(key ? a.k_out : a.q_out) + t * (key ? a.k_out_token_stride : a.q_out_token_stride) +
              hh * (key ? a.k_out_head_stride : a.q_out_head_stride) + at;
      P x = *(const P*)from, y = *(const P*)(from + apart);
      turn(x, y, tok, u);
      *(P*)to = x;
      *(P*)(to + apart) = y;
    }
  } else {
    constexpr int kAtOnce = at_once(sizeof(P));
    P x[kAtOnce], y[kAtOnce];
    auto place = [&](int tok, int h, int u, bool out) {
      const bool key = h >= a.n_heads;
      const int64_t ts = key ? (out ? a.k_out_token_stride : a.k_token_stride) : out ? a.q_out_token_stride : a.q_token_stride;
      const int64_t hs = key ? (out ? a.k_out_head_stride : a.k_head_stride) : out ? a.q_out_head_stride : a.q_head_stride;
      T* base = (T*)(key ? (out ? a.k_out : a.k) : out ? a.q_out : a.q);
      return base + (t0 + tok) * ts + (key ? h - a.n_heads : h) * hs + (kInterleaved ? 2 * u * V : u * V);
    };
    walk<kAtOnce>(n, H, half / V, s_on,
                  [&](int q, int tok, int h, int u) {
                    const T* from = place(tok, h, u, false);
                    x[q] = *(const P*)from, y[q] = *(const P*)(from + apart);
                  },
                  [&](int q, int tok, int h, int u) {
                    turn(x[q], y[q], tok, u);
                    T* to = place(tok, h, u, true);
                    *(P*)to = x[q], *(P*)(to + apart) = y[q];
                  });
  }
  if (wide == 16) copy_rest<uint4>(a, t0, n, s_on, sizeof(T));
  if (wide == 8) copy_rest<uint2>(a, t0, n, s_on, sizeof(T));
  if (wide == 4) copy_rest<uint32_t>(a, t0, n, s_on, sizeof(T));
  if (wide == 2) copy_rest<uint16_t>(a, t0, n, s_on, sizeof(T));
}

// The widest loads whose places all arguments allow, and tiles of so many tokens that every thread has some items to load at a
// time, but no fewer blocks than run at once.
Plan plan(const hx_rotate_args& a, int size) {
  const int half = a.rotary_dim / 2;
  const bool in_place = a.q_out == a.q && (!a.k || a.k_out == a.k);
  const int rest = in_place ? 0 : a.head_dim - a.rotary_dim;
  uint64_t all = 0;  // strides, in values
  if (a.n_tokens > 1) all |= a.q_token_stride | a.q_out_token_stride | (a.k ? a.k_token_stride | a.k_out_token_stride : 0);
  if (a.n_heads > 1) all |= a.q_head_stride | a.q_out_head_stride;
  if (a.n_kv_heads > 1) all |= a.k_head_stride | a.k_out_head_stride;
  all = all * size | (uint64_t)a.q | (uint64_t)a.q_out | (uint64_t)a.k | (uint64_t)(a.k ? a.k_out : nullptr);
  Plan p = {};
  p.vec = 16 / size;
  while (p.vec > 1 && (all % (p.vec * size) || half % p.vec)) p.vec /= 2;
  if (rest) {
    p.wide = 16;
    while ((all | a.rotary_dim * size | rest * size) % p.wide) p.wide /= 2;
  }
  const int heads = a.n_heads + a.n_kv_heads, lanes = std::max(1, kThreads / (half / p.vec));
  p.tile = std::min({kTile, (at_once(p.vec * size) * lanes + heads - 1) / heads, std::max(1, 16384 / (8 * half)), std::max(1, a.n_tokens / (4 * 152))});
  p.smem = p.tile * half * (int)sizeof(float2);
  return p;
}

template <class T, int V>
cudaError_t launch(const hx_rotate_args& a, const Plan& p, cudaStream_t s) {
  const unsigned blocks = (unsigned)((a.n_tokens + p.tile - 1) / p.tile);
  if (a.interleaved)
    hx_rotate_kernel<T, V, true><<<blocks, kThreads, p.smem, s>>>(a, p.tile, p.wide);
  else
    hx_rotate_kernel<T, V, false><<<blocks, kThreads, p.smem, s>>>(a, p.tile, p.wide);
  return cudaGetLastError();
}

template <class T>
cudaError_t launch_typed(const hx_rotate_args& a, cudaStream_t s) {
  const Plan p = plan(a, sizeof(T));
  if constexpr (sizeof(T) == 2)
    if (p.vec == 8) return launch<T, 8>(a, p, s);
  if (p.vec == 4) return launch<T, 4>(a, p, s);
  if (p.vec == 2) return launch<T, 2>(a, p, s);
  return launch<T, 1>(a, p, s);
}

}  // namespace

cudaError_t launch_rotate(const hx_rotate_args& a, cudaStream_t s) {
  if (a.dtype == HX_BF16) return launch_typed<__nv_bfloat16>(a, s);
  if (a.dtype == HX_F16) return launch_typed<__half>(a, s);
  return launch_typed<float>(a, s);
}

}  // namespace hx
