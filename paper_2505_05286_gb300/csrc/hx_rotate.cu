// hx_rotate.cu -- rotary positions of a step's queries and keys (hx_rotate).
//
// Pair (a, b) of a head becomes (a cos phi - b sin phi, a sin phi + b cos phi),
// phi = 2 pi * position * turns.  Turns a position are 64-bit fractions, so position * turns
// modulo 2^64 is the angle without loss, at any position; its upper 32 bits, less the nearest
// quarter turn, convert to 32-bit floating point within 2^-25 of a radian.
#include <algorithm>

#include "hx_step.cuh"

namespace hx {

namespace {

constexpr int kThreads = 256;

struct Plan {
  int vec;         // values of a load
  int units;       // loads of a head that one thread each takes: pairs of two, then values that are copied
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

template <class T, int V, bool kInterleaved>
__global__ void __launch_bounds__(1024) hx_rotate_kernel(const hx_rotate_args a, int units, int tile) {
  extern __shared__ float2 s_turn[];  // cos and sin, [tile][rotary_dim / 2]: two neighbours of every unit side by side
  __shared__ int64_t s_pos[16];
  __shared__ int s_on[16];
  const int half = a.rotary_dim / 2;
  const int64_t t0 = (int64_t)blockIdx.x * tile;
  const int n = (int)min((int64_t)tile, a.n_tokens - t0);
  for (int i = threadIdx.x / 32; i < n; i += blockDim.x / 32) {
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
  for (int i = threadIdx.x; i < n * half; i += blockDim.x) {
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
  const int lanes = blockDim.x / units;  // heads at a time
  const int u = threadIdx.x % units, first = threadIdx.x / units;
  if (first >= lanes) return;
  const int H = a.n_heads + a.n_kv_heads;
  const bool turned = u < half / V;
  // where the unit's values are in a head
  const int at = !turned ? a.rotary_dim + (u - half / V) * V : kInterleaved ? 2 * u * V : u * V;
  const int apart = kInterleaved ? V : half;
  using P = Pack<T, V>;
  for (int r = first; r < n * H; r += lanes) {
    const int tok = r / H, h = r - tok * H;
    if (!s_on[tok]) continue;
    const int64_t t = t0 + tok;
    const bool key = h >= a.n_heads;
    const int hh = key ? h - a.n_heads : h;
    const T* from = (const T*)(key ? a.k : a.q) + t * (key ? a.k_token_stride : a.q_token_stride) +
                    hh * (key ? a.k_head_stride : a.q_head_stride) + at;
    T* to = (T*)(key ? a.k_out : a.q_out) + t * (key ? a.k_out_token_stride : a.q_out_token_stride) +
            hh * (key ? a.k_out_head_stride : a.q_out_head_stride) + at;
    if (!turned) {
      *(P*)to = *(const P*)from;
      continue;
    }
    P x = *(const P*)from, y = *(const P*)(from + apart);
    const float2* cs = s_turn + tok * half;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      T& p = kInterleaved ? (2 * i < V ? x.v[2 * i % V] : y.v[2 * i % V]) : x.v[i];
      T& q = kInterleaved ? (2 * i + 1 < V ? x.v[(2 * i + 1) % V] : y.v[(2 * i + 1) % V]) : y.v[i];
      const float2 w = cs[((i / kSide) * (half / V) + u) * kSide + i % kSide];
      const float f = to_float(p), g = to_float(q);
      p = from_float<T>(f * w.x - g * w.y);
      q = from_float<T>(f * w.y + g * w.x);
    }
    *(P*)to = x;
    *(P*)(to + apart) = y;
  }
}

// The widest load whose places all arguments allow.
Plan plan(const hx_rotate_args& a, int size) {
  const int half = a.rotary_dim / 2;
  const bool in_place = a.q_out == a.q && (!a.k || a.k_out == a.k);
  const int rest = in_place ? 0 : a.head_dim - a.rotary_dim;
  uint64_t all = half | rest;
  if (a.n_tokens > 1)
    all |= a.q_token_stride | a.q_out_token_stride | (a.k ? a.k_token_stride | a.k_out_token_stride : 0);
  if (a.n_heads > 1) all |= a.q_head_stride | a.q_out_head_stride;
  if (a.n_kv_heads > 1) all |= a.k_head_stride | a.k_out_head_stride;
  const uint64_t base = (uint64_t)a.q | (uint64_t)a.q_out | (uint64_t)a.k | (uint64_t)(a.k ? a.k_out : nullptr);
  Plan p;
  p.vec = 16 / size;
  while (p.vec > 1 && (all % p.vec || base % (p.vec * size))) p.vec /= 2;
  p.units = half / p.vec + rest / p.vec;
  p.tile = 1;
  p.smem = p.tile * half * (int)sizeof(float2);
  return p;
}

template <class T, int V>
cudaError_t launch(const hx_rotate_args& a, const Plan& p, cudaStream_t s) {
  const int threads = std::max(kThreads, (p.units + 31) / 32 * 32);
  const unsigned blocks = (unsigned)((a.n_tokens + p.tile - 1) / p.tile);
  if (a.interleaved)
    hx_rotate_kernel<T, V, true><<<blocks, threads, p.smem, s>>>(a, p.units, p.tile);
  else
    hx_rotate_kernel<T, V, false><<<blocks, threads, p.smem, s>>>(a, p.units, p.tile);
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
