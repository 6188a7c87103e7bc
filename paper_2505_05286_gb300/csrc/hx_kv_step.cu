// hx_kv_step.cu -- the two kernels that put a step's tokens into the paged
// cache: its tables (hx_kv_map) and its keys and values (hx_kv_append).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>

#include "hx_kv.cuh"

namespace hx {
namespace {

constexpr int kMapThreads = 512;
constexpr int kMapChunk = 2048;  // tokens of one block

// What the rows before a row take, and in the same form what one row takes.
struct RowSum {
  long long tok, need, runs, gone;
  int live;  // rows with tokens
  __device__ RowSum& operator+=(const RowSum& o) {
    tok += o.tok, need += o.need, runs += o.runs, gone += o.gone, live += o.live;
    return *this;
  }
};

__device__ RowSum shfl_up(const RowSum& x, int d) {
  return {__shfl_up_sync(~0u, x.tok, d), __shfl_up_sync(~0u, x.need, d), __shfl_up_sync(~0u, x.runs, d),
          __shfl_up_sync(~0u, x.gone, d), __shfl_up_sync(~0u, x.live, d)};
}

struct Row {
  int held, add, tok;
  bool bad;
};

__device__ Row read_row(const hx_kv_map_args& a, int r) {
  Row w;
  w.held = a.held[r];
  w.add = a.add[r];
  w.tok = max(w.add, 0);
  const long long B = a.block_tokens;
  w.bad = w.held < 0 || w.add < -1 || ((long long)w.held + w.tok + B - 1) / B > a.table_width;
  return w;
}

__device__ RowSum sum_of(const Row& w, int B) {
  RowSum s = {w.tok, 0, 0, 0, w.tok > 0};
  if (w.bad) return s;
  const int old = (w.held + B - 1) / B;
  s.need = (w.held + w.tok + B - 1) / B - old;
  if (w.tok > 0) s.runs = (w.held + w.tok - 1) / B - w.held / B + 1;
  if (w.add < 0) s.gone = old;
  return s;
}

// Every block scans all rows (8 bytes each, from L2) and then writes its own
// kMapChunk tokens and kMapThreads rows: one launch, no block waits for another.  The
// cost of a step's tables is this scan's latency up to some hundred
// thousand tokens, and the slots' 8 bytes a token above.
__global__ void __launch_bounds__(kMapThreads) hx_kv_map_kernel(const hx_kv_map_args a) {
  __shared__ RowSum s_warp[kMapThreads / 32];
  __shared__ RowSum s_total;
  // the rows that own tokens of this chunk, at their rank among rows with tokens modulo
  // kMapChunk: they are consecutive and each owns a token of it
  __shared__ int s_start[kMapChunk], s_held[kMapChunk], s_row[kMapChunk], s_take[kMapChunk], s_run[kMapChunk];
  __shared__ int s_gone[kMapThreads];  // of the block's own rows: where their blocks go, -1: nowhere
  __shared__ int s_first, s_last, s_refused;
  __shared__ long long s_taken, s_zero;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int B = a.block_tokens, n = a.n_rows;
  const int per = (n + kMapThreads - 1) / kMapThreads;
  const int r0 = min(n, tid * per), r1 = min(n, r0 + per);
  const long long c0 = (long long)blockIdx.x * kMapChunk;
  const int own0 = blockIdx.x * kMapThreads;

  const long long cap = a.n_blocks;
  long long head = a.ring_state[0], free = a.ring_state[1];
  if (head < 0 || head >= cap) head = 0;
  free = min(max(free, 0LL), cap);

  RowSum mine = {};
  for (int r = r0; r < r1; ++r) mine += sum_of(read_row(a, r), B);
  RowSum upto = mine;
  for (int d = 1; d < 32; d <<= 1) {
    const RowSum o = shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 31) s_warp[warp] = upto;
  if (tid == 0) s_first = 0, s_last = -1, s_refused = 0, s_taken = 0;
  s_gone[tid] = -1;
  __syncthreads();
  if (warp == 0) {
    RowSum w = lane < kMapThreads / 32 ? s_warp[lane] : RowSum{};
    for (int d = 1; d < 32; d <<= 1) {
      const RowSum o = shfl_up(w, d);
      if (lane >= d) w += o;
    }
    if (lane < kMapThreads / 32) s_warp[lane] = w;
    if (lane == 31) s_total = w, s_zero = w.runs;
  }
  __syncthreads();
  const RowSum total = s_total;
  RowSum at = warp ? s_warp[warp - 1] : RowSum{};
  at += upto;
  at.tok -= mine.tok, at.need -= mine.need, at.runs -= mine.runs, at.gone -= mine.gone, at.live -= mine.live;

  const long long c1 = min(c0 + kMapChunk, min(total.tok, (long long)a.n_tokens));
  int refused = 0;
  long long taken = 0;
  for (int r = r0; r < r1; ++r) {
    const Row w = read_row(a, r);
    const RowSum x = sum_of(w, B);
    const long long end = at.tok + w.tok;
    const bool no = w.bad || (w.tok > 0 && ((x.need > 0 && at.need + x.need > free) || end > a.n_tokens));
    const bool ok = !no && w.tok > 0;
    refused += no;
    if (ok) taken += x.need;
    if (w.tok > 0 && end > a.n_tokens) atomicMin(&s_zero, at.runs);
    if (r >= own0 && r - own0 < kMapThreads) {
      a.row_start[r] = (int)min(at.tok, (long long)a.n_tokens);
      a.kv_len[r] = no || w.add < 0 ? 0 : w.held + w.tok;
      if (x.gone) s_gone[r - own0] = (int)((head + free + at.gone) % cap);
    }
    if (w.tok > 0 && at.tok < c1 && end > c0) {
      const int i = at.live & (kMapChunk - 1);
      s_start[i] = (int)at.tok;
      s_held[i] = w.held;
      s_row[i] = ok ? r : -1;
      s_take[i] = ok ? (int)at.need : 0;
      s_run[i] = w.bad ? -1 : (int)min(at.runs, (long long)a.n_runs);
      if (at.tok <= c0) s_first = at.live;
      if (end >= c1) s_last = at.live;
    }
    at += x;
  }
  if (blockIdx.x == 0) {
    atomicAdd(&s_refused, refused);
    atomicAdd((unsigned long long*)&s_taken, (unsigned long long)taken);
  }
  __syncthreads();

  if (blockIdx.x == 0 && tid == 0) {
    a.row_start[n] = (int)min(total.tok, (long long)a.n_tokens);
    a.counts[0] = (int)min(total.tok, (long long)a.n_tokens);
    a.counts[1] = (int)min(total.runs, 0x7fffffffLL);
    a.counts[2] = s_refused;
    a.counts[3] = (int)s_taken;
    a.ring_state_out[0] = (head + s_taken) % cap;
    a.ring_state_out[1] = min(free - s_taken + total.gone, cap);
  }

  // ended rows give their blocks back
  for (int i = warp; i < kMapThreads && own0 + i < n; i += kMapThreads / 32) {
    const int to = s_gone[i];
    if (to < 0) continue;
    const int32_t* row = a.block_table + (own0 + i) * a.table_stride;
    const int blocks = (a.held[own0 + i] + B - 1) / B;
    for (int j = lane; j < blocks; j += 32) a.ring[(to + (long long)j) % cap] = row[j];
  }

  // the chunk's tokens
  for (long long t = c0 + tid; t < min(c0 + kMapChunk, (long long)a.n_tokens); t += kMapThreads) {
    if (t >= c1) {
      a.slots[t] = -1;
      continue;
    }
    int lo = s_first, hi = s_last;  // the last row that starts at or before t
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_start[mid & (kMapChunk - 1)] <= t) lo = mid;
      else hi = mid - 1;
    }
    const int i = lo & (kMapChunk - 1);
    const int start = s_start[i], held = s_held[i], r = s_row[i];
    if (r < 0) {
      a.slots[t] = -1;
      if (s_run[i] >= 0) {  // a refused row's runs stay empty
        const long long pos = (long long)held + (t - start);
        const long long at_run = s_run[i] + pos / B - held / B;
        if ((pos % B == 0 || t == start) && at_run < a.n_runs) ((int4*)a.runs)[at_run] = int4{0, 0, 0, 0};
      }
      continue;
    }
    const int pos = held + (int)(t - start), blk = pos / B, off = pos % B, old = (held + B - 1) / B;
    const bool first = off == 0 || t == start;
    int id;
    if (blk >= old) {
      id = a.ring[(head + s_take[i] + (blk - old)) % cap];
      if (first) a.block_table[r * a.table_stride + blk] = id;
    } else {
      id = a.block_table[r * a.table_stride + blk];
    }
    a.slots[t] = (unsigned)id < (unsigned)a.n_blocks ? (int64_t)id * B + off : -1;
    if (first) {
      const int next = i + 1;
      const int end = lo < s_last ? s_start[next & (kMapChunk - 1)] : -1;
      // a row's end: where the next one starts, or for the chunk's last row from its own length
      const int left = (end >= 0 ? end : (int)min((long long)start + a.add[r], (long long)a.n_tokens)) - (int)t;
      const int at_run = s_run[i] + blk - held / B;
      if (at_run < a.n_runs) ((int4*)a.runs)[at_run] = int4{(int)t, min(B - off, left), id, off};
    }
  }
  for (long long i = min(s_zero, (long long)a.n_runs) + (long long)blockIdx.x * kMapThreads + tid; i < a.n_runs;
       i += (long long)gridDim.x * kMapThreads)
    ((int4*)a.runs)[i] = int4{0, 0, 0, 0};
}

// ---------------------------------------------------------------- append

template <class T>
struct Unpack;
template <>
struct Unpack<__nv_bfloat16> {
  static constexpr int n = 8;
  __device__ static void get(const uint4& u, float* f) {
    const __nv_bfloat162* h = (const __nv_bfloat162*)&u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = __bfloat1622float2(h[i]);
      f[2 * i] = x.x, f[2 * i + 1] = x.y;
    }
  }
};
template <>
struct Unpack<__half> {
  static constexpr int n = 8;
  __device__ static void get(const uint4& u, float* f) {
    const __half2* h = (const __half2*)&u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = __half22float2(h[i]);
      f[2 * i] = x.x, f[2 * i + 1] = x.y;
    }
  }
};
template <>
struct Unpack<float> {
  static constexpr int n = 4;
  __device__ static void get(const uint4& u, float* f) {
    f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
  }
};

// The exponent of the smallest power of two, -100 at least, by which amax
// fits 448 = 1.75 * 2^8: amax = m * 2^e with 1 <= m < 2 fits 2^(e-8) if m <= 1.75.
__device__ int scale_exponent(float amax) {
  const unsigned u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return max(e, -100);
}

__device__ float exp2i(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

__device__ uint32_t pack4(const float* f) {
  const unsigned lo = __nv_cvt_float2_to_fp8x2(float2{f[0], f[1]}, __NV_SATFINITE, __NV_E4M3);
  const unsigned hi = __nv_cvt_float2_to_fp8x2(float2{f[2], f[3]}, __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

__device__ void unpack4(uint32_t u, float* f) {
  const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)u, __NV_E4M3);
  const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u >> 16), __NV_E4M3);
  const float2 a = __half22float2(*(const __half2*)&lo), b = __half22float2(*(const __half2*)&hi);
  f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y;
}

// One block of threads writes one run's tokens of one head, K or V: the largest
// size first, then the values (read again, from L1), then, if the scale grew,
// the block's older tokens.
template <class T>
__global__ void __launch_bounds__(128) hx_kv_append_kernel(const hx_kv_cache c, const hx_kv_new a) {
  constexpr int kN = Unpack<T>::n;
  __shared__ float s_max[4];
  const int tid = threadIdx.x;
  const int H = c.n_kv_heads, D = c.head_dim, B = c.block_tokens;
  const unsigned which = blockIdx.x & 1, rest = blockIdx.x >> 1;
  const int h = rest % H;
  const int4 run = ((const int4*)a.runs)[rest / H];
  const int t0 = run.x, n = run.y, blk = run.z, off = run.w;
  if (n <= 0 || t0 < 0 || (long long)t0 + n > a.n_tokens || off < 0 || n > B || off > B - n ||
      (unsigned)blk >= (unsigned)c.n_blocks)
    return;
  const int64_t ts = which ? a.v_token_stride : a.k_token_stride, hs = which ? a.v_head_stride : a.k_head_stride;
  const T* x = (const T*)(which ? a.v : a.k) + t0 * ts + h * hs;
  uint8_t* to = (uint8_t*)(which ? c.v : c.k) + blk * c.block_stride + (int64_t)h * B * D;
  float* scale = (which ? c.v_scale : c.k_scale) + blk * c.scale_stride + h;

  const int units = D / kN;
  float amax = 0;
  for (int i = tid; i < n * units; i += 128) {
    float f[kN];
    Unpack<T>::get(*(const uint4*)(x + (i / units) * ts + (i % units) * kN), f);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const float s = fabsf(f[j]);
      if (s < INFINITY) amax = fmaxf(amax, s);
    }
  }
  for (int d = 16; d; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, d));
  if ((tid & 31) == 0) s_max[tid >> 5] = amax;
  const float was = off ? *scale : 0.f;
  __syncthreads();
  amax = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  const float need = exp2i(scale_exponent(amax)), now = fmaxf(was, need);
  const float inv = 1.f / now;  // exact for a power of two
  for (int i = tid; i < n * units; i += 128) {
    float f[kN];
    Unpack<T>::get(*(const uint4*)(x + (i / units) * ts + (i % units) * kN), f);
    uint32_t w[kN / 4];
#pragma unroll
    for (int j = 0; j < kN; ++j) f[j] *= inv;
#pragma unroll
    for (int j = 0; j < kN / 4; ++j) w[j] = pack4(f + 4 * j);
    uint8_t* p = to + (off + i / units) * D + (i % units) * kN;
    if constexpr (kN == 8) *(uint2*)p = uint2{w[0], w[1]};
    else *(uint32_t*)p = w[0];
  }
  if (now > was && off) {
    const float ratio = was * inv;
    for (int i = tid; i < off * D / 4; i += 128) {
      float f[4];
      unpack4(((uint32_t*)to)[i], f);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] *= ratio;
      ((uint32_t*)to)[i] = pack4(f);
    }
  }
  if (tid == 0 && now != was) *scale = now;
}

}  // namespace

cudaError_t launch_kv_map(const hx_kv_map_args& a, cudaStream_t s) {
  const int by_token = (int)(((int64_t)a.n_tokens + kMapChunk - 1) / kMapChunk);
  const int by_row = (a.n_rows + kMapThreads - 1) / kMapThreads;
  hx_kv_map_kernel<<<std::max(by_token, by_row), kMapThreads, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_kv_append(const hx_kv_cache& c, const hx_kv_new& a, cudaStream_t s) {
  const int64_t all = 2 * (int64_t)a.n_runs * c.n_kv_heads;
  if (all > 0x7fffffff) return cudaErrorInvalidValue;
  const unsigned grid = (unsigned)all;
  if (a.dtype == HX_BF16) hx_kv_append_kernel<__nv_bfloat16><<<grid, 128, 0, s>>>(c, a);
  else if (a.dtype == HX_F16) hx_kv_append_kernel<__half><<<grid, 128, 0, s>>>(c, a);
  else hx_kv_append_kernel<float><<<grid, 128, 0, s>>>(c, a);
  return cudaGetLastError();
}

}  // namespace hx
