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
constexpr int kMapChunk = 2048;  // tokens at a time
constexpr int kMapBlocks = 3 * 152;  // as many as run at a time (512 threads of 40 registers): each scans the rows once

// What the rows before a row take, and in the same form what one row takes.  Sums stop at
// kFull, above every limit that they are compared with: malformed lengths cannot overflow
// them, and stopping sums may still be added in any order.
constexpr uint32_t kFull = 0x7fffffffu;
struct RowSum {
  uint32_t tok, need, runs, gone, live;  // live: rows with tokens
  __device__ RowSum& operator+=(const RowSum& o) {
    tok = min(tok + o.tok, kFull), need = min(need + o.need, kFull), runs = min(runs + o.runs, kFull);
    gone = min(gone + o.gone, kFull), live += o.live;
    return *this;
  }
};

__device__ RowSum shfl_up(const RowSum& x, int d) {
  return {__shfl_up_sync(~0u, x.tok, d), __shfl_up_sync(~0u, x.need, d), __shfl_up_sync(~0u, x.runs, d),
          __shfl_up_sync(~0u, x.gone, d), __shfl_up_sync(~0u, x.live, d)};
}
// Of a warp's lanes up to and with each, and without it.
__device__ RowSum scan(const RowSum& x, int lane, RowSum* before) {
  RowSum s = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const RowSum o = shfl_up(s, d);
    if (lane >= d) s += o;
  }
  *before = shfl_up(s, 1);
  if (lane == 0) *before = RowSum{};
  return s;
}

struct Row {
  int held, add, tok;
  bool bad;
};

__device__ Row read_row(const hx_kv_map_args& a, int r, int shift) {
  Row w;
  w.held = a.held[r];
  w.add = a.add[r];
  w.tok = max(w.add, 0);
  // table_width is at most 2^23: a row that fits it has 32-bit positions
  w.bad = w.held < 0 || w.add < -1 || (((int64_t)w.held + w.tok + (1 << shift) - 1) >> shift) > a.table_width;
  return w;
}

__device__ RowSum sum_of(const Row& w, int shift) {
  RowSum s = {(uint32_t)w.tok, 0, 0, 0, w.tok > 0};
  if (w.bad) return s;
  const int old = (w.held + (1 << shift) - 1) >> shift;
  s.need = ((w.held + w.tok + (1 << shift) - 1) >> shift) - old;
  if (w.tok > 0) s.runs = ((w.held + w.tok - 1) >> shift) - (w.held >> shift) + 1;
  if (w.add < 0) s.gone = old;
  return s;
}

// Every block scans all rows (8 bytes each, from L2) and then writes its own kMapThreads rows and
// its chunks of kMapChunk tokens: one launch, no block waits for another.  A
// step's tables cost this scan's latency (16 rows 3.7 us, 1024 rows 11 us with their launch), and from some hundred
// thousand tokens on the search for each token's row and its 8 bytes: 777 prompts of 2.8 million
// tokens 21 us, 1.25 TB/s into L2 (a scan for each chunk, in three times the blocks: 25 us).
__global__ void __launch_bounds__(kMapThreads) hx_kv_map_kernel(const hx_kv_map_args a, int shift, int chunks) {
  __shared__ RowSum s_warp[kMapThreads / 32], s_before[kMapThreads / 32];
  __shared__ RowSum s_total;
  // the rows that own tokens of this chunk, at their rank among rows with tokens modulo
  // kMapChunk: they are consecutive and each owns a token of it
  __shared__ int s_start[kMapChunk], s_held[kMapChunk], s_row[kMapChunk], s_take[kMapChunk], s_run[kMapChunk];
  __shared__ int s_gone[kMapThreads];  // of the block's own rows: where their blocks go, -1: nowhere
  __shared__ int s_first, s_last, s_refused;
  __shared__ uint32_t s_taken, s_zero;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int B = 1 << shift, n = a.n_rows;
  const int per = (n + kMapThreads - 1) / kMapThreads;
  const int r0 = min(n, tid * per), r1 = min(n, r0 + per);
  const int own0 = blockIdx.x * kMapThreads;

  // the ring: places are head + x with x < cap, taken back by cap where they pass it
  const uint32_t cap = a.n_blocks;
  const int64_t head64 = a.ring_state[0], free64 = a.ring_state[1];
  const uint32_t head = head64 < 0 || head64 >= cap ? 0 : (uint32_t)head64;
  const uint32_t free = (uint32_t)min(max(free64, (int64_t)0), (int64_t)cap);
  const auto place = [&](uint32_t x) {  // x < 2 cap
    const uint32_t y = head + (x >= cap ? x - cap : x);
    return y >= cap ? y - cap : y;
  };

  RowSum mine = {};
  for (int r = r0; r < r1; ++r) mine += sum_of(read_row(a, r, shift), shift);
  RowSum at;
  const RowSum upto = scan(mine, lane, &at);
  if (lane == 31) s_warp[warp] = upto;
  if (tid == 0) s_first = 0, s_last = -1, s_refused = 0, s_taken = 0;
  s_gone[tid] = -1;
  __syncthreads();
  if (warp == 0) {
    RowSum before;
    const RowSum w = scan(lane < kMapThreads / 32 ? s_warp[lane] : RowSum{}, lane, &before);
    if (lane < kMapThreads / 32) s_before[lane] = before;
    if (lane == 31) s_total = w, s_zero = w.runs;
  }
  __syncthreads();
  const RowSum total = s_total;
  at += s_before[warp];
  const RowSum base = at;

  const uint32_t n_tok = a.n_tokens;
  int64_t c0 = (int64_t)blockIdx.x * kMapChunk, c1 = min(c0 + kMapChunk, (int64_t)min(total.tok, n_tok));
  // a row's entry among those of the chunk's tokens
  const auto enter = [&](int r, const Row& w, const RowSum& at, uint32_t end, bool ok) {
    if (w.tok > 0 && at.tok < c1 && end > c0) {
      const int i = at.live & (kMapChunk - 1);
      s_start[i] = (int)at.tok;
      s_held[i] = w.held;
      s_row[i] = ok ? r : -1;
      s_take[i] = ok ? (int)at.need : 0;
      s_run[i] = w.bad ? -1 : (int)min(at.runs, (uint32_t)a.n_runs);
      if (at.tok <= c0) s_first = at.live;
      if (end >= c1) s_last = at.live;
    }
  };
  const auto refuse = [&](const Row& w, const RowSum& x, const RowSum& at, uint32_t end) {
    return w.bad || (w.tok > 0 && ((x.need > 0 && at.need + x.need > free) || end > n_tok));
  };
  int refused = 0;
  uint32_t taken = 0;
  for (int r = r0; r < r1; ++r) {
    const Row w = read_row(a, r, shift);
    const RowSum x = sum_of(w, shift);
    const uint32_t end = min(at.tok + (uint32_t)w.tok, kFull);
    const bool no = refuse(w, x, at, end);
    const bool ok = !no && w.tok > 0;
    refused += no;
    if (ok) taken += x.need;
    if (w.tok > 0 && end > n_tok) atomicMin(&s_zero, at.runs);
    if (r >= own0 && r - own0 < kMapThreads) {
      a.row_start[r] = (int)min(at.tok, n_tok);
      a.kv_len[r] = no || w.add < 0 ? 0 : w.held + w.tok;
      if (x.gone) s_gone[r - own0] = (int)place(free + at.gone % cap);
    }
    enter(r, w, at, end, ok);
    at += x;
  }
  if (blockIdx.x == 0) {
    refused = __reduce_add_sync(~0u, refused);
    taken = __reduce_add_sync(~0u, taken);
    if (lane == 0) atomicAdd(&s_refused, refused), atomicAdd(&s_taken, taken);
  }
  __syncthreads();

  if (blockIdx.x == 0 && tid == 0) {
    a.row_start[n] = (int)min(total.tok, n_tok);
    *(int4*)a.counts = int4{(int)min(total.tok, n_tok), (int)total.runs, s_refused, (int)s_taken};
    a.ring_state_out[0] = place(s_taken);
    a.ring_state_out[1] = min((int64_t)free - s_taken + total.gone, (int64_t)cap);
  }

  // ended rows give their blocks back
  for (int i = warp; i < kMapThreads && own0 + i < n; i += kMapThreads / 32) {
    const int to = s_gone[i];
    if (to < 0) continue;
    const int32_t* row = a.block_table + (own0 + i) * a.table_stride;
    const int blocks = (a.held[own0 + i] + B - 1) >> shift;
    for (int j = lane; j < blocks; j += 32) {
      const uint32_t y = to + (uint32_t)j % cap;
      a.ring[y >= cap ? y - cap : y] = row[j];
    }
  }

  // the chunk's tokens, and those of the next chunks of this block: what the scan gave stands for all of them
  for (int chunk = blockIdx.x;;) {
    const int64_t stop = min(c0 + kMapChunk, (int64_t)n_tok);
    for (int64_t t = c0 + tid; t < stop; t += kMapThreads) {
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
      const int64_t pos64 = (int64_t)held + (t - start);
      if (r < 0) {
        a.slots[t] = -1;
        if (s_run[i] >= 0) {  // a refused row's runs stay empty
          const int64_t at_run = s_run[i] + (pos64 >> shift) - (held >> shift);
          if (((pos64 & (B - 1)) == 0 || t == start) && at_run < a.n_runs) ((int4*)a.runs)[at_run] = int4{0, 0, 0, 0};
        }
        continue;
      }
      const int pos = (int)pos64, blk = pos >> shift, off = pos & (B - 1), old = (held + B - 1) >> shift;
      const bool first = off == 0 || t == start;
      int id;
      if (blk >= old) {
        id = a.ring[place(s_take[i] + (blk - old))];
        if (first) a.block_table[r * a.table_stride + blk] = id;
      } else {
        id = a.block_table[r * a.table_stride + blk];
      }
      a.slots[t] = (unsigned)id < (unsigned)a.n_blocks ? ((int64_t)id << shift) + off : -1;
      if (first) {
        const int end = lo < s_last ? s_start[(i + 1) & (kMapChunk - 1)] : -1;
        // a row's end: where the next one starts, or for the chunk's last row from its own length
        const int left = (end >= 0 ? end : (int)min((int64_t)start + a.add[r], (int64_t)n_tok)) - (int)t;
        const int at_run = s_run[i] + blk - (held >> shift);
        if (at_run < a.n_runs) ((int4*)a.runs)[at_run] = int4{(int)t, min(B - off, left), id, off};
      }
    }
    chunk += gridDim.x;
    if (chunk >= chunks) break;
    c0 = (int64_t)chunk * kMapChunk, c1 = min(c0 + kMapChunk, (int64_t)min(total.tok, n_tok));
    __syncthreads();
    if (tid == 0) s_first = 0, s_last = -1;
    __syncthreads();
    if (base.tok < c1 && base.tok + mine.tok > c0) {
      at = base;
      for (int r = r0; r < r1; ++r) {
        const Row w = read_row(a, r, shift);
        const RowSum x = sum_of(w, shift);
        const uint32_t end = min(at.tok + (uint32_t)w.tok, kFull);
        enter(r, w, at, end, w.tok > 0 && !refuse(w, x, at, end));
        at += x;
      }
    }
    __syncthreads();
  }
  for (int64_t i = min(s_zero, (uint32_t)a.n_runs) + (int64_t)blockIdx.x * kMapThreads + tid; i < a.n_runs;
       i += (int64_t)gridDim.x * kMapThreads)
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

// A team of TW warps writes one run's tokens of one head, K or V, in one pass over them: 32
// values a lane (16 in a row, twice) stay in registers while their largest size is found, a whole
// block of the cache being TW * 1024 values.  Bound by reading the tokens and writing them back in 8
// bits where a step brings prompts, by latency where it brings single tokens.  If the scale grew, the
// block's older tokens follow.  Prompts of 33325 tokens in all, 8 heads of 128 in bf16: 37.6 us, 5.4 TB/s, 81 % of a copy;
// 301 requests, 12 heads of 64 in f16, blocks of 16: 13.7 us, 4.0 TB/s; 16 single tokens 2.7 us.
constexpr int kAppendWarps = 4;

template <class T, int TW>
__global__ void __launch_bounds__(32 * (TW > kAppendWarps ? TW : kAppendWarps)) hx_kv_append_kernel(const hx_kv_cache c, const hx_kv_new a,
                                                                                                   int d_shift) {
  constexpr int kN = Unpack<T>::n;  // values of a 16-byte load
  constexpr int kTeams = TW > kAppendWarps ? 1 : kAppendWarps / TW;
  __shared__ float s_max[kTeams][TW];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, team = warp / TW, part = warp % TW;
  const int D = 1 << d_shift, B = c.block_tokens;
  const unsigned item = blockIdx.x * kTeams + team;  // run, head, K or V
  const unsigned which = item & 1, rest = item >> 1, run_no = rest / c.n_kv_heads;
  const int h = rest % c.n_kv_heads;
  int4 run = {0, 0, 0, 0};
  if (run_no < (unsigned)a.n_runs) run = ((const int4*)a.runs)[run_no];
  const int t0 = run.x, blk = run.z, off = run.w;
  int n = run.y;
  if (n <= 0 || t0 < 0 || (int64_t)t0 + n > a.n_tokens || off < 0 || n > B || off > B - n || (unsigned)blk >= (unsigned)c.n_blocks) n = 0;
  const int64_t ts = which ? a.v_token_stride : a.k_token_stride, hs = which ? a.v_head_stride : a.k_head_stride;
  const T* x = (const T*)(which ? a.v : a.k) + t0 * ts + h * hs;

  // values part * 1024 + 512 u + 16 lane and on
  uint4 raw[2][16 / kN];
  float amax = 0;
  float* scale_at = (which ? c.v_scale : c.k_scale) + blk * c.scale_stride + h;
  const float was = n && off ? *scale_at : 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = part * 1024 + 512 * u + 16 * lane, tok = i >> d_shift;
#pragma unroll
    for (int y = 0; y < 16 / kN; ++y)
      raw[u][y] = tok < n ? *(const uint4*)(x + tok * ts + (i & (D - 1)) + y * kN) : uint4{0, 0, 0, 0};
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int y = 0; y < 16 / kN; ++y) {
      float f[kN];
      Unpack<T>::get(raw[u][y], f);
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        const float s = fabsf(f[j]);
        if (s < INFINITY) amax = fmaxf(amax, s);
      }
    }
  amax = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(amax)));  // sizes order as integers
  if constexpr (TW > 1) {
    if (lane == 0) s_max[team][part] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < TW; ++w) amax = fmaxf(amax, s_max[team][w]);
  }
  if (n == 0) return;
  const float now = fmaxf(was, exp2i(scale_exponent(amax)));
  const float inv = 1.f / now;  // exact for a power of two
  uint8_t* to = (uint8_t*)(which ? c.v : c.k) + blk * c.block_stride + (((int64_t)h * B) << d_shift);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = part * 1024 + 512 * u + 16 * lane;
    if ((i >> d_shift) >= n) break;
    uint32_t w[4];
#pragma unroll
    for (int y = 0; y < 16 / kN; ++y) {
      float f[kN];
      Unpack<T>::get(raw[u][y], f);
#pragma unroll
      for (int j = 0; j < kN; ++j) f[j] *= inv;
#pragma unroll
      for (int j = 0; j < kN / 4; ++j) w[y * (kN / 4) + j] = pack4(f + 4 * j);
    }
    *(uint4*)(to + (off << d_shift) + i) = uint4{w[0], w[1], w[2], w[3]};
  }
  if (now > was && off) {
    const float ratio = was * inv;
    for (int i = 32 * part + lane; i < (off << d_shift) / 4; i += 32 * TW) {
      float f[4];
      unpack4(((uint32_t*)to)[i], f);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] *= ratio;
      ((uint32_t*)to)[i] = pack4(f);
    }
  }
  if (part == 0 && lane == 0 && now != was) *scale_at = now;
}

template <class T, int TW>
cudaError_t launch_team(const hx_kv_cache& c, const hx_kv_new& a, cudaStream_t s) {
  constexpr int kTeams = TW > kAppendWarps ? 1 : kAppendWarps / TW;
  const unsigned items = 2u * (unsigned)a.n_runs * (unsigned)c.n_kv_heads;
  hx_kv_append_kernel<T, TW><<<(items + kTeams - 1) / kTeams, 32 * (TW > kAppendWarps ? TW : kAppendWarps), 0, s>>>(
      c, a, c.head_dim == 128 ? 7 : 6);
  return cudaGetLastError();
}

template <class T>
cudaError_t launch_append(const hx_kv_cache& c, const hx_kv_new& a, cudaStream_t s) {
  switch (c.block_tokens * c.head_dim / 1024) {
    case 1: return launch_team<T, 1>(c, a, s);
    case 2: return launch_team<T, 2>(c, a, s);
    case 4: return launch_team<T, 4>(c, a, s);
    case 8: return launch_team<T, 8>(c, a, s);
    default: return launch_team<T, 16>(c, a, s);
  }
}

}  // namespace

cudaError_t launch_kv_map(const hx_kv_map_args& a, cudaStream_t s) {
  const int by_token = (int)(((int64_t)a.n_tokens + kMapChunk - 1) / kMapChunk);
  const int by_row = (a.n_rows + kMapThreads - 1) / kMapThreads;
  int shift = 4;
  while ((1 << shift) < a.block_tokens) ++shift;
  const int rounds = std::max(1, (by_token + kMapBlocks - 1) / kMapBlocks);
  hx_kv_map_kernel<<<std::max((by_token + rounds - 1) / rounds, by_row), kMapThreads, 0, s>>>(a, shift, by_token);
  return cudaGetLastError();
}

cudaError_t launch_kv_append(const hx_kv_cache& c, const hx_kv_new& a, cudaStream_t s) {
  if (a.dtype == HX_BF16) return launch_append<__nv_bfloat16>(c, a, s);
  if (a.dtype == HX_F16) return launch_append<__half>(c, a, s);
  return launch_append<float>(c, a, s);
}

}  // namespace hx
