// hx_kv_attend.cu -- attention of a step's tokens over the paged 8-bit cache.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "hx_kv.cuh"

namespace hx {
namespace {

constexpr int kTile = 128;

__device__ float value_of(uint8_t b) {
  const __half_raw h = __nv_cvt_fp8_to_halfraw(b, __NV_E4M3);
  return __half2float(*(const __half*)&h);
}

__device__ float block_reduce(float x, bool sum, float* s) {
  for (int d = 16; d; d >>= 1) {
    const float o = __shfl_xor_sync(~0u, x, d);
    x = sum ? x + o : fmaxf(x, o);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
  __syncthreads();
  return sum ? s[0] + s[1] + s[2] + s[3] : fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
}

// One block of threads per token and head: a thread per position for the
// scores of a tile, then a thread per column for the weighted values, with
// the running maximum and sum of the softmax.
template <class T>
__global__ void __launch_bounds__(kTile) hx_kv_attend_kernel(const hx_kv_cache c, const hx_kv_query a) {
  __shared__ float s_q[128], s_p[kTile], s_red[4], s_o[kTile];
  __shared__ int64_t s_at[kTile];
  __shared__ float s_vs[kTile];
  const int tid = threadIdx.x, D = c.head_dim, B = c.block_tokens;
  const int t = blockIdx.x / a.n_heads, hq = blockIdx.x % a.n_heads, h = hq / (a.n_heads / c.n_kv_heads);

  int lo = 0, hi = a.n_rows;  // the last row that starts at or before t
  while (lo + 1 < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.row_start[mid] <= t) lo = mid;
    else hi = mid;
  }
  const int r = lo, first = a.row_start[r], end = a.row_start[r + 1], n = end - first;
  int kv = t >= first && t < end ? min(max(a.kv_len[r], 0), (int)min((int64_t)a.table_width * B, (int64_t)0x7fffffff)) : 0;
  const int p = kv - n + (t - first);
  int j1 = a.causal ? min(kv, p + 1) : kv, j0 = a.window ? max(0, p - a.window + 1) : 0;
  if (a.max_q && n > a.max_q) j1 = 0;

  const T* q = (const T*)a.q + t * a.q_token_stride + hq * a.q_head_stride;
  if (tid < D) s_q[tid] = (float)q[tid];
  float m = -INFINITY, l = 0, o = 0;
  const int d = tid % D, part = tid / D, parts = kTile / D;
  __syncthreads();
  for (int base = j0; base < j1; base += kTile) {
    const int j = base + tid;
    float s = -INFINITY;
    int64_t at = -1;
    if (j < j1) {
      const int blk = a.block_table[r * a.table_stride + j / B];
      if ((unsigned)blk < (unsigned)c.n_blocks) {
        at = blk * c.block_stride + ((int64_t)h * B + j % B) * D;
        const uint8_t* k = (const uint8_t*)c.k + at;
        float x = 0;
        for (int e = 0; e < D; ++e) x += s_q[e] * value_of(k[e]);
        s = x * c.k_scale[blk * c.scale_stride + h] * a.sm_scale;
        s_vs[tid] = c.v_scale[blk * c.scale_stride + h];
      }
    }
    s_at[tid] = at;
    const float top = fmaxf(m, block_reduce(s, false, s_red));
    const float e = at >= 0 && top > -INFINITY ? expf(s - top) : 0.f;
    s_p[tid] = e;
    const float keep = top > -INFINITY ? expf(m - top) : 1.f;
    l = l * keep + block_reduce(e, true, s_red);
    o *= keep;
    m = top;
    for (int i = part; i < min(kTile, j1 - base); i += parts)
      if (s_at[i] >= 0) o += s_p[i] * (value_of(((const uint8_t*)c.v)[s_at[i] + d]) * s_vs[i]);
    __syncthreads();
  }
  s_o[tid] = o;
  __syncthreads();
  if (tid < D) {
    for (int i = 1; i < parts; ++i) o += s_o[tid + i * D];
    ((T*)a.out)[t * a.out_token_stride + hq * a.out_head_stride + tid] = (T)(l > 0 ? o / l : isnan(l) ? l : 0.f);
  }
  if (tid == 0 && a.lse) a.lse[(int64_t)t * a.n_heads + hq] = l > 0 || isnan(l) ? m + logf(l) : -INFINITY;
}

}  // namespace

int64_t kv_attend_workspace(const hx_kv_cache&, const hx_kv_query&) { return 0; }

cudaError_t launch_kv_attend(const hx_kv_cache& c, const hx_kv_query& a, cudaStream_t s) {
  const int64_t grid = (int64_t)a.n_tokens * a.n_heads;
  if (grid > 0x7fffffff) return cudaErrorInvalidValue;
  if (a.dtype == HX_BF16) hx_kv_attend_kernel<__nv_bfloat16><<<(unsigned)grid, kTile, 0, s>>>(c, a);
  else hx_kv_attend_kernel<__half><<<(unsigned)grid, kTile, 0, s>>>(c, a);
  return cudaGetLastError();
}

}  // namespace hx
