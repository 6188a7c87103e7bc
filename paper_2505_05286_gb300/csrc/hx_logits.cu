// hx_logits.cu -- from a step's logits to its tokens (hx_adjust, hx_sample).
//
// Both kernels adjust logits in the same way.  A block has a stretch of one row's
// vocabulary; a word for each of its tokens in shared memory says how often the
// token was written, whether it was read in the prompt, and which entry of
// the row's biases is its last: whole numbers, so that the order in
// which threads add to them is of no matter.
#include <algorithm>
#include <cmath>

#include "hx_step.cuh"

namespace hx {

namespace {

constexpr int kThreads = 512;

// ---------------------------------------------------------------- adjusting

// A token's word: times written (19 bits), read in the prompt (1), number of its bias entry from 1 (12).
constexpr uint32_t kTimes = (1u << 19) - 1, kRead = 1u << 19;
constexpr int kBiasShift = 20;
static_assert(HX_MAX_HISTORY <= kTimes && HX_MAX_BIAS < 1 << (32 - kBiasShift), "fields of a token's word");

struct Row {
  float repetition, presence, frequency;
  const uint32_t* mask;   // or null
  const float* bias;      // entry 1 is bias[0]
};

// Words of the tokens [e0, e0 + n) of row r; all threads of the block call.
__device__ Row begin_row(const hx_rules& r, int row, int e0, int n, uint32_t* word) {
  Row o = {1.f, 0.f, 0.f, nullptr, nullptr};
  for (int i = threadIdx.x; i < n; i += blockDim.x) word[i] = 0;
  __syncthreads();
  if (r.bias_start) {
    const int b0 = max(0, min(r.bias_start[row], r.n_bias));
    const int b1 = min(min(max(b0, r.bias_start[row + 1]), r.n_bias), b0 + HX_MAX_BIAS);
    o.bias = r.bias_value + b0;
    for (int j = b0 + threadIdx.x; j < b1; j += blockDim.x) {
      const unsigned at = (unsigned)r.bias_token[j] - (unsigned)e0;
      if (at < (unsigned)n) atomicMax(&word[at], (uint32_t)(j - b0 + 1) << kBiasShift);
    }
    __syncthreads();
  }
  if (r.history) {
    if (r.repetition) o.repetition = r.repetition[row];
    if (r.presence) o.presence = r.presence[row];
    if (r.frequency) o.frequency = r.frequency[row];
    const int len = min(r.length[row], r.history_width);
    const int read = r.prompt_len ? r.prompt_len[row] : 0;
    const int32_t* h = r.history + row * r.history_stride;
    for (int i = threadIdx.x; i < len; i += blockDim.x) {
      const unsigned at = (unsigned)h[i] - (unsigned)e0;
      if (at < (unsigned)n) {
        if (i < read)
          atomicOr(&word[at], kRead);
        else
          atomicAdd(&word[at], 1u);
      }
    }
    __syncthreads();
  }
  if (r.mask) {
    const int m = r.mask_row ? r.mask_row[row] : row;
    if ((unsigned)m < (unsigned)r.n_masks) o.mask = r.mask + m * r.mask_stride;
  }
  return o;
}

// Each operation is rounded by itself: the same logits give the same adjusted ones wherever they are adjusted.
__device__ float adjusted(const Row& o, float x, uint32_t word, int e) {
  if (word & (kTimes | kRead)) {
    const uint32_t times = word & kTimes;
    x = x > 0.f ? __fdiv_rn(x, o.repetition) : __fmul_rn(x, o.repetition);
    if (times) x = __fsub_rn(x, __fadd_rn(__fmul_rn(o.frequency, (float)times), o.presence));
  }
  if (word >> kBiasShift) x = __fadd_rn(x, o.bias[(word >> kBiasShift) - 1]);
  if (o.mask && !(o.mask[e >> 5] >> (e & 31) & 1)) x = -INFINITY;
  return x;
}

constexpr int kAdjustStretch = 8192;

template <class T, class U>
__global__ void __launch_bounds__(kThreads) hx_adjust_kernel(const hx_logits x, const hx_rules r, U* out, int64_t out_stride, int blocks) {
  __shared__ uint32_t word[kAdjustStretch];
  const int row = blockIdx.x / blocks, e0 = (blockIdx.x - row * blocks) * kAdjustStretch, n = min(kAdjustStretch, x.n_vocab - e0);
  const Row o = begin_row(r, row, e0, n, word);
  const T* from = (const T*)x.x + row * x.stride + e0;
  U* to = out + row * out_stride + e0;
  for (int i = threadIdx.x; i < n; i += kThreads) to[i] = from_float<U>(adjusted(o, to_float(from[i]), word[i], e0 + i));
}

template <class T>
cudaError_t adjust_typed(const hx_logits& x, const hx_rules& r, void* out, int64_t out_stride, int32_t out_dtype, cudaStream_t s) {
  const int blocks = (x.n_vocab + kAdjustStretch - 1) / kAdjustStretch;
  const unsigned grid = (unsigned)x.n_rows * blocks;
  if (out_dtype == HX_F32)
    hx_adjust_kernel<T, float><<<grid, kThreads, 0, s>>>(x, r, (float*)out, out_stride, blocks);
  else
    hx_adjust_kernel<T, T><<<grid, kThreads, 0, s>>>(x, r, (T*)out, out_stride, blocks);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_adjust(const hx_logits& x, const hx_rules& r, void* out, int64_t out_stride, int32_t out_dtype, cudaStream_t s) {
  if (x.dtype == HX_BF16) return adjust_typed<__nv_bfloat16>(x, r, out, out_stride, out_dtype, s);
  if (x.dtype == HX_F16) return adjust_typed<__half>(x, r, out, out_stride, out_dtype, s);
  return adjust_typed<float>(x, r, out, out_stride, out_dtype, s);
}

}  // namespace hx
