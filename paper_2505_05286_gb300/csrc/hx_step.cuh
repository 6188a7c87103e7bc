// hx_step.cuh -- what the translation units of the operators on either side of
// the cache share (include/hxstep.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "hxstep.h"

namespace hx {

// Sets the calling thread's last error message and returns `code` (hx_api.cu).
int report(int code, const char* msg) noexcept;

cudaError_t launch_rotate(const hx_rotate_args& a, cudaStream_t s);
cudaError_t launch_adjust(const hx_logits& x, const hx_rules& r, void* out, int64_t out_stride, int32_t out_dtype, cudaStream_t s);
cudaError_t launch_sample(const hx_logits& x, const hx_rules& r, const hx_pick& p, cudaStream_t s);
int64_t sample_workspace(const hx_logits& x, const hx_pick& p);

// N values of T that are loaded and stored together.
template <class T, int N>
struct alignas(sizeof(T) * N) Pack {
  T v[N];
};

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(__half x) { return __half2float(x); }
__device__ inline float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T>
__device__ T from_float(float x);
template <>
__device__ inline float from_float<float>(float x) { return x; }
template <>
__device__ inline __half from_float<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ inline __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

}  // namespace hx
