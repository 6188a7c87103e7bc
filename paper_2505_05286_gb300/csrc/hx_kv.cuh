// hx_kv.cuh -- what the translation units of the serving step's cache
// operators share: launchers, and how blocks and lengths are checked.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "hxkv.h"

namespace hx {

// Sets the calling thread's last error message and returns `code` (hx_api.cu).
int report(int code, const char* msg) noexcept;

cudaError_t launch_kv_map(const hx_kv_map_args& a, cudaStream_t s);
cudaError_t launch_kv_append(const hx_kv_cache& c, const hx_kv_new& a, cudaStream_t s);
cudaError_t launch_kv_attend(const hx_kv_cache& c, const hx_kv_query& a, cudaStream_t s);
int64_t kv_attend_workspace(const hx_kv_cache& c, const hx_kv_query& a);

}  // namespace hx
