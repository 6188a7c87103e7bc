// hx_logits.cu -- logits adjusted by what holds for their rows (hx_adjust).
#include "hx_logits.cuh"

namespace hx {

namespace {

template <class T, class U, bool kWords>
__global__ void __launch_bounds__(kRowThreads) hx_adjust_kernel(const hx_logits x, const hx_rules r, U* out, int64_t out_stride, int blocks) {
  __shared__ alignas(16) uint32_t word[kWords ? kStretch : 4];
  using R = RowOf<T>;
  constexpr int kVec = R::kVec;
  const int row = blockIdx.x / blocks, p0 = (blockIdx.x - row * blocks) * kStretch;
  const R from(x, row);
  U* to = out + row * out_stride;
  // whether the row's out has its places where its logits have theirs
  const bool wide = ((uintptr_t)(to - from.shift) & 15) == 0;
  float v[kEach];
#pragma unroll
  for (int u = 0; u < kEach / kVec; ++u) from.load(p0 / kVec + u * kRowThreads + threadIdx.x, v + u * kVec);
  const RowRules o = begin_row(r, row, p0, from.shift, x.n_vocab, word);
#pragma unroll
  for (int u = 0; u < kEach / kVec; ++u) {
    const int i = u * kRowThreads + threadIdx.x, vec = p0 / kVec + i, e = from.token(vec);
    from.adjust(o, vec, kWords ? word + i * kVec : nullptr, v + u * kVec);
    U y[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) y[j] = from_float<U>(v[u * kVec + j]);
    if (wide && from.whole(e)) {
      constexpr int kStore = 16 / sizeof(U);
#pragma unroll
      for (int j = 0; j < kVec; j += kStore) {
        Pack<U, kStore> s;
#pragma unroll
        for (int i = 0; i < kStore; ++i) s.v[i] = y[j + i];
        *(Pack<U, kStore>*)(to + e + j) = s;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if ((unsigned)(e + j) < (unsigned)x.n_vocab) to[e + j] = y[j];
    }
  }
}

template <class T, class U>
cudaError_t launch(const hx_logits& x, const hx_rules& r, void* out, int64_t out_stride, cudaStream_t s) {
  const int blocks = stretches(x.n_vocab, RowOf<T>::kVec);
  const unsigned grid = (unsigned)x.n_rows * blocks;
  if (r.history || r.bias_start)
    hx_adjust_kernel<T, U, true><<<grid, kRowThreads, 0, s>>>(x, r, (U*)out, out_stride, blocks);
  else
    hx_adjust_kernel<T, U, false><<<grid, kRowThreads, 0, s>>>(x, r, (U*)out, out_stride, blocks);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_adjust(const hx_logits& x, const hx_rules& r, void* out, int64_t out_stride, int32_t out_dtype, cudaStream_t s) {
  const bool same = out_dtype == x.dtype;
  if (x.dtype == HX_BF16)
    return same ? launch<__nv_bfloat16, __nv_bfloat16>(x, r, out, out_stride, s) : launch<__nv_bfloat16, float>(x, r, out, out_stride, s);
  if (x.dtype == HX_F16) return same ? launch<__half, __half>(x, r, out, out_stride, s) : launch<__half, float>(x, r, out, out_stride, s);
  return launch<float, float>(x, r, out, out_stride, s);
}

}  // namespace hx
