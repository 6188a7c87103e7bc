// hx_logits.cu -- logits adjusted by what holds for their rows (hx_adjust).
//
// Every logit is read once and written once, 16 at a time by a thread.  A mask is applied to pairs of 16-bit logits as
// they are; tokens with a word (hx_logits.cuh) are written again behind that, one by one.  256 rows of 131072 logits in bf16, a mask
// alone: 26 us, 5.2 TB/s, 77 % of a copy; with histories of 1500 to 6400 tokens and biases: 51 us, bound by instructions, of which a
// third read the histories, which each block of a row does; one row of 32000: 4.7 us, five loads that wait for one another.
#include <type_traits>

#include "hx_logits.cuh"

namespace hx {

namespace {

// A block has kTurns stretches of a row one after the other, and the words of all of them.
template <class T, class U, bool kWords, int kTurns>
__global__ void __launch_bounds__(kRowThreads, kWords ? 3 : 4) hx_adjust_kernel(const hx_logits x, const hx_rules r, U* out, int64_t out_stride, int blocks) {
  extern __shared__ __align__(16) uint32_t word[];
  using R = RowOf<T>;
  constexpr int kVec = R::kVec, kPlaces = kTurns * kStretch;
  const int row = blockIdx.x / blocks, p0 = (blockIdx.x - row * blocks) * kPlaces;
  const R from(x, row);
  if (p0 >= x.n_vocab + from.shift) return;  // a stretch that only rows beginning elsewhere have
  U* to = out + row * out_stride;
  // whether the row's out has its places where its logits have theirs
  const bool wide = ((uintptr_t)(to - from.shift) & 15) == 0;
  const RowRules o(r, row);
  Pack<T, kVec> raw[kEach / kVec];
#pragma unroll
  for (int u = 0; u < kEach / kVec; ++u) raw[u] = from.load(p0 / kVec + u * kRowThreads + threadIdx.x);
  if (kWords) o.count<kPlaces>(p0, from.shift, x.n_vocab, word);
  for (int turn = 0; turn < kTurns; ++turn) {
    const int at = turn * kStretch;  // of the block's places
    uint32_t rest = 0;               // places of allowed tokens with a word
#pragma unroll
    for (int u = 0; u < kEach / kVec; ++u) {
      const int i = u * kRowThreads + threadIdx.x, vec = (p0 + at) / kVec + i, e = from.token(vec);
      const uint32_t bits = o.mask ? from.allowed(o.mask, vec) : ~0u;
      if (kWords && e < x.n_vocab) rest |= (R::worded(word + at + i * kVec) & bits) << u * kVec;
      U y[kVec];
      if (sizeof(T) == 2 && std::is_same<T, U>::value) {
        // only the mask, on pairs of values as they are
        constexpr uint32_t kLeast = std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;  // -infinity
        uint32_t* pair = (uint32_t*)&raw[u];
#pragma unroll
        for (int j = 0; j < kVec / 2; ++j) {
          const uint32_t keep = ((bits >> 2 * j & 1) | (bits >> (2 * j + 1) & 1) << 16) * 0xffffu;
          pair[j] = (pair[j] & keep) | (kLeast & ~keep);
        }
#pragma unroll
        for (int j = 0; j < kVec; ++j) y[j] = *(const U*)&raw[u].v[j];
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) y[j] = bits >> j & 1 ? from_float<U>(to_float(raw[u].v[j])) : from_float<U>(-INFINITY);
      }
      if (kTurns > 1 && turn + 1 < kTurns) raw[u] = from.load(vec + kStretch / kVec);
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
    if (kWords)
      for (; rest; rest &= rest - 1) {
        const int j = __ffs(rest) - 1, i = at + (j / kVec * kRowThreads + threadIdx.x) * kVec + j % kVec, e = p0 + i - from.shift;
        // in place, an allowed token's logit is still as it was
        to[e] = from_float<U>(adjusted(o, to_float(from.first[e]), word[i]));
      }
  }
}

template <class T, class U, bool kWords, int kTurns>
cudaError_t launch_turns(const hx_logits& x, const hx_rules& r, void* out, int64_t out_stride, cudaStream_t s) {
  const int blocks = stretches(x, kTurns * kStretch);
  constexpr int kSmem = kWords ? 4 * kTurns * kStretch : 0;
  const auto kernel = hx_adjust_kernel<T, U, kWords, kTurns>;
  if (kSmem > 48 << 10)
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem)) return e;
  kernel<<<(unsigned)x.n_rows * blocks, kRowThreads, kSmem, s>>>(x, r, (U*)out, out_stride, blocks);
  return cudaGetLastError();
}

template <class T, class U>
cudaError_t launch(const hx_logits& x, const hx_rules& r, void* out, int64_t out_stride, cudaStream_t s) {
  if (!r.history && !r.bias_start) return launch_turns<T, U, false, 1>(x, r, out, out_stride, s);
  // Two stretches a block, and every block reads half as often what holds for its row: 256 rows of 131072, all rules, 59 -> 51 us; not
  // where there are no more blocks than run at a time (16 rows: 13 -> 15) or one stretch is the row (4000 rows of 500: 61 -> 84).
  if (x.n_vocab > kStretch && (int64_t)x.n_rows * stretches(x, 2 * kStretch) > 3 * 152) return launch_turns<T, U, true, 2>(x, r, out, out_stride, s);
  return launch_turns<T, U, true, 1>(x, r, out, out_stride, s);
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
