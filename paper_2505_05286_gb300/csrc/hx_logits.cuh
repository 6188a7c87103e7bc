// hx_logits.cuh -- how a row of logits is read and adjusted (hx_adjust, hx_sample).
//
// A row's logits are read 16 bytes at a time.  A row may begin anywhere: places are counted
// from the 16-byte boundary at or before its first logit, token e being at place e + shift.
// A block has a stretch of kStretch places; a word for each in shared memory says how often the
// token was written, whether it was read in the prompt, and which entry of
// the row's biases is its last: whole numbers, so that the order in
// which threads add to them is of no matter.
#pragma once

#include <cmath>

#include "hx_step.cuh"

namespace hx {

constexpr int kRowThreads = 512;
constexpr int kStretch = 8192;                       // places of a block
constexpr int kEach = kStretch / kRowThreads;        // of a thread

// A token's word: times written (19 bits), read in the prompt (1), number of its bias entry from 1 (12).
constexpr uint32_t kTimes = (1u << 19) - 1, kRead = 1u << 19;
constexpr int kBiasShift = 20;
static_assert(HX_MAX_HISTORY <= kTimes && HX_MAX_BIAS < 1 << (32 - kBiasShift), "fields of a token's word");

struct RowRules {
  float repetition, presence, frequency;
  const uint32_t* mask;   // or null
  const float* bias;      // entry 1 is bias[0]
};

// Words of places [p0, p0 + kStretch) of row r; all threads of the block call.
__device__ inline RowRules begin_row(const hx_rules& r, int row, int p0, int shift, int n_vocab, uint32_t* word) {
  RowRules o = {1.f, 0.f, 0.f, nullptr, nullptr};
  const int e0 = p0 - shift;
  auto place = [&](int token) { return (unsigned)token < (unsigned)n_vocab ? (unsigned)(token - e0) : ~0u; };
  if (r.mask) {
    const int m = r.mask_row ? r.mask_row[row] : row;
    if ((unsigned)m < (unsigned)r.n_masks) o.mask = r.mask + m * r.mask_stride;
  }
  if (!r.bias_start && !r.history) return o;
#pragma unroll
  for (int i = 0; i < kEach / 4; ++i) ((uint4*)word)[threadIdx.x + i * kRowThreads] = uint4{0, 0, 0, 0};
  __syncthreads();
  if (r.bias_start) {
    const int b0 = max(0, min(r.bias_start[row], r.n_bias));
    const int b1 = min(min(max(b0, r.bias_start[row + 1]), r.n_bias), b0 + HX_MAX_BIAS);
    o.bias = r.bias_value + b0;
    for (int j = b0 + threadIdx.x; j < b1; j += kRowThreads) {
      const unsigned at = place(r.bias_token[j]);
      if (at < kStretch) atomicMax(&word[at], (uint32_t)(j - b0 + 1) << kBiasShift);
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
    for (int i = threadIdx.x; i < len; i += kRowThreads) {
      const unsigned at = place(h[i]);
      if (at < kStretch) {
        if (i < read)
          atomicOr(&word[at], kRead);
        else
          atomicAdd(&word[at], 1u);
      }
    }
    __syncthreads();
  }
  return o;
}

// Each operation is rounded by itself: the same logits give the same adjusted ones wherever they are adjusted.
__device__ inline float adjusted(const RowRules& o, float x, uint32_t word) {
  if (word & (kTimes | kRead)) {
    const uint32_t times = word & kTimes;
    x = x > 0.f ? __fdiv_rn(x, o.repetition) : __fmul_rn(x, o.repetition);
    if (times) x = __fsub_rn(x, __fadd_rn(__fmul_rn(o.frequency, (float)times), o.presence));
  }
  if (word >> kBiasShift) x = __fadd_rn(x, o.bias[(word >> kBiasShift) - 1]);
  return x;
}

// One row as loads of 16 bytes.
template <class T>
struct RowOf {
  static constexpr int kVec = 16 / sizeof(T);
  const T* first;   // token 0
  int shift, n_vocab;
  __device__ RowOf(const hx_logits& x, int row) : first((const T*)x.x + row * x.stride), n_vocab(x.n_vocab) {
    shift = (int)((uintptr_t)first % 16 / sizeof(T));
  }
  __device__ int token(int vec) const { return vec * kVec - shift; }  // of a load's first place
  __device__ bool whole(int e) const { return e >= 0 && e + kVec <= n_vocab; }
  // Load `vec` of the row; places that are no token are -infinity.
  __device__ void load(int vec, float* x) const {
    const int e = token(vec);
    if (whole(e)) {
      const Pack<T, kVec> v = *(const Pack<T, kVec>*)(first + e);
#pragma unroll
      for (int j = 0; j < kVec; ++j) x[j] = to_float(v.v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < kVec; ++j) x[j] = (unsigned)(e + j) < (unsigned)n_vocab ? to_float(first[e + j]) : -INFINITY;
    }
  }
  // A load's values adjusted; `word` are its places', or null.
  __device__ void adjust(const RowRules& o, int vec, const uint32_t* word, float* x) const {
    const int e = token(vec);
    if (word) {
      alignas(16) uint32_t w[kVec];
      uint32_t any = 0;
#pragma unroll
      for (int j = 0; j < kVec; j += 4) *(uint4*)(w + j) = *(const uint4*)(word + j);
#pragma unroll
      for (int j = 0; j < kVec; ++j) any |= w[j];
      if (any) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) x[j] = adjusted(o, x[j], w[j]);
      }
    }
    if (o.mask) {
      uint32_t bits = 0;
      if (whole(e)) {
        bits = __funnelshift_r(o.mask[e >> 5], o.mask[(e + kVec - 1) >> 5], e & 31);
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          if ((unsigned)(e + j) < (unsigned)n_vocab) bits |= (o.mask[(e + j) >> 5] >> ((e + j) & 31) & 1) << j;
      }
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (!(bits >> j & 1)) x[j] = -INFINITY;
    }
  }
};

// Stretches of a row, wherever it begins.
inline int stretches(int n_vocab, int vec) { return (n_vocab + vec - 1 + kStretch - 1) / kStretch; }

}  // namespace hx
