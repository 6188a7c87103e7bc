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

// What holds for one row, as its first loads give it: all of them are on their way at once.
struct RowRules {
  float repetition, presence, frequency;
  const uint32_t* mask;     // or null
  const float* bias;        // entry 1 is bias[0]
  const int32_t* history;
  const int32_t* bias_token;
  int n_bias, length, read;

  __device__ RowRules(const hx_rules& r, int row) {
    const int b0 = r.bias_start ? r.bias_start[row] : 0, b1 = r.bias_start ? r.bias_start[row + 1] : 0;
    const int len = r.history ? r.length[row] : 0;
    read = r.history && r.prompt_len ? r.prompt_len[row] : 0;
    repetition = r.history && r.repetition ? r.repetition[row] : 1.f;
    presence = r.history && r.presence ? r.presence[row] : 0.f;
    frequency = r.history && r.frequency ? r.frequency[row] : 0.f;
    const int m = r.mask && r.mask_row ? r.mask_row[row] : row;
    mask = r.mask && (unsigned)m < (unsigned)r.n_masks ? r.mask + m * r.mask_stride : nullptr;
    const int first = max(0, min(b0, r.n_bias));
    n_bias = min(min(max(first, b1), r.n_bias) - first, HX_MAX_BIAS);
    bias = r.bias_value + first;
    bias_token = r.bias_token + first;
    length = min(len, r.history_width);
    history = r.history + row * r.history_stride;
  }

  // Words of places [p0, p0 + kPlaces) up to the load with the last token; all threads of the block call.
  template <int kPlaces>
  __device__ void count(int p0, int shift, int n_vocab, uint32_t* word) const {
    // the stretch's tokens are [e0, e0 + span), the first at word[at0]
    const int e0 = max(p0 - shift, 0), at0 = e0 - (p0 - shift);
    const unsigned span = (unsigned)max(min(kPlaces - at0, n_vocab - e0), 0);
#pragma unroll
    for (int i = 4 * (int)threadIdx.x; i < kPlaces; i += 4 * kRowThreads)
      if (i - 4 * (int)threadIdx.x < (int)span + at0) *(uint4*)(word + i) = uint4{0, 0, 0, 0};
    enter(word + at0, span, [&](int token) { return (uint32_t)(token - e0); });
  }

  // Enters what the row's lists hold in words that the threads have cleared: token t's is word[where(t)], if that is below n.
  template <class Where>
  __device__ void enter(uint32_t* word, unsigned n, Where where) const {
    // 16 bytes a load from the boundary at or before the row's first entry, every block of the row reads all of it: one pair of
    // loads is on its way while the last is counted
    const int before = (int)((uintptr_t)history % 16 / 4);
    auto load = [&](int i) {
      int4 t = {-1, -1, -1, -1};
      if (i >= 0 && i + 4 <= length) {
        t = *(const int4*)(history + i);
      } else if (i + 4 > 0 && i < length) {
        if (i >= 0) t.x = history[i];
        if (i + 1 >= 0 && i + 1 < length) t.y = history[i + 1];
        if (i + 2 >= 0 && i + 2 < length) t.z = history[i + 2];
        if (i + 3 < length) t.w = history[i + 3];
      }
      return t;
    };
    constexpr int kStep = 4 * kRowThreads;
    int i0 = 4 * (int)threadIdx.x - before;
    int4 a = load(i0), b = load(i0 + kStep);  // while the words are cleared and the biases entered
    __syncthreads();
    if (n_bias > 0) {
      for (int j = threadIdx.x; j < n_bias; j += kRowThreads) {
        const uint32_t at = where(bias_token[j]);
        if (at < n) atomicMax(&word[at], (uint32_t)(j + 1) << kBiasShift);
      }
    }
    __syncthreads();  // a maximum with what is counted already would not be one of entries
    // without a branch: of a warp's tokens hardly ever none is in the stretch
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(word);
    auto add = [&](int token) {
      const uint32_t at = where(token);
      asm volatile("{.reg .pred p;\n\tsetp.lt.u32 p, %0, %1;\n\t@p red.shared.add.u32 [%2], 1;}" ::"r"(at), "r"(n), "r"(base + 4 * at) : "memory");
    };
    auto see = [&](int token) {
      const uint32_t at = where(token);
      asm volatile("{.reg .pred p;\n\tsetp.lt.u32 p, %0, %1;\n\t@p red.shared.or.b32 [%2], %3;}" ::"r"(at), "r"(n), "r"(base + 4 * at), "r"(kRead) : "memory");
    };
    auto count4 = [&](int i, const int4& t) {
      if (i >= read) {
        add(t.x), add(t.y), add(t.z), add(t.w);
      } else if (i + 4 <= read) {
        see(t.x), see(t.y), see(t.z), see(t.w);
      } else {
        see(t.x);
        i + 1 < read ? see(t.y) : add(t.y);
        i + 2 < read ? see(t.z) : add(t.z);
        add(t.w);
      }
    };
    while (i0 < length) {
      const int4 a2 = load(i0 + 2 * kStep), b2 = load(i0 + 3 * kStep);
      count4(i0, a);
      if (i0 + kStep < length) count4(i0 + kStep, b);
      a = a2, b = b2;
      i0 += 2 * kStep;
    }
    __syncthreads();
  }
};

// Few tokens have a word: 3 of 100 after 4000 tokens of 131072, but hardly a warp has none among its 256.  So every thread takes
// its own words one after the other, and the warp as many turns as the lane that has the most, where adjusting
// all places of a load with a word in it took 900 instructions a thread (256 rows of 131072, all rules: 75 us; so 56).
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
  __device__ Pack<T, kVec> load(int vec) const {
    const int e = token(vec);
    if (whole(e)) return *(const Pack<T, kVec>*)(first + e);
    Pack<T, kVec> v;
#pragma unroll
    for (int j = 0; j < kVec; ++j) v.v[j] = (unsigned)(e + j) < (unsigned)n_vocab ? first[e + j] : from_float<T>(-INFINITY);
    return v;
  }
  // Which of a load's places the row's mask allows, one bit each.
  __device__ uint32_t allowed(const uint32_t* mask, int vec) const {
    const int e = token(vec);
    if (whole(e)) return __funnelshift_r(mask[e >> 5], mask[(e + kVec - 1) >> 5], e & 31);
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      if ((unsigned)(e + j) < (unsigned)n_vocab) bits |= (mask[(e + j) >> 5] >> ((e + j) & 31) & 1) << j;
    return bits;
  }
  // Which of a load's words there is anything in, one bit each.
  __device__ static uint32_t worded(const uint32_t* word) {
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < kVec; j += 4) {
      const uint4 w = *(const uint4*)(word + j);
      bits |= (w.x ? 1u : 0u) << j | (w.y ? 2u : 0u) << j | (w.z ? 4u : 0u) << j | (w.w ? 8u : 0u) << j;
    }
    return bits;
  }
};

// Stretches of any of the rows.
inline int stretches(const hx_logits& x, int places = kStretch) {
  const int size = x.dtype == HX_F32 ? 4 : 2;
  const bool even = (uintptr_t)x.x % 16 == 0 && (x.n_rows == 1 || x.stride * size % 16 == 0);  // all begin at a boundary
  return (x.n_vocab + (even ? 0 : 16 / size - 1) + places - 1) / places;
}

}  // namespace hx
