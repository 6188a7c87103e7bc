// hx_sample.cu -- from a step's logits to its tokens (hx_sample).
//
// What the filters leave of a row is a beginning of its order, the larger logits first; the picked
// token is the winner of a race within it: the largest x / T - log(e), e exponential, wins in
// proportion to exp(x / T).  Two launches:
//
//   scan   blocks of 512 threads have 8192 logits each, 16 in a thread's registers, read once.  Every warp's 512 tokens, a segment, leave their
//          first token, the sum of their weights and their race's winner, whether the filters leave it or not; where filters go by
//          the order, a block counts its tokens or sums their weights in bins of 1/16 of x / T;
//   pick   a block for each row adds up the segments.  From the bins it sees which tokens the filters leave for sure: those of
//          the bins before the one in which a filter ends.  The best of the segments' winners that are left for sure is nearly the row's: only
//          the few segments whose winner scores more, or as much but for rounding, can hold a better one, and are read again.
//
// Where the race turns on a token of the bin in which a filter ends, that bin is resolved: the range of its tokens' keys
// is cut in parts until few are left, which are sorted and cut exactly where the filter says.  Where no
// segment's winner is left, all that are left race, in the segments whose first token is, or where there are too many in the row.
//
// Sums that decide where an order is cut are of whole numbers, so that no order of additions is of matter;
// those of the log-probability are 32-bit sums in a fixed order, without the first token, whose
// weight is 1: the logarithm of a share near 1 keeps its bits.
//
// 256 rows of 131072 logits in bf16: the likeliest tokens 35 us (reading the logits takes 10), by temperature alone
// 58 us (3.5 TB/s: the noise is twice the logits), by min-p 68 us, by top-k 76 to 112 us, by top-p 82 to 153 us (median of ten inputs 128): the
// scan 60, bound by instructions (60 for a logit, 19 of them for its bin), the pick 22, a chain of barriers, or up to 90 where
// a row has to be read again.  One row of 32000: 11.4 us.
#include <algorithm>

#include "hx_logits.cuh"

namespace hx {

namespace {

typedef unsigned long long u64;

constexpr int kWarps = kRowThreads / 32;
constexpr int kSegment = kStretch / kWarps;  // places of a warp
constexpr int kBins = kRowThreads;           // a thread each
constexpr float kBinsPerUnit = 16.f;
constexpr int kWeightBits = 18;              // a weight within its bin: 8192 of them stay below 2^32
constexpr int kList = 4096;                  // tokens of a bin that are kept at once
constexpr int kShort = 128;                  // of them that are sorted
constexpr int kMaxStretches = 64;
// Segments that are read again, where not the whole row is: four segments take as long as a stretch of sixteen (top-k of 256 rows: 90 us,
// with up to 128 of them 111).
constexpr int kMostAgain = 32;
constexpr int kMostNear = 256;               // tokens in them whose scores are next to the best
static_assert((HX_MAX_VOCAB + 8 + kStretch - 1) / kStretch <= kMaxStretches, "stretches of a row");
static_assert(kMostNear <= kRowThreads, "tokens next to the best by threads");
static_assert(kShort <= kRowThreads, "tokens of a short list by threads");

struct Pick {
  int k;
  float T, p, m;
  __device__ bool by_order() const { return T > 0.f && (k > 0 || p < 1.f); }  // with noise
};

// What a warp leaves of its segment.
struct alignas(16) Segment {
  u64 top;         // key of its first token, 0: no token takes part
  float sum;       // the other tokens' weights, of the first one's; NaN if a logit is
  float score;     // the race's best, in units of log 2, of the first token's weight
  int token;       // that has it
  float token_x;
  int pad[2];
};

struct Work {
  Segment* segment;   // [rows][stretches][kWarps]
  Pick* pick;         // [rows] the parameters as the scan read them
  unsigned* bins;     // [rows][stretches][2][kBins]: tokens, and sums of their weights
  int64_t bytes;
};

// The order of the tokens: larger keys first.  x is not NaN and not -0.
__device__ u64 key_of(float x, int e) {
  const uint32_t u = __float_as_uint(x);
  return (u64)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~e;
}
__device__ float x_of(u64 key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ int token_of(u64 key) { return (int)~(uint32_t)key; }
__device__ u64 key_of(double x) {
  const u64 u = (u64)__double_as_longlong(x);
  return u >> 63 ? ~u : u | 1ull << 63;
}

// 32-bit numbers in the order of whole ones; of NaN the result is of no matter.
__device__ uint32_t order(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ float unorder(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

__device__ u64 warp_max(u64 x) {
  const uint32_t hi = __reduce_max_sync(~0u, (uint32_t)(x >> 32));
  const uint32_t lo = __reduce_max_sync(~0u, (uint32_t)(x >> 32) == hi ? (uint32_t)x : 0u);
  return (u64)hi << 32 | lo;
}
__device__ float warp_sum(float x) {
  for (int d = 16; d; d /= 2) x = __fadd_rn(x, __shfl_xor_sync(~0u, x, d));
  return x;
}

// All threads of the block call these; `room` is one number a warp.
__device__ u64 block_max(u64 x, u64* room) {
  x = warp_max(x);
  __syncthreads();
  if (threadIdx.x % 32 == 0) room[threadIdx.x / 32] = x;
  __syncthreads();
  return warp_max(room[threadIdx.x % kWarps]);
}
__device__ float block_max(float x, uint32_t* room) {
  const uint32_t u = __reduce_max_sync(~0u, order(x));
  __syncthreads();
  if (threadIdx.x % 32 == 0) room[threadIdx.x / 32] = u;
  __syncthreads();
  return unorder(__reduce_max_sync(~0u, room[threadIdx.x % kWarps]));
}
__device__ float block_sum(float x, float* room) {
  x = warp_sum(x);
  __syncthreads();
  if (threadIdx.x % 32 == 0) room[threadIdx.x / 32] = x;
  __syncthreads();
  const float y = threadIdx.x % 32 < kWarps ? room[threadIdx.x % kWarps] : 0.f;
  return warp_sum(y);
}
// The sum over the threads before this one.
template <class N>
__device__ N block_before(N x, N* room) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  N in = x;
  for (int d = 1; d < 32; d *= 2) {
    const N y = __shfl_up_sync(~0u, in, d);
    if (lane >= d) in += y;
  }
  __syncthreads();
  if (lane == 31) room[warp] = in;
  __syncthreads();
  N all = lane < kWarps ? room[lane] : N(0);
  for (int d = 1; d < kWarps; d *= 2) {
    const N y = __shfl_up_sync(~0u, all, d);
    if (lane >= d) all += y;
  }
  const N before = __shfl_sync(~0u, all, warp > 0 ? warp - 1 : 0);
  return (warp > 0 ? before : N(0)) + in - x;
}

__device__ float clean(float x) { return __fadd_rn(x, 0.f); }  // -0 is 0

// 2^x and log2(x) of the special function unit: 2^-22 relative, and 2^-22 relative or absolute near 1; numbers below 2^-126 are 0.
__device__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ float log2_fast(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Scores in 32 bits, in units of log 2.  One near the largest, s, is off by less than half of this difference: a difference of logits over T, which
// is at most |s| and the logarithm of a number of 2^-126 (126), is rounded four times (2^-22 of it, 6e-5 with |s| up to 128), the logarithm is
// off by 2^-22 of 126 (3e-5), their sum is rounded (8e-6), and the scan puts a number in the place of five bits of a segment's
// score, which is up to 126 however small s is: 31 * 2^-17 = 2.4e-4, or 2^-18 of a larger one.
__device__ float near_score(float best) { return best - (1e-3f + fabsf(best) * 0x1p-16f); }

// x / T below that of the row's (or segment's) first token.
struct Scale {
  float top, T, unit, inv_bin;
  float zero = 0.f;     // where the grid of bins begins
  bool coarse = false;  // at the first token itself
  float first;          // the first token's place on it
  int first_bin;
  static constexpr float kMagic = 12582912.f;  // 1.5 * 2^23

  __device__ Scale(float top, float t) : top(top), T(t > 0.f ? t : 1.f) {
    // within what keeps products with 0 and infinity what they should be
    unit = fminf(fmaxf(1.44269504f / T, 0x1p-149f), 1e30f);
    inv_bin = kBinsPerUnit / T;
    first = __fmul_rn(top, inv_bin);
    first_bin = __float_as_int(__fmaf_rn(top, inv_bin, kMagic));
  }
  // Whether the grid has steps of 1 / 2 at least where the first token is, and numbers at all.  A row asks for less than its stretches
  // do: one that has no bins because its grid is not fine lies far below a row whose grid is.
  __device__ bool fine(float below = 4e6f) const { return fabsf(first) < below; }
  __device__ void begin_at_top() { zero = top, coarse = true, first = 0.f, first_bin = __float_as_int(kMagic); }
  // log2 of the weight
  __device__ float below(float x) const { return x == top ? 0.f : __fmul_rn(__fsub_rn(x, top), unit); }
  // Bins lie on a grid of x / T that is the same for all stretches of a row, of the whole numbers of 1 / kBinsPerUnit and what
  // rounds to them: what lies between two numbers' bins is the same from either.  Added to 1.5 * 2^23, x / T is rounded to a whole number that
  // stands in the sum's last bits; what is far down differs by more than there are bins, whatever stands there.  The last bin
  // holds all that is further down.
  // `share`: the weight within its bin, of that of the bin's middle, in 1 / 2^kWeightBits: exp(d / 16), |d| <= 1 / 2, by the series to
  // its third power, off by 2^-24 of it.  The last bin's tokens, all below e^-31 of the first's, have none.
  __device__ int bin(float x, unsigned* share = nullptr) const {
    if (coarse && (x == top || top == INFINITY)) {
      if (share) *share = x == top ? 1u << kWeightBits : 0u;
      return x == top ? 0 : kBins - 1;
    }
    unsigned s;
    const unsigned b = min(bin_or_more(x, &s), (unsigned)(kBins - 1));
    if (share) *share = b < kBins - 1 ? s : 0u;
    return (int)b;
  }
  // The same without what tells the last bin from those behind it, where the grid is not at the first token.
  __device__ unsigned bin_or_more(float x, unsigned* share = nullptr) const {
    constexpr float k1 = (float)(1 << kWeightBits), k = 1.f / kBinsPerUnit;
    const float z = __fsub_rn(x, zero), m = __fmaf_rn(z, inv_bin, kMagic), d = __fmaf_rn(z, inv_bin, -__fsub_rn(m, kMagic));
    const float f = __fmaf_rn(__fmaf_rn(__fmaf_rn(d, k1 * k * k * k / 6, k1 * k * k / 2), d, k1 * k), d, k1 + 8388608.f);
    if (share) *share = __float_as_uint(f) & 0x7fffffu;
    return (unsigned)first_bin - (unsigned)__float_as_int(m);
  }
  __device__ unsigned share(float x) const {
    unsigned s;
    bin(x, &s);
    return s;
  }
  // A score in 32 bits, in units of log 2; a number that is not fit never wins, nor what weighs nothing beside an infinite logit.
  __device__ float score(float x, float e) const {
    const float s = __fsub_rn(below(x), log2_fast(e));
    return e >= 0x1p-126f && e < INFINITY && (x == top || top < INFINITY) ? s : -INFINITY;
  }
};

__device__ void add_shared(uint32_t at, unsigned x, unsigned bin) {
  asm volatile("{.reg .pred p;\n\tsetp.lt.u32 p, %2, %3;\n\t@p red.shared.add.u32 [%0], %1;}" ::"r"(at), "r"(x), "r"(bin), "n"(kBins - 1) : "memory");
}

// The score that decides, in 64 bits.  (Not inline: few calls, many registers.)
__device__ __noinline__ u64 exact_score(float top, float T, float x, float e) {
  const double z = x == top ? 0. : ((double)x - (double)top) / (double)T;
  return key_of(z - log((double)e));
}

// kNoise: whether there is any; without, no row races.  (One kernel for both, that asks for the noise beside the temperature, takes 35 us
// where this one takes 31: 256 rows of 131072 logits with noise of which none races.)
template <class T, bool kWords, bool kNoise>
__global__ void __launch_bounds__(kRowThreads, kWords ? 2 : 3) hx_sample_scan(const hx_logits in, const hx_rules r, const hx_pick p, const Work w, int blocks) {
  __shared__ alignas(16) uint32_t word[kWords ? kStretch : 4];
  __shared__ unsigned bin_n[kBins], bin_w[kBins];
  __shared__ uint32_t warp_top[kWarps];
  __shared__ Pick s_pick;
  using R = RowOf<T>;
  constexpr int kVec = R::kVec;
  const int row = blockIdx.x / blocks, stretch = blockIdx.x - row * blocks, p0 = stretch * kStretch;
  const int t = threadIdx.x, lane = t % 32, warp = t / 32;
  Pick pick;
  pick.k = p.top_k ? p.top_k[row] : p.all_top_k;
  pick.T = p.temperature ? p.temperature[row] : p.all_temperature;
  pick.p = p.top_p ? p.top_p[row] : p.all_top_p;
  pick.m = p.min_p ? p.min_p[row] : p.all_min_p;
  if (t == 0) {
    s_pick = pick;
    if (stretch == 0) w.pick[row] = pick;
  }
  bin_n[t] = bin_w[t] = 0;
  const R from(in, row);
  if (kNoise && pick.T > 0.f) {
    // the noise is asked for now and read when the logits are done: a line for each of some threads
    const int e = p0 - from.shift + 32 * t;
    if (t < kStretch / 32 && (unsigned)e < (unsigned)in.n_vocab)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(p.noise + row * p.noise_stride + e));
  }
  // a warp's places are one after the other; load u of a lane is at place(u) of the stretch
  auto place = [&](int u) { return warp * kSegment + (u * 32 + lane) * kVec; };
  Pack<T, kVec> raw[kEach / kVec];
#pragma unroll
  for (int u = 0; u < kEach / kVec; ++u) raw[u] = from.load((p0 + place(u)) / kVec);
  const RowRules o(r, row);
  if (kWords) o.count<kStretch>(p0, from.shift, in.n_vocab, word);
  float x[kEach], top = -INFINITY;
#pragma unroll
  for (int u = 0; u < kEach / kVec; ++u) {
    const int at = place(u), vec = (p0 + at) / kVec;
#pragma unroll
    for (int j = 0; j < kVec; ++j) x[u * kVec + j] = to_float(raw[u].v[j]);
    if (kWords && from.token(vec) < in.n_vocab) {
      const uint32_t worded = R::worded(word + at);
      for (uint32_t rest = worded; rest; rest &= rest - 1) {
        const int j = at + __ffs(rest) - 1, e = p0 + j - from.shift;
        word[j] = __float_as_uint(adjusted(o, to_float(from.first[e]), word[j]));
      }
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (worded >> j & 1) x[u * kVec + j] = __uint_as_float(word[at + j]);
    }
    if (o.mask) {
      const uint32_t bits = from.allowed(o.mask, vec);
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (!(bits >> j & 1)) x[u * kVec + j] = -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) top = fmaxf(top, x[u * kVec + j]);
  }
  top = clean(unorder(__reduce_max_sync(~0u, order(top))));
  Segment s = {};
  if (top > -INFINITY) {
    Scale scale(top, pick.T);
    float base = top;
    if (top == INFINITY) {  // beside it the others weigh nothing
      base = 0.f;
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (x[i] == x[i]) x[i] = x[i] == INFINITY ? 0.f : -INFINITY;
    }
    const bool race = kNoise && pick.T > 0.f;
    const float* noise = p.noise + row * p.noise_stride - from.shift + p0;  // by place
    const int first_token = p0 + warp * kSegment - from.shift;
    const bool plain = ((uintptr_t)noise & 15) == 0 && first_token >= 0 && first_token + kSegment <= in.n_vocab;
    float part = 0.f, best = -INFINITY, e[kEach];
    uint32_t ties = 0;
    if (race) {
      if (plain) {
#pragma unroll
        for (int u = 0; u < kEach / 4; ++u) {
          const float4 v = *(const float4*)(noise + place(4 * u / kVec) + 4 * u % kVec);
          e[4 * u] = v.x, e[4 * u + 1] = v.y, e[4 * u + 2] = v.z, e[4 * u + 3] = v.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int at = place(i / kVec) + i % kVec;
          e[i] = (unsigned)(p0 + at - from.shift) < (unsigned)in.n_vocab ? noise[at] : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const float below = __fmul_rn(__fsub_rn(x[i], base), scale.unit), weight = exp2_fast(below);
        const bool tie = x[i] == base;
        part = __fadd_rn(part, tie ? 0.f : weight);
        ties |= tie ? 1u << i : 0u;
        // a score with its logit's number from 1 in its last bits: infinite ones (noise 0 or infinite, logits of -infinity) become
        // NaN by it, which loses, as does a negative noise's
        const float f = __fsub_rn(below, log2_fast(e[i]));
        best = fmaxf(best, __uint_as_float((__float_as_uint(f) & ~31u) | (unsigned)(i + 1)));
      }
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const float weight = exp2_fast(__fmul_rn(__fsub_rn(x[i], base), scale.unit));
        const bool tie = x[i] == base;
        part = __fadd_rn(part, tie ? 0.f : weight);
        ties |= tie ? 1u << i : 0u;
      }
    }
    auto token = [&](int i) { return p0 - from.shift + place(i / kVec) + i % kVec; };  // of x[i]
    const uint32_t first = __reduce_min_sync(~0u, ties ? (uint32_t)token(__ffs(ties) - 1) : ~0u);
    s.top = key_of(top, (int)first);
    s.sum = warp_sum(part) + (float)((int)__reduce_add_sync(~0u, (unsigned)__popc(ties)) - 1);
    s.score = -INFINITY, s.token = -1;
    const uint32_t most = __reduce_max_sync(~0u, order(best));
    if (race && unorder(most) > -INFINITY) {
      const int best_i = (int)(__float_as_uint(best) & 31u) - 1;
      const uint32_t mine = order(best) == most ? (uint32_t)token(best_i) : ~0u, e = __reduce_min_sync(~0u, mine);
      float best_x = x[0];
#pragma unroll
      for (int i = 1; i < kEach; ++i)
        if (i == best_i) best_x = x[i];
      s.score = unorder(most), s.token = (int)e;
      s.token_x = __shfl_sync(~0u, best_x, __ffs(__ballot_sync(~0u, mine == e)) - 1);
      if (top == INFINITY) s.token_x = top;
    }
  } else {
    bool nan = false;
#pragma unroll
    for (int i = 0; i < kEach; ++i) nan |= x[i] != x[i];
    s.sum = __any_sync(~0u, nan) ? NAN : 0.f;
    s.token = -1;
  }
  if (lane == 0) warp_top[warp] = order(top);
  __syncthreads();
  pick = s_pick;  // for all threads the same, whatever becomes of the parameters meanwhile: there are barriers behind
  if (kNoise && pick.by_order()) {
    const Scale scale(unorder(__reduce_max_sync(~0u, warp_top[lane % kWarps])), pick.T);
    const bool fine = scale.fine(), by_k = pick.k > 0, by_p = pick.p < 1.f;
    if (fine && top < INFINITY) {
      // without branches: of a warp's tokens hardly ever none is entered.  (Logits of -infinity are in the last bin, which nothing reads;
      // so are all of a stretch whose grid is not the row's.)
      const uint32_t n0 = (uint32_t)__cvta_generic_to_shared(bin_n), w0 = (uint32_t)__cvta_generic_to_shared(bin_w);
      if (by_k) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const unsigned b = scale.bin_or_more(x[i]);
          add_shared(n0 + 4 * b, 1u, b);
        }
      }
      if (by_p) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          unsigned share;
          const unsigned b = scale.bin_or_more(x[i], &share);
          add_shared(w0 + 4 * b, share, b);
        }
      }
    }
    __syncthreads();
    unsigned* bins = w.bins + ((int64_t)row * blocks + stretch) * 2 * kBins;
    if (by_k) bins[t] = bin_n[t];
    if (by_p) bins[kBins + t] = bin_w[t];
  }
  if (lane == 0) w.segment[((int64_t)row * blocks + stretch) * kWarps + warp] = s;
}

// ---------------------------------------------------------------- the row's pick

struct Shared {
  u64 room[kWarps];
  u64 list[kList];          // keys
  u64 sorted[kShort];
  u64 mass_total;
  u64 border_mass, base_mass;
  float room_f[kWarps];
  uint32_t room_n[kWarps];
  unsigned bin_n[kBins], bin_lo[kBins], bin_hi[kBins];
  uint32_t stretch_top[kMaxStretches];
  int away[kMaxStretches];  // bins from the row's first token to the stretch's, kBins: no token
  int at, last, n_list, n_again, unsure;
  unsigned base_count;
  int again[kMostAgain];    // segments
  uint8_t slot[kMaxStretches * kWarps];
  int n_near;
  float near_score[kMostNear], near_x[kMostNear];
  int near_token[kMostNear];
};

// A row's logits once more, adjusted; f(x, token) for each that takes part.  All threads of the block call.
template <class T, bool kWords>
struct RowAgain {
  RowOf<T> row;
  RowRules rules;
  uint32_t* word;
  int blocks;

  // Those from `least` to `most`.
  template <class F>
  __device__ void each(float least, float most, F f) const {
    constexpr int kVec = RowOf<T>::kVec, kLoads = kEach / kVec;
    Pack<T, kVec> raw[kLoads];
    auto load = [&](int c) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) raw[u] = row.load(c * (kStretch / kVec) + u * kRowThreads + threadIdx.x);
    };
    load(0);
    for (int c = 0; c < blocks; ++c) {
      const int p0 = c * kStretch;
      if (kWords) rules.template count<kStretch>(p0, row.shift, row.n_vocab, word);
      uint32_t rest = 0;  // the places that may be
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int i = u * kRowThreads + threadIdx.x, vec = p0 / kVec + i;
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
          const float x = to_float(raw[u].v[j]);
          bits |= x >= least && x <= most ? 1u << j : 0u;
        }
        if (row.token(vec) < row.n_vocab) {
          if (kWords) bits |= RowOf<T>::worded(word + i * kVec);
          if (bits && rules.mask) bits &= row.allowed(rules.mask, vec);
          rest |= bits << u * kVec;
        }
      }
      if (c + 1 < blocks) load(c + 1);
      // one after the other, so that f is here once
      for (; rest; rest &= rest - 1) {
        const int j = __ffs(rest) - 1, i = (j / kVec * kRowThreads + threadIdx.x) * kVec + j % kVec, e = p0 + i - row.shift;
        if ((unsigned)e >= (unsigned)row.n_vocab) continue;
        float x = to_float(row.first[e]);
        if (kWords && word[i]) x = adjusted(rules, x, word[i]);
        if (x >= least && x <= most && x > -INFINITY) f(clean(x), e);
      }
      if (kWords) __syncthreads();  // the words are the next stretch's
    }
  }
  // Segments list[0, n), a place of each for every thread and four segments at a time; f(x, token, noise), the noise read only if
  // there is one.  slot: room for a byte for each of the row's segments.
  template <class F>
  __device__ void segments(const int* list, int n, uint8_t* slot, const float* noise, F f) const {
    static_assert(kSegment % kRowThreads == 0, "places of a segment by threads");
    constexpr int kAtOnce = kStretch / kSegment;  // whose words there is room for
    for (int i0 = 0; i0 < n; i0 += kAtOnce) {
      const int m = min(kAtOnce, n - i0);
      if (kWords) {
        for (int i = threadIdx.x; i < blocks * kWarps; i += kRowThreads) slot[i] = 255;
        __syncthreads();
        if (threadIdx.x < m) slot[list[i0 + threadIdx.x]] = (uint8_t)threadIdx.x;
        for (int i = 4 * (int)threadIdx.x; i < m * kSegment; i += 4 * kRowThreads) *(uint4*)(word + i) = uint4{0, 0, 0, 0};
        __syncthreads();
        rules.enter(word, m * kSegment, [&](int token) {
          const int place = token + row.shift;
          return (unsigned)token < (unsigned)row.n_vocab ? (uint32_t)slot[place / kSegment] * kSegment + place % kSegment : ~0u;
        });
      }
      for (int at = threadIdx.x; at < kSegment; at += kRowThreads)
#pragma unroll 1
        for (int j = 0; j < m; j += 4) {
          float x[4], z[4];
          int e[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            e[q] = j + q < m ? list[i0 + j + q] * kSegment + at - row.shift : -1;
            const bool is = (unsigned)e[q] < (unsigned)row.n_vocab && (!rules.mask || rules.mask[e[q] >> 5] >> (e[q] & 31) & 1);
            x[q] = is ? to_float(row.first[e[q]]) : -INFINITY;
            z[q] = is && noise ? noise[e[q]] : 0.f;
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (kWords && x[q] != -INFINITY) {
              const uint32_t w = word[(j + q) * kSegment + at];
              if (w) x[q] = adjusted(rules, x[q], w);
            }
            if (x[q] > -INFINITY) f(clean(x[q]), e[q], z[q]);
          }
        }
      if (kWords) __syncthreads();
    }
  }
};

// The whole number at or above p * all, at least 1.
__device__ u64 part_of(float p, u64 all) {
  if (!(p > 0.f)) return 1;
  const u64 f = __float2ull_rn(p * 0x1p63f);  // p < 1 has 24 bits: exact above 2^-40
  const u64 hi = __umul64hi(all, f), lo = all * f;
  const u64 up = (hi << 1 | lo >> 63) + ((lo << 1) != 0);
  return max(up, (u64)1);
}

struct Picker {
  Shared& s;
  Scale& scale;
  float one;               // 2^shift: weights of 1 / 2^kWeightBits of the first token's bin in whole numbers

  __device__ u64 mass_of_bin(int b) const { return __float2ull_rn(exp2f((float)b * (-1.44269504f / kBinsPerUnit)) * one); }
  __device__ u64 mass(float x) const {
    unsigned share;
    const int b = scale.bin(x, &share);
    return share * mass_of_bin(b);
  }

  // Adds a token of this weight to a bin of the row's.
  __device__ void count(int bin, unsigned w) {
    atomicAdd(&s.bin_n[bin], 1u);
    const unsigned was = atomicAdd(&s.bin_lo[bin], w);
    if (was + w < was) atomicAdd(&s.bin_hi[bin], 1u);
  }

  // Sorts s.sorted[0, n), the largest first.
  __device__ void sort(int n) {
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += kRowThreads) s.sorted[i] = 0;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
      for (int d = run / 2; d; d /= 2) {
        for (int i = threadIdx.x; i < size / 2; i += kRowThreads) {
          const int a = (i & ~(d - 1)) * 2 + (i & (d - 1)), b = a + d;
          const u64 x = s.sorted[a], y = s.sorted[b];
          if ((x < y) == ((a & run) == 0)) s.sorted[a] = y, s.sorted[b] = x;
        }
        __syncthreads();
      }
  }

  // The key at which the sum over the order (of tokens, or of their mass) first reaches target, the tokens of bin `bin` being
  // those in question, `base` what is before them.  Leaves the mass up to there in s.border_mass.  read(f): f for all tokens that may
  // be in the bin.
  template <class Read>
  __device__ u64 border(bool by_mass, u64 target, int bin, u64 base, u64 base_mass, Read read) {
    const int t = threadIdx.x;
    u64 lo = 0, hi = ~0ull;   // keys in question
    unsigned left = 0;
    // cuts their range in parts, of the tokens that `all` goes through, and keeps the one in which the sum reaches target
    auto cut = [&](u64 a, u64 b, auto all) {  // the largest of ~key and of key among the thread's
      lo = ~block_max(a, s.room), hi = block_max(b, s.room);
      int shift = 0;
      while (((hi - lo) >> shift) >= kBins) ++shift;
      __syncthreads();
      s.bin_n[t] = s.bin_lo[t] = s.bin_hi[t] = 0;
      __syncthreads();
      all([&](u64 key) {
        if (key >= lo && key <= hi) count((int)((hi - key) >> shift), scale.share(x_of(key)));
      });
      __syncthreads();
      const unsigned mine_n = s.bin_n[t];
      const u64 mine_w = ((u64)s.bin_hi[t] << 32 | s.bin_lo[t]) * mass_of_bin(bin);
      const u64 before_n = block_before<u64>(mine_n, s.room), before_w = block_before<u64>(mine_w, s.room);
      // the last part that has any if none reaches it: fewer tokens than asked for
      if (t == 0) s.at = 0;
      __syncthreads();
      if (mine_n) atomicMax(&s.at, t);
      __syncthreads();
      const int last = s.at;
      __syncthreads();
      const u64 before = base + (by_mass ? before_w : before_n), mine = by_mass ? mine_w : mine_n;
      if (before < target && (before + mine >= target || t == last) && t <= last)
        s.at = t, s.base_mass = base_mass + before_w, s.base_count = (unsigned)before_n, s.border_mass = mine_n;
      __syncthreads();
      base = by_mass ? s.base_mass : base + s.base_count, base_mass = s.base_mass;
      left = (unsigned)s.border_mass;
      hi -= (u64)s.at << shift;
      const u64 least = hi - ((1ull << shift) - 1);
      if (least > lo && least <= hi) lo = least;
      __syncthreads();
    };
    for (int turn = 0; turn < 16; ++turn) {
      // into the list
      u64 a = 0, b = 0;
      __syncthreads();
      if (t == 0) s.n_list = 0;
      __syncthreads();
      read([&](float x, int e) {
        const u64 key = key_of(x, e);
        if (key < lo || key > hi || scale.bin(x) != bin) return;
        a = max(a, ~key), b = max(b, key);
        const int at = atomicAdd(&s.n_list, 1);
        if (at < kList) s.list[at] = key;
      });
      __syncthreads();
      left = (unsigned)s.n_list;
      if (left <= kList) break;
      cut(a, b, [&](auto f) {
        read([&](float x, int e) {
          if (scale.bin(x) == bin) f(key_of(x, e));
        });
      });
    }
    // in the list
    const int n = min(s.n_list, kList);
    for (int turn = 0; left > kShort && turn < 16; ++turn) {
      u64 a = 0, b = 0;
      for (int i = t; i < n; i += kRowThreads) {
        const u64 key = s.list[i];
        if (key >= lo && key <= hi) a = max(a, ~key), b = max(b, key);
      }
      cut(a, b, [&](auto f) {
        for (int i = t; i < n; i += kRowThreads) f(s.list[i]);
      });
    }
    // in order
    __syncthreads();
    if (t == 0) s.n_list = 0;
    __syncthreads();
    for (int i = t; i < n; i += kRowThreads) {
      const u64 key = s.list[i];
      if (key < lo || key > hi) continue;
      const int at = atomicAdd(&s.n_list, 1);
      if (at < kShort) s.sorted[at] = key;
    }
    __syncthreads();
    const int m = min(s.n_list, kShort);
    sort(m);
    return along(m, by_mass, target, base, base_mass);
  }

  // The same over the sorted tokens alone.  Without any (a row that has fewer tokens than asked for and none in its last bin), all before
  // them are left, with their mass.
  __device__ u64 along(int m, bool by_mass, u64 target, u64 base, u64 base_mass) {
    const int t = threadIdx.x;
    const u64 mine = t < m ? mass(x_of(s.sorted[t])) : 0, w = base_mass + block_before<u64>(mine, s.room);
    if (t == 0) s.last = m, s.border_mass = base_mass;
    __syncthreads();
    const u64 before = by_mass ? w : base + t, after = by_mass ? w + mine : base + t + 1;
    if (t < m && before < target && (after >= target || t == m - 1)) s.last = t + 1, s.border_mass = w + mine;
    __syncthreads();
    return s.last > 0 ? s.sorted[s.last - 1] : 0;
  }
};

template <class T, bool kWords>
__global__ void __launch_bounds__(kRowThreads, 2) hx_sample_pick(const hx_logits in, const hx_rules r, const hx_pick p, const Work w, int blocks) {
  extern __shared__ __align__(16) uint32_t word[];
  __shared__ Shared s;
  const int row = blockIdx.x, t = threadIdx.x;
  const Segment* seg = w.segment + (int64_t)row * blocks * kWarps;
  const int n_seg = blocks * kWarps;
  constexpr int kMine = (kMaxStretches * kWarps + kRowThreads - 1) / kRowThreads;  // segments of a thread
  if (t < kMaxStretches) s.stretch_top[t] = 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched as the scan's last blocks end
  const Pick pick = w.pick[row];
  __syncthreads();
  // add up the segments
  u64 top = 0;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int i = t + j * kRowThreads;
    if (i < n_seg) {
      const u64 k = seg[i].top;
      top = max(top, k);
      if (k) atomicMax(&s.stretch_top[i / kWarps], (uint32_t)(k >> 32));
    }
  }
  top = block_max(top, s.room);
  Scale scale(x_of(top), pick.T);
  float part = 0.f;  // of the others' weights
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int i = t + j * kRowThreads;
    if (i >= n_seg) continue;
    const Segment g = seg[i];
    const float x = x_of(g.top);
    if (!g.top || g.top == top)
      part += g.sum;
    else if (scale.top < INFINITY || x == scale.top)
      part += (g.sum + 1.f) * exp2_fast(scale.below(x));
    else if (g.sum != g.sum)
      part += g.sum;
  }
  const float others = block_sum(part, s.room_f);
  int token = token_of(top);
  float token_x = scale.top;
  const float* noise = p.noise + row * p.noise_stride;
  if (top && p.noise && pick.T > 0.f) {
    RowAgain<T, kWords> again = {RowOf<T>(in, row), RowRules(r, row), word, blocks};
    Picker a{s, scale, 1.f};
    const float log_least = !(pick.m > 0.f) ? -INFINITY : pick.m < 1.f ? log2f(pick.m) : pick.m > 1.f ? INFINITY : 0.f;
    const bool by_order = pick.by_order();
    bool by_k = false, by_p = false;
    u64 mass = 0, mass_before = 0, total = 0;
    auto bin_at = [&](u64 target) {  // where the sum of the bins' masses reaches it
      __syncthreads();
      if (t == 0) s.at = kBins - 1;
      __syncthreads();
      if (mass_before < target && mass_before + mass >= target) s.at = t;
      __syncthreads();
      return s.at;
    };
    int sure = kBins, out = kBins;  // tokens of bins before `sure` are left, of those behind `out` they are not
    int bin_k = kBins - 1;
    unsigned n_before = 0, n = 0;
    if (by_order) {
      // bins of the whole row: of its stretches'; where the grid is too coarse for them (T is small), of its tokens', from
      // the first token down
      const bool fine = scale.fine(3.9e6f);
      if (t < blocks) s.away[t] = !s.stretch_top[t] ? kBins : fine ? scale.bin(clean(unorder(s.stretch_top[t]))) : 0;
      s.bin_n[t] = s.bin_lo[t] = s.bin_hi[t] = 0;
      __syncthreads();
      u64 sum_w = 0;
      if (fine) {
        const unsigned* bins = w.bins + (int64_t)row * blocks * 2 * kBins + t;
        auto add = [&](int which, auto& sum) {  // eight stretches' loads on their way at a time
          for (int c0 = 0; c0 < blocks; c0 += 8) {
            unsigned v[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const int c = c0 + q, away = c < blocks ? s.away[c] : kBins;
              v[q] = t >= away && t < kBins - 1 ? bins[(c * 2 + which) * kBins - away] : 0u;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) sum += v[q];
          }
        };
        if (pick.k > 0) add(0, n);
        if (pick.p < 1.f) add(1, sum_w);
      } else {
        scale.begin_at_top();
        again.each(-INFINITY, INFINITY, [&](float x, int) {
          unsigned share;
          const int b = scale.bin(x, &share);
          a.count(b, share);
        });
        __syncthreads();
        if (t < kBins - 1) n = s.bin_n[t], sum_w = (u64)s.bin_hi[t] << 32 | s.bin_lo[t];
      }
      n_before = block_before<unsigned>(n, s.room_n);
      // as many bits for the sums as fit
      const float about = block_sum(exp2f((float)t * (-1.44269504f / kBinsPerUnit)) * (float)sum_w, s.room_f);
      const int bits = min(44, 60 - (int)(__float_as_uint(fmaxf(about, 1.f)) >> 23) + 127);
      a.one = __uint_as_float((uint32_t)(127 + max(bits, 0)) << 23);
      mass = sum_w * a.mass_of_bin(t);
      mass_before = block_before<u64>(mass, s.room);
      if (t == kBins - 1) s.mass_total = mass_before + mass;
      if (t == 0) s.at = kBins - 1;
      __syncthreads();
      total = s.mass_total;
      by_k = pick.k > 0, by_p = pick.p < 1.f;
      u64 least = total, most = total;  // mass that p is of
      if (by_k) {
        // the last bin if there are fewer tokens before it (or in all)
        if (n_before < (unsigned)pick.k && (n_before + n >= (unsigned)pick.k || t == kBins - 1))
          s.at = t, s.base_mass = mass_before, s.border_mass = mass_before + mass;
        __syncthreads();
        bin_k = s.at, least = s.base_mass, most = s.border_mass;
        sure = out = bin_k;
      }
      if (by_p) {
        const int bin_p = bin_at(min(part_of(pick.p, most), most));
        const int from = by_k ? bin_at(min(part_of(pick.p, least), max(least, (u64)1))) : bin_p;
        sure = min(sure, from), out = min(out, bin_p);
      }
    }
    u64 border = 0;  // once they are resolved, the last token that the filters by order leave
    bool resolved = !by_k && !by_p;
    // 1: the filters leave it, 0: they do not, -1: it is in a bin where they end
    auto left = [&](float x, u64 key) {
      if (key == top) return 1;
      if (scale.below(x) < log_least) return 0;
      if (resolved) return key >= border ? 1 : 0;
      const int b = scale.bin(x);
      return b < sure ? 1 : b > out ? 0 : -1;
    };
    u64 mine = 0, mine_at = 0;
    auto take = [&](float x, int e) {
      const u64 f = exact_score(scale.top, scale.T, x, noise[e]);
      if (f > mine || (f == mine && (u64)(uint32_t)~e << 32 > (mine_at | 0xffffffffu))) mine = f, mine_at = (u64)(uint32_t)~e << 32 | __float_as_uint(x);
    };
    // lists the segments that f holds for; whether there is room for them
    auto list_segments = [&](auto f) {
      __syncthreads();
      if (t == 0) s.n_again = 0, s.unsure = 0, s.n_near = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        const int i = t + j * kRowThreads;
        if (i < n_seg && f(seg[i])) {
          const int at = atomicAdd(&s.n_again, 1);
          if (at < kMostAgain) s.again[at] = i;
        }
      }
      __syncthreads();
      return s.n_again <= kMostAgain;
    };
    auto score_of = [&](const Segment& g) {
      return g.token < 0 || (scale.top == INFINITY && g.token_x < INFINITY) ? -INFINITY : g.score + scale.below(x_of(g.top));
    };
    bool found = false;
    while (true) {
      float best = -INFINITY, unsure = -INFINITY;
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        const int i = t + j * kRowThreads;
        if (i >= n_seg) continue;
        const Segment g = seg[i];
        const float f = score_of(g);
        if (f == -INFINITY) continue;
        const int l = left(g.token_x, key_of(g.token_x, g.token));
        if (l > 0) best = fmaxf(best, f);
        if (l < 0) unsure = fmaxf(unsure, f);
      }
      best = block_max(best, s.room_n);
      unsure = block_max(unsure, s.room_n);
      // where no winner is left, all that are left race: in the segments whose first token is
      const bool none = resolved && best == -INFINITY;
      const float near = none ? -INFINITY : near_score(best);
      found = none ? list_segments([&](const Segment& g) { return g.top && left(x_of(g.top), g.top) > 0; })
                   : best > -INFINITY && unsure < near && list_segments([&](const Segment& g) { return score_of(g) >= near; });
      if (found) {
        again.segments(s.again, s.n_again, s.slot, noise, [&](float x, int e, float z) {
          const float f = scale.score(x, z);
          if (f < near || f == -INFINITY) return;
          const int l = left(x, key_of(x, e));
          if (l < 0) s.unsure = 1;
          if (l <= 0) return;
          const int at = atomicAdd(&s.n_near, 1);
          if (at < kMostNear) s.near_score[at] = f, s.near_x[at] = x, s.near_token[at] = e;
        });
        __syncthreads();
        const int n_near = s.n_near;
        found = !s.unsure && n_near <= kMostNear;
        if (found) {
          const float f = t < n_near ? s.near_score[t] : -INFINITY, least = near_score(block_max(f, s.room_n));
          const bool is = t < n_near && f >= least;
          const int many = __syncthreads_count(is);
          if (is && many == 1) mine = 1, mine_at = (u64)(uint32_t)~s.near_token[t] << 32 | __float_as_uint(s.near_x[t]);
          if (is && many > 1) take(s.near_x[t], s.near_token[t]);
        }
      }
      if (found || resolved) break;
      // resolve the filters
      auto end = [&](bool by_mass, u64 target, int bin) {
        __syncthreads();
        if (t == bin) s.base_count = n_before, s.base_mass = mass_before;
        __syncthreads();
        const u64 m0 = s.base_mass, base = by_mass ? m0 : s.base_count;
        // the bin's tokens are between these: bin - 1 and bin + 1 bins further down than the first token, but for roundings
        const float step = scale.T / kBinsPerUnit, slack = fabsf(scale.top) * 0x1p-20f;
        const bool finite = scale.top < INFINITY;
        const float least = finite && bin < kBins - 1 ? scale.top - ((float)(bin + 2) * step + slack) : -INFINITY;
        const float most = finite && bin > 2 ? scale.top - ((float)(bin - 2) * step - slack) : INFINITY;
        const bool few = list_segments([&](const Segment& g) { return g.top && scale.bin(x_of(g.top)) <= bin; });
        return a.border(by_mass, target, bin, base, m0, [&](auto f) {
          if (few)
            again.segments(s.again, s.n_again, s.slot, nullptr, [&](float x, int e, float) { f(x, e); });
          else
            again.each(least, most, f);
        });
      };
      u64 of = total;
      if (by_k) {
        border = end(false, (u64)pick.k, bin_k);
        of = s.border_mass;
      }
      if (by_p) {
        const u64 target = min(part_of(pick.p, of), max(of, (u64)1));
        border = max(border, end(true, target, bin_at(target)));
      }
      resolved = true;
    }
    if (!found) {
      // more than there is room for: the race of all that are left
      float fast = -INFINITY;
      const float least = border ? x_of(border) : -INFINITY;
      again.each(least, INFINITY, [&](float x, int e) {
        if (left(x, key_of(x, e)) > 0) fast = fmaxf(fast, scale.score(x, noise[e]));
      });
      const float near = near_score(block_max(fast, s.room_n));
      const bool any = fast > -INFINITY && fast >= near;
      again.each(least, INFINITY, [&](float x, int e) {
        if (any && left(x, key_of(x, e)) > 0 && scale.score(x, noise[e]) >= near) take(x, e);
      });
    }
    const u64 high = block_max(mine, s.room);
    const u64 low = block_max(mine && mine == high ? mine_at : 0, s.room);
    if (high) token = (int)~(uint32_t)(low >> 32), token_x = __uint_as_float((uint32_t)low);
  }
  if (t == 0) {
    p.token[row] = top ? token : -1;
    if (p.logprob) {
      const double y = token_x == scale.top ? 0. : ((double)token_x - (double)scale.top) / (double)scale.T;
      p.logprob[row] = others != others ? NAN : top ? (float)(y - log1p((double)others)) : -INFINITY;
    }
  }
}

// The parts of a call's workspace.
Work work_of(const hx_logits& x, const hx_pick& p, void* at) {
  const int64_t blocks = (int64_t)x.n_rows * stretches(x);
  Work w = {};
  char* base = (char*)at;
  auto part = [&](int64_t bytes) {
    void* here = base + w.bytes;
    w.bytes += (bytes + 255) / 256 * 256;
    return here;
  };
  w.segment = (Segment*)part(blocks * kWarps * (int64_t)sizeof(Segment));
  w.pick = (Pick*)part(x.n_rows * (int64_t)sizeof(Pick));
  if (p.noise && (p.top_k || p.top_p || p.all_top_k > 0 || p.all_top_p < 1.f)) w.bins = (unsigned*)part(blocks * 2 * kBins * 4);
  return w;
}

template <class T, bool kWords>
cudaError_t launch(const hx_logits& x, const hx_rules& r, const hx_pick& p, cudaStream_t s) {
  const Work w = work_of(x, p, p.workspace);
  const int blocks = stretches(x);
  const auto scan = p.noise ? hx_sample_scan<T, kWords, true> : hx_sample_scan<T, kWords, false>;
  scan<<<(unsigned)x.n_rows * blocks, kRowThreads, 0, s>>>(x, r, p, w, blocks);
  if (cudaError_t e = cudaGetLastError()) return e;
  constexpr int kSmem = kWords ? 4 * kStretch : 0;
  const auto kernel = hx_sample_pick<T, kWords>;
  if (kWords)
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem)) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(x.n_rows);
  cfg.blockDim = kRowThreads;
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, x, r, p, w, blocks);
}

template <class T>
cudaError_t sample_typed(const hx_logits& x, const hx_rules& r, const hx_pick& p, cudaStream_t s) {
  return r.history || r.bias_start ? launch<T, true>(x, r, p, s) : launch<T, false>(x, r, p, s);
}

}  // namespace

int64_t sample_workspace(const hx_logits& x, const hx_pick& p) { return work_of(x, p, nullptr).bytes; }

cudaError_t launch_sample(const hx_logits& x, const hx_rules& r, const hx_pick& p, cudaStream_t s) {
  if (x.dtype == HX_BF16) return sample_typed<__nv_bfloat16>(x, r, p, s);
  if (x.dtype == HX_F16) return sample_typed<__half>(x, r, p, s);
  return sample_typed<float>(x, r, p, s);
}

}  // namespace hx
