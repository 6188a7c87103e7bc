// hx_sample.cu -- from a step's logits to its tokens (hx_sample).
//
// What the filters leave of a row is a beginning of its order, the larger logits first; the picked
// token is the winner of a race within it: the largest x / T - log(e), e exponential, wins in
// proportion to exp(x / T).  Two launches:
//
//   scan   blocks of 512 threads have 8192 logits each, 16 in a thread's registers, read once.  Each finds its stretch's first
//          token, the sum of its weights and, where nothing is filtered, the race's winner; where something is, it counts its tokens
//          and sums their weights in bins of 1/16 of x / T;
//   pick   a block for each row adds up the stretches.  From the bins it sees how far down the order the filters can
//          reach: the tokens of those bins are read again, sorted, cut exactly where the filters say, and raced.  Where they
//          are too many for one list, the last bin is cut by its keys until what is left fits, and the race reads the row.
//
// Sums that decide where an order is cut are of whole numbers, so that no order of additions is of matter;
// those of the log-probability are 32-bit sums of 16 weights, added up in a fixed order.
#include <algorithm>

#include "hx_logits.cuh"

namespace hx {

namespace {

typedef unsigned long long u64;

constexpr int kWarps = kRowThreads / 32;
constexpr int kBins = kRowThreads;     // a thread each
constexpr float kBinsPerUnit = 16.f;
constexpr int kWeightBits = 18;        // a weight within its bin: 8192 of them stay below 2^32
constexpr int kList = 2048;            // tokens of a row that are sorted at once
constexpr int kMaxStretches = 64;
static_assert((HX_MAX_VOCAB + 8 + kStretch - 1) / kStretch <= kMaxStretches, "stretches of a row");
static_assert(kList % kRowThreads == 0, "tokens of a list by threads");

// What a stretch's block leaves for the row's.
struct alignas(16) Record {
  u64 top;       // key of its first token, 0: no token takes part
  float sum;     // weights, of its first token's
  int nan;
  int token;     // the race's winner, -1: none
  float token_x;
  int count;     // tokens that take part
  int k;         // the row's parameters, as this block read them
  float T, p, m;
  int pad;
};

struct Work {
  Record* record;     // [rows][stretches]
  unsigned* bin_n;    // [rows][stretches][kBins]: tokens, and sums of their weights
  unsigned* bin_w;
  float* x;           // [rows][places] adjusted logits, or null: the row's own
  int places;
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

__device__ u64 warp_max(u64 x) {
  for (int d = 16; d; d /= 2) x = max(x, __shfl_xor_sync(~0u, x, d));
  return x;
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

// x / T below that of the row's (or stretch's) first token.
struct Scale {
  float top, T, inv, inv_bin;
  float zero = 0.f;   // where the grid of bins begins
  __device__ Scale(float top, float t) : top(top), T(t > 0.f ? t : 1.f) {
    inv = 1.f / T;
    inv_bin = kBinsPerUnit / T;
  }
  // Whether the grid has steps of 1 / 2 at least where the first token is.
  __device__ bool fine() const { return fabsf(top * inv_bin) < 4e6f; }
  __device__ float below(float x) const { return x == top ? 0.f : fmaxf(__fmul_rn(__fsub_rn(x, top), inv), -1e30f); }
  __device__ float weight(float x) const { return exp2f(__fmul_rn(below(x), 1.44269504f)); }
  // Bins lie on a grid of x / T that is the same for all stretches of a row: what lies between two numbers' bins is the
  // same from either.  The last bin holds all that is further down.
  __device__ float grid(float x) const { return floorf(__fmul_rn(__fsub_rn(x, zero), inv_bin)); }
  __device__ int bin(float x) const { return x == top ? 0 : (int)fminf(__fsub_rn(grid(top), grid(x)), (float)(kBins - 1)); }
  // The weight within its bin, of that of the bin's upper edge; the last bin's tokens, all below e^-31 of the first's, have none.
  __device__ unsigned share(float x, int bin) const {
    const float z = __fsub_rn(x, zero), y = __fmul_rn(z, inv_bin), rest = __fmaf_rn(z, inv_bin, -y);
    const float down = fminf(fmaxf(__fsub_rn(__fsub_rn(__fadd_rn(floorf(y), 1.f), y), rest), 0.f), 1.f);
    return bin < kBins - 1 ? __float2uint_rn(exp2f(__fmul_rn(down, -1.44269504f / kBinsPerUnit)) * (float)(1 << kWeightBits)) : 0u;
  }
  __device__ u64 exact(float x, float e) const {
    const double z = x == top ? 0. : ((double)x - (double)top) / (double)T;
    return key_of(z - log((double)e));
  }
  // The same in 32 bits; a number that is not fit never wins, nor what weighs nothing beside an infinite logit.
  __device__ float score(float x, float e) const {
    return e > 0.f && e < INFINITY && (x == top || top < INFINITY) ? __fsub_rn(below(x), logf(e)) : -INFINITY;
  }
  // Scores in 32 bits are off by less than this difference; those so near the largest are formed in 64.
  __device__ static float near(float best) { return best - (2e-4f + fabsf(best) * 0x1p-19f); }
};

struct Pick {
  int k;
  float T, p, m;
  __device__ bool cut() const { return T > 0.f && (k > 0 || p < 1.f || m > 0.f); }
};

__device__ float clean(float x) { return __fadd_rn(x, 0.f); }  // -0 is 0

template <class T, bool kWords>
__global__ void __launch_bounds__(kRowThreads) hx_sample_scan(const hx_logits in, const hx_rules r, const hx_pick p, const Work w, int blocks) {
  __shared__ alignas(16) uint32_t word[kWords ? kStretch : 4];
  __shared__ alignas(16) u64 room[kWarps];
  __shared__ alignas(16) float room_f[kWarps];
  __shared__ int room_n[kWarps];
  __shared__ unsigned bin_n[kBins], bin_w[kBins];
  __shared__ Pick s_pick;
  using R = RowOf<T>;
  constexpr int kVec = R::kVec;
  const int row = blockIdx.x / blocks, stretch = blockIdx.x - row * blocks, p0 = stretch * kStretch, t = threadIdx.x;
  if (t == 0) {
    s_pick.k = p.top_k ? p.top_k[row] : p.all_top_k;
    s_pick.T = !p.noise ? 0.f : p.temperature ? p.temperature[row] : p.all_temperature;
    s_pick.p = p.top_p ? p.top_p[row] : p.all_top_p;
    s_pick.m = p.min_p ? p.min_p[row] : p.all_min_p;
  }
  bin_n[t] = bin_w[t] = 0;
  const R from(in, row);
  float x[kEach];
#pragma unroll
  for (int u = 0; u < kEach / kVec; ++u) from.load(p0 / kVec + u * kRowThreads + t, x + u * kVec);
  const RowRules o(r, row);
  if (kWords) o.count<kStretch>(p0, from.shift, in.n_vocab, word);
  auto token = [&](int i) { return from.token(p0 / kVec + i / kVec * kRowThreads + t) + i % kVec; };  // of x[i]
  float best = -INFINITY;
  int best_e = 0, count = 0;
  bool nan = false;
#pragma unroll
  for (int u = 0; u < kEach / kVec; ++u) {
    const int i = u * kRowThreads + t, vec = p0 / kVec + i;
    if (kWords && from.token(vec) < in.n_vocab) {
      const uint32_t worded = R::worded(word + i * kVec);
      for (uint32_t rest = worded; rest; rest &= rest - 1) {
        const int j = i * kVec + __ffs(rest) - 1, e = p0 + j - from.shift;
        word[j] = __float_as_uint(adjusted(o, to_float(from.first[e]), word[j]));
      }
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (worded >> j & 1) x[u * kVec + j] = __uint_as_float(word[i * kVec + j]);
    }
    const uint32_t bits = o.mask ? from.allowed(o.mask, vec) : ~0u;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      float& v = x[u * kVec + j];
      if (!(bits >> j & 1)) v = -INFINITY;
      if (v != v) nan = true, v = -INFINITY;
      v = clean(v);
      if (v > best) best = v, best_e = token(u * kVec + j);
      count += v > -INFINITY;
    }
  }
  const u64 top = block_max(best > -INFINITY ? key_of(best, best_e) : 0, room);
  nan = __syncthreads_or(nan);
  const Pick pick = s_pick;
  Record* rec = w.record + (int64_t)row * blocks + stretch;
  const Scale s(x_of(top), pick.T);
  float sum = 0.f;
  int token_out = -1;
  float token_x = 0.f;
  if (top) {
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (x[i] > -INFINITY) part += s.weight(x[i]);
    sum = block_sum(part, room_f);
    if (pick.cut()) {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (x[i] > -INFINITY) {
          const int b = s.bin(x[i]);
          atomicAdd(&bin_n[b], 1u);
          const unsigned share = s.share(x[i], b);
          if (share) atomicAdd(&bin_w[b], share);
        }
      for (int d = 16; d; d /= 2) count += __shfl_xor_sync(~0u, count, d);
      if (t % 32 == 0) room_n[t / 32] = count;
      __syncthreads();
      const int64_t at = ((int64_t)row * blocks + stretch) * kBins + t;
      w.bin_n[at] = bin_n[t], w.bin_w[at] = bin_w[t];
      count = 0;
      for (int i = 0; i < kWarps; ++i) count += room_n[i];
    } else if (pick.T > 0.f) {
      const float* noise = p.noise + row * p.noise_stride;
      float e[kEach], fast = -INFINITY;
#pragma unroll
      for (int i = 0; i < kEach; ++i) e[i] = x[i] > -INFINITY ? noise[token(i)] : 0.f;
#pragma unroll
      for (int i = 0; i < kEach; ++i) fast = fmaxf(fast, s.score(x[i], e[i]));
      const u64 all = block_max(fast > -INFINITY ? key_of(fast, 0) : 0, room);
      if (all) {
        const float near = Scale::near(x_of(all));
        u64 mine = 0;
        int mine_e = 0;
        float mine_x = 0.f;
        if (fast >= near) {
#pragma unroll 1
          for (int i = 0; i < kEach; ++i) {
            // by its place again: an index that is not known when compiled would put x and e in memory
            float v = x[0], f = e[0];
#pragma unroll
            for (int j = 1; j < kEach; ++j)
              if (i == j) v = x[j], f = e[j];
            if (s.score(v, f) < near) continue;
            const u64 key = s.exact(v, f);
            if (key > mine) mine = key, mine_e = token(i), mine_x = v;
          }
        }
        const u64 high = block_max(mine, room);
        const u64 low = block_max(mine && mine == high ? (u64)(uint32_t)~mine_e << 32 | __float_as_uint(mine_x) : 0, room);
        token_out = (int)~(uint32_t)(low >> 32), token_x = __uint_as_float((uint32_t)low);
      }
    }
  }
  if (w.x && pick.cut()) {
    float* to = w.x + (int64_t)row * w.places;
#pragma unroll
    for (int u = 0; u < kEach / 4; ++u) {
      const int at = p0 + (u * 4 / kVec * kRowThreads + t) * kVec + u * 4 % kVec;
      if (at < w.places) *(float4*)(to + at) = float4{x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]};
    }
  }
  if (t == 0) {
    Record c = {top, sum, nan, token_out, token_x, count, pick.k, pick.T, pick.p, pick.m, 0};
    *rec = c;
  }
}

// ---------------------------------------------------------------- the row's pick

struct Shared {
  u64 room[kWarps];
  u64 list[kList];          // keys
  u64 mass_total;
  u64 border_mass, base_mass;
  float room_f[kWarps];
  unsigned room_n[kWarps];
  unsigned bin_n[kBins], bin_lo[kBins], bin_hi[kBins];
  int away[kMaxStretches];  // bins from the row's first token to the stretch's, kBins: no token
  int found, at, last, n_list;
  unsigned base_count, bin_count;
};

// A row's logits, adjusted, as loads of several; f(x, token) for each that takes part.
template <class T>
struct RowAgain {
  RowOf<T> row;
  const float* x;   // adjusted and stored by place, or null
  int places;
  template <class F>
  __device__ void each(int p0, int p1, F f) const {
    constexpr int kVec = RowOf<T>::kVec;
    const int end = min(p1, places);
    for (int q = p0 + threadIdx.x * kVec; q < end; q += kRowThreads * kVec) {
      float v[kVec];
      if (x) {
#pragma unroll
        for (int j = 0; j < kVec; j += 4) {
          const float4 a = *(const float4*)(x + q + j);
          v[j] = a.x, v[j + 1] = a.y, v[j + 2] = a.z, v[j + 3] = a.w;
        }
      } else {
        row.load(q / kVec, v);
      }
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (v[j] > -INFINITY) f(clean(v[j]), q - row.shift + j);
    }
  }
};

// Smallest number whose share of 2^64 parts p is of `all`: the whole number at or above p * all.
__device__ u64 part_of(float p, u64 all) {
  if (!(p > 0.f)) return 1;
  const u64 f = __float2ull_rn(p * 0x1p63f);  // p < 1 has 24 bits: exact above 2^-40
  const u64 hi = __umul64hi(all, f), lo = all * f;
  const u64 up = (hi << 1 | lo >> 63) + ((lo << 1) != 0);
  return max(up, (u64)1);
}

template <class T>
struct Picker {
  Shared& s;
  Scale& scale;
  const RowAgain<T>& row;
  float one;               // 2^shift: weights of 1 / 2^kWeightBits of the first token's bin in whole numbers

  __device__ u64 mass_of_bin(int b) const { return __float2ull_rn(exp2f((float)b * (-1.44269504f / kBinsPerUnit)) * one); }
  __device__ u64 mass(float x, int b) const { return scale.share(x, b) * mass_of_bin(b); }

  // Adds a token of this weight to a bin of the row's.
  __device__ void count(int bin, unsigned w) {
    atomicAdd(&s.bin_n[bin], 1u);
    const unsigned was = atomicAdd(&s.bin_lo[bin], w);
    if (was + w < was) atomicAdd(&s.bin_hi[bin], 1u);
  }

  // Sorts s.list[0, n), the largest first.
  __device__ void sort(int n) {
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += kRowThreads) s.list[i] = 0;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
      for (int d = run / 2; d; d /= 2) {
        for (int i = threadIdx.x; i < size / 2; i += kRowThreads) {
          const int a = i / d * 2 * d + i % d, b = a + d;
          const u64 x = s.list[a], y = s.list[b];
          if ((x < y) == ((a & run) == 0)) s.list[a] = y, s.list[b] = x;
        }
        __syncthreads();
      }
  }

  // Collects the tokens that f holds for.  Returns their number (at most kList are kept).
  template <class F>
  __device__ void collect(int p0, int p1, F f) {
    row.each(p0, p1, [&](float x, int e) {
      if (f(x, e)) {
        const int at = atomicAdd(&s.n_list, 1);
        if (at < kList) s.list[at] = key_of(x, e);
      }
    });
  }

  // The key at which the sum over the order (of tokens, or of their mass) first reaches target, the tokens of bin `bin` being
  // those in question, `base` what is before them.  Leaves the mass up to there in s.border_mass.
  __device__ u64 border(bool by_mass, u64 target, int bin, unsigned n, u64 base, u64 base_mass) {
    const int t = threadIdx.x;
    u64 lo = 0, hi = ~0ull;
    for (int turn = 0; n > kList && turn < 16; ++turn) {
      u64 a = 0, b = 0;  // the largest of ~key and of key
      row.each(0, row.places, [&](float x, int e) {
        const u64 key = key_of(x, e);
        if (key >= lo && key <= hi && scale.bin(x) == bin) a = max(a, ~key), b = max(b, key);
      });
      lo = ~block_max(a, s.room), hi = block_max(b, s.room);
      int shift = 0;
      while (((hi - lo) >> shift) >= kBins) ++shift;
      __syncthreads();
      s.bin_n[t] = s.bin_lo[t] = s.bin_hi[t] = 0;
      __syncthreads();
      row.each(0, row.places, [&](float x, int e) {
        const u64 key = key_of(x, e);
        if (key < lo || key > hi || scale.bin(x) != bin) return;
        count((int)((hi - key) >> shift), scale.share(x, bin));
      });
      __syncthreads();
      const unsigned mine_n = s.bin_n[t];
      const u64 mine_w = ((u64)s.bin_hi[t] << 32 | s.bin_lo[t]) * mass_of_bin(bin);
      const u64 before_n = block_before<u64>(mine_n, s.room), before_w = block_before<u64>(mine_w, s.room);
      if (t == 0) s.at = -1;
      __syncthreads();
      const u64 before = base + (by_mass ? before_w : before_n), mine = by_mass ? mine_w : mine_n;
      if (before < target && before + mine >= target) {
        s.at = t, s.bin_count = mine_n, s.base_mass = base_mass + before_w, s.base_count = (unsigned)before_n;
      }
      __syncthreads();
      if (s.at < 0) break;  // no token reaches it: cannot be, as the sums are of the same whole numbers
      base = by_mass ? s.base_mass : base + s.base_count, base_mass = s.base_mass;
      n = s.bin_count;
      hi -= (u64)s.at << shift;
      const u64 least = hi - ((1ull << shift) - 1);
      if (least > lo && least <= hi) lo = least;
      __syncthreads();
    }
    if (t == 0) s.n_list = 0;
    __syncthreads();
    collect(0, row.places, [&](float x, int e) {
      const u64 key = key_of(x, e);
      return key >= lo && key <= hi && scale.bin(x) == bin;
    });
    __syncthreads();
    const int m = min(s.n_list, kList);
    sort(m);
    return along(m, by_mass, target, base, base_mass);
  }

  // The same over the sorted list alone.  s.last is the number of tokens up to there.
  __device__ u64 along(int m, bool by_mass, u64 target, u64 base, u64 base_mass) {
    constexpr int kMine = kList / kRowThreads;
    const int t = threadIdx.x;
    u64 part[kMine], sum = 0;
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
      const int i = t * kMine + j;
      const float x = i < m ? x_of(s.list[i]) : 0.f;
      part[j] = i < m ? mass(x, scale.bin(x)) : 0;
      sum += part[j];
    }
    u64 w = base_mass + block_before<u64>(sum, s.room);
    if (t == 0) s.last = m, s.border_mass = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
      const int i = t * kMine + j;
      const u64 before = by_mass ? w : base + i;
      w += part[j];
      const u64 after = by_mass ? w : base + i + 1;
      if (i < m && ((before < target && after >= target) || (i == m - 1 && after < target))) s.last = i + 1, s.border_mass = w;
    }
    __syncthreads();
    return s.last > 0 ? s.list[s.last - 1] : 0;
  }
};

template <class T>
__global__ void __launch_bounds__(kRowThreads) hx_sample_pick(const hx_logits in, const hx_pick p, const Work w, int blocks) {
  __shared__ Shared s;
  const int row = blockIdx.x, t = threadIdx.x, lane = t % 32;
  const Record* rec = w.record + (int64_t)row * blocks;
  // every warp adds up the stretches by itself
  u64 top = 0;
  bool nan = false;
  for (int c = lane; c < blocks; c += 32) top = max(top, rec[c].top), nan |= rec[c].nan != 0;
  top = warp_max(top);
  nan = __any_sync(~0u, nan);
  const Pick pick = {rec[0].k, rec[0].T, rec[0].p, rec[0].m};
  Scale scale(x_of(top), pick.T);
  const bool cut = top && pick.cut();
  double sum = 0.;
  if (t < 32) {
    for (int c = lane; c < blocks; c += 32)
      if (rec[c].top) {
        const float x = x_of(rec[c].top);
        if (scale.top < INFINITY || x == scale.top) sum += x == scale.top ? (double)rec[c].sum : (double)rec[c].sum * exp(((double)x - (double)scale.top) / (double)scale.T);
      }
    for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
  }
  u64 best = 0;       // the race's best score, in 64 bits
  int token = token_of(top);
  float token_x = scale.top;
  const float* noise = p.noise + row * p.noise_stride;
  if (cut) {
    RowAgain<T> again = {RowOf<T>(in, row), w.x ? w.x + (int64_t)row * w.places : nullptr, w.places};
    Picker<T> a{s, scale, again, 1.f};
    // bins of the whole row: of its stretches'; where the grid is too coarse for them (T is small), of its tokens', from
    // the first token down
    const bool fine = scale.fine();
    if (t < blocks) {
      const u64 first = rec[t].top;
      s.away[t] = !first ? kBins : fine ? scale.bin(x_of(first)) : 0;
    }
    s.bin_n[t] = s.bin_lo[t] = s.bin_hi[t] = 0;
    __syncthreads();
    unsigned n = 0;
    u64 sum_w = 0;
    int all = 0;
    for (int c = 0; c < blocks; ++c) {
      const int b = t - s.away[c];
      if (s.away[c] < kBins) all += rec[c].count;
      if (fine && b >= 0 && t < kBins - 1) {
        const int64_t at = ((int64_t)row * blocks + c) * kBins + b;
        n += w.bin_n[at], sum_w += w.bin_w[at];
      }
    }
    if (!fine) {
      scale.zero = scale.top;
      again.each(0, w.places, [&](float x, int e) {
        const int b = scale.bin(x);
        a.count(b, scale.share(x, b));
      });
      __syncthreads();
      if (t < kBins - 1) n = s.bin_n[t], sum_w = (u64)s.bin_hi[t] << 32 | s.bin_lo[t];
    }
    unsigned n_before = block_before<unsigned>(n, s.room_n);
    if (t == kBins - 1) n = (unsigned)all - n_before;  // all that is further down
    // as many bits for the sums as fit
    const float about = block_sum(exp2f((float)t * (-1.44269504f / kBinsPerUnit)) * (float)sum_w, s.room_f);
    const int bits = min(44, 60 - (int)(__float_as_uint(fmaxf(about, 1.f)) >> 23) + 127);
    a.one = __uint_as_float((uint32_t)(127 + max(bits, 0)) << 23);
    const u64 mass = sum_w * a.mass_of_bin(t);
    const u64 mass_before = block_before<u64>(mass, s.room);
    if (t == kBins - 1) s.mass_total = mass_before + mass;
    if (t == 0) s.at = kBins - 1, s.last = kBins - 1;
    __syncthreads();
    const u64 total = s.mass_total;
    const bool by_k = pick.k > 0 && pick.k < all, by_p = pick.p < 1.f;
    const u64 want = by_p ? min(part_of(pick.p, total), total) : 0;
    // the bins that k and p end in (p of all mass)
    if (by_k && n_before < (unsigned)pick.k && n_before + n >= (unsigned)pick.k) s.at = t;
    if (by_p && mass_before < want && mass_before + mass >= want) s.last = t;
    __syncthreads();
    const int bin_k = s.at, bin_p = s.last;
    int reach = by_k ? bin_k : by_p ? bin_p : kBins - 1;
    if (pick.m > 0.f && !(by_k && by_p)) {
      // what has at least m of the first token's weight is no further down than this
      const float far = -logf(pick.m) * kBinsPerUnit + 3.f;
      reach = min(reach, far < (float)kBins ? max((int)far, 0) : kBins - 1);
    }
    const float log_least = pick.m > 0.f ? logf(pick.m) : -INFINITY;
    __syncthreads();
    if (t == reach) s.bin_count = n_before + n;
    if (t == 0) s.n_list = 0;
    __syncthreads();
    float fast = -INFINITY;
    if (s.bin_count <= kList) {
      // all that the filters can leave fits the list
      for (int c = 0; c < blocks; ++c)
        if (s.away[c] <= reach)
          a.collect(c * kStretch, (c + 1) * kStretch, [&](float x, int e) { return scale.bin(x) <= reach; });
      __syncthreads();
      const int m = min(s.n_list, kList);
      a.sort(m);
      int left = m;
      u64 of = total;
      if (by_k && reach == bin_k) {
        a.along(m, false, (u64)pick.k, 0, 0);
        left = s.last, of = s.border_mass;
        __syncthreads();
      }
      if (by_p) {
        a.along(left, true, min(part_of(pick.p, of), of), 0, 0);
        left = min(left, s.last);
        __syncthreads();
      }
      constexpr int kMine = kList / kRowThreads;
      float e[kMine];
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        const int i = t + j * kRowThreads;
        e[j] = 0.f;
        if (i < left) {
          const float x = x_of(s.list[i]);
          if (i == 0 || !(scale.below(x) < log_least)) e[j] = noise[token_of(s.list[i])];
        }
      }
#pragma unroll
      for (int j = 0; j < kMine; ++j)
        if (e[j] != 0.f) fast = fmaxf(fast, scale.score(x_of(s.list[t + j * kRowThreads]), e[j]));
      const u64 most = block_max(fast > -INFINITY ? key_of(fast, 0) : 0, s.room);
      if (most) {
        const float near = Scale::near(x_of(most));
        u64 mine = 0, at = 0;
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
          if (e[j] == 0.f) continue;
          const u64 key = s.list[t + j * kRowThreads];
          if (scale.score(x_of(key), e[j]) < near) continue;
          const u64 f = scale.exact(x_of(key), e[j]);
          if (f > mine || (f == mine && (uint32_t)key > (uint32_t)(at >> 32))) mine = f, at = key << 32 | __float_as_uint(x_of(key));
        }
        best = block_max(mine, s.room);
        const u64 low = block_max(mine && mine == best ? at : 0, s.room);
        token = (int)~(uint32_t)(low >> 32), token_x = __uint_as_float((uint32_t)low);
      }
    } else {
      u64 border = 0, of = total;
      auto start = [&](int bin) {  // what lies before a bin
        __syncthreads();
        if (t == bin) s.bin_count = n, s.base_count = n_before, s.base_mass = mass_before;
        __syncthreads();
      };
      if (by_k) {
        start(bin_k);
        const unsigned c = s.bin_count, c0 = s.base_count;
        const u64 m0 = s.base_mass;
        border = a.border(false, (u64)pick.k, bin_k, c, c0, m0);
        of = s.border_mass;
        __syncthreads();
      }
      if (by_p) {
        const u64 target = min(part_of(pick.p, of), of);
        if (t == 0) s.at = bin_k;
        __syncthreads();
        if (mass_before < target && mass_before + mass >= target) s.at = t;
        __syncthreads();
        const int bin = s.at;
        start(bin);
        const unsigned c = s.bin_count;
        const u64 m0 = s.base_mass;
        border = max(border, a.border(true, target, bin, c, m0, m0));
        __syncthreads();
      }
      auto kept = [&](float x, u64 key) { return key >= border && (key == top || !(scale.below(x) < log_least)); };
      again.each(0, w.places, [&](float x, int e) {
        if (kept(x, key_of(x, e))) fast = fmaxf(fast, scale.score(x, noise[e]));
      });
      const u64 most = block_max(fast > -INFINITY ? key_of(fast, 0) : 0, s.room);
      if (most) {
        const float near = Scale::near(x_of(most));
        u64 mine = 0, at = 0;
        if (fast >= near)
          again.each(0, w.places, [&](float x, int e) {
            if (!kept(x, key_of(x, e)) || scale.score(x, noise[e]) < near) return;
            const u64 f = scale.exact(x, noise[e]);
            if (f > mine) mine = f, at = (u64)(uint32_t)~e << 32 | __float_as_uint(x);
          });
        best = block_max(mine, s.room);
        const u64 low = block_max(mine && mine == best ? at : 0, s.room);
        token = (int)~(uint32_t)(low >> 32), token_x = __uint_as_float((uint32_t)low);
      }
    }
  } else if (top && pick.T > 0.f && t < 32) {
    u64 mine = 0, at = 0;
    for (int c = lane; c < blocks; c += 32)
      if (rec[c].token >= 0) {
        const u64 f = scale.score(rec[c].token_x, noise[rec[c].token]) > -INFINITY ? scale.exact(rec[c].token_x, noise[rec[c].token]) : 0;
        if (f > mine) mine = f, at = (u64)(uint32_t)~rec[c].token << 32 | __float_as_uint(rec[c].token_x);
      }
    best = warp_max(mine);
    const u64 low = warp_max(mine && mine == best ? at : 0);
    if (best) token = (int)~(uint32_t)(low >> 32), token_x = __uint_as_float((uint32_t)low);
  }
  if (t == 0) {
    p.token[row] = top ? token : -1;
    if (p.logprob) {
      const double y = token_x == scale.top ? 0. : ((double)token_x - (double)scale.top) / (double)scale.T;
      p.logprob[row] = nan ? NAN : top ? (float)(y - log(sum)) : -INFINITY;
    }
  }
}

bool may_cut(const hx_pick& p) { return p.noise && (p.top_k || p.top_p || p.min_p || p.all_top_k > 0 || p.all_top_p < 1.f || p.all_min_p > 0.f); }

// The parts of a call's workspace.
Work work_of(const hx_logits& x, const hx_rules& r, const hx_pick& p, void* at) {
  const int vec = x.dtype == HX_F32 ? 4 : 8;
  const int64_t blocks = (int64_t)x.n_rows * stretches(x);
  Work w = {};
  char* base = (char*)at;
  auto part = [&](int64_t bytes) {
    void* here = base + w.bytes;
    w.bytes += (bytes + 255) / 256 * 256;
    return here;
  };
  w.places = (x.n_vocab + 2 * vec - 2) / vec * vec;
  w.record = (Record*)part(blocks * (int64_t)sizeof(Record));
  if (may_cut(p)) {
    w.bin_n = (unsigned*)part(blocks * kBins * 4);
    w.bin_w = (unsigned*)part(blocks * kBins * 4);
    if (r.history || r.bias_start || r.mask) w.x = (float*)part((int64_t)x.n_rows * w.places * 4);
  }
  return w;
}

template <class T>
cudaError_t sample_typed(const hx_logits& x, const hx_rules& r, const hx_pick& p, cudaStream_t s) {
  const Work w = work_of(x, r, p, p.workspace);
  const int blocks = stretches(x);
  const unsigned grid = (unsigned)x.n_rows * blocks;
  if (r.history || r.bias_start)
    hx_sample_scan<T, true><<<grid, kRowThreads, 0, s>>>(x, r, p, w, blocks);
  else
    hx_sample_scan<T, false><<<grid, kRowThreads, 0, s>>>(x, r, p, w, blocks);
  if (cudaError_t e = cudaGetLastError()) return e;
  hx_sample_pick<T><<<x.n_rows, kRowThreads, 0, s>>>(x, p, w, blocks);
  return cudaGetLastError();
}

}  // namespace

int64_t sample_workspace(const hx_logits& x, const hx_rules& r, const hx_pick& p) { return work_of(x, r, p, nullptr).bytes; }

cudaError_t launch_sample(const hx_logits& x, const hx_rules& r, const hx_pick& p, cudaStream_t s) {
  if (x.dtype == HX_BF16) return sample_typed<__nv_bfloat16>(x, r, p, s);
  if (x.dtype == HX_F16) return sample_typed<__half>(x, r, p, s);
  return sample_typed<float>(x, r, p, s);
}

}  // namespace hx
