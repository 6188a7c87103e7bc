// hx_kv_attend.cu -- attention of a step's tokens over the paged 8-bit cache:
// requests of few rows (a row: one token and query head of a kv head's group),
// which is every request that decodes.
#include <algorithm>
#include <type_traits>

#include "hx_kv_attend.cuh"

namespace hx {
namespace {

// out = softmax(c q k^T) v for up to 8 or 16 rows that share their keys: bound by
// reading the cache once.  An item is one request and kv head; its tokens are cut
// into tiles of kTokens, and all items' tiles, laid end to end, are dealt out to the blocks in
// equal stretches, whatever the lengths.  Two warps of a block fetch, keys and values
// (tile copies into a ring of kStages), the others compute, each on its own tiles with its own running
// maximum, sum and rows x D sums, joined where an item ends.  An item that
// several blocks share leaves partial results, joined by a second kernel in a fixed order, so
// that a result never depends on the order in which blocks run.
//
// Tokens are the matrix instructions' 16 rows and the few rows their 8 columns:
// S^T = K Q^T, O^T = V^T P^T.  So eight rows waste nothing (16 x 8 x 16 the other way round would
// compute 16), and the sums take half the registers, which lets 12 computing warps reside on an SM.
//
// 48 requests of 32000 tokens, 32 heads on 8 of 128: 505 us, 6.4 TB/s, 95 % of a copy.  500 requests of 437 to
// 18133 tokens, 28 heads on 4 of 64, blocks of 16: 224 us, 4.0 TB/s: instructions, of which a column of 64 takes as
// many for its softmax as one of 128.  One request of 5065 tokens: 14.8 us, latency.
constexpr int kRows = 16;  // most rows of an item
constexpr int kStageBytes = 8192;
constexpr int kTileBytes = kStageBytes / 2;

// D: head dim, NR: rows in eights.
template <int D, int NR>
struct Shape {
  static constexpr int kTokens = kTileBytes / D;  // of a tile: 32 or 64
  static constexpr int kGroups = kTokens / 16;    // 16 tokens lie in one block of the cache
  static constexpr int kWarps = NR * D <= 128 ? 6 : 4;  // computing warps, by the registers of their sums
  static constexpr int kThreads = 32 * (kWarps + 2);
  static constexpr int kMergeRow = D + 4;         // floats; padded against bank conflicts
  static constexpr int kMergeBytes = 4 * 8 * NR * kMergeRow * 4;
  static constexpr int kStages = (106 * 1024 - kMergeBytes) / kStageBytes;
  static constexpr int kSmem = kStages * kStageBytes + kMergeBytes + 1024;
};

// Where a tile of keys or of values lies, its scales, and which of its groups of 16 tokens are fetched.
struct __align__(16) Tile {
  float scale[4];  // (values': times kSumDown)
  int id[4];  // blocks of the cache, -1: not fetched
  int y;      // row in the tile map
  uint32_t bytes, valid;
};
// Tiles are looked up kAhead at a time, and a tile is read no later than kStages after it.
constexpr int kAhead = 16, kTiles = 32;

// What an item costs a block beside its tiles (joining the warps' sums), in tiles.
constexpr int kItemCost = 3;

// The length of an item, 0: it is not this kernel's.  It begins with kItemCost places without a tile, so that
// stretches with many items have fewer tiles.  An item that sees nothing, with any number of rows,
// has no others, but is dealt out, so that its zeros are written.
template <int D>
__device__ __forceinline__ int length_of(const AttendArgs& a, const Request& q, int* first_tile) {
  constexpr int NT = kTileBytes / D;
  *first_tile = 0;
  if (q.n == 0) return 0;
  if (q.kv == 0) return kItemCost;
  if (q.n * a.group > a.few_rows) return 0;
  *first_tile = see_from(a, q, 0) / NT;
  return kItemCost + (q.kv + NT - 1) / NT - *first_tile;
}

// A place in the sequence of all items.
template <int D>
struct Place {
  int r, h, o, length, first_tile;
  Request q;
  __device__ void load(const AttendArgs& a) {
    q = request(a, r);
    length = length_of<D>(a, q, &first_tile);
  }
  // Steps by d places; false past the last request.
  __device__ bool step(const AttendArgs& a, int d) {
    o += d;
    while (o >= length) {
      o -= length;
      if (length && ++h < a.n_kv_heads) continue;
      h = 0;
      do {
        if (++r >= a.n_rows) return false;
        load(a);
      } while (!length);
    }
    return true;
  }
};

template <int kThreads>
__device__ __forceinline__ void sync_consumers() {
  asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
}

// The 8 x 8 matrix of 16-bit values that a warp holds, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <class T>
__device__ __forceinline__ float2 to_float2(uint32_t u);
template <>
__device__ __forceinline__ float2 to_float2<__half>(uint32_t u) {
  return __half22float2(*(const __half2*)&u);
}
template <>
__device__ __forceinline__ float2 to_float2<__nv_bfloat16>(uint32_t u) {
  return __bfloat1622float2(*(const __nv_bfloat162*)&u);
}
template <class T>
__device__ __forceinline__ uint32_t from_float2(float x, float y);
template <>
__device__ __forceinline__ uint32_t from_float2<__half>(float x, float y) {
  return pack_half(x, y);
}
template <>
__device__ __forceinline__ uint32_t from_float2<__nv_bfloat16>(float x, float y) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *(const uint32_t*)&h;
}

// Writes zeros and -inf for `rows` rows of an item (all of them: any number).
template <class T>
__device__ void write_empty(const AttendArgs& a, int D, const Request& q, int h, int tid, int threads) {
  const int64_t rows = (int64_t)q.n * a.group;
  const int units = D / 8;
  for (int64_t i = tid; i < rows * units; i += threads) {
    const int64_t x = i / units;
    const int token = q.first + (int)(x / a.group), head = h * a.group + (int)(x % a.group);
    *(uint4*)((T*)a.out + token * a.out_token_stride + head * a.out_head_stride + (i % units) * 8) = uint4{0, 0, 0, 0};
    if (i % units == 0 && a.lse) a.lse[(int64_t)token * a.n_heads + head] = -INFINITY;
  }
}

// One thread of the warp, the same each time; what it does, the hardware takes from uniform registers.
__device__ __forceinline__ bool elected() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p;
}

// A fetching warp, of keys (V = 0) or of values: looks tiles up, a lane each, one batch ahead of the
// copies that it issues.  A look-up is two loads that depend on one another (block number, its
// scale); they are placed before and halfway through the copies of the batch before, which hide them.
template <int D, int NR, int V>
__device__ void produce(const AttendArgs& a, const CUtensorMap* map, Place<D> at, int count, uint8_t* ring, Tile* tiles,
                        uint64_t* full, uint64_t* empty, volatile int* dead) {
  using S = Shape<D, NR>;
  const int lane = threadIdx.x & 31;
  const int block = 1 << a.block_shift;
  const int box = min(block, S::kTokens), pieces = S::kTokens / box;
  int stage = 0;
  uint32_t turn = 0;
  bool more = at.step(a, lane), tile = false;
  int id[4] = {-1, -1, -1, -1}, y = 0, h = 0;
  float scale[4];
  uint32_t bytes = 0, valid = 0;

  const auto look_up = [&](int base) {
    tile = more && lane < kAhead && base + lane < count && at.o >= kItemCost;
#pragma unroll
    for (int p = 0; p < 4; ++p) id[p] = -1;
    if (tile) {
      const int pos = (at.first_tile + at.o - kItemCost) * S::kTokens;
      const int32_t* row = a.block_table + at.r * a.table_stride + (pos >> a.block_shift);
      h = at.h;
      y = h * block + (pos & (block - 1));
#pragma unroll
      for (int p = 0; p < 4; ++p)
        if (p < pieces && pos + p * box < at.q.kv) id[p] = row[p];
    }
    if (more) more = at.step(a, kAhead);
  };
  const auto scales = [&] {
    bytes = valid = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      float x = 0.f;
      if ((unsigned)id[p] < (unsigned)a.n_blocks) {
        x = (V ? a.v_scale : a.k_scale)[id[p] * a.scale_stride + h];
        bytes += box * D;
      } else {
        id[p] = -1;
      }
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g)
        if (g * 16 / box == p) {
          scale[g] = x;
          if (id[p] >= 0) valid |= 1u << g;
        }
    }
  };
  // Tiles are numbered, places without one are not: `number` is the next batch's first.
  int number = 0;
  const auto store = [&]() -> int {
    const unsigned who = __ballot_sync(~0u, tile);
    if (tile) {
      Tile& x = tiles[(number + __popc(who & ((1u << lane) - 1))) & (kTiles - 1)];
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g) x.scale[g] = V ? scale[g] * kSumDown : scale[g];
#pragma unroll
      for (int p = 0; p < 4; ++p) x.id[p] = id[p];
      x.y = y, x.bytes = bytes, x.valid = valid;
    }
    __syncwarp();
    return __popc(who);
  };
  // The whole warp goes through the loop, and one elected thread issues: with the loop inside that thread's
  // branch the operands leave the uniform registers (48 requests of 32000 tokens 705 us against 535).
  const auto issue = [&](int from, int to) -> bool {
    for (int k = from; k < to; ++k) {
      const Tile& x = tiles[k & (kTiles - 1)];
      const int at_y = x.y;
      const uint32_t expect = x.bytes;
      const int4 ids = *(const int4*)x.id;
      uint8_t* dst = ring + stage * kStageBytes + V * kTileBytes;
      if (!__all_sync(~0u, bar_wait(&empty[2 * stage + V], (turn & 1) ^ 1, dead))) return false;
      uint64_t* const landed = &full[2 * (2 * stage + V) + (turn & 1)];
      if (elected()) {
        bar_expect(landed, expect);
        if (ids.x >= 0) tile_load(dst, map, landed, 0, at_y, ids.x);
        if (pieces > 1) {
          if (ids.y >= 0) tile_load(dst + box * D, map, landed, 0, at_y, ids.y);
          if (ids.z >= 0) tile_load(dst + 2 * box * D, map, landed, 0, at_y, ids.z);
          if (ids.w >= 0) tile_load(dst + 3 * box * D, map, landed, 0, at_y, ids.w);
        }
      }
      __syncwarp();
      if (++stage == S::kStages) stage = 0, ++turn;
    }
    return true;
  };

  look_up(0);
  scales();
  for (int base = 0; base < count;) {
    const int have = store();
    base += kAhead;
    const bool next = base < count;
    if (next) look_up(base);
    if (!issue(number, number + have / 2)) return;
    if (next) scales();
    if (!issue(number + have / 2, number + have)) return;
    number += have;
  }
}

// Where the four threads of a row find their values in a tile.  Rows of D
// bytes lie in shared memory with their 16-byte units permuted by the tile copy
// (by the row's low bits); column n of a matrix instruction is token order(n) of eight, so that
// both the keys' 16-byte reads and the values' fall on different banks.
template <int D>
__device__ __forceinline__ int order(int n) {
  return ((D == 128 ? 0x37156240u : 0x67542310u) >> (4 * n)) & 7;
}

template <int D, int NR, class T>
__device__ void consume(const AttendArgs& a, Place<D> at, int count, const uint8_t* ring, const Tile (*tiles)[kTiles],
                        uint64_t* full, uint64_t* empty, volatile int* dead, float* merge, float (*s_ml)[kRows][2]) {
  using S = Shape<D, NR>;
  constexpr int NT = S::kTokens, KJ = D / 64, ND = D / 16, W = S::kWarps;
  // a maximum may lag by this factor of two: the weights then reach 2^8, far from f16's limit, and
  // most tiles need neither the maximum over the warp nor new factors
  constexpr float kLag = 8.f;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, q4 = lane & 3;
  const int tn = order<D>(n), ta = order<D>(2 * q4), tb = order<D>(2 * q4 + 1);
  // the permutation of 16-byte units in the rows of this thread's key and two values
  const int swk = D == 128 ? tn : (tn >> 1) & 3;
  const int swa = D == 128 ? ta : (ta >> 1) & 3, swb = D == 128 ? tb : (tb >> 1) & 3;

  int it = 0;  // tiles fetched so far, over all items
  int stage = warp, left = warp;  // this warp's next: its place in the ring, and its number less `it`
  uint32_t turn = 0;
  // Tiles land in any order, and the tile before this one in its place is another warp's, which need not have
  // landed: a barrier tells a phase from the one before it only.  So a place has two of them, for its tiles
  // by turns; the tile two before has been used, or this one would not have been asked for.
  const auto landed = [&](int x) { return bar_wait(&full[2 * x + (turn & 1)], turn >> 1 & 1, dead); };
  bool more = true;
  while (more && count > 0) {
    // this block's places of the item, and its tiles among them
    const int places = min(count, at.length - at.o), tile0 = max(0, at.o - kItemCost);
    const int seg = places - (at.o ? 0 : kItemCost);
    const Request q = at.q;
    const int rows = q.n * a.group;
    if (q.kv == 0) {
      write_empty<T>(a, D, q, at.h, threadIdx.x, 32 * W);
      count -= places;
      more = at.step(a, places);
      continue;
    }

    // q of row n (of each eight) in f16, scaled by a power of two so that no value leaves f16's range: exact down to
    // 2^-14 of the row's largest, what lies below is off by 2^-25 of that at most
    uint32_t bq[NR][KJ * 4][2];
    float c[NR][2];  // factors of the scores of rows 2 q4 and 2 q4 + 1, and what those rows see
    int lo[NR][2], hi[NR][2];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int row = n + 8 * r, token = row / a.group;
      const bool real = row < rows;
      const T* p = (const T*)a.q + (q.first + token) * a.q_token_stride + (at.h * a.group + row % a.group) * a.q_head_stride;
      uint4 raw[KJ][2];
#pragma unroll
      for (int j = 0; j < KJ; ++j)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          raw[j][u] = real ? *(const uint4*)(p + 16 * (q4 + 4 * j) + 8 * u) : uint4{0, 0, 0, 0};
      float amax = 0;
#pragma unroll
      for (int j = 0; j < KJ; ++j)
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float2 f = to_float2<T>(((const uint32_t*)raw[j])[u]);
          amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
      amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
      int e = 0;
      if (amax > 0 && amax < INFINITY) e = max((int)(__float_as_uint(amax) >> 23) - 127, -126);
      const float down = __uint_as_float((unsigned)(127 - e) << 23);
#pragma unroll
      for (int j = 0; j < KJ; ++j)
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float2 f = to_float2<T>(((const uint32_t*)raw[j])[u]);
          bq[r][4 * j + (u >> 1)][u & 1] = pack_half(f.x * down, f.y * down);
        }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int col = 2 * q4 + x, i = (col + 8 * r) / a.group;
        c[r][x] = a.sm_scale_log2 * __uint_as_float((unsigned)(127 + __shfl_sync(~0u, e, 4 * col)) << 23);
        lo[r][x] = col + 8 * r < rows ? see_from(a, q, i) : 0;
        hi[r][x] = col + 8 * r < rows ? see_to(a, q, i) : 0;
      }
    }
    // where every row sees everything: [all_lo, all_hi); where any sees something: [any_lo, any_hi)
    const int any_lo = see_from(a, q, 0), any_hi = q.kv;
    const int all_lo = see_from(a, q, q.n - 1), all_hi = see_to(a, q, 0);

    float acc[NR][ND][4];  // column tiles of 16 values by 8 rows
    float m[NR][2], l[NR][2];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
#pragma unroll
      for (int i = 0; i < ND; ++i) acc[r][i][0] = acc[r][i][1] = acc[r][i][2] = acc[r][i][3] = 0;
      m[r][0] = m[r][1] = -INFINITY, l[r][0] = l[r][1] = 0;
    }
    for (; left < seg; left += W) {
      // (a place whose tile has not been waited for to its end must not be filled again)
      const bool keys = landed(2 * stage);
      const uint8_t* kt = ring + stage * kStageBytes;
      const uint8_t* vt = kt + kTileBytes;
      const Tile& key_tile = tiles[0][(it + left) & (kTiles - 1)];
      const Tile& value_tile = tiles[1][(it + left) & (kTiles - 1)];
      const int pos = (at.first_tile + tile0 + left) * NT;
      const uint32_t valid = key_tile.valid;
      const bool whole = valid == (1u << S::kGroups) - 1 && pos >= all_lo && pos + NT <= all_hi;

      // scores: of group g, tokens tn and tn + 8 by rows 2 q4 and 2 q4 + 1
      float s[S::kGroups][NR][4];
      float top[NR][2];
#pragma unroll
      for (int r = 0; r < NR; ++r) top[r][0] = top[r][1] = -INFINITY;
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
        for (int r = 0; r < NR; ++r) s[g][r][0] = s[g][r][1] = s[g][r][2] = s[g][r][3] = 0;
      // two groups' products in turn: each waits for its own last one only
#pragma unroll
      for (int g0 = 0; g0 < S::kGroups; g0 += 2)
#pragma unroll
        for (int j = 0; j < KJ; ++j) {
          uint4 k[2][2];
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const uint8_t* p = kt + (16 * (g0 + g) + tn) * D + (((q4 + 4 * j) ^ swk) << 4);
            k[g][0] = *(const uint4*)p, k[g][1] = *(const uint4*)(p + 8 * D);
          }
#pragma unroll
          for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const uint32_t u0 = ((const uint32_t*)&k[g][0])[w], u1 = ((const uint32_t*)&k[g][1])[w];
              const uint32_t ak[4] = {cvt2(u0), cvt2(u1), cvt2_hi(u0), cvt2_hi(u1)};
#pragma unroll
              for (int r = 0; r < NR; ++r) mma16816(s[g0 + g][r], ak, bq[r][4 * j + w][0], bq[r][4 * j + w][1]);
            }
        }
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g) {
        const float ks = key_tile.scale[g];
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            s[g][r][y] *= ks * c[r][y & 1];
            if (!whole) {
              const int p = pos + 16 * g + tn + 4 * (y & 2);
              if (p < lo[r][y & 1] || p >= hi[r][y & 1] || !(valid >> g & 1)) s[g][r][y] = -INFINITY;
            }
            top[r][y & 1] = fmaxf(top[r][y & 1], s[g][r][y]);
          }
      }
      fence_async();
      __syncwarp();
      if (lane == 0 && keys) bar_arrive(&empty[2 * stage]);
      // values of tokens ta, tb, ta + 8, tb + 8 of each group, D / 8 columns each: on their way while the
      // softmax is done, and their place free again
      const bool values = landed(2 * stage + 1);
      uint32_t vw[S::kGroups][4][D / 32];
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const uint8_t* p = vt + (16 * g + 8 * (y >> 1) + (y & 1 ? tb : ta)) * D;
          const int sw = y & 1 ? swb : swa;
          if constexpr (D == 128) *(uint4*)vw[g][y] = *(const uint4*)(p + ((n ^ sw) << 4));
          else *(uint2*)vw[g][y] = *(const uint2*)(p + (((n >> 1) ^ sw) << 4) + ((n & 1) << 3));
        }
      float value_scale[S::kGroups];
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g) value_scale[g] = value_tile.scale[g];
      fence_async();
      __syncwarp();
      if (lane == 0 && values) bar_arrive(&empty[2 * stage + 1]);
      bool late = false;
#pragma unroll
      for (int r = 0; r < NR; ++r) late |= top[r][0] > m[r][0] + kLag || top[r][1] > m[r][1] + kLag;
      float keep[NR][2];
      const bool moved = __any_sync(~0u, late);
      if (moved) {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float z = fmaxf(m[r][x], top[r][x]);
            z = fmaxf(z, __shfl_xor_sync(~0u, z, 4));
            z = fmaxf(z, __shfl_xor_sync(~0u, z, 8));
            z = fmaxf(z, __shfl_xor_sync(~0u, z, 16));
            keep[r][x] = z == -INFINITY ? 1.f : ex2(m[r][x] - z);
            m[r][x] = z;
            l[r][x] *= keep[r][x];
          }
      }
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float base = m[r][x] == -INFINITY ? 0.f : m[r][x];
#pragma unroll
          for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
            for (int y = x; y < 4; y += 2) {
              s[g][r][y] = ex2(s[g][r][y] - base);
              l[r][x] += s[g][r][y];
            }
        }

      if (moved) {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int d = 0; d < ND; ++d)
            acc[r][d][0] *= keep[r][0], acc[r][d][1] *= keep[r][1], acc[r][d][2] *= keep[r][0], acc[r][d][3] *= keep[r][1];
      }
      // A scale that is infinite or no number reaches the rows that see something of its group, and no others.
      bool odd = false;
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g) odd |= !(fabsf(value_scale[g]) < INFINITY);
      if (odd) {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            bool none = false;
#pragma unroll
            for (int g = 0; g < S::kGroups; ++g)
              none |= !(fabsf(value_scale[g]) < INFINITY) && pos + 16 * g + 16 > lo[r][x] && pos + 16 * g < hi[r][x];
#pragma unroll
            for (int d = 0; d < ND; ++d)
              if (none) acc[r][d][x] = acc[r][d][2 + x] = NAN;
          }
#pragma unroll
        for (int g = 0; g < S::kGroups; ++g)
          if (!(fabsf(value_scale[g]) < INFINITY)) value_scale[g] = 0.f;
      }
      uint32_t bp[S::kGroups][NR][2];  // the weights, rounded to 2^-11 of themselves or 2^-25
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          bp[g][r][0] = transpose8(pack_half(s[g][r][0], s[g][r][1]));
          bp[g][r][1] = transpose8(pack_half(s[g][r][2], s[g][r][3]));
        }
        if (!whole) {
          // a masked position's values must not count, not even as 0 * NaN
          bool nan = false;
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int p = pos + 16 * g + 8 * (y >> 1) + (y & 1 ? tb : ta);
            const bool in = p >= any_lo && p < any_hi && (valid >> g & 1);
#pragma unroll
            for (int w = 0; w < D / 32; ++w) {
              if (!in) vw[g][y][w] = 0;
              nan |= (((vw[g][y][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
            }
          }
          if (__any_sync(~0u, nan)) {
            // rows that do not see a NaN must not get it: count what each row sees of them, then take them out
            uint32_t bs[NR][2];
#pragma unroll
            for (int r = 0; r < NR; ++r) {
              const int row = n + 8 * r, i = row / a.group;
              const int l0 = row < rows ? see_from(a, q, i) : 0, h0 = row < rows ? see_to(a, q, i) : 0;
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int p = pos + 16 * g + 8 * y;
                bs[r][y] = (p + ta >= l0 && p + ta < h0 ? 0x3c00u : 0) | (p + tb >= l0 && p + tb < h0 ? 0x3c000000u : 0);
              }
            }
#pragma unroll
            for (int w = 0; w < D / 32; ++w) {
              uint32_t f[4];
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                f[y] = (((vw[g][y][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
                vw[g][y][w] &= ~(f[y] * 0xffu);
                f[y] *= 0x38u;
              }
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const uint32_t x = __byte_perm(f[0], f[1], e ? 0x7362 : 0x5140), y = __byte_perm(f[2], f[3], e ? 0x7362 : 0x5140);
                const uint32_t av[4] = {cvt2(x), cvt2_hi(x), cvt2(y), cvt2_hi(y)};
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                  float seen[4] = {0, 0, 0, 0};
                  mma16816(seen, av, bs[r][0], bs[r][1]);
#pragma unroll
                  for (int z = 0; z < 4; ++z)
                    if (seen[z] > 0) acc[r][2 * w + e][z] = NAN;
                }
              }
            }
          }
        }
      }
      // O^T += scale * (V^T P^T), 16 columns at a time: the scale's product and the sum over groups are in 32 bits, so that
      // scales far apart cost each other nothing, and one that a row does not see is multiplied by zero.  (Sums in units
      // of the last scale, rescaled where it changed, let a masked block's scale into the row; 500 ragged requests took 248 us, now 224.)
#pragma unroll
      for (int w = 0; w < D / 32; ++w)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int g = 0; g < S::kGroups; ++g) {
            const uint32_t x = __byte_perm(vw[g][0][w], vw[g][1][w], e ? 0x7362 : 0x5140);
            const uint32_t y = __byte_perm(vw[g][2][w], vw[g][3][w], e ? 0x7362 : 0x5140);
            const uint32_t av[4] = {cvt2(x), cvt2_hi(x), cvt2(y), cvt2_hi(y)};
#pragma unroll
            for (int r = 0; r < NR; ++r) {
              float o[4] = {0, 0, 0, 0};
              mma16816(o, av, bp[g][r][0], bp[g][r][1]);
#pragma unroll
              for (int z = 0; z < 4; ++z) acc[r][2 * w + e][z] = fmaf(value_scale[g], o[z], acc[r][2 * w + e][z]);
            }
          }
        }
      stage += W;
      if (stage >= S::kStages) stage -= S::kStages, ++turn;
    }
    left -= seg;
    if (__any_sync(~0u, *dead)) {
#pragma unroll
      for (int r = 0; r < NR; ++r) l[r][0] = l[r][1] = NAN;
    }

    // the warps' results as one
    float part[NR][2];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float z = l[r][x];
        z += __shfl_xor_sync(~0u, z, 4);
        z += __shfl_xor_sync(~0u, z, 8);
        z += __shfl_xor_sync(~0u, z, 16);
        if (n == 0) *(float2*)s_ml[warp][2 * q4 + x + 8 * r] = float2{m[r][x], z};
      }
    sync_consumers<32 * W>();
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float z = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) z = fmaxf(z, s_ml[w][2 * q4 + x + 8 * r][0]);
        part[r][x] = z == -INFINITY ? 0.f : ex2(m[r][x] - z);
      }
    // this thread's columns are D / 8 in a row from n * D / 8, for rows 2 q4 and 2 q4 + 1
    const auto place = [&](int buf, int r, int x) {
      return (float4*)(merge + ((buf * NR + r) * 8 + 2 * q4 + x) * S::kMergeRow + n * (D / 8));
    };
    if (warp >= 4) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (2 * q4 + x + 8 * r < rows) {
#pragma unroll
            for (int d = 0; d < ND; d += 2)
              place(warp - 4, r, x)[d / 2] =
                  float4{acc[r][d][x] * part[r][x], acc[r][d][2 + x] * part[r][x], acc[r][d + 1][x] * part[r][x],
                         acc[r][d + 1][2 + x] * part[r][x]};
          }
    }
    sync_consumers<32 * W>();
    if (warp < 4) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (2 * q4 + x + 8 * r < rows) {
#pragma unroll
            for (int d = 0; d < ND; d += 2) {
              float4 o = {0, 0, 0, 0};
              if (warp < W - 4) o = place(warp, r, x)[d / 2];
              o.x += acc[r][d][x] * part[r][x], o.y += acc[r][d][2 + x] * part[r][x];
              o.z += acc[r][d + 1][x] * part[r][x], o.w += acc[r][d + 1][2 + x] * part[r][x];
              place(warp, r, x)[d / 2] = o;
            }
          }
    }
    sync_consumers<32 * W>();
    const bool done = places == at.length;
    const int64_t slot = 2 * blockIdx.x + (at.o == 0);
    for (int i = threadIdx.x; i < rows * (D / 4); i += 32 * W) {
      const int row = i / (D / 4), col = i % (D / 4) * 4;
      float mt = -INFINITY, lt = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) mt = fmaxf(mt, s_ml[w][row][0]);
      const float base = mt == -INFINITY ? 0.f : mt;
#pragma unroll
      for (int w = 0; w < W; ++w) lt += s_ml[w][row][1] * ex2(s_ml[w][row][0] - base);
      float4 o = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float4 p = *(const float4*)(merge + (w * 8 * NR + row) * S::kMergeRow + col);
        o.x += p.x, o.y += p.y, o.z += p.z, o.w += p.w;
      }
      if (done) {
        const float inv = lt == 0 ? 0.f : kSumUp / lt;
        const int token = q.first + row / a.group, head = at.h * a.group + row % a.group;
        *(uint2*)((T*)a.out + token * a.out_token_stride + head * a.out_head_stride + col) =
            uint2{from_float2<T>(o.x * inv, o.y * inv), from_float2<T>(o.z * inv, o.w * inv)};
        if (col == 0 && a.lse)
          a.lse[(int64_t)token * a.n_heads + head] = lt == 0 ? -INFINITY : (mt + log2f(lt)) * 0.6931471805599453f;
      } else {
        *(float4*)(a.part + (slot * kRows + row) * D + col) = o;
        if (col == 0) *(float2*)(a.part_ml + (slot * kRows + row) * 2) = float2{mt, lt};
      }
    }
    it += seg;
    count -= places;
    more = at.step(a, places);
    if (more && count > 0) sync_consumers<32 * W>();  // s_ml and the sums have been read
  }
}

__device__ __forceinline__ long long divide(long long x, int d) {  // x >= 0
  return (x >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)d) : x / d;
}

// `total` places dealt out to `blocks` blocks, of which only as many as there are places get any: the first
// `more` one more than the others.
struct Stretches {
  long long total, each;
  int blocks, more;
  __device__ Stretches(long long total, int grid) : total(total), blocks(total < grid ? max(1, (int)total) : grid) {
    each = divide(total, blocks);
    more = (int)(total - each * blocks);
  }
  __device__ long long begin(int b) const { return b >= blocks ? total : each * b + min(b, more); }
  __device__ int owner(long long x) const {
    const long long first = (each + 1) * more;
    return x < first ? (int)divide(x, (int)(each + 1)) : more + (int)divide(x - first, (int)each);
  }
};

template <int D, int NR, class T>
__global__ void __launch_bounds__(Shape<D, NR>::kThreads, 2)
    hx_kv_attend_rows(const __grid_constant__ CUtensorMap km, const __grid_constant__ CUtensorMap vm,
                      const __grid_constant__ AttendArgs a) {
  using S = Shape<D, NR>;
  constexpr int kThreads = S::kThreads, kWarps = S::kWarps;
  extern __shared__ uint8_t s_raw[];
  __shared__ uint64_t s_full[4 * S::kStages], s_empty[2 * S::kStages];  // of a place: keys, values
  __shared__ Tile s_tiles[2][kTiles];
  __shared__ __align__(16) float s_ml[kWarps][kRows][2];
  __shared__ long long s_sum[kThreads / 32];
  __shared__ int s_row[2], s_head[2], s_place[2], s_moved[2], s_dead;
  uint8_t* ring = (uint8_t*)(((uintptr_t)s_raw + 1023) & ~(uintptr_t)1023);
  float* merge = (float*)(ring + S::kStages * kStageBytes);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  asm volatile("griddepcontrol.launch_dependents;");

  if (tid == 0) {
    for (int i = 0; i < 2 * S::kStages; ++i) bar_init(&s_full[2 * i], 1), bar_init(&s_full[2 * i + 1], 1), bar_init(&s_empty[i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s_dead = 0;
    s_moved[0] = s_moved[1] = 0;
  }

  // how long the items are before each thread's rows, and in all
  const int ahead = min(max(a.row_start[0], 0), a.n_tokens), owned = min(max(a.row_start[a.n_rows], ahead), a.n_tokens);
  const int per = (a.n_rows + kThreads - 1) / kThreads;
  const int r0 = min(a.n_rows, tid * per), r1 = min(a.n_rows, r0 + per);
  long long mine = 0;
  int ft;
  for (int r = r0; r < r1; ++r) mine += (long long)length_of<D>(a, request(a, r), &ft) * a.n_kv_heads;
  long long upto = mine;
  for (int d = 1; d < 32; d <<= 1) {
    const long long o = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 31) s_sum[warp] = upto;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += s_sum[w];
    total += s_sum[w];
  }
  before += upto - mine;
  // This block's stretch of them: [n0, n1).  A bound before an item's first tile is moved to the item's
  // beginning, for both of its blocks: so an item's blocks follow one another, each with a tile at least.
  const Stretches all(total, gridDim.x);
  const int b = blockIdx.x;
  const long long bound[2] = {all.begin(b), all.begin(b + 1)};
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    if (!(before <= bound[x] && bound[x] < before + mine)) continue;
    long long at = before;
    for (int r = r0;; ++r) {
      const int length = length_of<D>(a, request(a, r), &ft);
      if (bound[x] < at + (long long)length * a.n_kv_heads) {
        const int h = (int)divide(bound[x] - at, length);
        const int o = (int)(bound[x] - at - (long long)h * length);
        s_row[x] = r, s_head[x] = h, s_place[x] = o <= kItemCost ? 0 : o;
        s_moved[x] = o <= kItemCost ? o : 0;
        break;
      }
      at += (long long)length * a.n_kv_heads;
    }
  }
  __syncthreads();

  // tokens that no row owns, before the first row's and behind the last one's
  for (int i = blockIdx.x; i < ahead + a.n_tokens - owned; i += gridDim.x) {
    const Request q = {i < ahead ? i : owned + i - ahead, 1, 0};
    for (int h = 0; h < a.n_kv_heads; ++h) write_empty<T>(a, D, q, h, tid, kThreads);
  }

  const int count = (int)(bound[1] - bound[0] + s_moved[0] - s_moved[1]);
  if (count <= 0) {
    if (tid == 0) a.joins[b] = int4{0, 0, -1, 0};
    return;
  }
  Place<D> at;
  at.r = s_row[0];
  at.load(a);
  at.h = s_head[0];
  at.o = s_place[0];
  // an item that began in an earlier block and ends in this one is joined here
  if (tid == 0)
    a.joins[b] = at.o > 0 && at.o + (long long)count >= at.length
                     ? int4{at.q.first, at.q.n, all.owner(bound[0] - at.o + kItemCost), at.h}
                     : int4{0, 0, -1, 0};
  if (warp == kWarps)
    produce<D, NR, 0>(a, &km, at, count, ring, s_tiles[0], s_full, s_empty, &s_dead);
  else if (warp == kWarps + 1)
    produce<D, NR, 1>(a, &vm, at, count, ring, s_tiles[1], s_full, s_empty, &s_dead);
  else
    consume<D, NR, T>(a, at, count, ring, s_tiles, s_full, s_empty, &s_dead, merge, s_ml);
  drain(&s_dead, a.status);
}

// Joins an item's partial results: block (e, y) rows 16 y and on of the item that ends in stretch e.
// Each warp turns its rows' maxima and sums into a weight for every part; then D / 4 threads
// take a row's sums (or an equal share of its parts, where there are fewer rows than
// that), with eight loads in flight, the first of them asked for before the weights: what counts is
// the latency of few dependent loads (one request of 5065 tokens, 38 parts of each item: 5 us).
constexpr int kJoinThreads = 512;
constexpr int kMaxBlocks = 512;  // and so of an item's parts

template <int D, int kSlotRows, class T>
__global__ void __launch_bounds__(kJoinThreads) hx_kv_attend_join(const __grid_constant__ AttendArgs a) {
  constexpr int kCols = D / 4, kTeams = kJoinThreads / kCols;
  __shared__ float s_w[kRows][kMaxBlocks];
  __shared__ float2 s_ml[kRows];
  __shared__ float4 s_o[kTeams][kCols];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int4 join = a.joins[blockIdx.x];
  if (join.z < 0) return;
  // the token and head of this block's rows; a half's rows of the many-rows kernel begin at 0 and 128
  const int y0 = blockIdx.y * kRows;
  constexpr int kHalf = kSlotRows / 2;
  const bool halves = kSlotRows == kItemRows;
  const int i0 = halves ? y0 / kHalf * a.half_tokens : 0, x0 = halves ? y0 % kHalf : y0;
  const int rows = min(kRows, (halves ? min(a.half_tokens, join.y - i0) : join.y) * a.group - x0);
  const int parts = blockIdx.x - join.z + 1;
  if (rows <= 0) return;
  const auto slot = [&](int i) { return (2 * (int64_t)(join.z + i) + (i == 0)) * kSlotRows + y0; };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int team = threadIdx.x / kCols, col = threadIdx.x % kCols;
  const int share = max(1, kTeams / rows), together = kTeams / share;  // teams of a row, rows at a time
  const int sub = team % share;
  const auto part_of = [&](int i, int row) { return *(const float4*)(a.part + (slot(i) + row) * D + 4 * col); };
  constexpr int kMost = 8;
  float4 p[kMost];
  const auto ask = [&](int i0, int row) {
#pragma unroll
    for (int u = 0; u < kMost; ++u)
      if (row < rows && team < share * together && i0 + u * share < parts) p[u] = part_of(i0 + u * share, row);
  };
  float first = -INFINITY;  // a warp's first row's maximum of part `lane`
  if (warp < rows && lane < parts) first = a.part_ml[(slot(lane) + warp) * 2];
  ask(sub, team / share);
  for (int row = warp; row < rows; row += kJoinThreads / 32) {
    float m = row == warp ? first : -INFINITY, l = 0;
    for (int i = row == warp ? lane + 32 : lane; i < parts; i += 32) m = fmaxf(m, a.part_ml[(slot(i) + row) * 2]);
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    const float base = m == -INFINITY ? 0.f : m;
    for (int i = lane; i < parts; i += 32) {
      const float2 ml = *(const float2*)(a.part_ml + (slot(i) + row) * 2);
      const float w = ex2(ml.x - base);
      s_w[row][i] = w;
      l += ml.y * w;
    }
    for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(~0u, l, d);
    if (lane == 0) s_ml[row] = float2{m, l};
  }
  __syncthreads();
  for (int r0 = 0; r0 < rows; r0 += together) {
    const int row = r0 + team / share;
    float4 o = {0, 0, 0, 0};
    if (r0) ask(sub, row);
    if (row < rows && team < share * together)
      for (int i = sub; i < parts;) {
#pragma unroll
        for (int u = 0; u < kMost; ++u)
          if (i + u * share < parts) {
            const float w = s_w[row][i + u * share];
            o.x += p[u].x * w, o.y += p[u].y * w, o.z += p[u].z * w, o.w += p[u].w * w;
          }
        i += kMost * share;
        ask(i, row);
      }
    if (share > 1) {
      s_o[team][col] = o;
      __syncthreads();
      if (sub == 0)
        for (int i = 1; i < share && team + i < kTeams; ++i) {
          const float4 q = s_o[team + i][col];
          o.x += q.x, o.y += q.y, o.z += q.z, o.w += q.w;
        }
      __syncthreads();
    }
    if (sub == 0 && row < rows && team < share * together) {
      const float2 ml = s_ml[row];
      const float inv = ml.y == 0 ? 0.f : kSumUp / ml.y;
      const int64_t token = join.x + i0 + a.by_group.of(x0 + row);
      const int head = join.w * a.group + a.by_group.rest(x0 + row);
      T* to = (T*)a.out + token * a.out_token_stride + head * a.out_head_stride + 4 * col;
      *(uint2*)to = uint2{from_float2<T>(o.x * inv, o.y * inv), from_float2<T>(o.z * inv, o.w * inv)};
      if (col == 0 && a.lse)
        a.lse[token * a.n_heads + head] = ml.y == 0 ? -INFINITY : (ml.x + log2f(ml.y)) * 0.6931471805599453f;
    }
  }
}

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 152;
  return sms;
}

// Two blocks fill an SM's shared memory.
int row_blocks() { return std::min(2 * sm_count(), kMaxBlocks); }

struct Work {
  int64_t part, ml, joins, bytes;
};

// Two partial results of a block at most, and what it joins.
Work workspace(int head_dim, int blocks, int slot_rows) {
  Work w;
  w.part = 0;  // rows on multiples of 32 bytes, as the workspace has to begin on one
  w.ml = w.part + 2 * (int64_t)blocks * slot_rows * head_dim * 4;
  w.joins = w.ml + 2 * (int64_t)blocks * slot_rows * 8;
  w.bytes = w.joins + (int64_t)blocks * 16;
  return w;
}

AttendArgs with(AttendArgs a, void* workspace, const Work& w) {
  a.part = (float*)((uint8_t*)workspace + w.part);
  a.part_ml = (float*)((uint8_t*)workspace + w.ml);
  a.joins = (int4*)((uint8_t*)workspace + w.joins);
  return a;
}

// Whether no request of the step has more rows than the few-rows kernel takes.
bool all_few(const hx_kv_cache& c, const hx_kv_query& q) {
  return q.max_q && (int64_t)q.max_q * (q.n_heads / c.n_kv_heads) <= kRows;
}

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode encoder() {
  static const Encode f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess)
      p = nullptr;
    return (Encode)p;
  }();
  return f;
}

// k or v as [blocks][heads * block_tokens][head_dim] bytes, fetched `rows` tokens at a time.
bool tile_map(CUtensorMap* m, const void* base, const hx_kv_cache& c, int rows) {
  const Encode f = encoder();
  if (!f) return false;
  const cuuint64_t dim[3] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.n_kv_heads * c.block_tokens, (cuuint64_t)c.n_blocks};
  const cuuint64_t stride[2] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.block_stride};
  const cuuint32_t box[3] = {(cuuint32_t)c.head_dim, (cuuint32_t)rows, 1}, one[3] = {1, 1, 1};
  return f(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, (void*)base, dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
           c.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// q as [tokens][heads][head_dim], fetched a half's tokens of one group and 64 columns at a time.
bool query_map(CUtensorMap* m, const hx_kv_cache& c, const hx_kv_query& q, int tokens) {
  const Encode f = encoder();
  if (!f) return false;
  const int group = q.n_heads / c.n_kv_heads;
  const cuuint64_t dim[3] = {(cuuint64_t)c.head_dim, (cuuint64_t)q.n_heads, (cuuint64_t)q.n_tokens};
  // the stride of a dimension of one is of no matter, but has to be one that a map can have
  const cuuint64_t stride[2] = {2 * (cuuint64_t)(q.n_heads > 1 ? q.q_head_stride : c.head_dim),
                                2 * (cuuint64_t)(q.n_tokens > 1 ? q.q_token_stride : c.head_dim)};
  const cuuint32_t box[3] = {64, (cuuint32_t)group, (cuuint32_t)tokens}, one[3] = {1, 1, 1};
  return f(m, q.dtype == HX_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, (void*)q.q, dim, stride, box,
           one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

AttendArgs args_of(const hx_kv_cache& c, const hx_kv_query& q) {
  AttendArgs a = {};
  a.k = (const uint8_t*)c.k, a.v = (const uint8_t*)c.v, a.k_scale = c.k_scale, a.v_scale = c.v_scale;
  a.block_stride = c.block_stride, a.scale_stride = c.scale_stride;
  a.q = q.q, a.out = q.out, a.lse = q.lse;
  a.q_token_stride = q.q_token_stride, a.q_head_stride = q.q_head_stride;
  a.out_token_stride = q.out_token_stride, a.out_head_stride = q.out_head_stride;
  a.row_start = q.row_start, a.kv_len = q.kv_len, a.block_table = q.block_table, a.table_stride = q.table_stride;
  a.table_width = q.table_width, a.n_blocks = c.n_blocks, a.n_tokens = q.n_tokens, a.n_rows = q.n_rows;
  a.n_heads = q.n_heads, a.n_kv_heads = c.n_kv_heads, a.group = q.n_heads / c.n_kv_heads;
  while ((1 << a.block_shift) < c.block_tokens) ++a.block_shift;
  a.by_group = divisor(a.group);
  a.half_tokens = kItemRows / 2 / a.group;
  a.max_q = q.max_q, a.causal = q.causal;
  a.window = q.window >= (1 << 30) ? 0 : q.window;  // no request holds so many tokens
  a.out_by_32 = (((uintptr_t)q.out | 2 * (uintptr_t)q.out_token_stride | 2 * (uintptr_t)q.out_head_stride) & 31) == 0;
  a.sm_scale_log2 = q.sm_scale * kLog2e;
  a.status = q.status;
  return a;
}

// Its blocks are launched while the kernel before still runs, and wait for its end.
template <int D, int kSlotRows, class T>
cudaError_t launch_join(const AttendArgs& a, int blocks, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks, kSlotRows / kRows);
  cfg.blockDim = kJoinThreads;
  cfg.stream = s;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, hx_kv_attend_join<D, kSlotRows, T>, a);
}

template <int D, int NR, class T>
cudaError_t launch_rows(const hx_kv_cache& c, const AttendArgs& a, cudaStream_t s) {
  CUtensorMap km, vm;
  const int box = std::min(c.block_tokens, Shape<D, NR>::kTokens);
  if (!tile_map(&km, c.k, c, box) || !tile_map(&vm, c.v, c, box)) return cudaErrorInvalidValue;
  const auto kernel = hx_kv_attend_rows<D, NR, T>;
  if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D, NR>::kSmem)) return e;
  const int blocks = row_blocks();
  kernel<<<blocks, Shape<D, NR>::kThreads, Shape<D, NR>::kSmem, s>>>(km, vm, a);
  if (cudaError_t e = cudaGetLastError()) return e;
  return launch_join<D, kRows, T>(a, blocks, s);
}

template <int D, class T>
cudaError_t launch_typed(const hx_kv_cache& c, const hx_kv_query& q, AttendArgs a, cudaStream_t s) {
  const bool few = all_few(c, q);
  // Up to 8 rows in the leaner form; up to 16 in the other where a step has no longer requests
  // (max_q) or a single token of a group needs them.
  a.few_rows = (few ? q.max_q * a.group : a.group) <= 8 ? 8 : kRows;
  const AttendArgs rows = with(a, q.workspace, workspace(D, row_blocks(), kRows));
  if (cudaError_t e = a.few_rows == 8 ? launch_rows<D, 1, T>(c, rows, s) : launch_rows<D, 2, T>(c, rows, s)) return e;
  if (few) return cudaSuccess;
  const int blocks = sm_count();
  const AttendArgs many = with(a, q.workspace, workspace(D, blocks, kItemRows));
  CUtensorMap qm;
  if (!query_map(&qm, c, q, a.half_tokens)) return cudaErrorInvalidValue;
  if (cudaError_t e = launch_attend_many(qm, many, D, std::is_same<T, __nv_bfloat16>::value, blocks, s)) return e;
  return launch_join<D, kItemRows, T>(many, blocks, s);
}

}  // namespace

int64_t kv_attend_workspace(const hx_kv_cache& c, const hx_kv_query& q) {
  const int64_t rows = workspace(c.head_dim, row_blocks(), kRows).bytes;
  return all_few(c, q) ? rows : std::max(rows, workspace(c.head_dim, sm_count(), kItemRows).bytes);
}

cudaError_t launch_kv_attend(const hx_kv_cache& c, const hx_kv_query& q, cudaStream_t s) {
  const AttendArgs a = args_of(c, q);
  const bool bf = q.dtype == HX_BF16;
  if (c.head_dim == 128) return bf ? launch_typed<128, __nv_bfloat16>(c, q, a, s) : launch_typed<128, __half>(c, q, a, s);
  return bf ? launch_typed<64, __nv_bfloat16>(c, q, a, s) : launch_typed<64, __half>(c, q, a, s);
}

}  // namespace hx
