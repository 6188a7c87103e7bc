// hx_kv_attend_many.cu -- attention of a step's tokens over the paged 8-bit cache:
// requests of many rows (a row: one token and query head of a kv head's group), which
// is a prompt or a chunk of one.
#include <algorithm>
#include <type_traits>

#include "hx_kv_attend.cuh"

namespace hx {
namespace {

// Bound by the tensor cores: 4 D operations per row and visible token.  An item is two halves of
// one request and kv head, each as many whole tokens as give 128 rows at most (the height of
// a tcgen05 accumulator); the tokens it sees come in tiles of 128, and all items' tiles, laid end to end, are
// dealt out to one block per SM in equal stretches (items that blocks share are joined by a
// second kernel).  In a block,
//   1 warp looks the tiles up and has them copied to shared memory as they are,
//   4 warps turn their e4m3 into 16 bits in the layout that tcgen05 reads: keys into q's type, values
//     into f16, both exact (both halves use each: the conversion is paid once for 256 rows),
//   1 thread has an item's q copied as soon as the last item's products have read theirs,
//   1 thread issues the products: S = Q K^T into tensor memory, O += P V with P read from
//     tensor memory, the halves alternating, so that one half's products run while the other's
//     softmax does,
//   2 x 4 warps do a half's softmax, a row to a thread, and write P over S.
// Tensor memory (512 columns): S, P of the halves at 0 and 128, O at 256 and 256 + D.
// Four prompts of 5600 tokens, 32 heads on 8 of 128 in bf16: 1125 us, 945 TFLOP/s, 50 % of a plain product's rate; a
// tile takes some 4000 cycles where its products take 2048: a half's softmax, values and scores follow one another.
//
// By turns (kTurns): where no request of the step has more tokens than a half (max_q says so), the second half
// would have nothing to do.  Then both halves have the same rows, one takes the even tiles and the other the odd ones, and the
// first half's threads join the two: 64 requests of 1 to 5 tokens at 810 to 11507, 32 heads on 8 of 128, 221 -> 191 us;
// a chunk of 30 at 24001 47 -> 40 us.  As a branch in one kernel it cost prompts 4 %.
//
// Scales: a score is s * ks * c, and a value's scale vs goes into the weight, P = exp2(s ks c +
// log2(vs) - m) with m within kLag of the largest of those exponents so far.  So P in f16 is accurate
// relative to the row's largest weight times scale (a token below 2^-25 of that adds nothing to O), however far apart scales lie.  The softmax's sum l is that of
// P 2^ref / vs, in units of 2^(m - ref) where ref is the power of two of a scale of the item, as long as all its scales lie
// within 2^kNear of that.  Past this P may be zero where its share of l is not: from the first such tile on l is
// summed from the scores alone, in units of 2^ml with a maximum of its own (64 blocks of zeros, as hx_kv_append leaves them
// under 2^-100, beside one under 2^20: the result was too large by what they weigh).
constexpr int kHalf = 128;
constexpr int kKv = 128;       // tokens of a tile
constexpr int kGroups = kKv / 16;
constexpr int kConvWarp = 8, kMmaWarp = 12, kFetchWarp = 13, kQueryWarp = 14;
constexpr int kManyThreads = 32 * (kQueryWarp + 1);
constexpr float kNear = 16.f;  // what l loses of P below 2^-126 is then less than 2^-90 of it, by its exponents' rounding 2^-20
constexpr int kNanList = 8;
constexpr int kNanLists = 8;  // the conversion may be four items ahead of a half that still writes one out

template <int D>
struct Many {
  static constexpr int kQBytes = kHalf * D * 2;   // one half's q
  static constexpr int kTile = kKv * D * 2;       // K or V in f16
  static constexpr int kRaw = kKv * D;            // K or V as it is in the cache
  static constexpr int kTiles = 2 * kQBytes + 4 * kTile + 2 * kRaw;
};

struct Segment {  // a stretch of one item's tiles
  int r, h, mt;           // request, kv head, which tokens
  int t, tiles;           // the next tile, and how many the item has
  int first_tile;
  int items;              // of the request, for one kv head
  Request q;
  int i0;                 // its first token in the request
  int lo0, hi0, lo1, hi1; // tokens that any row of a half sees (no arrays: an index that is not
                          // constant would put them into local memory)
  bool empty;             // nothing visible, or not to be computed: zeros
};

__device__ __forceinline__ bool many(const AttendArgs& a, const Request& q) {
  return q.kv > 0 && q.n * a.group > a.few_rows;
}
__device__ __forceinline__ int items_of(const AttendArgs& a, const Request& q) {
  return (q.n + 2 * a.half_tokens - 1) / (2 * a.half_tokens);
}
// First and end tile of item mt of a request (at least one, to write its zeros).
__device__ __forceinline__ void item_span(const AttendArgs& a, const Request& q, int mt, int* t0, int* t1, bool* empty) {
  const int i0 = mt * 2 * a.half_tokens, i1 = min(i0 + 2 * a.half_tokens, q.n);
  const int lo = see_from(a, q, i0), hi = see_to(a, q, i1 - 1);
  *empty = hi <= lo;
  *t0 = *empty ? 0 : lo / kKv;
  *t1 = *empty ? 1 : (hi + kKv - 1) / kKv;
}
__device__ __forceinline__ int item_tiles(const AttendArgs& a, const Request& q, int mt) {
  int t0, t1;
  bool e;
  item_span(a, q, mt, &t0, &t1, &e);
  return t1 - t0;
}
__device__ __forceinline__ long long warp_sum(long long x) {
  for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
  return x;
}
// Tiles of a request's items for one kv head, for the 32 rows of a warp's lanes: a request of few
// items by its lane, one of many by all lanes together.
__device__ long long tiles_per_head(const AttendArgs& a, const Request& q, bool real) {
  const int lane = threadIdx.x & 31, items = real && many(a, q) ? items_of(a, q) : 0;
  long long sum = 0;
  if (items <= 8)
    for (int mt = 0; mt < items; ++mt) sum += item_tiles(a, q, mt);
  for (unsigned big = __ballot_sync(~0u, items > 8); big; big &= big - 1) {
    const int src = __ffs(big) - 1;
    const Request o = {__shfl_sync(~0u, q.first, src), __shfl_sync(~0u, q.n, src), __shfl_sync(~0u, q.kv, src)};
    const int n = items_of(a, o);
    long long part = 0;
    for (int mt = lane; mt < n; mt += 32) part += item_tiles(a, o, mt);
    part = warp_sum(part);
    if (lane == src) sum = part;
  }
  return sum;
}

template <bool kTurns>
__device__ __forceinline__ void load_item(const AttendArgs& a, Segment& s) {
  int t0, t1;
  item_span(a, s.q, s.mt, &t0, &t1, &s.empty);
  s.first_tile = t0;
  s.tiles = t1 - t0;
  s.i0 = s.mt * 2 * a.half_tokens;
  s.lo0 = see_from(a, s.q, s.i0);
  s.hi0 = see_to(a, s.q, min(s.i0 + a.half_tokens, s.q.n) - 1);
  if (kTurns) {
    s.lo1 = s.lo0, s.hi1 = s.hi0;
    return;
  }
  s.lo1 = s.hi1 = 0;
  if (s.i0 + a.half_tokens < s.q.n) {
    s.lo1 = see_from(a, s.q, s.i0 + a.half_tokens);
    s.hi1 = see_to(a, s.q, min(s.i0 + 2 * a.half_tokens, s.q.n) - 1);
  }
}
// To the next item; false past the last.
template <bool kTurns>
__device__ __forceinline__ bool next_item(const AttendArgs& a, Segment& s) {
  s.t = 0;
  if (++s.mt < s.items) {
    load_item<kTurns>(a, s);
    return true;
  }
  s.mt = 0;
  if (++s.h < a.n_kv_heads) {
    load_item<kTurns>(a, s);
    return true;
  }
  s.h = 0;
  do {
    if (++s.r >= a.n_rows) return false;
    s.q = request(a, s.r);
  } while (!many(a, s.q));
  s.items = items_of(a, s.q);
  load_item<kTurns>(a, s);
  return true;
}
template <bool kTurns>
__device__ __forceinline__ bool active(const Segment& s, int half, int tile) {
  if (kTurns && (tile & 1) != half) return false;
  return tile * kKv < (half ? s.hi1 : s.hi0) && (tile + 1) * kKv > (half ? s.lo1 : s.lo0);
}

// ---- tcgen05

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// A 64-bit descriptor of an operand in shared memory, 128-byte rows permuted in 16-byte units by the
// row's low three bits; lead: bytes between panels of 64 columns (rows of values only).
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
// f16 x f16 or bf16 x bf16 with 32-bit sums, M = 128; b_rows: B is stored with its N side contiguous.
__host__ __device__ constexpr uint32_t instruction(int n, bool b_rows, bool bf16) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0) | (b_rows ? 1u << 16 : 0) | (uint32_t)(n / 8) << 17 | (uint32_t)(128 / 16) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a),
      "l"(b), "r"(idesc), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d), "r"(a),
      "l"(b), "r"(idesc), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void tm_load(uint32_t addr, uint32_t* r) {  // 32 columns
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_load16(uint32_t addr, uint32_t* r) {  // 16 columns
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
      "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_store8(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two 32-bit values at once.
__device__ __forceinline__ float2 both(float x) { return float2{x, x}; }
__device__ __forceinline__ float2 pair(uint32_t x, uint32_t y) { return float2{__uint_as_float(x), __uint_as_float(y)}; }
__device__ __forceinline__ uint64_t bits(float2 x) { return (uint64_t)__float_as_uint(x.y) << 32 | __float_as_uint(x.x); }
__device__ __forceinline__ float2 floats(uint64_t x) { return pair((uint32_t)x, (uint32_t)(x >> 32)); }
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(x)), "l"(bits(y)), "l"(bits(z)));
  return floats(r);
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(x)), "l"(bits(y)));
  return floats(r);
}
// What a tile's groups of 16 tokens are scaled by: {ks, log2 vs, 2^ref / vs, -}, and which of them exist; kFar: the
// item's scales lie far apart.
constexpr uint32_t kFar = 1u << 31;
struct TileInfo {
  float4 g[kGroups];
  uint32_t valid;
};

// The barriers and small shared state of a block.
struct Shared {
  uint64_t raw_full[2], raw_empty[2];  // of keys and values as they come
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], o_full[2], go[2], ended[2][2];  // go and ended: of even and odd items
  TileInfo info[8];
  int nan_count[kNanLists];
  float ref[kNanLists];  // by items, as the lists are
  int nan_pos[kNanLists][kNanList];
  long long sum[kManyThreads / 32];
  long long skip;  // tiles of the item before this block's stretch
  int row, head, mt, dead;
  uint32_t tmem;
  float2 ml[kHalf];  // the second half's ml and l, where both have the same rows
  signed char up[kHalf];  // and its m - ml, -128: it holds nothing
};

// The end of a stretch: `count` tiles from s.t on that lie in s's item.
#define HX_SEGMENTS(s, count)                                                                       \
  for (int seg = min((count), (s).tiles - (s).t); (count) > 0;                                      \
       (count) -= seg, (s).t += seg, seg = (count) > 0 && next_item<kTurns>(a, (s)) ? min((count), (s).tiles - (s).t) : (count))

template <class T>
__device__ __forceinline__ float2 two(uint32_t u) {
  if constexpr (std::is_same<T, __half>::value) return __half22float2(*(const __half2*)&u);
  else return __bfloat1622float2(*(const __nv_bfloat162*)&u);
}
template <class T>
__device__ __forceinline__ uint32_t pack(float x, float y) {
  if constexpr (std::is_same<T, __half>::value) return pack_half(x, y);
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *(const uint32_t*)&h;
}

// ---- the fetching warp

// Lane g looks up the block of a tile's 16 tokens g, a tile ahead; the lanes whose block begins
// there (or is the tile's first) have it copied.
template <int D, bool kTurns>
__device__ void fetch(const AttendArgs& a, Segment s, int count, Shared* sh, uint8_t* raw) {
  const int lane = threadIdx.x & 31, block = 1 << a.block_shift;
  const int tokens = min(block, kKv);  // of a copy
  const bool copies = lane < kGroups && (16 * lane & (tokens - 1)) == 0;
  volatile int* dead = &sh->dead;
  int id = -1, pos = 0, h = 0;
  float ref = 0;
  bool has_ref = false, far = false;  // of the item
  int item = 0;
  const auto look_up = [&] {
    pos = (s.first_tile + s.t) * kKv + 16 * lane;
    h = s.h;
    id = lane < kGroups && pos < max(s.hi0, s.hi1) ? a.block_table[s.r * a.table_stride + (pos >> a.block_shift)] : -1;
  };
  const auto skip_empty = [&] {  // items that see nothing have one tile, and nothing in it
    while (count > 0 && s.empty)
      if (--count > 0) next_item<kTurns>(a, s);
  };
  skip_empty();
  if (count > 0) look_up();
  for (int it = 0; count > 0; ++it) {
    const bool ok = (unsigned)id < (unsigned)a.n_blocks;
    const uint32_t valid = __ballot_sync(~0u, ok);
    const int64_t at = id * a.block_stride + ((int64_t)h * block + (pos & (block - 1))) * D;
    float ks = 0, vs = 0;
    if (ok) ks = a.k_scale[id * a.scale_stride + h], vs = a.v_scale[id * a.scale_stride + h];
    const bool seen = ok && pos + 16 > s.lo0;  // by any row of the item
    bool last = false;                         // of its tiles here
    --count;
    if (count > 0 && ++s.t == s.tiles) {
      last = true;
      next_item<kTurns>(a, s);
      skip_empty();
    }
    if (count > 0) look_up();
    const uint32_t bytes = (uint32_t)__popc(__ballot_sync(~0u, ok && copies)) * tokens * D;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      if (!__all_sync(~0u, bar_wait(&sh->raw_empty[v], (it & 1) ^ 1, dead))) return;
      if (v == 0) {
        TileInfo& info = sh->info[it & 7];
        const float lv = log2f(vs);  // rounded, which the sum takes out again; -inf: the values are zeros
        const uint32_t who = __ballot_sync(~0u, seen && fabsf(lv) < INFINITY);
        if (who && !has_ref) ref = rintf(__shfl_sync(~0u, lv, __ffs(who) - 1)), has_ref = true;
        const bool near = fabsf(lv - ref) <= kNear;
        far |= __any_sync(~0u, seen && !near);
        if (lane < kGroups) info.g[lane] = float4{ks, lv, near ? exp2f(ref - lv) : 1.f, 0.f};
        if (lane == 0) info.valid = valid | (far ? kFar : 0), sh->ref[item & (kNanLists - 1)] = ref;
        if (last) has_ref = far = false, ++item;
        __syncwarp();
      }
      if (lane == 0) bar_expect(&sh->raw_full[v], bytes);
      __syncwarp();
      if (ok && copies) bulk_load(raw + v * Many<D>::kRaw + 16 * lane * D, (v ? a.v : a.k) + at, tokens * D, &sh->raw_full[v]);
    }
  }
}

// ---- the converting warps

// What has not been copied (no such block) is converted as it lies there: its scores are masked, and its
// values are numbers times weights of zero.
template <int D, class T, bool kTurns>
__device__ void convert(const AttendArgs& a, Segment s, int count, Shared* sh, const uint8_t* raw, uint8_t* kbuf) {
  // 8 bytes a lane: a lane's 8 f16 are one 16-byte unit, and eight lanes' units lie on different banks
  constexpr int kLanes = D / 8;            // lanes of a token
  constexpr int kPer = 32 / kLanes;        // tokens of a warp's load
  constexpr int kLoads = 32 / kPer;        // loads of a warp's 32 tokens
  const int tid = threadIdx.x - 32 * kConvWarp, warp = tid >> 5, lane = tid & 31;
  const int unit = lane % kLanes, sub = lane / kLanes;
  volatile int* dead = &sh->dead;
  int seg_no = 0, it = 0;
  // a tile's f16 rows: panels of 64 columns, 128-byte rows, 16-byte units permuted
  uint8_t* const row0 = kbuf + (unit >> 3) * (kKv * 128) + (32 * warp + sub) * 128;
  const auto put = [&](int offset, uint4 h, int j) {
    const int tok = j * kPer;
    *(uint4*)(row0 + offset + tok * 128 + (((unit & 7) ^ ((tok + sub) & 7)) << 4)) = h;
  };
  const auto halves = [](const uint2& u) { return uint4{cvt2(u.x), cvt2_hi(u.x), cvt2(u.y), cvt2_hi(u.y)}; };
  const auto key = [&](const uint2& u) {
    uint4 h = halves(u);
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      uint32_t* w = (uint32_t*)&h;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float2 f = two<__half>(w[y]);
        w[y] = pack<__nv_bfloat16>(f.x, f.y);
      }
    }
    return h;
  };
  const auto take = [&](int v, uint2* u) {
    const bool landed = bar_wait(&sh->raw_full[v], it & 1, dead);
    const uint8_t* from = raw + v * Many<D>::kRaw + (32 * warp + sub) * D + unit * 8;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) u[j] = *(const uint2*)(from + j * kPer * D);
    fence_async();
    __syncwarp();
    if (lane == 0 && landed) bar_arrive(&sh->raw_empty[v]);  // else its copy may be on its way still
  };
  HX_SEGMENTS(s, count) {
    if (s.empty) continue;
    const int list = seg_no & (kNanLists - 1);
    if (tid == 0) sh->nan_count[list] = 0;
    asm volatile("bar.sync 1, 128;" ::: "memory");
    for (int i = 0; i < seg && !__any_sync(~0u, *dead); ++i, ++it) {
      const int st = it & 1;
      const uint32_t phase = (it >> 1) & 1;
      uint2 u[kLoads];
      take(0, u);
      bar_wait(&sh->k_empty[st], phase ^ 1, dead);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) put(st * Many<D>::kTile, key(u[j]), j);
      fence_async();
      bar_arrive(&sh->k_full[st]);
      take(1, u);
      bar_wait(&sh->v_empty[st], phase ^ 1, dead);
      const auto nans = [](uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };
      uint32_t any = 0;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) any |= ((u[j].x & 0x7f7f7f7fu) + 0x01010101u) | ((u[j].y & 0x7f7f7f7fu) + 0x01010101u);
      if (any & 0x80808080u) {
        // a NaN would reach rows that do not see it (0 * NaN): taken out here, and put
        // into the rows that see it at their end
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          if (!(nans(u[j].x) | nans(u[j].y))) continue;
          u[j].x &= ~((nans(u[j].x) >> 7) * 0xffu);
          u[j].y &= ~((nans(u[j].y) >> 7) * 0xffu);
          const int tok = 32 * warp + j * kPer + sub, p = (s.first_tile + s.t + i) * kKv + tok;
          if (p < max(s.hi0, s.hi1) && (sh->info[it & 7].valid >> (tok >> 4) & 1)) {
            const int n = atomicAdd(&sh->nan_count[list], 1);
            if (n < kNanList) sh->nan_pos[list][n] = p;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < kLoads; ++j) put((2 + st) * Many<D>::kTile, halves(u[j]), j);
      fence_async();
      bar_arrive(&sh->v_full[st]);
    }
    ++seg_no;
  }
}

// ---- the query warp

// A half's q: rows of token and head of the group, as they lie in q; what lies past the request
// or past q is not used.
template <int D, bool kTurns>
__device__ void queries(const AttendArgs& a, const CUtensorMap* qm, Segment s, int count, Shared* sh, uint8_t* qbuf) {
  const uint32_t bytes = (uint32_t)(a.half_tokens * a.group) * D * 2;
  volatile int* dead = &sh->dead;
  int seg_no = 0;
  HX_SEGMENTS(s, count) {
    if (s.empty) continue;
    for (int half = 0; half < 2; ++half) {
      const int token = s.q.first + s.i0 + (kTurns ? 0 : half * a.half_tokens);
#pragma unroll
      for (int x = 0; x < D; x += 64) tile_prefetch(qm, x, s.h * a.group, token);
    }
    for (int half = 0; half < 2; ++half) {
      const int token = s.q.first + s.i0 + (kTurns ? 0 : half * a.half_tokens);
      if (!bar_wait(&sh->q_empty[half], (seg_no & 1) ^ 1, dead) || *dead) return;
      bar_expect(&sh->q_full[half], bytes);
#pragma unroll
      for (int x = 0; x < D; x += 64)
        tile_load(qbuf + half * Many<D>::kQBytes + x / 64 * (kHalf * 128), qm, &sh->q_full[half], x, s.h * a.group, token);
    }
    ++seg_no;
  }
}

// ---- the issuing warp

// One thread of the warp, the same each time; what it does, the hardware takes from uniform registers.
__device__ __forceinline__ bool elected() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p;
}

template <int D, class T, bool kTurns>
__device__ void issue(const AttendArgs& a, Segment s, int count, Shared* sh, const uint8_t* qbuf, const uint8_t* kbuf,
                      const uint8_t* vbuf) {
  const uint32_t tm = sh->tmem;
  const uint64_t q0 = operand(smem_addr(qbuf), 16), k0 = operand(smem_addr(kbuf), 16), v0 = operand(smem_addr(vbuf), kKv * 128);
  uint32_t n_s[2] = {0, 0};  // products P V issued per half
  int it = 0, seg_no = 0;
  volatile int* dead = &sh->dead;
  const auto issued = [&](int half) { return half ? n_s[1] : n_s[0]; };
  const auto scores = [&](int half, int st) {
    // S's columns hold the half's last P; the order of products with different sums is not promised
    if (issued(half)) bar_wait(&sh->o_full[half], (issued(half) - 1) & 1, dead);
    tc_fence_after();
    if (elected()) {
      const uint64_t q = q0 + half * (Many<D>::kQBytes >> 4), k = k0 + st * (Many<D>::kTile >> 4);
#pragma unroll
      for (int x = 0; x < D / 16; ++x) {
        const uint32_t o = ((x >> 2) * (128 * 128) + (x & 3) * 32) >> 4;
        mma_ss(tm + half * kKv, q + o, k + o, instruction(kKv, false, std::is_same<T, __nv_bfloat16>::value), x > 0);
      }
      tc_commit(&sh->s_full[half]);
    }
    __syncwarp();
  };
  const auto values = [&](int half, int st, bool add) {
    bar_wait(&sh->p_full[half], issued(half) & 1, dead);
    tc_fence_after();
    if (elected()) {
      const uint64_t v = v0 + st * (Many<D>::kTile >> 4);
#pragma unroll
      for (int x = 0; x < kKv / 16; ++x)
        mma_ts(tm + 256 + half * D, tm + half * kKv + 8 * x, v + x * (2048 >> 4), instruction(D, true, false), add || x > 0);
      tc_commit(&sh->o_full[half]);
    }
    __syncwarp();
    n_s[0] += half == 0, n_s[1] += half == 1;
  };
  const auto commit = [&](uint64_t* bar) {
    if (elected()) tc_commit(bar);
    __syncwarp();
  };
  HX_SEGMENTS(s, count) {
    if (s.empty) continue;
    const int tile0 = s.first_tile + s.t;
    // the item before the last has been written out, and this one may begin
    if (seg_no >= 2) {
      bar_wait(&sh->ended[0][seg_no & 1], ((seg_no - 2) >> 1) & 1, dead);
      bar_wait(&sh->ended[1][seg_no & 1], ((seg_no - 2) >> 1) & 1, dead);
    }
    if ((threadIdx.x & 31) == 0) bar_arrive(&sh->go[seg_no & 1]);
    if (kTurns) {
      // a half's next tile is the one after next
      bar_wait(&sh->q_full[0], seg_no & 1, dead), bar_wait(&sh->q_full[1], seg_no & 1, dead);
      uint32_t had = 0;  // the halves whose O holds something
#pragma unroll 1
      for (int i = -2; i < seg && !__any_sync(~0u, *dead); ++i) {
        const int tile = tile0 + i, half = tile & 1, st = (it + i) & 1;
        if (i >= 0) {
          bar_wait(&sh->v_full[st], ((it + i) >> 1) & 1, dead);
          if (active<kTurns>(s, half, tile)) {
            values(half, st, had >> half & 1);
            had |= 1u << half;
          }
          commit(&sh->v_empty[st]);
        }
        if (i + 2 >= seg) continue;
        bar_wait(&sh->k_full[st], ((it + i + 2) >> 1) & 1, dead);
        if (active<kTurns>(s, half, tile + 2)) scores(half, st);
        commit(&sh->k_empty[st]);
        if (i + 3 == seg) commit(&sh->q_empty[0]), commit(&sh->q_empty[1]);
      }
      it += seg;
      ++seg_no;
      continue;
    }
    bool has[2] = {false, false};  // a half's O holds something
    bar_wait(&sh->k_full[it & 1], (it >> 1) & 1, dead);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      bar_wait(&sh->q_full[half], seg_no & 1, dead);
      if (active<kTurns>(s, half, tile0)) scores(half, it & 1);
      if (seg == 1) commit(&sh->q_empty[half]);
    }
    commit(&sh->k_empty[it & 1]);
    for (int i = 0; i < seg && !__any_sync(~0u, *dead); ++i, ++it) {
      const int tile = tile0 + i, st = it & 1;
      const bool more = i + 1 < seg;
      bar_wait(&sh->v_full[st], (it >> 1) & 1, dead);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (active<kTurns>(s, half, tile)) {
          values(half, st, has[half]);
          has[half] = true;
        }
        if (half == 1) commit(&sh->v_empty[st]);
        if (more) {
          if (half == 0) bar_wait(&sh->k_full[st ^ 1], ((it + 1) >> 1) & 1, dead);
          if (active<kTurns>(s, half, tile + 1)) scores(half, st ^ 1);
          if (i + 2 == seg) commit(&sh->q_empty[half]);
        }
      }
      if (more) commit(&sh->k_empty[st ^ 1]);
    }
    ++seg_no;
  }
}

// ---- the softmax warps

// N 32-bit values in a row, 32 bytes at a time where their place allows it: a thread's own row, of which each store
// then fills whole sectors.
template <int N>
__device__ __forceinline__ void store32(void* p, const uint32_t* w, bool wide) {
  if (wide) {
#pragma unroll
    for (int y = 0; y < N; y += 8)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"((uint32_t*)p + y), "r"(w[y]), "r"(w[y + 1]),
                   "r"(w[y + 2]), "r"(w[y + 3]), "r"(w[y + 4]), "r"(w[y + 5]), "r"(w[y + 6]), "r"(w[y + 7])
                   : "memory");
  } else {
#pragma unroll
    for (int y = 0; y < N; y += 4) *(uint4*)((uint32_t*)p + y) = uint4{w[y], w[y + 1], w[y + 2], w[y + 3]};
  }
}

template <int D, class T, bool kTurns>
__device__ void softmax(const AttendArgs& a, Segment s, int count, Shared* sh) {
  constexpr float kLag = 10.f;  // of f16's 2^16
  const int half = threadIdx.x >> 7, row = threadIdx.x & 127;
  const uint32_t lanes = (threadIdx.x & 96) << 16;
  const uint32_t ts = sh->tmem + lanes + half * kKv, to = sh->tmem + lanes + 256 + half * D;
  int it = 0, seg_no = 0;
  uint32_t n_s = 0;
  volatile int* dead = &sh->dead;
  HX_SEGMENTS(s, count) {
    const int first = s.i0 + (kTurns ? 0 : half * a.half_tokens);
    const int i = first + a.by_group.of(row);  // the row's token in its request
    const bool real = row < a.half_tokens * a.group && i < s.q.n;
    if (s.empty) {
      if (real && !(kTurns && half)) {
        const int64_t token = s.q.first + i;
        const int head = s.h * a.group + a.by_group.rest(row);
        T* out = (T*)a.out + token * a.out_token_stride + head * a.out_head_stride;
#pragma unroll
        for (int y = 0; y < D / 8; ++y) *(uint4*)(out + 8 * y) = uint4{0, 0, 0, 0};
        if (a.lse) a.lse[token * a.n_heads + head] = -INFINITY;
      }
      continue;
    }
    __all_sync(~0u, bar_wait(&sh->go[seg_no & 1], (seg_no >> 1) & 1, dead));
    const int lo = real ? see_from(a, s.q, i) : 0, hi = real ? see_to(a, s.q, i) : 0;
    // what all rows of the half see: [all_lo, all_hi); rows without a token do not matter
    const int last = min(first + a.half_tokens, s.q.n) - 1;
    const int all_lo = last < first ? 0 : see_from(a, s.q, last), all_hi = last < first ? 0 : see_to(a, s.q, first);
    const float c = a.sm_scale_log2;
    const float* ref = &sh->ref[seg_no & (kNanLists - 1)];
    float m = 0, l = 0, ml = -INFINITY;
    bool has = false, fresh = true;  // fresh: the row has seen nothing yet
    bool apart = false;              // l has a maximum of its own, ml
    for (int j = 0; j < seg && !__any_sync(~0u, *dead); ++j, ++it) {
      const int tile = s.first_tile + s.t + j;
      if (!active<kTurns>(s, half, tile)) continue;
      const int pos = tile * kKv;
      const TileInfo& info = sh->info[it & 7];
      bar_wait(&sh->s_full[half], n_s & 1, dead);
      tc_fence_after();
      const uint32_t valid = info.valid;
      if (!has) m = *ref;  // near the first exponents, so that they are rounded as the scores themselves are
      if ((valid & kFar) && !apart) {
        apart = true;
        if (l != 0) ml = m - *ref;
      }
      const bool whole = valid == (1u << kGroups) - 1 && pos >= all_lo && pos + kKv <= all_hi;
      // what this row sees of 32 tokens
      const auto sees = [&](int ch) -> uint32_t {
        const int p = pos + 32 * ch, f = min(max(lo - p, 0), 32), e = min(max(hi - p, 0), 32);
        if (f >= e) return 0;
        const uint32_t range = (0xffffffffu >> (32 - (e - f))) << f;
        const uint32_t have = valid >> (2 * ch);
        return range & ((have & 1 ? 0xffffu : 0) | (have & 2 ? 0xffff0000u : 0));
      };
      // 32 tokens at a time, P over the S that has been read.  m need not be the maximum: a row moves its m
      // (by a whole number) only when a weight would pass 2^kLag, and then what it has written of this tile
      // and O follow.
      const auto weigh = [&](auto kind) {
        constexpr bool masked = decltype(kind)::value > 0, far = decltype(kind)::value > 1;
#pragma unroll 1
        for (int ch = 0; ch < 4; ++ch) {
          uint32_t v[32];
          tm_load(ts + 32 * ch, v);
          const uint32_t see = masked ? sees(ch) : 0;
          if constexpr (far) {
            float top = -INFINITY;
#pragma unroll
            for (int y = 0; y < 32; ++y)
              if (see >> y & 1) top = fmaxf(top, __uint_as_float(v[y]) * (info.g[2 * ch + (y >> 4)].x * c));
            if (top > ml && top < INFINITY) {
              const float up = ceilf(top);
              l *= ex2(ml - up);
              ml = up;
            }
            const float base = ml == -INFINITY ? 0.f : ml;
#pragma unroll
            for (int y = 0; y < 32; ++y)
              if (see >> y & 1) l += ex2(fmaf(__uint_as_float(v[y]), info.g[2 * ch + (y >> 4)].x * c, -base));
          }
          float4 z[2];
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            z[g] = info.g[2 * ch + g];
            const float2 f = both(z[g].x * c), b = both(z[g].y - m);
#pragma unroll
            for (int y = 16 * g; y < 16 * g + 16; y += 2) {
              float2 s2 = fma2(pair(v[y], v[y + 1]), f, b);
              if (masked && !(see >> y & 1)) s2.x = -INFINITY;
              if (masked && !(see >> (y + 1) & 1)) s2.y = -INFINITY;
              top[y / 2 % 4] = fmaxf(top[y / 2 % 4], fmaxf(s2.x, s2.y));
              v[y] = __float_as_uint(s2.x), v[y + 1] = __float_as_uint(s2.y);
            }
          }
          const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
          const bool late = real && (fresh ? most > -INFINITY : most > kLag);
          if (__any_sync(~0u, late)) {
            const float by = late && most < INFINITY ? ceilf(most) : 0.f;
            const float keep = fresh ? 1.f : ex2(-by);  // nothing has been kept while nothing was seen
            fresh &= !late;
            m += by;
            if (!far) l *= keep;
#pragma unroll
            for (int y = 0; y < 32; ++y) v[y] = __float_as_uint(__uint_as_float(v[y]) - by);
            tm_stored();
            uint32_t w[16];
#pragma unroll 1
            for (int o = 0; o < 16 * ch; o += 16) {
              tm_load16(ts + o, w);
#pragma unroll
              for (int y = 0; y < 16; ++y) {
                // in 32 bits: the factor alone may be too small for f16 where its product with a weight is not
                const float2 e = __half22float2(*(const __half2*)&w[y]);
                w[y] = pack_half(e.x * keep, e.y * keep);
              }
              tm_store16(ts + o, w);
            }
            if (has) {
#pragma unroll 1
              for (int o = 0; o < D; o += 16) {
                tm_load16(to + o, w);
#pragma unroll
                for (int y = 0; y < 16; ++y) w[y] = __float_as_uint(__uint_as_float(w[y]) * keep);
                tm_store16(to + o, w);
              }
            }
          }
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            float2 part[2] = {{0, 0}, {0, 0}};
            uint32_t w[8];
#pragma unroll
            for (int y = 0; y < 16; y += 2) {
              const float2 e = {ex2(__uint_as_float(v[16 * g + y])), ex2(__uint_as_float(v[16 * g + y + 1]))};
              part[y / 2 % 2] = add2(part[y / 2 % 2], e);
              w[y / 2] = pack_half(e.x, e.y);
            }
            const float2 sum = add2(part[0], part[1]);
            if (!far) l = fmaf(sum.x + sum.y, z[g].z, l);
            tm_store8(ts + 16 * ch + 8 * g, w);
          }
        }
      };
      if (whole) weigh(std::integral_constant<int, 0>{});
      else if (!apart) weigh(std::integral_constant<int, 1>{});
      else weigh(std::integral_constant<int, 2>{});
      tm_stored();
      tc_fence_before();
      bar_arrive(&sh->p_full[half]);
      has = true;
      ++n_s;
    }

    if (has) {
      bar_wait(&sh->o_full[half], (n_s - 1) & 1, dead);
      tc_fence_after();
    }
    // O is in units of 2^m, l in units of 2^ml: so is what is stored of both
    // (what has seen nothing has not waited for ref either)
    if (fresh) m = -INFINITY;
    if (!apart && !fresh) ml = m - *ref;
    if (*dead) l = NAN;          // a wait gave up: what has been computed does not stand
    if (l == INFINITY) l = NAN;  // of an infinite score: exp(inf - inf), and not 1 / inf
    float up = m - ml, up1 = 0;  // what brings the halves' O there, powers of two
    bool holds = has && l != 0, holds1 = false;
    if (kTurns) {
      // the first half's threads join the two; a thread reaches the other half's row in tensor memory, its lane
      if (half) sh->ml[row] = float2{ml, l}, sh->up[row] = (signed char)(holds ? fminf(fmaxf(m - ml, -127.f), 127.f) : -128.f);
      tc_fence_before();
      __syncwarp();
      asm volatile("bar.sync 2, 256;" ::: "memory");
      tc_fence_after();
      if (half) {
        asm volatile("bar.sync 2, 256;" ::: "memory");
        bar_arrive(&sh->ended[half][seg_no & 1]);
        ++seg_no;
        continue;
      }
      const float2 other = sh->ml[row];
      const float most = fmaxf(ml, other.x), base = most > -INFINITY ? most : 0.f;
      up = m - base, up1 = sh->up[row] + other.x - base, holds1 = sh->up[row] != -128;
      l = l * ex2(ml - base) + other.y * ex2(other.x - base);
      ml = most;
    }
    const int64_t token = s.q.first + i;
    const int head = s.h * a.group + a.by_group.rest(row);
    T* out = (T*)a.out + token * a.out_token_stride + head * a.out_head_stride;
    const bool done = seg == s.tiles;
    const int64_t slot = 2 * blockIdx.x + (s.t == 0);
    float* part = a.part + (slot * kItemRows + half * kHalf + row) * D;
    const bool none = l == 0;
    const float nothing = l == l ? 0.f : NAN;
    const float inv = done ? (none ? 0.f : 1.f / l) : kSumDown;
    const auto factor = [&](float up) {  // 2^up * inv, in two steps: 2^up alone may leave the range
      up = fminf(fmaxf(up, -252.f), 252.f);
      const float part = rintf(0.5f * up);
      return ex2(part) * (ex2(up - part) * inv);
    };
    const float by = factor(up), by1 = factor(up1);
#pragma unroll 1
    for (int ch = 0; ch < D; ch += 32) {
      uint32_t u[32];
      tm_load(to + ch, u);
#pragma unroll
      for (int y = 0; y < 32; ++y) u[y] = __float_as_uint(holds ? __uint_as_float(u[y]) * by : nothing);
      if (kTurns) {
        uint32_t w[32];
        tm_load(to + D + ch, w);
#pragma unroll
        for (int y = 0; y < 32; ++y)
          u[y] = __float_as_uint(__uint_as_float(u[y]) + (holds1 ? __uint_as_float(w[y]) * by1 : 0.f));
      }
      if (!real) continue;
      if (done) {
        uint32_t w[16];
#pragma unroll
        for (int y = 0; y < 16; ++y) w[y] = pack<T>(__uint_as_float(u[2 * y]), __uint_as_float(u[2 * y + 1]));
        store32<16>(out + ch, w, a.out_by_32);
      } else {
        store32<32>(part + ch, u, true);
      }
    }
    if (kTurns) {
      tc_fence_before();
      __syncwarp();
      asm volatile("bar.sync 2, 256;" ::: "memory");
    }
    // NaN among the values that this row sees
    const int nans = has || kTurns ? sh->nan_count[seg_no & (kNanLists - 1)] : 0;
    if (nans && real) {
      const int p0 = max(lo, (s.first_tile + s.t) * kKv), p1 = min(hi, (s.first_tile + s.t + seg) * kKv);
      const bool listed = nans <= kNanList;
#pragma unroll 1
      for (int e = listed ? 0 : p0; e < (listed ? nans : p1); ++e) {
        const int p = listed ? sh->nan_pos[seg_no & (kNanLists - 1)][e] : e;
        if (p < p0 || p >= p1) continue;
        const int id = a.block_table[s.r * a.table_stride + (p >> a.block_shift)];
        if ((unsigned)id >= (unsigned)a.n_blocks) continue;
        const int block = 1 << a.block_shift;
        const uint8_t* v = a.v + id * a.block_stride + ((int64_t)s.h * block + (p & (block - 1))) * D;
#pragma unroll 1
        for (int y = 0; y < D; ++y) {
          if ((v[y] & 0x7f) != 0x7f) continue;
          if (done) out[y] = (T)NAN;
          else part[y] = NAN;
        }
      }
    }
    if (real) {
      if (!done) *(float2*)(a.part_ml + (slot * kItemRows + half * kHalf + row) * 2) = float2{ml, l};
      else if (a.lse) a.lse[token * a.n_heads + head] = none ? -INFINITY : (ml + log2f(l)) * 0.6931471805599453f;
    }
    tc_fence_before();
    bar_arrive(&sh->ended[half][seg_no & 1]);
    ++seg_no;
  }
}

template <int D, class T, bool kTurns>
__global__ void __launch_bounds__(kManyThreads, 1) hx_kv_attend_many(
    const __grid_constant__ CUtensorMap qm, const __grid_constant__ AttendArgs a) {
  // all but the last few of the 227 KB; the tiles first, for their alignment
  extern __shared__ __align__(1024) uint8_t s_mem[];
  uint8_t* const qbuf = s_mem;
  uint8_t* const kbuf = qbuf + 2 * Many<D>::kQBytes;
  uint8_t* const vbuf = kbuf + 2 * Many<D>::kTile;
  uint8_t* const raw = vbuf + 2 * Many<D>::kTile;
  Shared& sh = *(Shared*)(raw + 2 * Many<D>::kRaw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  asm volatile("griddepcontrol.launch_dependents;");
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      bar_init(&sh.raw_full[i], 1), bar_init(&sh.raw_empty[i], 4);
      bar_init(&sh.k_full[i], 128), bar_init(&sh.v_full[i], 128);
      bar_init(&sh.k_empty[i], 1), bar_init(&sh.v_empty[i], 1);
      bar_init(&sh.q_full[i], 1), bar_init(&sh.q_empty[i], 1), bar_init(&sh.s_full[i], 1);
      bar_init(&sh.ended[i][0], 128), bar_init(&sh.ended[i][1], 128);
      bar_init(&sh.p_full[i], 128), bar_init(&sh.o_full[i], 1);
    }
    bar_init(&sh.go[0], 1), bar_init(&sh.go[1], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.dead = 0;
    sh.row = -1;
  }

  // this block's stretch of all tiles: each warp adds up its rows', and the one that holds the
  // stretch's first looks it up
  const int per = ((a.n_rows + kManyThreads - 1) / kManyThreads) * 32;  // rows of a warp
  const int w0 = warp * per, w1 = min(a.n_rows, w0 + per);
  const auto row_tiles = [&](int r) {
    const bool real = r < w1;
    const Request q = real ? request(a, r) : Request{0, 0, 0};
    return tiles_per_head(a, q, real);
  };
  long long mine = 0;
  for (int r = w0; r < w1; r += 32) mine += row_tiles(r + lane);
  mine = warp_sum(mine) * a.n_kv_heads;
  if (lane == 0) sh.sum[warp] = mine;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kManyThreads / 32; ++w) {
    if (w < warp) before += sh.sum[w];
    total += sh.sum[w];
  }
  const long long G = max(1LL, min((long long)gridDim.x, total)), b = blockIdx.x;
  const long long n0 = b < G ? total * b / G : 0, n1 = b < G ? total * (b + 1) / G : 0;
  if (n0 < n1 && before <= n0 && n0 < before + mine) {
    for (int r = w0; r < w1; r += 32) {
      const long long head = row_tiles(r + lane), x = head * a.n_kv_heads;
      long long upto = x;
      for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += o;
      }
      const unsigned past = __ballot_sync(~0u, n0 < before + upto);
      if (!past) {
        before += __shfl_sync(~0u, upto, 31);
        continue;
      }
      const int src = __ffs(past) - 1;
      const long long per_head = __shfl_sync(~0u, head, src);
      long long skip = n0 - before - __shfl_sync(~0u, upto - x, src);
      const int h = (int)(skip / per_head);
      skip -= h * per_head;
      const Request q = request(a, r + src);
      const int items = items_of(a, q);
      for (int mt = 0; mt < items; mt += 32) {
        const int tiles = mt + lane < items ? item_tiles(a, q, mt + lane) : 0;
        int sum = tiles;
        for (int d = 1; d < 32; d <<= 1) {
          const int o = __shfl_up_sync(~0u, sum, d);
          if (lane >= d) sum += o;
        }
        const unsigned in = __ballot_sync(~0u, skip < sum);
        if (!in) {
          skip -= __shfl_sync(~0u, sum, 31);
          continue;
        }
        const int y = __ffs(in) - 1;
        skip -= __shfl_sync(~0u, sum - tiles, y);
        if (lane == 0) sh.row = r + src, sh.head = h, sh.mt = mt + y, sh.skip = skip;
        break;
      }
      break;
    }
  }
  __syncthreads();
  if (sh.row < 0) {
    if (tid == 0) a.joins[b] = int4{0, 0, -1, 0};
    return;
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sh.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  Segment s;
  s.r = sh.row;
  s.q = request(a, s.r);
  s.items = items_of(a, s.q);
  s.h = sh.head;
  s.mt = sh.mt;
  const long long skip = sh.skip;
  load_item<kTurns>(a, s);
  s.t = (int)skip;
  int count = (int)(n1 - n0);
  if (tid == 0) {
    // an item that began in an earlier block and ends in this one is joined here
    int4 join = {0, 0, -1, 0};
    if (skip > 0 && skip + count >= s.tiles) {
      const long long f0 = n0 - skip;
      long long c = f0 * G / total;
      while (total * (c + 1) / G <= f0) ++c;
      while (total * c / G > f0) --c;
      join = int4{s.q.first + s.i0, min(s.q.n - s.i0, 2 * a.half_tokens), (int)c, s.h};
    }
    a.joins[b] = join;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp < kConvWarp) softmax<D, T, kTurns>(a, s, count, &sh);
  else if (warp < kMmaWarp) convert<D, T, kTurns>(a, s, count, &sh, raw, kbuf);
  else if (warp == kMmaWarp) issue<D, T, kTurns>(a, s, count, &sh, qbuf, kbuf, vbuf);
  else if (warp == kFetchWarp) fetch<D, kTurns>(a, s, count, &sh, raw);
  else if (lane == 0) queries<D, kTurns>(a, &qm, s, count, &sh, qbuf);
  __syncwarp();
  drain(&sh.dead, a.status);
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sh.tmem) : "memory");
}

template <int D, class T, bool kTurns>
cudaError_t launch(const CUtensorMap& qm, const AttendArgs& a, int blocks, cudaStream_t s) {
  constexpr int kSmem = Many<D>::kTiles + (int)sizeof(Shared);
  static_assert(kSmem <= 227 * 1024, "shared memory of a block");
  const auto kernel = hx_kv_attend_many<D, T, kTurns>;
  if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem)) return e;
  kernel<<<blocks, kManyThreads, kSmem, s>>>(qm, a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_many(const CUtensorMap& qm, const AttendArgs& a, int head_dim, bool bf16, int blocks, cudaStream_t s) {
  const bool turns = a.max_q > 0 && a.max_q <= a.half_tokens;
  const auto typed = [&](auto d, auto type) {
    using T = decltype(type);
    return turns ? launch<decltype(d)::value, T, true>(qm, a, blocks, s) : launch<decltype(d)::value, T, false>(qm, a, blocks, s);
  };
  const std::integral_constant<int, 64> d64{};
  const std::integral_constant<int, 128> d128{};
  if (head_dim == 128) return bf16 ? typed(d128, __nv_bfloat16{}) : typed(d128, __half{});
  return bf16 ? typed(d64, __nv_bfloat16{}) : typed(d64, __half{});
}

}  // namespace hx
