// hx_kv_attend.cuh -- device helpers of the attention kernels: barriers and tile
// copies with bounded waits, e4m3 to f16, the rows of a request.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "hx_kv.cuh"

namespace hx {

constexpr float kLog2e = 1.4426950408889634f;
// Sums of weighted values are kept, and left to the join, in units of 2^kSumUnit: before they are divided by the softmax's sum
// they are larger than a result by up to 2^30 tokens and the 2^8 or 2^10 by which a maximum may lag.
constexpr int kSumUnit = 20;
constexpr float kSumUp = 1 << kSumUnit, kSumDown = 1 / kSumUp;
constexpr int kItemRows = 256;  // places for rows of an item of the many-rows kernel: two halves of 128

// Division by a divisor known on the host (Granlund and Montgomery's invariant
// division): x / d for 0 <= x < 2^31.
struct Divisor {
  uint32_t mul, shift;
  int32_t d;
#ifdef __CUDACC__
  __device__ __forceinline__ int of(int x) const { return (int)((__umulhi((uint32_t)x, mul) + (uint32_t)x) >> shift); }
  __device__ __forceinline__ int rest(int x) const { return x - of(x) * d; }
#endif
};
inline Divisor divisor(int32_t d) {
  uint32_t s = 0;
  while ((1u << s) < (uint32_t)d) ++s;
  return {(uint32_t)((((1ull << s) - (uint32_t)d) << 32) / (uint32_t)d + 1), s, d};
}

// What the kernels read of hx_kv_cache and hx_kv_query.
struct AttendArgs {
  const uint8_t* k;
  const uint8_t* v;
  const float* k_scale;
  const float* v_scale;
  int64_t block_stride, scale_stride;
  const void* q;
  void* out;
  float* lse;
  int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
  const int32_t* row_start;
  const int32_t* kv_len;
  const int32_t* block_table;
  int64_t table_stride;
  int32_t table_width, n_blocks, n_tokens, n_rows, n_heads, n_kv_heads, group;
  int32_t block_shift, max_q, causal, window;
  int32_t out_by_32;    // whether out's rows lie on multiples of 32 bytes
  int32_t few_rows;     // requests of so many rows at most are the few-rows kernel's
  Divisor by_group;     // rows to tokens
  int32_t half_tokens;  // of an item's half in the many-rows kernel: 128 / group
  float sm_scale_log2;  // sm_scale * log2(e): scores are exponents of two
  float* part;          // partial results of items that several blocks share
  float* part_ml;
  int4* joins;          // [blocks] of the item that ends in the block's stretch: its first token, its tokens, the block where
                        // it begins (-1: nothing to join), its kv head
  int32_t* status;      // set to 1 if a wait gives up, or NULL
};

// Launches the many-rows kernel (hx_kv_attend_many.cu) on `blocks` blocks.
cudaError_t launch_attend_many(const CUtensorMap& qm, const AttendArgs& a, int head_dim, bool bf16, int blocks, cudaStream_t s);

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint64_t* b, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(b)), "r"(bytes) : "memory");
}
// Between a thread's own reads and writes of shared memory and those of copies and products, whichever come
// first.  An arrival alone does not wait for loads that are still under way: the copy that it lets
// begin could write under them.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(smem_addr(b)), "r"(parity)
      : "memory");
  return ok;
}
// Waits for a phase, but not for ever: after kWaitCycles (about two seconds; 0: a phase that is not over yet is not
// waited for) it gives up, says so in *dead, and from then on no wait of the block waits.  What a warp has computed stands only if
// *dead is still 0 behind its last wait: whoever gives up says so before it arrives anywhere.  And a barrier that bytes may
// still be due at is not armed again: nobody arrives where that would be asked for.
#ifndef HX_KV_WAIT_CYCLES
#define HX_KV_WAIT_CYCLES 4000000000LL
#endif
constexpr long long kWaitCycles = HX_KV_WAIT_CYCLES;
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile int* dead) {
  if constexpr (kWaitCycles == 0) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(smem_addr(b)), "r"(parity)
        : "memory");
    if (!ok) *dead = 1;
    return ok;
  }
  if (bar_try(b, parity)) return true;
  const long long t0 = clock64();
  do {
#pragma unroll 1  // there are many waits: unrolled, they crowd the instruction cache
    for (int i = 0; i < 32; ++i)
      if (bar_try(b, parity)) return true;
  } while (!*dead && clock64() - t0 < kWaitCycles);
  *dead = 1;
  return false;
}
// Before a block that gave up ends: says so to the caller, and leaves its own copies in flight the time to land.
__device__ __forceinline__ void drain(volatile int* dead, int32_t* status) {
  if (!*dead) return;
  if (status) *status = 1;
  const long long t0 = clock64();
  while (clock64() - t0 < 20000000LL) __nanosleep(1000);
}

__device__ __forceinline__ void tile_load(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
          smem_addr(dst)),
      "l"(map), "r"(smem_addr(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

__device__ __forceinline__ void tile_prefetch(const CUtensorMap* map, int x, int y, int z) {  // into L2
  asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(map), "r"(x), "r"(y), "r"(z)
               : "memory");
}

// `bytes` (a multiple of 16) in a row, both sides 16-byte aligned.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_addr(dst)),
               "l"(src), "r"(bytes), "r"(smem_addr(bar))
               : "memory");
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two e4m3 bytes to two f16 (exact).
__device__ __forceinline__ uint32_t cvt2(uint32_t two) {
  uint32_t h;
  asm("{\n.reg .b16 l;\ncvt.u16.u32 l, %1;\ncvt.rn.f16x2.e4m3x2 %0, l;\n}\n" : "=r"(h) : "r"(two));
  return h;
}
__device__ __forceinline__ uint32_t cvt2_hi(uint32_t four) {
  uint32_t h;
  asm("{\n.reg .b16 l, u;\nmov.b32 {l, u}, %1;\ncvt.rn.f16x2.e4m3x2 %0, u;\n}\n" : "=r"(h) : "r"(four));
  return h;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  uint32_t h;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(hi), "f"(lo));
  return h;
}

// d += a b, 16 x 8 x 16, f16 with 32-bit sums.
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// One request's part in the step, its lengths brought into range.
struct Request {
  int first, n, kv;  // its first token, its tokens in the step, the tokens it holds
};
__device__ __forceinline__ Request request(const AttendArgs& a, int r) {
  Request q;
  q.first = min(max(a.row_start[r], 0), a.n_tokens);
  q.n = min(max(a.row_start[r + 1], q.first), a.n_tokens) - q.first;
  const int64_t room = (int64_t)a.table_width << a.block_shift;
  q.kv = (int)min((int64_t)max(a.kv_len[r], 0), room);
  if (a.max_q && q.n > a.max_q) q.kv = 0;
  return q;
}

// [lo, hi) of token i of a request.
__device__ __forceinline__ int see_from(const AttendArgs& a, const Request& q, int i) {
  return a.window ? max(0, q.kv - q.n + i - a.window + 1) : 0;
}
__device__ __forceinline__ int see_to(const AttendArgs& a, const Request& q, int i) {
  return a.causal ? min(q.kv, max(0, q.kv - q.n + i + 1)) : q.kv;
}

}  // namespace hx
