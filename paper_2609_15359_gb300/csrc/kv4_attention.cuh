// kv4_attention.cuh -- what the two forms of attention over the 4-bit cache share: their arguments,
// how work is dealt out, and small device helpers.
#pragma once

#include <atomic>

#include "kv4.cuh"

namespace maps {

// Requests up to which every block deals out the units for itself; beyond, a kernel of one block does it for all (64 requests of
// 300 tokens: 18 us themselves, 25 with the kernel; 512: 52, 58; 2,048: 173, 178).
constexpr int kMaxLocalB = 2048;

// Lets a kernel have `bytes` of dynamic shared memory, once for each device.  `current` receives the device.
template <auto kKernel>
int allow_smem(size_t bytes, int *current = nullptr) {
  static std::atomic<uint64_t> done;
  int dev = 0;
  MAPS_TRY(cuda_ok(cudaGetDevice(&dev)));
  if (current != nullptr) *current = dev;
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return MAPS_OK;
  MAPS_TRY(cuda_ok(cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes))));
  done.fetch_or(bit, std::memory_order_relaxed);
  return MAPS_OK;
}

constexpr int kMaxGrid = kCtrlBytes - 64;
inline int attn_grid() { return sm_count() < kMaxGrid ? sm_count() : kMaxGrid; }

struct Part;

// Tokens a request can have: places a unit or a step past them are still counted in 32 bits.
constexpr int32_t kMaxLen = 0x7fffffff - 1023;

struct AttnArgs {
  int32_t B, Hq, Hkv, S;
  int64_t T, n_blocks, max_blocks;
  const void *q;
  int64_t q_row, q_head, o_row, o_head;
  const int64_t *off;
  const int32_t *len, *table;
  const uint8_t *cache;
  float scale;
  int32_t causal, window, wide;
  int64_t block_bytes;  // of all heads
  int32_t block_groups, block_shift;  // groups of a block, and their logarithm where they are a power of two, else -1
  void *out;
  float *lse;
  void *starts;        // where each worker starts, and the units in all, where a block does not find out for itself
  uint32_t *units;
  uint32_t *arrived;   // a byte for each block: blocks that have brought their part of the item it begins
  float *parts;        // [grid][2] parts of items that cross blocks
  // the form for many queries
  int32_t few_rows;       // a request with more query rows to a KV head may go there (0: none does)
  void *many_starts;      // where each block starts, and the units in all
  uint32_t *many_units;
  float *many_parts;      // [grid][2]
  Part *many_open;        // [grid] the item that a block begins and does not end
  int32_t *status;
};

// What of an item a warp, or a block, has: the item's first unit and its units (0: none), its queries' first row, rows, head and row tile.
struct Part {
  int64_t q0;
  uint32_t id, tiles;
  int32_t rows, h, rt;
};

__device__ __forceinline__ bool length_ok(const AttnArgs &a, int32_t n) { return n >= 0 && n <= kMaxLen && n <= a.max_blocks * a.S; }

// ---------------------------------------------------------------------------- small device helpers
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Sleeps for up to 20 us where the phase is not over: polling costs the other warps issue slots.
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000u) : "memory");
  return ok != 0;
}
constexpr uint32_t kTries = 1u << 18;
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t tries = kTries) {  // bounded; tries >= 1
  uint32_t i = 0;
  do
    if (bar_try(bar, parity)) return true;
  while (++i < tries);
  return false;
}
// The same for a warp, whose lanes go on, or give up, together.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint32_t tries = kTries) { return __all_sync(0xffffffffu, bar_wait(bar, parity, tries)); }
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  uint32_t y;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}

// A word's eight codes as four pairs of half numbers, in five operations: a bare code is the
// subnormal number code * 2^-24, four bits higher it is code * 2^-20, and the tensor core multiplies
// both exactly.  The odd pairs' factor of 16 is taken off in the other operand (keys) or the sum (values).
struct Codes {
  uint32_t x[4];  // codes (r, r + 4)
};
__device__ __forceinline__ Codes codes_of(uint32_t w) {
  const uint32_t v = w >> 8;
  return {{w & 0x000f000fu, w & 0x00f000f0u, v & 0x000f000fu, v & 0x00f000f0u}};
}
constexpr float kEven = 16777216.0f, kOdd = 1048576.0f;  // 2^24, 2^20

// How the units are dealt out: worker w, a warp, has units start(w) .. start(w + 1) - 1.
struct Deal {
  uint32_t units, used, per, more;  // used: workers that get units, the first ones
  __device__ __forceinline__ Deal(uint32_t U, uint32_t workers) : units(U), used(U < workers ? U : workers), per(0), more(0) {
    if (used) per = U / used, more = U % used;
  }
  __device__ __forceinline__ uint32_t start(uint32_t w) const { return w >= used ? units : per * w + min(w, more); }
  __device__ __forceinline__ uint32_t worker(uint32_t u) const { return u < more * (per + 1) ? u / (per + 1) : more + (u - more * (per + 1)) / per; }
};

// Query rows x keys x KV heads of all requests that may go to the form for many queries, up to which none does: its queries,
// parts and joins cost 40 us and more whatever the lengths (a window, which lessens both forms' work, is left out of account).
// 128 channels, one request of 256 rows and 4,096 tokens (8 million): 44 us with few, 76 with many; four of 128 rows
// (17 million) 63, 58; 32 of 128 rows and 500 tokens (16 million) 76, 73; four of 256 rows (34 million) 100, 69.
constexpr uint64_t kFewPairs = uint64_t(1) << 24;

// The rows over which a request of this call goes to the form for many queries; 0: none does.  All kN threads call it.
template <int kN>
__device__ __forceinline__ int32_t many_over(const AttnArgs &a) {
  if (a.few_rows == 0) return 0;
  __shared__ unsigned long long s_pairs;
  if (threadIdx.x == 0) s_pairs = 0;
  __syncthreads();
  const int64_t group = a.Hq / a.Hkv;
  uint64_t pairs = 0;
  for (int b = threadIdx.x; b < a.B; b += kN) {
    const int64_t q0 = a.off[b], q1 = a.off[b + 1], rows = (q1 - q0) * group;
    const int32_t n = a.len[b];
    if (!length_ok(a, n) || q0 < 0 || q1 < q0 || q1 > a.T || rows <= a.few_rows) continue;
    pairs += min(static_cast<uint64_t>(rows) * static_cast<uint64_t>(n), uint64_t(1) << 32);
  }
  if (pairs) atomicAdd(&s_pairs, static_cast<unsigned long long>(pairs));
  __syncthreads();
  return s_pairs > kFewPairs / a.Hkv ? a.few_rows : 0;
}

// The form for many queries (kv4_attention_many.cu).
bool attn_many_dim(int D);
void attn_many_carve(Carve &c, AttnArgs &a, int32_t B, int D);
int attn_many(int32_t dtype, int D, const AttnArgs &a, cudaStream_t s);

// maps_test_attention_withhold for attention over lists (kv4_attention_blocks.cu).
int attn_lists_withhold(int32_t block, uint32_t tries);

}  // namespace maps
