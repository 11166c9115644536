// kv4_attention_many.cu -- attention over the paged 4-bit KV cache, form for many queries a request
// (chunks of prompts): the products dominate, so they run on tcgen05.
//
// A block takes 256 query rows (queries x heads of one KV head) as two tiles of 128 and passes over the
// keys they see in steps of 128.  Per step and tile, S = Q K^T and O += P V are 128 x 128 x D products
// with their results in tensor memory; P replaces S there, as halves, and is the second product's operand.
//
//   warps 0-3, 4-7   softmax of a tile, a row a thread: S from tensor memory, running maximum and sum, P back;
//                    they rescale O when the maximum has grown by more than 2^8, and write it out at the end
//   warps 8-11       the values' codes to operands in shared memory, one step deep
//   warp 15          the same of the keys, two deep: a step's keys may be wanted a second time (below)
//   warp 12          issues the products; the two tiles alternate, so that one's softmax runs beside the other's products
//   warp 13          bulk copies of the cache's records, up to three steps ahead
//   warp 14          walks the block's items and tells the others what each is; in their registers it would cost the
//                    inner loops, which need little of it, a fifth of theirs
//
// Keys enter the first product as bare codes (subnormal halves, exact; the odd pairs' factor of 16 is taken
// off in Q) and s, z come in with the row's sum of Q in 32 bits, as in the form for few queries: two packed
// operations for two scores.  Values become halves of their own: v 2^-E with a power of two of their token's, so any
// magnitude fits and a value keeps 11 bits.  2^E goes with the weight, so that what enters the running maximum is a weight times
// its value, and rows that a query hardly weighs, or does not see, take no bits from the others however large they are.  That is
// one packed addition for two scores (753 -> 783 us below); with a power of two common to a step, value rows 2^16 times
// the others left later steps' weights below half's range.  The whole scale on the weights would be three operations a score.
//
// Bound.  A step's four products take the tensor cores about 2,200 cycles at D = 128 where nothing else runs, but a step
// takes 6,800: each tile's chain of softmax (some 3,500 cycles: scores, weights, the tile's vote, P) and products (3,100 from P to the
// next S, which replaces P), in which the products take two and a half times as long to issue as alone.  The tensor
// cores' pipe is active 24 % of the time, and issue slots are 46 % taken.  Six chunks of 1,024 queries, 32 heads on 8, behind 1,500
// to 9,000 tokens: 783 us, 552 TFLOP/s of 432 GFLOP (0.29 of the measured dense rate); with 64 channels 636.  S in halves of 64 keys, the first beside
// P, so that the softmax need not wait for the sums, was 894 us: more and smaller products for the same thread.
//
// Split.  As in the other form, a call's steps are dealt out to the blocks in equal runs, whatever the
// lengths; what a run begins or ends inside of is left as parts, which a second kernel joins.
#include "kv4_attention.cuh"
#include "maps_bench.h"

namespace maps {
namespace {

constexpr int kThreads = 512;
constexpr int kItemUnits = 3;  // what an item costs besides its steps, in steps: its queries, its output, the pipeline's start
constexpr int kRows = 256, kTok = 128, kStepGroups = kTok / kGroup;
constexpr int kRing = 3;  // steps of the cache's records under way or waiting

// Test aid (maps_test_attention_withhold): the block whose keys are never said to be there (-1: none), so that the waits of all
// its warps run out, and the tries after which a wait gives up.
__constant__ int32_t c_withheld = -1;
__constant__ uint32_t c_tries = kTries;
__device__ __forceinline__ bool one_wait(uint32_t bar, uint32_t parity) { return bar_wait(bar, parity, c_tries); }
__device__ __forceinline__ bool all_wait(uint32_t bar, uint32_t parity) { return warp_wait(bar, parity, c_tries); }

struct MReq {
  int64_t q0;
  int32_t n, n_q, row_tiles;
};

__device__ __forceinline__ MReq many_request(const AttnArgs &a, int b) {
  MReq r;
  const int64_t q0 = a.off[b], q1 = a.off[b + 1];
  int64_t m = q1 - q0;
  int32_t n = a.len[b];
  if (!length_ok(a, n) || q0 < 0 || m < 0 || q1 > a.T) n = 0, m = 0;  // the other form has reported it
  const int64_t rows = m * (a.Hq / a.Hkv);
  r.q0 = q0;
  r.n = n;
  r.n_q = static_cast<int32_t>(m);
  r.row_tiles = n > 0 && rows > a.few_rows ? static_cast<int32_t>((rows + kRows - 1) / kRows) : 0;
  return r;
}

// The tokens lo .. hi - 1 that a row tile's queries see between them (lo to 16), and its units: kItemUnits for itself, and its steps.
__device__ __forceinline__ int span(const AttnArgs &a, const MReq &r, int rt, int32_t &lo, int32_t &hi) {
  const int group = a.Hq / a.Hkv;
  const int first = rt * kRows / group, last = min(r.n_q - 1, (rt * kRows + kRows - 1) / group);
  const int64_t shift = static_cast<int64_t>(r.n) - r.n_q;
  hi = a.causal ? static_cast<int32_t>(max(int64_t(0), shift + last + 1)) : r.n;
  const int64_t from = a.window > 0 ? shift + first - a.window + 1 : 0;
  lo = from > 0 ? static_cast<int32_t>(min(from, static_cast<int64_t>(hi))) / kGroup * kGroup : 0;
  return kItemUnits + (hi > lo ? (hi - lo + kTok - 1) / kTok : 0);
}

struct ManyStart {
  MReq r;
  int32_t b;
  uint32_t rest;
};

// What the warps are told of an item, or of what a block has of it.
struct Seg {
  int64_t q0;
  int32_t steps;         // -1: no further item
  int32_t token, hi;     // the first step's first token, and the end of those that any of the rows see
  int32_t n, n_q, rows;  // of the request; rows of all its tiles
  int32_t b, h, rt;
  int32_t second;        // whether the second tile has rows
  int32_t whole;
  uint32_t id, tiles;    // the item's first unit and its units
};
constexpr int kSegs = 4;  // under way or told ahead
constexpr int kHearers = 15;

template <int kN, class Put>
__device__ __forceinline__ uint32_t many_plan(const AttnArgs &a, uint32_t blocks, uint32_t w0, uint32_t w1, Put put) {
  __shared__ uint64_t s_warp[kN / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int run = (a.B + kN - 1) / kN, b0 = min(tid * run, a.B), b1 = min(b0 + run, a.B);
  auto units_of = [&](const MReq &r) {
    uint64_t all = 0;
    int32_t lo, hi;
    for (int t = 0; t < r.row_tiles; ++t) all += span(a, r, t, lo, hi);
    return all * a.Hkv;
  };
  uint64_t mine = 0;
  for (int b = b0; b < b1; ++b) mine += units_of(many_request(a, b));
  uint64_t x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  uint64_t at = x - mine, U = 0;
  for (int w = 0; w < kN / 32; ++w) {
    const uint64_t y = s_warp[w];
    if (w < warp) at += y;
    U += y;
  }
  if (U >= 1ull << 31) {  // more than one call's worth of work
    if (tid == 0) flag_error(a.status, MAPS_E_RANGE);
    return 0;
  }
  const Deal deal(static_cast<uint32_t>(U), blocks);
  if (mine > 0 && at < deal.start(w1) && at + mine > deal.start(w0)) {
    for (int b = b0; b < b1; ++b) {
      const MReq r = many_request(a, b);
      const uint32_t lo = static_cast<uint32_t>(at), n = static_cast<uint32_t>(units_of(r));
      at += n;
      if (n == 0) continue;
      uint32_t w = max(deal.worker(lo), w0);
      if (deal.start(w) < lo) ++w;
      for (; w < min(w1, deal.used) && deal.start(w) < lo + n; ++w) put(w, ManyStart{r, b, deal.start(w) - lo});
    }
  }
  return static_cast<uint32_t>(U);
}

__global__ void __launch_bounds__(1024) attn_many_plan_kernel(const AttnArgs a, uint32_t blocks) {
  pdl_prologue();
  const uint32_t U = many_over<1024>(a) == 0 ? 0 : many_plan<1024>(a, blocks, 0, blocks, [&](uint32_t w, const ManyStart &s) { static_cast<ManyStart *>(a.many_starts)[w] = s; });
  if (threadIdx.x == 0) *a.many_units = U;
}

// ---------------------------------------------------------------------------- tensor memory, products, packed arithmetic
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Operands in shared memory are rows of 64 halves (128 bytes) in the 128-byte swizzle, 8 rows to 1,024 bytes:
// the low word of a descriptor is the address, the high word the same for all.
__device__ __forceinline__ uint32_t rows_desc(uint32_t addr) { return (addr >> 4 & 0x3fffu) | 1u << 16; }
constexpr uint32_t kDescHigh = 64u | 1u << 14 | 2u << 29;
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t A, uint32_t B, uint32_t idesc, uint32_t add) {
  asm volatile("{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %4, 0;\nmov.b64 a, {%1, %5};\nmov.b64 b, {%2, %5};\n"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d), "r"(A), "r"(B), "r"(idesc), "r"(add), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t A, uint32_t B, uint32_t idesc, uint32_t add) {
  asm volatile("{\n.reg .pred p;\n.reg .b64 b;\nsetp.ne.b32 p, %4, 0;\nmov.b64 b, {%2, %5};\n"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d), "r"(A), "r"(B), "r"(idesc), "r"(add), "r"(kDescHigh) : "memory");
}
// Instruction: halves in, 32-bit sums, 128 rows, N columns, both operands along the depth.
__host__ __device__ constexpr uint32_t idesc_of(int N) { return (1u << 4) | (static_cast<uint32_t>(N / 8) << 17) | (8u << 24); }

#define MAPS_R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define MAPS_W8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
__device__ __forceinline__ void tm_load16(uint32_t addr, uint32_t *x) {  // a row a thread
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];" : MAPS_R8(x, 0), MAPS_R8(x, 8) : "r"(addr) : "memory");
}
// 16 rows and 32 columns as the four-lanes-a-row fragments of a warp-level product: registers 4 i .. 4 i + 3 are columns
// 8 i + 2 (lane % 4) and the next, of row lane / 4 and of row lane / 4 + 8.
__device__ __forceinline__ void tm_load_frag(uint32_t addr, uint32_t *x) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];" : MAPS_R8(x, 0), MAPS_R8(x, 8) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_load_frag2(uint32_t addr, uint32_t *x) {  // 16 columns
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];" : MAPS_R8(x, 0) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_store_frag(uint32_t addr, const uint32_t *x) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x4.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::MAPS_W8(x, 0), MAPS_W8(x, 8), "r"(addr) : "memory");
}
// The same of 16 columns as halves, two to a word: register 2 i is row lane / 4, register 2 i + 1 the row 8 on.
__device__ __forceinline__ void tm_store_halves(uint32_t addr, const uint32_t *x) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x2.b32 [%4], {%0,%1,%2,%3};" ::"r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(addr) : "memory");
}
// The loads' registers pass through the wait, so that nothing uses them ahead of it.
#define MAPS_RW8(x, i) "+r"(x[i]), "+r"(x[i + 1]), "+r"(x[i + 2]), "+r"(x[i + 3]), "+r"(x[i + 4]), "+r"(x[i + 5]), "+r"(x[i + 6]), "+r"(x[i + 7])
__device__ __forceinline__ void tm_wait16(uint32_t *x) { asm volatile("tcgen05.wait::ld.sync.aligned;" : MAPS_RW8(x, 0), MAPS_RW8(x, 8)::"memory"); }
__device__ __forceinline__ void tm_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

union F2 {
  uint64_t v;
  float f[2];
  uint32_t u[2];
};
__device__ __forceinline__ uint64_t two(float x, float y) {
  F2 r;
  r.f[0] = x, r.f[1] = y;
  return r.v;
}
__device__ __forceinline__ uint64_t mul2(uint64_t x, uint64_t y) {
  uint64_t z;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(z) : "l"(x), "l"(y));
  return z;
}
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) {
  uint64_t z;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(z) : "l"(x), "l"(y));
  return z;
}
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t w) {
  uint64_t z;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(z) : "l"(x), "l"(y), "l"(w));
  return z;
}


template <int D>
struct Lay {  // shared memory, from a 1,024-byte boundary
  static constexpr int kTile = 128 * D * 2;          // Q of a tile, K or V of a step
  static constexpr int kStep = kStepGroups * kv4_group_bytes(D);  // records
  static constexpr int kQ = 0, kK = 2 * kTile, kV = 4 * kTile, kRingAt = 5 * kTile;
  // [4][64][2] of two tokens: {scale, scale, zero, zero} of the keys, {exponent, exponent, and 2 to minus them} of the values
  static constexpr int kPar = kRingAt + kRing * kStep;
  static constexpr int kRow = kPar + 4 * kTok * 16;  // [256] a row's sum, what a score is to be multiplied by, and the keys that it sees
  static constexpr int kNan = kRow + kRows * 16;     // [4][4] bits: values that are not finite
  static constexpr int kAgain = kNan + 64;           // [2] a tile's scores are wanted again
  static constexpr int kBars = kAgain + 8;
  static constexpr int kSegAt = kBars + 8 * (2 * kRing + 14 + 2 * kSegs);
  static constexpr int kBytes = kSegAt + kSegs * static_cast<int>(sizeof(Seg));
  static constexpr int kPart = kRows * D + 2 * kRows;  // floats of a part: sums, maxima, totals
};
static_assert(Lay<128>::kBytes + 1024 + 512 <= 227 * 1024, "shared memory");
template <int D>
constexpr bool lay_aligned() {  // to what is read and written there at once
  using L = Lay<D>;
  return L::kK % 1024 == 0 && L::kV % 1024 == 0 && L::kRingAt % 16 == 0 && L::kStep % 16 == 0 && L::kPar % 16 == 0 && L::kRow % 16 == 0 && L::kNan % 16 == 0 &&
         L::kAgain % 4 == 0 && L::kBars % 8 == 0 && L::kSegAt % alignof(Seg) == 0;
}
static_assert(lay_aligned<64>() && lay_aligned<128>(), "alignment");

// Weights are halves against the largest weight times value so far, which counts as 2^kBias: what is 2^21 times smaller still
// has 11 bits.  They may exceed it by 2^kSlack before the sums are rescaled at the next step, and by 2^kMost at all, for half's range.
constexpr float kBias = 7.0f, kSlack = 6.0f, kMost = 8.75f;

// A token's values are left out of the product where they are no finite numbers: held as NaN, or, at places that no query
// sees, whatever lies there.  0 times what is not finite would reach every row.  (Halves: the largest may round past 32 bits.)
__device__ __forceinline__ bool value_finite(float2 p) { return fabsf(fmaf(7.5f, p.x, 0.5f * p.y)) < INFINITY && fabsf(p.y) < INFINITY; }
// The power of two by which they are taken out: v 2^-E is in 2^14 .. 2^15, or less where the row is tiny or zero.
__device__ __forceinline__ int value_exponent(float2 p) {
  return max(static_cast<int>(__float_as_uint(fmaxf(fabsf(0.5f * p.y), fabsf(fmaf(7.5f, p.x, 0.5f * p.y)))) >> 23) - 140, -60);
}

// Whether any of a tile's 128 threads says so; barrier `id` of the block.
__device__ __forceinline__ bool tile_any(int id, bool x) {
  uint32_t y;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 q, %1, 0;\nbarrier.cta.red.or.pred p, %2, 128, q;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(y) : "r"(static_cast<uint32_t>(x)), "r"(id) : "memory");
  return y != 0;
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1) attn_many_kernel(const AttnArgs a) {
  using L = Lay<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ ManyStart s_start;
  __shared__ uint32_t s_tmem;
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t base = smem_u32(smem), bars = base + L::kBars;
  // barriers
  auto step_full = [&](int i) { return bars + 8 * i; };  // a step's records are in the ring, and have been read
  auto step_free = [&](int i) { return bars + 8 * (kRing + i); };
  const uint32_t b0 = bars + 16 * kRing, v_full = b0, v_free = b0 + 8;
  auto k_full = [&](int i) { return b0 + 16 + 8 * i; };
  auto k_free = [&](int i) { return b0 + 32 + 8 * i; };
  auto q_full = [&](int t) { return b0 + 48 + 8 * t; };
  auto s_full = [&](int t) { return b0 + 64 + 8 * t; };
  auto p_full = [&](int t) { return b0 + 80 + 8 * t; };
  auto o_full = [&](int t) { return b0 + 96 + 8 * t; };
  auto seg_full = [&](int i) { return b0 + 112 + 8 * i; };
  auto seg_free = [&](int i) { return b0 + 112 + 8 * kSegs + 8 * i; };

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_prologue();
  uint32_t U;
  const uint32_t me = blockIdx.x;
  if (a.B <= kMaxLocalB) {
    U = many_over<kThreads>(a) == 0 ? 0 : many_plan<kThreads>(a, gridDim.x, me, me + 1, [&](uint32_t, const ManyStart &s) { s_start = s; });
    if (me == 0 && tid == 0) *a.many_units = U;  // for the kernel that joins
  } else {
    U = *a.many_units;
    if (me < U && tid == 0) s_start = static_cast<const ManyStart *>(a.many_starts)[me];
  }
  if (tid == 0) a.many_open[me].tiles = 0;
  if (U == 0) return;  // no request here has many queries
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) reinterpret_cast<int *>(smem + L::kAgain)[i] = 0;
    for (int i = 0; i < kRing; ++i) bar_init(step_full(i), kStepGroups), bar_init(step_free(i), 5);
    bar_init(v_full, 4), bar_init(v_free, 1);
    for (int i = 0; i < 2; ++i) {
      bar_init(k_full(i), 1), bar_init(k_free(i), 1);
      bar_init(q_full(i), 4), bar_init(s_full(i), 2), bar_init(p_full(i), 4), bar_init(o_full(i), 1);
    }
    for (int i = 0; i < kSegs; ++i) bar_init(seg_full(i), 1), bar_init(seg_free(i), kHearers);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const Deal deal(U, gridDim.x);
  const uint32_t u0 = deal.start(me), u1 = deal.start(me + 1);
  const uint32_t tmem = s_tmem;  // 0
  const int group = a.Hq / a.Hkv;
  const float sl2 = a.scale * 1.4426950408889634f, k_sign = a.scale < 0.0f ? -1.0f : 1.0f;

  // the next item: waits for it, and says whether there is one; then what it is, and that this warp is done with it
  uint32_t n_seg = 0;
  // where a step's records lie in the ring, and the parity of the round
  int place = 0;
  uint32_t round = 0;
  auto ring_on = [&]() {
    if (++place == kRing) place = 0, round ^= 1u;
  };
  auto more = [&](bool ok) { return ok && reinterpret_cast<const Seg *>(smem + L::kSegAt)[n_seg % kSegs].steps >= 0; };
  auto hear = [&](bool &ok) { return more(ok = all_wait(seg_full(n_seg % kSegs), n_seg / kSegs & 1)); };
  auto hear_alone = [&](bool &ok) { return more(ok = one_wait(seg_full(n_seg % kSegs), n_seg / kSegs & 1)); };
  auto told = [&]() -> const Seg & { return reinterpret_cast<const Seg *>(smem + L::kSegAt)[n_seg % kSegs]; };
  auto done = [&]() { bar_arrive(seg_free(n_seg++ % kSegs)); };  // by one lane

  if (warp < 8) {
    // ======================================================================== softmax
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;  // 32 lanes of tensor memory to a warp
    const uint32_t s_at = tmem + lanes + t * 128, o_at = tmem + lanes + 256 + t * 128;
    uint32_t c = 0, n_s = 0, n_o = 0;  // steps, scores and sums so far
    // A wait that has run out in one warp ends the four warps of its tile together, at their next vote: a warp that left alone
    // would leave the others in a barrier without an end.  So between votes a failure is carried on.
    bool ok = true, failed = false;
    for (;;) {
      const bool another = ok && hear(ok);
      ok = !tile_any(1 + t, !ok);
      if (!ok || !another) break;
      const Seg &w = told();
      const int steps = w.steps, tok_at = w.token;
      if (t == 1 && !w.second) {
        c += steps;
        __syncwarp();
        if (lane == 0) bar_arrive(seg_free(n_seg % kSegs));
        ++n_seg;
        continue;
      }
      float4 *row_of = reinterpret_cast<float4 *>(smem + L::kRow) + t * 128;
      const int R = w.rt * kRows + t * 128 + row;
      const bool there = R < w.rows;
      {
        int32_t lo = 0, hi = 0x7fffffff;  // a row that is none sees everything; nobody reads it
        if (there) {
          const int64_t pos = static_cast<int64_t>(w.n) - w.n_q + R / group;
          hi = pos < 0 ? 0 : a.causal ? static_cast<int32_t>(pos) + 1 : w.n;
          if (a.window > 0 && pos - a.window + 1 > 0) lo = static_cast<int32_t>(pos - a.window + 1);
        }
        reinterpret_cast<int2 *>(row_of + row)[1] = make_int2(lo, hi);
      }
      if (steps > 0) {
        // ---- the warp's 32 rows of Q, D/8 lanes to a row, each row scaled by a power of two to fill half's range; 8 channels
        // in the order of the codes.  Small loops here and below: what is met once an item is not in the instruction cache.
        constexpr int kLanes = D / 8, kAt = 32 / kLanes;
        const int rows = w.rows, h0 = w.h * group;
        const int64_t q0 = w.q0;
        constexpr int kBatch = 8;  // loads under way at once
#pragma unroll 1
        for (int x0 = 0; x0 < kLanes; x0 += kBatch) {
          uint4 raws[kBatch];
#pragma unroll
          for (int x = 0; x < kBatch; ++x) {
            const int Rx = w.rt * kRows + t * 128 + (warp & 3) * 32 + (x0 + x) * kAt + lane / kLanes;
            raws[x] = make_uint4(0, 0, 0, 0);
            if (Rx < rows) {
              const T *src = static_cast<const T *>(a.q) + (q0 + Rx / group) * a.q_row + (h0 + Rx % group) * a.q_head + 8 * (lane % kLanes);
              if (a.wide) {
                raws[x] = *reinterpret_cast<const uint4 *>(src);
              } else {
                T *z = reinterpret_cast<T *>(&raws[x]);
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = src[e];
              }
            }
          }
#pragma unroll
          for (int x = 0; x < kBatch; ++x) {
            const int r = (warp & 3) * 32 + (x0 + x) * kAt + lane / kLanes, at = lane % kLanes;
            const T *y = reinterpret_cast<const T *>(&raws[x]);
            float q[8], top = 0.0f, sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) q[e] = Cvt<T>::to(y[e]), top = fmaxf(top, fabsf(q[e]));
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const int ef = min(max(static_cast<int>(__float_as_uint(top) >> 23), 20), 254);
            const float up = __uint_as_float(static_cast<uint32_t>(268 - ef) << 23);
#pragma unroll
            for (int e = 0; e < 8; ++e) q[e] *= up, sum += q[e];
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const uint4 z = make_uint4(pack_half(q[0], q[4]), pack_half(q[1] * 0.0625f, q[5] * 0.0625f), pack_half(q[2], q[6]),
                                       pack_half(q[3] * 0.0625f, q[7] * 0.0625f));
            *reinterpret_cast<uint4 *>(smem + L::kQ + t * L::kTile + at / 8 * 16384 + r * 128 + ((at % 8 ^ (r & 7)) << 4)) = z;
            if (at == 0)
              *reinterpret_cast<float2 *>(row_of + r) =
                  make_float2(sum, fmaxf(fabsf(sl2) * __uint_as_float(static_cast<uint32_t>(ef - 14) << 23), 1.17549435e-38f));
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive(q_full(t));
      }
      __syncwarp();
      // From here on a thread has the columns of its place among four lanes, of four rows: a key's scale and zero are
      // then read once for four rows, where a thread for each row would have every warp read them all.
      float fsum[4], funit[4], fm[4], fl[4], top[4];
      bool pending = false;  // a row's maximum has grown, and the sums are to follow before the next step's weights
      int32_t flo[4], fhi[4];
      int32_t all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 x = row_of[(warp & 3) * 32 + 8 * e + (lane >> 2)];
        fsum[e] = x.x * x.y;
        funit[e] = x.y;
        flo[e] = __float_as_int(x.z);
        fhi[e] = __float_as_int(x.w);
        fm[e] = top[e] = -INFINITY;
        fl[e] = 0.0f;
        all_lo = max(all_lo, flo[e]);
        all_hi = min(all_hi, fhi[e]);
      }
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        all_lo = max(all_lo, __shfl_xor_sync(0xffffffffu, all_lo, o));
        all_hi = min(all_hi, __shfl_xor_sync(0xffffffffu, all_hi, o));
      }

      for (int j = 0; j < steps; ++j, ++c) {
        const int buf = c & 3;
        ok = all_wait(s_full(t), n_s & 1);
        ++n_s;
        tc_after();
        const uint4 *par = reinterpret_cast<const uint4 *>(smem + L::kPar + buf * kTok * 16);
        const int32_t tok0 = tok_at + j * kTok;
        const bool every = tok0 >= all_lo && tok0 + kTok <= all_hi;
        // S is taken in eighths of 16 keys.  x[4 h + 2 i + e]: columns 8 i .. of row 2 h + e; what a weight times its value is,
        // as a power of two, in place of their products.
        auto load = [&](uint64_t *x, int k) {
          tm_load_frag2(s_at + 16 * k, reinterpret_cast<uint32_t *>(x));
          tm_load_frag2(s_at + (16u << 16) + 16 * k, reinterpret_cast<uint32_t *>(x) + 8);
        };
        auto landed = [](uint64_t *x) { tm_wait16(reinterpret_cast<uint32_t *>(x)); };
        auto scores = [&](auto all, uint64_t *x, int k) {  // all: every row sees every key
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int at = 2 * (8 * k + 4 * i + (lane & 3));
            const uint4 p = par[at];
            const uint2 q = *reinterpret_cast<const uint2 *>(par + at + 1);
            F2 s, z, ve;
            s.u[0] = p.x, s.u[1] = p.y, z.u[0] = p.z, z.u[1] = p.w, ve.u[0] = q.x, ve.u[1] = q.y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint64_t &y = x[4 * (e >> 1) + 2 * i + (e & 1)];
              y = fma2(mul2(s.v, two(funit[e], funit[e])), y, fma2(z.v, two(fsum[e], fsum[e]), ve.v));
              if (!decltype(all)::value) {
                const int tok = tok0 + 16 * k + 8 * i + 2 * (lane & 3);
                F2 v;
                v.v = y;
                if (tok < flo[e] || tok >= fhi[e]) v.f[0] = -INFINITY;
                if (tok + 1 < flo[e] || tok + 1 >= fhi[e]) v.f[1] = -INFINITY;
                y = v.v;
              }
            }
          }
        };
        auto larger = [&](const uint64_t *x) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              F2 y;
              y.v = x[4 * (e >> 1) + 2 * i + (e & 1)];
              asm("max.f32 %0, %0, %1, %2;" : "+f"(top[e]) : "f"(y.f[0]), "f"(y.f[1]));
            }
        };
        auto join_top = [&]() {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 1));
            top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 2));
          }
        };
        // the sums so far to the maxima in top, where larger: the product before has to be done
        auto rescale = [&]() {
          if (j > 0 && !all_wait(o_full(t), (n_o - 1) & 1)) failed = true;
          tc_after();
          float f[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float mn = fmaxf(fm[e], top[e]);
            f[e] = mn == -INFINITY ? 1.0f : ex2(fm[e] - mn);
            fl[e] *= f[e];
            fm[e] = mn;
          }
#pragma unroll 1
          for (int k = 0; k < 2 * D; k += 32) {
            uint32_t o[16];
            const int h = k >= D;
            const uint32_t at = o_at + (h ? (16u << 16) + k - D : k);
            tm_load_frag(at, o);
            tm_wait16(o);
            const float g0 = h ? f[2] : f[0], g1 = h ? f[3] : f[1];
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * (e >> 1 & 1 ? g1 : g0));
            tm_store_frag(at, o);
          }
        };
        if (ok && j == 0) {
          // the first step finds its maxima before its weights
#pragma unroll 1
          for (int k = 0; k < 8; ++k) {
            uint64_t x[8];
            load(x, k);
            landed(x);
            scores(No{}, x, k);
            larger(x);
          }
          join_top();
#pragma unroll
          for (int e = 0; e < 4; ++e) fm[e] = top[e];
        } else if (ok && pending) {
          rescale();
        }
        // Weights against the maxima so far, in the place of the scores that have been read.  A row that has grown past what
        // a half can hold, and with it the whole tile, has its scores computed again.
        uint64_t total[4];
        auto weigh = [&](auto all) {
          float ref[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ref[e] = kBias - (fm[e] == -INFINITY ? 0.0f : fm[e]);
            total[e] = 0;
            top[e] = -INFINITY;
          }
          // a loop of one quarter: the warps of all kinds together have to fit the instruction cache
#pragma unroll 1
          for (int k = 0; k < 8; ++k) {
            uint64_t z[8];
            load(z, k);
            landed(z);
            scores(all, z, k);
            larger(z);
            uint32_t p[8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint64_t weight = reinterpret_cast<const uint64_t *>(par)[4 * (8 * k + 4 * i + (lane & 3)) + 3];  // without the value
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int at = 4 * (e >> 1) + 2 * i + (e & 1);
                F2 v;
                v.v = add2(z[at], two(ref[e], ref[e]));
                v.f[0] = ex2(v.f[0]);
                v.f[1] = ex2(v.f[1]);
                total[e] = fma2(v.v, weight, total[e]);
                p[at] = pack_half(v.f[0], v.f[1]);
              }
            }
            tm_store_halves(s_at + 8 * k, p);
            tm_store_halves(s_at + (16u << 16) + 8 * k, p + 4);
          }
          join_top();
        };
        if (ok) {
          if (every)
            weigh(Yes{});
          else
            weigh(No{});
        }
        bool again = false;
        pending = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          again |= top[e] > fm[e] + kMost || (fm[e] == -INFINITY && top[e] > fm[e]);
          pending |= top[e] > fm[e] + kSlack;
        }
        pending = __any_sync(0xffffffffu, pending);
        if (tile_any(1 + t, again || !ok || failed)) {  // every warp of the tile comes here once for every wait on s_full
          ok = !tile_any(1 + t, !ok || failed);
          if (!ok) break;
          rescale();
          if (lane == 0 && (warp & 3) == 0) reinterpret_cast<volatile int *>(smem + L::kAgain)[t] = 1;
          pending = false;
          tm_wait_store();  // the weights have to be there before the next scores take their place
          tc_before();
          __syncwarp();
          if (lane == 0) bar_arrive(p_full(t));
          --j, --c;  // the same step
          continue;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          F2 y;
          y.v = total[e];
          fl[e] += y.f[0] + y.f[1];
        }
        // A value that is not finite is left out of the product.  A row that sees one is marked, in the place of what a score is to be
        // multiplied by, which is in registers: its output is NaN, its sum of weights is not.
        const uint4 nans = reinterpret_cast<const uint4 *>(smem + L::kNan)[buf];
        if (nans.x | nans.y | nans.z | nans.w) {
#pragma unroll 1
          for (int col = 0; col < kTok; ++col) {
            const uint32_t word = col < 32 ? nans.x : col < 64 ? nans.y : col < 96 ? nans.z : nans.w;
            if (!(word >> (col & 31) & 1u)) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (tok0 + col >= flo[e] && tok0 + col < fhi[e]) row_of[(warp & 3) * 32 + 8 * e + (lane >> 2)].y = NAN;
          }
        }
        tm_wait_store();
        tc_before();
        __syncwarp();
        if (lane == 0) bar_arrive(p_full(t));
        ++n_o;
      }
      if (!ok) break;

      // ---- the item's rows, or this block's part of them; a row a thread again
      const int64_t i = w.q0 + (there ? R / group : 0);
      const int hq = w.h * group + (there ? R % group : 0);
      float m = -INFINITY, l = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        fl[e] += __shfl_xor_sync(0xffffffffu, fl[e], 1);
        fl[e] += __shfl_xor_sync(0xffffffffu, fl[e], 2);
        const float x = __shfl_sync(0xffffffffu, fm[e], (lane & 7) * 4), y = __shfl_sync(0xffffffffu, fl[e], (lane & 7) * 4);
        if (lane >> 3 == e) m = x, l = y;
      }
      const bool whole = w.whole;
      const uint32_t id = w.id;
      if (steps > 0) {
        ok = all_wait(o_full(t), (n_o - 1) & 1);
        if (!ok) continue;  // to the vote
        tc_after();
      }
      __syncwarp();
      const bool nan = steps > 0 && isnan(row_of[row].y);
      const float f = nan ? NAN : whole ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;
      T *dst = static_cast<T *>(a.out) + i * a.o_row + hq * a.o_head;
      const int at = t * 128 + row;
      float *part = a.many_parts + (static_cast<int64_t>(me) * 2 + (id < u0 ? 0 : 1)) * L::kPart;
#pragma unroll 1
      for (int k = 0; k < D; k += 16) {
        uint32_t o[16];
        if (steps > 0) {
          tm_load16(o_at + k, o);
          tm_wait16(o);
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = 0;
        }
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = f == 0.0f ? 0.0f : __uint_as_float(o[e]) * f;
        if (!whole) {
#pragma unroll
          for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4 *>(part + at * D + k + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        } else if (there) {
          T y[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) y[e] = Cvt<T>::from(v[e]);
          if (a.wide) {
#pragma unroll
            for (int e = 0; e < 16; e += 8) *reinterpret_cast<uint4 *>(dst + k + e) = *reinterpret_cast<const uint4 *>(y + e);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) dst[k + e] = y[e];
          }
        }
      }
      if (!whole) {
        part[kRows * D + at] = m - kBias;
        part[kRows * D + kRows + at] = l;
        if (tid == 0 && id >= u0) a.many_open[me] = {w.q0, id, w.tiles, w.rows, w.h, w.rt};
      } else if (there && a.lse) {
        a.lse[i * a.Hq + hq] = l == 0.0f ? -INFINITY : (m - kBias + log2f(l)) * 0.6931471805599453f;
      }
      tc_before();  // the sums have been read, before the next item's first product
      __syncwarp();
      if (lane == 0) bar_arrive(seg_free(n_seg % kSegs));
      ++n_seg;
    }
    if (!ok && lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
  } else if (warp < 12) {
    // ======================================================================== values
    const int w4 = warp - 8;
    uint32_t c = 0;
    bool ok = true;
    while (hear(ok)) {
      const int steps = told().steps, tok_at = told().token, hi = told().hi;
      for (int j = 0; j < steps; ++j, ++c) {
        ok = all_wait(step_full(place), round);
        if (!ok) break;
        const int32_t tok0 = tok_at + j * kTok;
        auto record = [&](int g) -> const uint8_t * { return smem + L::kRingAt + place * L::kStep + g * kv4_group_bytes(D); };
        // ---- scales and zeros of the lane's 4 tokens, two side by side, against each value's own power of two; those left out are zero
        const uint4 v4 = *reinterpret_cast<const uint4 *>(record(lane >> 2) + 16 * D + 64 + (lane & 3) * 16);
        const uint32_t vp[4] = {v4.x, v4.y, v4.z, v4.w};
        uint32_t vs[2], vz[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float2 p0 = kv4_param(vp[2 * e]), p1 = kv4_param(vp[2 * e + 1]);
          const int32_t tok = tok0 + 4 * lane + 2 * e;
          if (tok >= hi || !value_finite(p0)) p0 = make_float2(0.0f, 0.0f);
          if (tok + 1 >= hi || !value_finite(p1)) p1 = make_float2(0.0f, 0.0f);
          const float d0 = __uint_as_float(static_cast<uint32_t>(127 - value_exponent(p0)) << 23), d1 = __uint_as_float(static_cast<uint32_t>(127 - value_exponent(p1)) << 23);
          vs[e] = pack_half(p0.x * d0, p1.x * d1);
          vz[e] = pack_half(p0.y * d0, p1.y * d1);
        }
        ok = all_wait(v_free, (c & 1) ^ 1);
        if (!ok) break;
        uint8_t *V = smem + L::kV;
#pragma unroll 1
        for (int g = w4; g < kStepGroups; g += 4) {
          const uint8_t *rec = record(g);
          // ---- values: a lane has 4 channels of 8 tokens, which are 16 bytes of each channel's row
#pragma unroll 1
          for (int hh = 0; hh < (D == 128 ? 2 : 1); ++hh) {
            const int h = D == 128 ? hh : lane >> 4;
            const int cg = D == 128 ? lane >> 2 : (lane >> 1) & 7, b = D == 128 ? lane & 3 : lane & 1;
            const int f = D == 128 ? (cg >> 1) & 3 : ((cg >> 2) + 2 * h) & 3;  // the order of the four loads, for their banks
            uint32_t v[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] = *reinterpret_cast<const uint32_t *>(rec + 8 * D + (((h * 8 + cg) * 4 + (t ^ f)) * (D / 32) + b) * 4);
            if (f & 1) {
              uint32_t y = v[0];
              v[0] = v[1], v[1] = y;
              y = v[2], v[2] = v[3], v[3] = y;
            }
            if (f & 2) {
              uint32_t y = v[0];
              v[0] = v[2], v[2] = y;
              y = v[1], v[1] = v[3], v[3] = y;
            }
            const int turn = D == 128 ? b >> 1 | (cg & 1) << 1 : cg & 3;  // the order of the lane's channels, so that eight lanes write to eight different banks
            uint4 out[4];
            const __half2 off = __float2half2_rn(1024.0f);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const uint32_t su = __shfl_sync(0xffffffffu, vs[t & 1], 4 * g + 2 * h + (t >> 1)), zu = __shfl_sync(0xffffffffu, vz[t & 1], 4 * g + 2 * h + (t >> 1));
              const __half2 s = *reinterpret_cast<const __half2 *>(&su), z = *reinterpret_cast<const __half2 *>(&zu);
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const uint32_t code = ((v[t] >> (4 * (r ^ turn))) & 0x000f000fu) | 0x64006400u;  // 1024 + code
                const __half2 y = __hfma2(__hsub2(*reinterpret_cast<const __half2 *>(&code), off), s, z);
                reinterpret_cast<uint32_t *>(&out[r])[t] = *reinterpret_cast<const uint32_t *>(&y);
              }
            }
            const int t8 = 2 * g + h;  // 8 tokens of the step's 128
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int ch = cg * (D / 8) + 4 * b + (r ^ turn);
              *reinterpret_cast<uint4 *>(V + t8 / 8 * (D * 128) + ch * 128 + ((t8 % 8 ^ (ch & 7)) << 4)) = out[r];
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive(step_free(place)), bar_arrive(v_full);
        ring_on();
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) bar_arrive(seg_free(n_seg % kSegs));
      ++n_seg;
    }
    if (!ok && lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
  } else {
    if (warp == 12 && lane == 0) {
      // ====================================================================== products
      constexpr uint32_t kQK = idesc_of(kTok), kPV = idesc_of(D);
      uint32_t c = 0, n_q[2] = {0, 0}, n_p[2] = {0, 0};
      bool ok = true;
      // Tensor memory is taken whole, so it starts at 0.  The loops are short ones for the instruction cache's sake, which they
      // share with the softmax: straight-line code of its own for each tile and buffer 817 us (the chunks above), eight products
      // in a row 806, four 796, two 782, one 801.
      auto scores = [&](int t, int buf) {
        const uint32_t q = rows_desc(base + L::kQ + t * L::kTile), k_at = rows_desc(base + L::kK + buf * L::kTile);
#pragma unroll 2
        for (int k = 0; k < D / 16; ++k) {
          constexpr int kStep = 32 / 16, kBlock = 16384 / 16;  // of a descriptor's address
          const uint32_t off = k / 4 * kBlock + k % 4 * kStep;
          mma_ss(t * 128, q + off, k_at + off, kQK, k > 0);
        }
        tc_commit(s_full(t));
        bar_arrive(s_full(t));  // passes on what this thread has seen of the step: the keys' scales and zeros
      };
      auto sums = [&](int t, bool more) {
#pragma unroll 2
        for (int k = 0; k < kTok / 16; ++k)
          mma_ts(256 + t * 128, t * 128 + 8 * k, rows_desc(base + L::kV) + (k / 4 * (D * 8) + k % 4 * 2), kPV, more || k > 0);
        tc_commit(o_full(t));
      };
      while (hear_alone(ok)) {
        const int steps = told().steps, tiles = told().second ? 2 : 1;
        done();
        if (steps == 0) continue;
        for (int t = 0; t < tiles && ok; ++t) ok = one_wait(q_full(t), n_q[t]++ & 1);
        ok = ok && one_wait(k_full(c & 1), c >> 1 & 1);
        if (!ok) break;
        tc_after();
        for (int t = 0; t < tiles; ++t) scores(t, c & 1);
        for (int j = 0; j < steps && ok; ++j, ++c) {
          const int buf = c & 1;
          for (int t = 0; t < tiles; ++t) {
            for (;;) {
              ok = one_wait(p_full(t), n_p[t]++ & 1);
              if (!ok) break;
              tc_after();
              volatile int *again = reinterpret_cast<volatile int *>(smem + L::kAgain) + t;
              if (!*again) break;
              *again = 0;
              scores(t, buf);
            }
            if (!ok) break;
            if (t == tiles - 1) tc_commit(k_free(buf));  // nobody wants these scores again
            ok = t > 0 || one_wait(v_full, c & 1);
            if (!ok) break;
            tc_after();
            sums(t, j > 0);
            if (t == tiles - 1) tc_commit(v_free);
            if (j + 1 < steps) {
              if (t == 0) {
                ok = one_wait(k_full(buf ^ 1), (c + 1) >> 1 & 1);
                if (!ok) break;
                tc_after();
              }
              scores(t, buf ^ 1);
            }
          }
        }
      }
      if (!ok) flag_error(a.status, MAPS_E_TIMEOUT);
    } else if (warp == 13) {
      // ====================================================================== loads: a group a lane
      bool ok = true;
      while (hear(ok)) {
        const int steps = told().steps, tok_at = told().token, hi = told().hi, head_groups = told().h * a.block_groups;
        const int32_t *table = a.table + told().b * a.max_blocks;
        __syncwarp();
        if (lane == 0) bar_arrive(seg_free(n_seg % kSegs));
        ++n_seg;
        for (int j = 0; j < steps && ok; ++j) {
          if (lane < kStepGroups) {
            const int32_t tok = tok_at + j * kTok + lane * kGroup;
            bool load = tok < hi;
            int64_t at = 0;
            if (load) {
              const int32_t grp = tok / kGroup, page = a.block_shift >= 0 ? grp >> a.block_shift : grp / a.block_groups;
              const int32_t block = table[page];
              if (block < 0 || block >= a.n_blocks) {
                flag_error(a.status, MAPS_E_RANGE);
                load = false;
              }
              at = block * a.block_bytes + (head_groups + grp - page * a.block_groups) * static_cast<int64_t>(kv4_group_bytes(D));
            }
            ok = one_wait(step_free(place), round ^ 1u);
            if (ok) {
              bar_expect(step_full(place), load ? kv4_group_bytes(D) : 0);
              if (load) bulk_load(base + L::kRingAt + place * L::kStep + lane * kv4_group_bytes(D), a.cache + at, kv4_group_bytes(D), step_full(place));
            }
          }
          ok = __all_sync(0xffffffffu, ok);
          ring_on();
        }
        if (!ok) break;
      }
      if (!ok) {
        if (lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
        // let what is under way land: a step's barrier is over once all of it has
        for (int i = 0; i < kRing; ++i) (void)all_wait(step_full(i), 0), (void)all_wait(step_full(i), 1);
      }
    } else if (warp == 15) {
      // ====================================================================== keys
      uint32_t c = 0;
      bool ok = true;
      while (hear(ok)) {
        const int steps = told().steps, tok_at = told().token, hi = told().hi;
        for (int j = 0; j < steps; ++j, ++c) {
          const int buf = c & 1;
          ok = all_wait(step_full(place), round) && all_wait(k_free(buf), (c >> 1 & 1) ^ 1);
          if (!ok) break;
          const int32_t tok0 = tok_at + j * kTok;
          auto record = [&](int g) -> const uint8_t * { return smem + L::kRingAt + place * L::kStep + g * kv4_group_bytes(D); };
          uint8_t *K = smem + L::kK + buf * L::kTile;
#pragma unroll 1
          for (int g = 0; g < kStepGroups; ++g) {
            const uint8_t *rec = record(g);
            // ---- keys: a token's row, 8 channels to 16 bytes
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const int tr = half * 8 + (lane >> 2), t = lane & 3, row = g * kGroup + tr;
              uint32_t words[D / 32];
              if (D == 64)
                *reinterpret_cast<uint2 *>(words) = *reinterpret_cast<const uint2 *>(rec + tr * (D / 2) + t * (D / 8));
              else
                *reinterpret_cast<uint4 *>(words) = *reinterpret_cast<const uint4 *>(rec + tr * (D / 2) + t * (D / 8));
#pragma unroll
              for (int x = 0; x < D / 32; ++x) {
                // lanes of the second 64 channels take their words in another order, so that eight lanes write to eight different banks
                const bool other = D == 128 && (t & 2);
                const int y = other ? x ^ 2 : x;
                const Codes z = codes_of(D == 128 && other ? words[(x ^ 2) % (D / 32)] : words[x]);
                const int chunk = t * (D / 32) + y;
                *reinterpret_cast<uint4 *>(K + chunk / 8 * 16384 + row * 128 + ((chunk % 8 ^ (row & 7)) << 4)) = make_uint4(z.x[0], z.x[1], z.x[2], z.x[3]);
              }
            }
          }
          // ---- the values' powers of two, and those that are not finite, from 4 tokens a lane
          const uint4 v4 = *reinterpret_cast<const uint4 *>(record(lane >> 2) + 16 * D + 64 + (lane & 3) * 16);
          const uint32_t vp[4] = {v4.x, v4.y, v4.z, v4.w};
          uint32_t bad = 0;
          float ve[4], weight[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 p = kv4_param(vp[e]);
            const bool there = tok0 + 4 * lane + e < hi;
            const bool finite = value_finite(p);
            if (there && !finite) bad |= 1u << e;
            const int E = there && finite ? value_exponent(p) : -60;
            ve[e] = static_cast<float>(E);
            weight[e] = __uint_as_float(static_cast<uint32_t>(127 - E) << 23);
          }
          bad <<= (lane & 7) * 4;
#pragma unroll
          for (int o = 4; o > 0; o >>= 1) bad |= __shfl_xor_sync(0xffffffffu, bad, o);
          if ((lane & 7) == 0) reinterpret_cast<uint32_t *>(smem + L::kNan)[4 * (c & 3) + (lane >> 3)] = bad;
          // ---- keys' scales and zeros, two tokens side by side
          {
            const uint4 k4 = *reinterpret_cast<const uint4 *>(record(lane >> 2) + 16 * D + (lane & 3) * 16);
            const uint32_t kp[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              float2 p0 = kv4_param(kp[e]), p1 = kv4_param(kp[e + 1]);
              if (tok0 + 4 * lane + e >= hi) p0 = make_float2(0.0f, 0.0f);
              if (tok0 + 4 * lane + e + 1 >= hi) p1 = make_float2(0.0f, 0.0f);
              float4 *par = reinterpret_cast<float4 *>(smem + L::kPar + (c & 3) * kTok * 16) + 4 * lane + e;
              par[0] = make_float4(p0.x * (k_sign * kEven), p1.x * (k_sign * kEven), p0.y * k_sign, p1.y * k_sign);
              par[1] = make_float4(ve[e], ve[e + 1], weight[e], weight[e + 1]);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            bar_arrive(step_free(place));
            if (static_cast<int>(me) != c_withheld) bar_arrive(k_full(buf));
          }
          ring_on();
        }
        if (!ok) break;
        __syncwarp();
        if (lane == 0) bar_arrive(seg_free(n_seg % kSegs));
        ++n_seg;
      }
      if (!ok && lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
    } else if (warp == 14 && lane == 0) {
      // ====================================================================== the block's items
      bool ok = true;
      auto tell = [&](const Seg &x) {
        ok = one_wait(seg_free(n_seg % kSegs), (n_seg / kSegs & 1) ^ 1);
        if (!ok) return;
        reinterpret_cast<Seg *>(smem + L::kSegAt)[n_seg % kSegs] = x;
        bar_arrive(seg_full(n_seg++ % kSegs));
      };
      Seg x = {};
      if (u0 < u1) {
        MReq r = s_start.r;
        int32_t lo, hi;
        uint32_t all = 0, rest = s_start.rest;
        for (int t = 0; t < r.row_tiles; ++t) all += span(a, r, t, lo, hi);
        int b = s_start.b, h = static_cast<int>(rest / all), rt = 0, tiles;
        rest -= static_cast<uint32_t>(h) * all;
        while (rest >= static_cast<uint32_t>(tiles = span(a, r, rt, lo, hi))) rest -= tiles, ++rt;
        int tile = static_cast<int>(rest);
        for (uint32_t u = u0; ok;) {
          const int end = static_cast<int>(min(static_cast<uint32_t>(tiles), tile + (u1 - u)));  // of the block's units of the item
          x.q0 = r.q0, x.n = r.n, x.n_q = r.n_q, x.rows = r.n_q * group;
          x.steps = max(end - max(tile, kItemUnits), 0);
          x.token = lo + (max(tile, kItemUnits) - kItemUnits) * kTok, x.hi = hi;
          x.b = b, x.h = h, x.rt = rt;
          x.second = rt * kRows + 128 < x.rows;
          x.whole = tile == 0 && end == tiles;
          x.id = u - tile, x.tiles = tiles;
          tell(x);
          u += end - tile;
          if (u >= u1) break;
          tile = 0;
          if (++rt == r.row_tiles) {
            rt = 0;
            if (++h == a.Hkv) {
              h = 0;
              do r = many_request(a, ++b);
              while (r.row_tiles == 0);
            }
          }
          tiles = span(a, r, rt, lo, hi);
        }
      }
      x.steps = -1;
      if (ok) tell(x);
      if (!ok) flag_error(a.status, MAPS_E_TIMEOUT);
    }
    __syncwarp();
  }
  tc_before();
  __syncthreads();
  if (warp == 12) {
    tc_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// ---------------------------------------------------------------------------- the items that cross blocks
constexpr int kJoinRows = 64;  // of a block

template <class T, int D>
__global__ void __launch_bounds__(512) attn_many_join_kernel(const AttnArgs a, uint32_t blocks) {
  pdl_prologue();
  constexpr int kPart = Lay<D>::kPart;
  const uint32_t f = blockIdx.x;
  const Part item = a.many_open[f];
  if (item.tiles == 0) return;
  const Deal deal(*a.many_units, blocks);
  const uint32_t e = deal.worker(item.id + item.tiles - 1);
  const int group = a.Hq / a.Hkv;
  for (int x = 4 * threadIdx.x; x < kJoinRows * D; x += 4 * 512) {
    const int at = blockIdx.y * kJoinRows + x / D, d = x % D, R = item.rt * kRows + at;
    if (R >= item.rows) continue;
    float M = -INFINITY, den = 0.0f;
    float4 num = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t c = f; c <= e; ++c) {
      const float *p = a.many_parts + (static_cast<int64_t>(c) * 2 + (c == f)) * kPart;
      const float4 v = *reinterpret_cast<const float4 *>(p + at * D + d);
      const float mk = p[kRows * D + at], lk = p[kRows * D + kRows + at], top = fmaxf(M, mk);
      const float g = top == -INFINITY ? 1.0f : ex2(M - top), k = top == -INFINITY ? 0.0f : ex2(mk - top);
      M = top;
      num.x = fmaf(k, v.x, num.x * g), num.y = fmaf(k, v.y, num.y * g), num.z = fmaf(k, v.z, num.z * g), num.w = fmaf(k, v.w, num.w * g);
      den = fmaf(k, lk, den * g);
    }
    const int64_t i = item.q0 + R / group;
    const int hq = item.h * group + R % group;
    const float inv = den == 0.0f ? 0.0f : 1.0f / den;
    T *dst = static_cast<T *>(a.out) + i * a.o_row + hq * a.o_head + d;
    const T y[4] = {Cvt<T>::from(num.x * inv), Cvt<T>::from(num.y * inv), Cvt<T>::from(num.z * inv), Cvt<T>::from(num.w * inv)};
    if (a.wide) {
      *reinterpret_cast<uint2 *>(dst) = *reinterpret_cast<const uint2 *>(y);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) dst[k] = y[k];
    }
    if (d == 0 && a.lse) a.lse[i * a.Hq + hq] = den == 0.0f ? -INFINITY : (M + log2f(den)) * 0.6931471805599453f;
  }
}

template <class T, int D>
int launch(const AttnArgs &a, cudaStream_t s) {
  const unsigned grid = static_cast<unsigned>(attn_grid());
  const size_t smem = Lay<D>::kBytes + 1024;
  constexpr auto kernel = attn_many_kernel<T, D>;
  MAPS_TRY(allow_smem<kernel>(smem));
  if (a.B > kMaxLocalB) launch_pdl(attn_many_plan_kernel, 1, 1024, 0, s, a, grid);
  launch_pdl(kernel, grid, kThreads, smem, s, a);
  launch_pdl(attn_many_join_kernel<T, D>, dim3(grid, kRows / kJoinRows), 512, 0, s, a, grid);
  return launch_ok();
}

}  // namespace

bool attn_many_dim(int D) { return D == 64 || D == 128; }

void attn_many_carve(Carve &c, AttnArgs &a, int32_t B, int D) {
  const size_t grid = static_cast<size_t>(attn_grid()), part = D == 64 ? Lay<64>::kPart : Lay<128>::kPart;
  a.many_starts = c.take<ManyStart>(B > kMaxLocalB ? grid : 0);
  a.many_units = c.take<uint32_t>(1);
  a.many_open = c.take<Part>(grid);
  a.many_parts = c.take<float>(grid * 2 * part);
}

int attn_many(int32_t dtype, int D, const AttnArgs &a, cudaStream_t s) {
  if (dtype == MAPS_BF16) return D == 64 ? launch<__nv_bfloat16, 64>(a, s) : launch<__nv_bfloat16, 128>(a, s);
  return D == 64 ? launch<__half, 64>(a, s) : launch<__half, 128>(a, s);
}

}  // namespace maps

extern "C" int maps_test_attention_withhold(int32_t block, uint32_t spin_limit) {
  using namespace maps;
  const uint32_t tries = spin_limit == 0 ? kTries : spin_limit;
  MAPS_TRY(cuda_ok(cudaMemcpyToSymbol(c_withheld, &block, sizeof(block))));
  MAPS_TRY(cuda_ok(cudaMemcpyToSymbol(c_tries, &tries, sizeof(tries))));
  return attn_lists_withhold(block, tries);
}
