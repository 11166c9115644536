// kv4_attention_many.cu -- attention over the paged 4-bit KV cache, form for many queries a request
// (chunks of prompts): the products dominate, so they run on tcgen05.
//
// A block takes 256 query rows (queries x heads of one KV head) as two tiles of 128 and passes over the
// keys they see in steps of 128.  Per step and tile, S = Q K^T and O += P V are 128 x 128 x D products
// with their results in tensor memory; P replaces S there, as halves, and is the second product's operand.
//
//   warps 0-3, 4-7   softmax of a tile, a row a thread: S from tensor memory, running maximum and sum, P back;
//                    they rescale O when the maximum has grown by more than 2^8, and write it out at the end
//   warps 8-11       the cache's codes to operands in shared memory, two steps deep
//   warp 12          issues the products; the two tiles alternate, so that one's softmax runs beside the other's products
//   warp 13          bulk copies of the cache's records, a ring of groups ahead
//
// Keys enter the first product as bare codes (subnormal halves, exact; the odd pairs' factor of 16 is taken
// off in Q) and s, z come in with the row's sum of Q in 32 bits, as in the form for few queries: two packed
// operations for two scores.  Values become halves of their own: v 2^-E with a power of two common to the step's
// 128 tokens, so any magnitude fits and a value keeps 11 bits; the running sum carries its own exponent.
// Both would cost a score more work the other way round: a value's scale on the weights takes three operations
// a score and eight warps' registers, on the values two for two of them.
//
// Bound.  128 x 128 scores cost the tensor cores 1,024 cycles at D = 128, and the softmax warps about as many
// issue slots with packed arithmetic; shared memory is next, since each product reads its operands at full rate.
//
// Split.  As in the other form, a call's steps are dealt out to the blocks in equal runs, whatever the
// lengths; what a run begins or ends inside of is left as parts, which a second kernel joins.
#include "kv4_attention.cuh"

namespace maps {
namespace {

constexpr int kThreads = 512;
constexpr int kRows = 256, kTok = 128, kStepGroups = kTok / kGroup;
constexpr int kLaunchRegs = 128, kSoftmaxRegs = 184, kOperandRegs = 88, kOtherRegs = 56;  // of a thread, by warpgroup
constexpr int kRing = 14;  // groups of the cache under way or waiting

struct MReq {
  int64_t q0;
  int32_t n, n_q, row_tiles;
};

__device__ __forceinline__ MReq many_request(const AttnArgs &a, int b) {
  MReq r;
  const int64_t q0 = a.off[b], q1 = a.off[b + 1];
  int64_t m = q1 - q0;
  int32_t n = a.len[b];
  if (n < 0 || n > a.max_blocks * a.S || q0 < 0 || m < 0 || q1 > a.T) n = 0, m = 0;  // the other form has reported it
  const int64_t rows = m * (a.Hq / a.Hkv);
  r.q0 = q0;
  r.n = n;
  r.n_q = static_cast<int32_t>(m);
  r.row_tiles = n > 0 && rows > a.few_rows ? static_cast<int32_t>((rows + kRows - 1) / kRows) : 0;
  return r;
}

// The tokens lo .. hi - 1 that a row tile's queries see between them (lo to 16), and its units: one for itself, and its steps.
__device__ __forceinline__ int span(const AttnArgs &a, const MReq &r, int rt, int32_t &lo, int32_t &hi) {
  const int group = a.Hq / a.Hkv;
  const int first = rt * kRows / group, last = min(r.n_q - 1, (rt * kRows + kRows - 1) / group);
  const int64_t shift = static_cast<int64_t>(r.n) - r.n_q;
  hi = a.causal ? static_cast<int32_t>(max(int64_t(0), shift + last + 1)) : r.n;
  const int64_t from = a.window > 0 ? shift + first - a.window + 1 : 0;
  lo = from > 0 ? static_cast<int32_t>(min(from, static_cast<int64_t>(hi))) / kGroup * kGroup : 0;
  return 1 + (hi > lo ? (hi - lo + kTok - 1) / kTok : 0);
}

struct ManyStart {
  MReq r;
  int32_t b;
  uint32_t rest;
};

// A block's run of units, item by item.
struct Walk {
  MReq r;
  int32_t b, h, rt, tile, tiles, lo, hi;
  uint32_t u, u1;
  __device__ __forceinline__ Walk(const AttnArgs &a, const ManyStart &s, uint32_t u0, uint32_t u1) : r(s.r), b(s.b), h(0), rt(0), tile(0), tiles(0), lo(0), hi(0), u(u0), u1(u1) {
    if (u >= u1) return;
    uint32_t all = 0;
    for (int t = 0; t < r.row_tiles; ++t) all += span(a, r, t, lo, hi);
    h = static_cast<int32_t>(s.rest / all);
    uint32_t rest = s.rest - static_cast<uint32_t>(h) * all;
    while (rest >= static_cast<uint32_t>(tiles = span(a, r, rt, lo, hi))) rest -= tiles, ++rt;
    tile = static_cast<int32_t>(rest);
  }
  __device__ __forceinline__ bool more() const { return u < u1; }
  __device__ __forceinline__ int end() const { return static_cast<int>(min(static_cast<uint32_t>(tiles), tile + (u1 - u))); }  // of this run's units of the item
  __device__ __forceinline__ int first_step() const { return max(tile, 1) - 1; }
  __device__ __forceinline__ int steps() const { return end() - max(tile, 1); }
  __device__ __forceinline__ int rows(const AttnArgs &a) const { return r.n_q * (a.Hq / a.Hkv); }
  __device__ __forceinline__ bool second(const AttnArgs &a) const { return rt * kRows + 128 < rows(a); }  // whether the second tile has rows
  __device__ __forceinline__ void next(const AttnArgs &a) {
    u += end() - tile;
    if (u >= u1) return;
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
};

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
  const uint32_t U = many_plan<1024>(a, blocks, 0, blocks, [&](uint32_t w, const ManyStart &s) { static_cast<ManyStart *>(a.many_starts)[w] = s; });
  if (threadIdx.x == 0) *a.many_units = U;
}

// ---------------------------------------------------------------------------- tensor memory, products, packed arithmetic
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t A, uint64_t B, uint32_t idesc, uint32_t add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(A), "l"(B), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t A, uint64_t B, uint32_t idesc, uint32_t add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(A), "l"(B), "r"(idesc), "r"(add) : "memory");
}
// Descriptor of rows of 64 halves (128 bytes) in the 128-byte swizzle: 8 rows to 1,024 bytes.
__device__ __forceinline__ uint64_t rows_desc(uint32_t addr) {
  return static_cast<uint64_t>((addr >> 4) & 0x3fffu) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction: halves in, 32-bit sums, 128 rows, N columns, both operands along the depth.
__host__ __device__ constexpr uint32_t idesc_of(int N) { return (1u << 4) | (static_cast<uint32_t>(N / 8) << 17) | (8u << 24); }

#define MAPS_R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define MAPS_W8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
#define MAPS_32 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}"
__device__ __forceinline__ void tm_load32(uint32_t addr, uint32_t *x) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 " MAPS_32 ", [%32];" : MAPS_R8(x, 0), MAPS_R8(x, 8), MAPS_R8(x, 16), MAPS_R8(x, 24) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_store32(uint32_t addr, const uint32_t *x) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], " MAPS_32 ";" ::MAPS_W8(x, 0), MAPS_W8(x, 8), MAPS_W8(x, 16), MAPS_W8(x, 24), "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_load16(uint32_t addr, uint32_t *x) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];" : MAPS_R8(x, 0), MAPS_R8(x, 8) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t addr, const uint32_t *x) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::MAPS_W8(x, 0), MAPS_W8(x, 8), "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
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
  static constexpr int kQ = 0, kK = 2 * kTile, kV = 4 * kTile, kRingAt = 6 * kTile;
  static constexpr int kPar = kRingAt + kRing * kv4_group_bytes(D);  // [2][64] {scale, scale, zero, zero} of two keys
  static constexpr int kNan = kPar + 2 * kTok * 8;   // [2][4] bits: values held as NaN
  static constexpr int kExp = kNan + 32;             // [2] the step's exponent
  static constexpr int kBars = kExp + 16;
  static constexpr int kBytes = kBars + 8 * (2 * kRing + 12) + 16;
  static constexpr int kPart = kRows * D + 2 * kRows;  // floats of a part: sums, maxima, totals
};
static_assert(Lay<128>::kBytes + 1024 < 231 * 1024, "shared memory");
static_assert(Lay<128>::kBars % 8 == 0 && Lay<64>::kBars % 8 == 0 && Lay<128>::kPar % 16 == 0 && Lay<64>::kPar % 16 == 0, "alignment");

constexpr int kNoExp = -400;     // of a step without a value
constexpr float kSlack = 8.0f;   // powers of two that a weight may exceed 1 by before the sums are rescaled

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1) attn_many_kernel(const AttnArgs a) {
  using L = Lay<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ ManyStart s_start;
  __shared__ uint32_t s_tmem;
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t base = smem_u32(smem), bars = base + L::kBars;
  // barriers
  auto ring_full = [&](int i) { return bars + 8 * i; };
  auto ring_free = [&](int i) { return bars + 8 * (kRing + i); };
  const uint32_t b0 = bars + 16 * kRing;
  auto kv_full = [&](int i) { return b0 + 8 * i; };
  auto kv_free = [&](int i) { return b0 + 16 + 8 * i; };
  auto q_full = [&](int t) { return b0 + 32 + 8 * t; };
  auto s_full = [&](int t) { return b0 + 48 + 8 * t; };
  auto p_full = [&](int t) { return b0 + 64 + 8 * t; };
  auto o_full = [&](int t) { return b0 + 80 + 8 * t; };

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) bar_init(ring_full(i), 1), bar_init(ring_free(i), 4);
    for (int i = 0; i < 2; ++i) {
      bar_init(kv_full(i), 4), bar_init(kv_free(i), 1);
      bar_init(q_full(i), 4), bar_init(s_full(i), 1), bar_init(p_full(i), 4), bar_init(o_full(i), 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_prologue();
  uint32_t U;
  const uint32_t me = blockIdx.x;
  if (a.B <= kMaxLocalB) {
    U = many_plan<kThreads>(a, gridDim.x, me, me + 1, [&](uint32_t, const ManyStart &s) { s_start = s; });
    if (me == 0 && tid == 0) *a.many_units = U;  // for the kernel that joins
  } else {
    U = *a.many_units;
    if (me < U && tid == 0) s_start = static_cast<const ManyStart *>(a.many_starts)[me];
  }
  tc_before();
  __syncthreads();
  tc_after();
  const Deal deal(U, gridDim.x);
  const uint32_t u0 = deal.start(me), u1 = deal.start(me + 1);
  const uint32_t tmem = s_tmem;
  const int group = a.Hq / a.Hkv;
  const float sl2 = a.scale * 1.4426950408889634f, k_sign = a.scale < 0.0f ? -1.0f : 1.0f;
  if (tid == 0) a.many_open[me].tiles = 0;

  if (warp < 8) {
    // ======================================================================== softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;  // 32 lanes of tensor memory to a warp
    const uint32_t s_at = tmem + lanes + t * 128, o_at = tmem + lanes + 256 + t * 128;
    uint32_t c = 0, n_s = 0, n_o = 0;  // steps, scores and sums so far
    bool ok = true;
    for (Walk w(a, s_start, u0, u1); w.more() && ok; w.next(a)) {
      const int steps = w.steps(), rows = w.rows(a);
      if (t == 1 && !w.second(a)) {
        c += steps;
        continue;
      }
      const int R = w.rt * kRows + t * 128 + row;
      const bool there = R < rows;
      const int64_t i = w.r.q0 + (there ? R / group : 0);
      const int hq = w.h * group + (there ? R % group : 0);
      float m = -INFINITY, l = 0.0f, unit = 1.0f, sum = 0.0f;
      int run = kNoExp;
      int32_t row_lo = 0, row_hi = 0x7fffffff;  // a row that is none sees everything; nobody reads it
      if (there) {
        const int64_t pos = static_cast<int64_t>(w.r.n) - w.r.n_q + R / group;
        row_hi = pos < 0 ? 0 : a.causal ? static_cast<int32_t>(pos) + 1 : w.r.n;
        if (a.window > 0 && pos - a.window + 1 > 0) row_lo = static_cast<int32_t>(pos - a.window + 1);
      }
      if (steps > 0) {
        // ---- the row of Q, scaled by a power of two to fill half's range, to shared memory; 8 channels in the order of the codes
        const T *src = static_cast<const T *>(a.q) + i * a.q_row + hq * a.q_head;
        uint4 raw[D / 8];
        float top = 0.0f;
#pragma unroll
        for (int x = 0; x < D / 8; ++x) {
          raw[x] = make_uint4(0, 0, 0, 0);
          T *y = reinterpret_cast<T *>(&raw[x]);
          if (there) {
            if (a.wide) {
              raw[x] = *reinterpret_cast<const uint4 *>(src + 8 * x);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] = src[8 * x + e];
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(Cvt<T>::to(y[e])));
        }
        const int ef = min(max(static_cast<int>(__float_as_uint(top) >> 23), 20), 254);
        const float up = __uint_as_float(static_cast<uint32_t>(268 - ef) << 23);
        unit = fmaxf(fabsf(sl2) * __uint_as_float(static_cast<uint32_t>(ef - 14) << 23), 1.17549435e-38f);
#pragma unroll
        for (int x = 0; x < D / 8; ++x) {
          const T *y = reinterpret_cast<const T *>(&raw[x]);
          float q[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) q[e] = Cvt<T>::to(y[e]) * up, sum += q[e];
          const uint4 z = make_uint4(pack_half(q[0], q[4]), pack_half(q[1] * 0.0625f, q[5] * 0.0625f), pack_half(q[2], q[6]),
                                     pack_half(q[3] * 0.0625f, q[7] * 0.0625f));
          *reinterpret_cast<uint4 *>(smem + L::kQ + t * L::kTile + x / 8 * 16384 + row * 128 + ((x % 8 ^ (row & 7)) << 4)) = z;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive(q_full(t));
      }
      const uint64_t sum2 = two(sum, sum), unit2 = two(unit, unit);
      int32_t all_lo = row_lo, all_hi = row_hi;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        all_lo = max(all_lo, __shfl_xor_sync(0xffffffffu, all_lo, o));
        all_hi = min(all_hi, __shfl_xor_sync(0xffffffffu, all_hi, o));
      }

      for (int j = 0; j < steps; ++j, ++c) {
        const int buf = c & 1;
        ok = bar_wait(kv_full(buf), c >> 1 & 1) && bar_wait(s_full(t), n_s & 1);
        if (!ok) break;
        ++n_s;
        tc_after();
        uint64_t x[64];
#pragma unroll
        for (int k = 0; k < 4; ++k) tm_load32(s_at + 32 * k, reinterpret_cast<uint32_t *>(x) + 32 * k);
        tm_wait_load();
        const uint4 *par = reinterpret_cast<const uint4 *>(smem + L::kPar + buf * kTok * 8);
        const int32_t tok0 = w.lo + (w.first_step() + j) * kTok;
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        const bool every = tok0 >= all_lo && tok0 + kTok <= all_hi;
        const int c_lo = row_lo - tok0, c_hi = row_hi - tok0;
#pragma unroll
        for (int k = 0; k < 64; ++k) {
          const uint4 p = par[k];
          F2 s, z;
          s.u[0] = p.x, s.u[1] = p.y, z.u[0] = p.z, z.u[1] = p.w;
          F2 y;
          y.v = fma2(s.v, x[k], mul2(z.v, sum2));
          x[k] = y.v;
        }
        if (!every) {
#pragma unroll
          for (int k = 0; k < 64; ++k) {
            F2 y;
            y.v = x[k];
            if (2 * k < c_lo || 2 * k >= c_hi) y.f[0] = -INFINITY;
            if (2 * k + 1 < c_lo || 2 * k + 1 >= c_hi) y.f[1] = -INFINITY;
            x[k] = y.v;
          }
        }
#pragma unroll
        for (int k = 0; k < 64; ++k) {
          F2 y;
          y.v = x[k];
          top[k & 3] = fmaxf(top[k & 3], fmaxf(y.f[0], y.f[1]));
        }
        const float mt = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * unit;
        const int E = reinterpret_cast<const int *>(smem + L::kExp)[buf];
        if (j == 0) {
          m = mt;
          run = E;
        } else if (__any_sync(0xffffffffu, mt > m + kSlack || (m == -INFINITY && mt > m)) || E > run) {
          // ---- the sums to a new maximum or exponent: the product before has to be done
          ok = bar_wait(o_full(t), (n_o - 1) & 1);
          if (!ok) break;
          tc_after();
          const float mn = fmaxf(m, mt);
          const int en = max(run, E);
          const float down = mn == -INFINITY ? 1.0f : ex2(m - mn), f = down * ex2(static_cast<float>(run - en));
#pragma unroll
          for (int k = 0; k < D; k += 16) {
            uint32_t o[16];
            tm_load16(o_at + k, o);
            tm_wait_load();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tm_store16(o_at + k, o);
          }
          l *= down;
          m = mn;
          run = en;
        }
        const float lag = static_cast<float>(max(E - run, -60));  // this step's values lie so many powers of two lower
        const float ref = lag - (m == -INFINITY ? 0.0f : m);
        const uint64_t ref2 = two(ref, ref);
        uint64_t total[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t p[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            F2 y;
            y.v = fma2(x[32 * k + e], unit2, ref2);
            y.f[0] = ex2(y.f[0]);
            y.f[1] = ex2(y.f[1]);
            total[e & 1] = add2(total[e & 1], y.v);
            p[e] = pack_half(y.f[0], y.f[1]);
          }
          tm_store32(s_at + 32 * k, p);
        }
        F2 sums;
        sums.v = add2(total[0], total[1]);
        l = fmaf(sums.f[0] + sums.f[1], ex2(-lag), l);
        // a value held as NaN is left out of the product, and makes a row that sees it NaN here
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t bad = reinterpret_cast<const uint32_t *>(smem + L::kNan)[4 * buf + k];
          while (bad) {
            const int col = 32 * k + __ffs(bad) - 1;
            bad &= bad - 1;
            if (col >= c_lo && col < c_hi) l = NAN;
          }
        }
        tm_wait_store();
        tc_before();
        __syncwarp();
        if (lane == 0) bar_arrive(p_full(t));
        ++n_o;
      }
      if (!ok) break;

      // ---- the item's rows, or this block's part of them
      const bool whole = w.tile == 0 && w.end() == w.tiles;
      const uint32_t id = w.u - w.tile;
      if (steps > 0) {
        ok = bar_wait(o_full(t), (n_o - 1) & 1);
        if (!ok) break;
        tc_after();
      }
      if (whole) {
        const float f = l == 0.0f ? 0.0f : ex2(static_cast<float>(run)) / l;
        T *dst = static_cast<T *>(a.out) + i * a.o_row + hq * a.o_head;
#pragma unroll
        for (int k = 0; k < D; k += 32) {
          uint32_t o[32];
          if (steps > 0) {
            tm_load32(o_at + k, o);
            tm_wait_load();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0;
          }
          T y[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) y[e] = Cvt<T>::from(l == 0.0f ? 0.0f : __uint_as_float(o[e]) * f);
          if (there) {
            if (a.wide) {
#pragma unroll
              for (int e = 0; e < 32; e += 8) *reinterpret_cast<uint4 *>(dst + k + e) = *reinterpret_cast<const uint4 *>(y + e);
            } else {
#pragma unroll
              for (int e = 0; e < 32; ++e) dst[k + e] = y[e];
            }
          }
        }
        if (there && a.lse) a.lse[i * a.Hq + hq] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      } else {
        float *part = a.many_parts + (static_cast<int64_t>(me) * 2 + (id < u0 ? 0 : 1)) * L::kPart;
        const int at = t * 128 + row;
        const float f = run == kNoExp ? 0.0f : ex2(static_cast<float>(run));
#pragma unroll
        for (int k = 0; k < D; k += 32) {
          uint32_t o[32];
          if (steps > 0) {
            tm_load32(o_at + k, o);
            tm_wait_load();
          }
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (steps > 0) v = make_float4(__uint_as_float(o[e]) * f, __uint_as_float(o[e + 1]) * f, __uint_as_float(o[e + 2]) * f, __uint_as_float(o[e + 3]) * f);
            *reinterpret_cast<float4 *>(part + at * D + k + e) = v;
          }
        }
        part[kRows * D + at] = m;
        part[kRows * D + kRows + at] = l;
        if (tid == 0 && id >= u0) a.many_open[me] = {w.r.q0, id, static_cast<uint32_t>(w.tiles), rows, w.h, w.rt};
      }
      tc_before();  // the sums have been read, before the next item's first product
    }
    if (!ok && lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
  } else if (warp < 12) {
    // ======================================================================== codes to operands
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOperandRegs));
    const int w4 = warp - 8;
    uint32_t c = 0;
    bool ok = true;
    for (Walk w(a, s_start, u0, u1); w.more() && ok; w.next(a)) {
      const int steps = w.steps();
      for (int j = 0; j < steps; ++j, ++c) {
        const int buf = c & 1;
        ok = bar_wait(kv_free(buf), (c >> 1 & 1) ^ 1);
        for (int g = 0; g < kStepGroups && ok; ++g) {
          const uint32_t s = c * kStepGroups + g;
          ok = bar_wait(ring_full(s % kRing), s / kRing & 1);
        }
        if (!ok) break;
        const int32_t tok0 = w.lo + (w.first_step() + j) * kTok;
        auto record = [&](int g) -> const uint8_t * { return smem + L::kRingAt + ((c * kStepGroups + g) % kRing) * kv4_group_bytes(D); };
        // ---- the step's largest value, and the values held as NaN: every warp finds them, 4 tokens a lane
        const uint4 v4 = *reinterpret_cast<const uint4 *>(record(lane >> 2) + 16 * D + 64 + (lane & 3) * 16);
        const uint32_t vp[4] = {v4.x, v4.y, v4.z, v4.w};
        float big = 0.0f;
        uint32_t bad = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 p = kv4_param(vp[e]);
          if (tok0 + 4 * lane + e >= w.hi) continue;
          if (p.x != p.x || p.y != p.y)
            bad |= 1u << e;
          else
            big = fmaxf(big, fmaxf(fabsf(p.y), fabsf(fmaf(15.0f, p.x, p.y))));
        }
        bad <<= (lane & 7) * 4;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) bad |= __shfl_xor_sync(0xffffffffu, bad, o);
        // v 2^-E is below 2^15
        const int E = big == 0.0f ? kNoExp : max(static_cast<int>(__float_as_uint(big) >> 23) - 141, -112);
        const float down = big == 0.0f ? 0.0f : __uint_as_float(static_cast<uint32_t>(127 - E) << 23);
        if (w4 == 0) {
          if ((lane & 7) == 0) reinterpret_cast<uint32_t *>(smem + L::kNan)[4 * buf + (lane >> 3)] = bad;
          if (lane == 0) reinterpret_cast<int *>(smem + L::kExp)[buf] = E;
        }
        // ---- keys' scales and zeros, two tokens side by side
        {
          const int g = w4 + 4 * (lane >> 4), tau = lane & 15, at = g * kGroup + tau;
          float2 p = kv4_param(*reinterpret_cast<const uint32_t *>(record(g) + 16 * D + 4 * tau));
          if (tok0 + at >= w.hi) p = make_float2(0.0f, 0.0f);
          float *dst = reinterpret_cast<float *>(smem + L::kPar + buf * kTok * 8) + (at >> 1) * 4 + (at & 1);
          dst[0] = p.x * (k_sign * kEven);
          dst[2] = p.y * k_sign;
        }
        uint8_t *K = smem + L::kK + buf * L::kTile, *V = smem + L::kV + buf * L::kTile;
#pragma unroll 1
        for (int g = w4; g < kStepGroups; g += 4) {
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
          // ---- values: a lane has 4 channels of 8 tokens, which are 16 bytes of each channel's row
#pragma unroll
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
            const uint32_t *par = reinterpret_cast<const uint32_t *>(rec + 16 * D + 64) + 8 * h;
            uint4 out[4];
            const __half2 off = __float2half2_rn(1024.0f);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              float2 p0 = kv4_param(par[2 * t]), p1 = kv4_param(par[2 * t + 1]);
              const int32_t tok = tok0 + g * kGroup + 8 * h + 2 * t;
              if (tok >= w.hi || p0.x != p0.x || p0.y != p0.y) p0 = make_float2(0.0f, 0.0f);
              if (tok + 1 >= w.hi || p1.x != p1.x || p1.y != p1.y) p1 = make_float2(0.0f, 0.0f);
              const __half2 s = __floats2half2_rn(p0.x * down, p1.x * down), z = __floats2half2_rn(p0.y * down, p1.y * down);
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const uint32_t code = ((v[t] >> (4 * r)) & 0x000f000fu) | 0x64006400u;  // 1024 + code
                const __half2 y = __hfma2(__hsub2(*reinterpret_cast<const __half2 *>(&code), off), s, z);
                reinterpret_cast<uint32_t *>(&out[r])[t] = *reinterpret_cast<const uint32_t *>(&y);
              }
            }
            const int t8 = 2 * g + h;  // 8 tokens of the step's 128
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int ch = cg * (D / 8) + 4 * b + r;
              *reinterpret_cast<uint4 *>(V + t8 / 8 * (D * 128) + ch * 128 + ((t8 % 8 ^ (ch & 7)) << 4)) = out[r];
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane < kStepGroups) bar_arrive(ring_free((c * kStepGroups + lane) % kRing));
        if (lane == 0) bar_arrive(kv_full(buf));
      }
    }
    if (!ok && lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == 12 && lane == 0) {
      // ====================================================================== products
      constexpr uint32_t kQK = idesc_of(kTok), kPV = idesc_of(D);
      uint32_t c = 0, n_q[2] = {0, 0}, n_p[2] = {0, 0};
      bool ok = true;
      auto scores = [&](int t, int buf) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = k / 4 * 16384 + k % 4 * 32;
          mma_ss(tmem + t * 128, rows_desc(base + L::kQ + t * L::kTile + off), rows_desc(base + L::kK + buf * L::kTile + off), kQK, k > 0);
        }
        tc_commit(s_full(t));
      };
      for (Walk w(a, s_start, u0, u1); w.more() && ok; w.next(a)) {
        const int steps = w.steps(), tiles = w.second(a) ? 2 : 1;
        if (steps == 0) continue;
        for (int t = 0; t < tiles && ok; ++t) ok = bar_wait(q_full(t), n_q[t]++ & 1);
        ok = ok && bar_wait(kv_full(c & 1), c >> 1 & 1);
        if (!ok) break;
        tc_after();
        for (int t = 0; t < tiles; ++t) scores(t, c & 1);
        for (int j = 0; j < steps && ok; ++j, ++c) {
          const int buf = c & 1;
          for (int t = 0; t < tiles; ++t) {
            ok = bar_wait(p_full(t), n_p[t]++ & 1);
            if (!ok) break;
            tc_after();
#pragma unroll
            for (int k = 0; k < kTok / 16; ++k)
              mma_ts(tmem + 256 + t * 128, tmem + t * 128 + 8 * k, rows_desc(base + L::kV + buf * L::kTile + k / 4 * (D * 128) + k % 4 * 32), kPV, j > 0 || k > 0);
            tc_commit(o_full(t));
            if (t == tiles - 1) tc_commit(kv_free(buf));
            if (j + 1 < steps) {
              if (t == 0) {
                ok = bar_wait(kv_full(buf ^ 1), (c + 1) >> 1 & 1);
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
      uint32_t c = 0;
      bool ok = true;
      for (Walk w(a, s_start, u0, u1); w.more() && ok; w.next(a)) {
        const int steps = w.steps();
        for (int j = 0; j < steps && ok; ++j, ++c) {
          if (lane < kStepGroups) {
            const uint32_t s = c * kStepGroups + lane;
            const int32_t tok = w.lo + (w.first_step() + j) * kTok + lane * kGroup;
            bool load = tok < w.hi;
            int64_t at = 0;
            if (load) {
              const int32_t grp = tok / kGroup, page = a.block_shift >= 0 ? grp >> a.block_shift : grp / a.block_groups;
              const int32_t block = a.table[w.b * a.max_blocks + page];
              if (block < 0 || block >= a.n_blocks) {
                flag_error(a.status, MAPS_E_RANGE);
                load = false;
              }
              at = block * a.block_bytes + (w.h * a.block_groups + grp - page * a.block_groups) * static_cast<int64_t>(kv4_group_bytes(D));
            }
            ok = bar_wait(ring_free(s % kRing), (s / kRing & 1) ^ 1);
            if (ok) {
              bar_expect(ring_full(s % kRing), load ? kv4_group_bytes(D) : 0);
              if (load) bulk_load(base + L::kRingAt + s % kRing * kv4_group_bytes(D), a.cache + at, kv4_group_bytes(D), ring_full(s % kRing));
            }
          }
          ok = __all_sync(0xffffffffu, ok);
        }
      }
      if (!ok) {
        if (lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
        // let what is under way land: each place of the ring was last filled in this step's round or the one before
        for (int i = lane; i < kRing; i += 32) {
          (void)bar_wait(ring_full(i), (c * kStepGroups + kStepGroups - 1) / kRing & 1);
          (void)bar_wait(ring_full(i), ((c * kStepGroups + kStepGroups - 1) / kRing & 1) ^ 1);
        }
      }
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
constexpr int kJoinRows = 16;  // of a block

template <class T, int D>
__global__ void __launch_bounds__(256) attn_many_join_kernel(const AttnArgs a, uint32_t blocks) {
  pdl_prologue();
  constexpr int kPart = Lay<D>::kPart;
  const uint32_t f = blockIdx.x;
  const Part item = a.many_open[f];
  if (item.tiles == 0) return;
  const Deal deal(*a.many_units, blocks);
  const uint32_t e = deal.worker(item.id + item.tiles - 1);
  const int group = a.Hq / a.Hkv;
  for (int x = 4 * threadIdx.x; x < kJoinRows * D; x += 4 * 256) {
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
  auto kernel = attn_many_kernel<T, D>;
  // The register split below waits for ever where the block was launched with fewer than it adds up to.
  static_assert((2 * kSoftmaxRegs + kOperandRegs + kOtherRegs) * 128 == kThreads * kLaunchRegs, "register split");
  cudaFuncAttributes attr;
  MAPS_TRY(cuda_ok(cudaFuncGetAttributes(&attr, kernel)));
  if (attr.numRegs != kLaunchRegs) return cuda_ok(cudaErrorInvalidConfiguration);
  MAPS_TRY(cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem))));
  if (a.B > kMaxLocalB) launch_pdl(attn_many_plan_kernel, 1, 1024, 0, s, a, grid);
  launch_pdl(kernel, grid, kThreads, smem, s, a);
  launch_pdl(attn_many_join_kernel<T, D>, dim3(grid, kRows / kJoinRows), 256, 0, s, a, grid);
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
