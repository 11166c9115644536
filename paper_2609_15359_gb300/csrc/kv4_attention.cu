// kv4_attention.cu -- attention over the paged 4-bit KV cache, form for few queries a request.
//
// out_i = sum_j softmax_j(sm_scale q_i . k_j) v_j over the keys j that query i sees, with the
// running maximum and sum of the softmax, so the cache is passed over once.
//
// Bound.  A key and value of D channels are D + 8 bytes and serve the few query rows (queries x
// heads of one KV head) of one request, so the time is the cache's bytes; what has to keep up
// is turning 4-bit codes into tensor-core operands.  Codes are therefore never scaled: with
// k = s c + z, q . k = s (q . c) + z sum(q), and with weights p, sum p v = sum (p s) c + sum p z,
// so the matrix products run on the codes themselves, at one shift and one bit operation for
// two of them, with an offset that is taken off in 32 bits with the z term.  Scales then cost a
// few operations a token instead of D.
//
// Shape.  The products are transposed: 16 tokens (or 16 channels) are the 16 rows of an
// m16n8k16 step and 8 query rows its columns, so up to 8 rows waste nothing, and K and V
// are the register operand, straight from the cache's bytes by 16-byte loads from shared
// memory.  P crosses from the first product's result to the second's operand by an 8 x 8
// transpose between lanes.
//
// Split.  The call's work is cut into units of kTok tokens of one (request, KV head, tile of
// query rows).  Every warp of the grid takes an equal run of consecutive units, whatever
// the lengths, and streams its records of the cache through a ring of its own in shared
// memory with bulk copies, two or more stages ahead; nothing is waited for across warps until the end. What
// a run begins or ends inside of is joined afterwards: within the block through shared memory, across blocks
// by the last block to arrive, in the order of the keys, so results do not depend on timing.
#include "kv4.cuh"

namespace maps {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxLocalB = 2048;  // requests whose prefix of units a block sums up for itself

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
  void *out;
  float *lse;
  int64_t *prefix;     // [B + 1] units before each request, where a block does not sum it up
  uint32_t *arrived;   // a byte for each block: blocks that have brought their part of the item it begins
  float *parts;        // [grid][2] parts of items that cross blocks
  int32_t *status;
};

// ---------------------------------------------------------------------------- small device helpers
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {  // bounded
  for (uint32_t i = 0; i < kSpinLimit; ++i)
    if (bar_try(bar, parity)) return true;
  return false;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t y;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}
__device__ __forceinline__ float lo_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// Two keys' codes as 16-bit numbers, one shift and one bit operation for both.  bfloat16: 16 + code,
// the code in the mantissa's upper bits (128 + code would cost one shift less in four, and eight
// times the rounding error of a sum that the offset dominates).  half: code * 2^-24, the bare code
// being a subnormal number, which the tensor core multiplies exactly.
template <class T>
struct Key;
template <>
struct Key<__nv_bfloat16> {
  static constexpr float kOffset = 16.0f, kUnit = 1.0f;
  static constexpr int kParts = 1;  // 16-bit numbers that a weight is the sum of
  static __device__ __forceinline__ uint32_t two(uint32_t w, int r) {  // codes r and r + 4 of a word
    return ((r == 0 ? w << 3 : w >> (4 * r - 3)) & 0x00780078u) | 0x41804180u;
  }
  static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
template <>
struct Key<__half> {
  static constexpr float kOffset = 0.0f, kUnit = 16777216.0f;
  static constexpr int kParts = 2;  // a half output shows the rounding of a weight to 8 bits
  static __device__ __forceinline__ uint32_t two(uint32_t w, int r) { return (w >> (4 * r)) & 0x000f000fu; }
  static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
// Two values' codes as 128 + code in bfloat16, whatever the queries' type: a weight times a scale needs the range.
__device__ __forceinline__ uint32_t two_values(uint32_t w, int r) { return ((w >> (4 * r)) & 0x000f000fu) | 0x43004300u; }

// ---------------------------------------------------------------------------- the work, in units
template <int D, int NT>
struct Shape {
  static constexpr int kRows = 8 * NT;                       // query rows of a tile
  static constexpr int kGroups = D == 256 ? 2 : 4;           // groups of 16 tokens in a unit
  static constexpr int kTok = kGroups * kGroup;
  static constexpr int kBytes = kGroups * kv4_group_bytes(D);  // of a stage
  static constexpr int kStages = D == 64 ? 4 : 2;
  static constexpr int kPart = kRows * D + 2 * kRows;        // floats of a part: sums, maxima, totals
};

// What one request is for the kernel: queries, tokens, the first token any query sees (to 16), units.
struct Req {
  int32_t n, n_q, lo, tiles, row_tiles;
};
template <int kTok, int kRows>
__device__ __forceinline__ Req request(const AttnArgs &a, int b) {
  Req r;
  const int64_t q0 = a.off[b], q1 = a.off[b + 1];
  int32_t n = a.len[b];
  int64_t m = q1 - q0;
  if (n < 0 || n > a.max_blocks * a.S) {
    flag_error(a.status, MAPS_E_RANGE);
    n = 0;
  }
  if (q0 < 0 || m < 0 || q1 > a.T) {
    flag_error(a.status, MAPS_E_RANGE);
    m = 0;
  }
  r.n = n;
  r.n_q = static_cast<int32_t>(m);
  int64_t lo = 0;
  if (a.window > 0) lo = static_cast<int64_t>(n) - m - a.window + 1;
  r.lo = lo > 0 ? static_cast<int32_t>(lo) / kGroup * kGroup : 0;
  const int32_t span = r.n - r.lo;
  r.tiles = span > kTok ? (span + kTok - 1) / kTok : 1;
  r.row_tiles = static_cast<int32_t>((m * (a.Hq / a.Hkv) + kRows - 1) / kRows);
  return r;
}

// The prefix of units over the requests: each thread sums a run of them.
template <int kTok, int kRows, int kN>
__device__ __forceinline__ void sum_units(const AttnArgs &a, int64_t *prefix) {
  __shared__ int64_t s_warp[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.B + kN - 1) / kN, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  int64_t mine = 0;
  for (int b = b0; b < b1; ++b) {
    const Req r = request<kTok, kRows>(a, b);
    mine += static_cast<int64_t>(r.tiles) * r.row_tiles * a.Hkv;
  }
  int64_t x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  int64_t at = x - mine;
  for (int w = 0; w < warp; ++w) at += s_warp[w];
  for (int b = b0; b < b1; ++b) {
    prefix[b] = at;
    const Req r = request<kTok, kRows>(a, b);
    at += static_cast<int64_t>(r.tiles) * r.row_tiles * a.Hkv;
  }
  if (tid == kN - 1) prefix[a.B] = at;
  __syncthreads();
}

template <int kTok, int kRows>
__global__ void __launch_bounds__(1024) attn_plan_kernel(const AttnArgs a) {
  pdl_prologue();
  sum_units<kTok, kRows, 1024>(a, a.prefix);
}

// A place in the list of units: unit `tile` of the item (request b, KV head h, row tile rt).
struct Cursor {
  int32_t b, h, rt, tile;
  Req r;
  template <int kTok, int kRows>
  __device__ __forceinline__ void seek(const AttnArgs &a, const int64_t *prefix, int64_t u) {
    int lo = 0, hi = a.B;  // prefix[lo] <= u < prefix[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (prefix[mid] <= u)
        lo = mid;
      else
        hi = mid;
    }
    b = lo;
    r = request<kTok, kRows>(a, b);
    int64_t rest = u - prefix[b];
    const int64_t item = rest / r.tiles;
    tile = static_cast<int32_t>(rest - item * r.tiles);
    h = static_cast<int32_t>(item / r.row_tiles);
    rt = static_cast<int32_t>(item - static_cast<int64_t>(h) * r.row_tiles);
  }
  template <int kTok, int kRows>
  __device__ __forceinline__ void next_item(const AttnArgs &a) {
    tile = 0;
    if (++rt < r.row_tiles) return;
    rt = 0;
    if (++h < a.Hkv) return;
    h = 0;
    do {
      if (++b >= a.B) return;
      r = request<kTok, kRows>(a, b);
    } while (r.row_tiles == 0);
  }
};

// ---------------------------------------------------------------------------- the kernel
template <class T, int D, int NT>
__global__ void __launch_bounds__(kThreads, 1) attn_few_kernel(const AttnArgs a) {
  using Sh = Shape<D, NT>;
  constexpr int kSteps = D / 16, kWords = D / 32, kCh = D / 8;
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t *ring_all = smem;
  float *first_parts = reinterpret_cast<float *>(smem + kWarps * Sh::kStages * Sh::kBytes);
  uint64_t *bars = reinterpret_cast<uint64_t *>(first_parts + kWarps * Sh::kPart);
  int64_t *s_prefix = reinterpret_cast<int64_t *>(bars + kWarps * Sh::kStages);
  __shared__ int64_t s_id[2 * kWarps];     // an item's first unit, -1: no part here
  __shared__ int32_t s_tiles[2 * kWarps];  // its units
  __shared__ int32_t s_b[2 * kWarps], s_h[2 * kWarps], s_rt[2 * kWarps];
  __shared__ uint32_t s_last;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  uint8_t *ring = ring_all + warp * Sh::kStages * Sh::kBytes;
  const uint32_t ring32 = smem_u32(ring), bar32 = smem_u32(bars + warp * Sh::kStages);
  if (lane < Sh::kStages) bar_init(bar32 + 8 * lane, 1);
  if (lane < 2) s_id[2 * warp + lane] = -1;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  pdl_prologue();
  const int64_t *prefix = a.prefix;
  if (a.B <= kMaxLocalB) {
    sum_units<Sh::kTok, Sh::kRows, kThreads>(a, s_prefix);
    prefix = s_prefix;
  } else {
    __syncthreads();
  }

  const int64_t U = prefix[a.B], workers = static_cast<int64_t>(gridDim.x) * kWarps;
  const int64_t used = U < workers ? U : workers;  // warps that get units, the first ones
  auto start = [&](int64_t w) -> int64_t { return used == 0 ? 0 : w >= used ? U : U / used * w + min(w, U % used); };
  const int64_t me = static_cast<int64_t>(blockIdx.x) * kWarps + warp;
  const int64_t u0 = start(me), u1 = start(me + 1);
  const int group = a.Hq / a.Hkv;

  if (u0 < u1) {
    // The loads run ahead of the products by the ring's depth; lanes below kGroups move one group each.
    Cursor ahead = {};
    ahead.seek<Sh::kTok, Sh::kRows>(a, prefix, u0);
    Cursor at = ahead;
    int64_t issued = u0;
    int32_t block = -1;  // the next unit's block of this lane's group, fetched one step early
    auto fetch = [&]() {
      block = -1;
      const int32_t tok = ahead.r.lo + ahead.tile * Sh::kTok + lane * kGroup;
      if (issued < u1 && lane < Sh::kGroups && tok < ahead.r.n) block = a.table[ahead.b * a.max_blocks + tok / a.S];
    };
    auto issue = [&](int stage) {
      const int32_t tok = ahead.r.lo + ahead.tile * Sh::kTok + lane * kGroup;
      const bool mine = issued < u1 && lane < Sh::kGroups && tok < ahead.r.n;
      const bool good = mine && block >= 0 && block < a.n_blocks;
      if (mine && !good) flag_error(a.status, MAPS_E_RANGE);
      const uint32_t n = __popc(__ballot_sync(0xffffffffu, good));
      if (lane == 0) bar_expect(bar32 + 8 * stage, n * kv4_group_bytes(D));
      __syncwarp();
      if (good) {
        const int64_t rec = (static_cast<int64_t>(block) * a.Hkv + ahead.h) * (a.S / kGroup) + tok % a.S / kGroup;
        bulk_load(ring32 + stage * Sh::kBytes + lane * kv4_group_bytes(D), a.cache + rec * kv4_group_bytes(D), kv4_group_bytes(D), bar32 + 8 * stage);
      }
      if (issued < u1) {
        ++issued;
        if (++ahead.tile == ahead.r.tiles && issued < u1) ahead.next_item<Sh::kTok, Sh::kRows>(a);
        fetch();
      }
    };
    fetch();
#pragma unroll
    for (int s = 0; s < Sh::kStages; ++s) issue(s);

    int stage = 0;
    uint32_t parity = 0;
    bool alive = true;
    for (int64_t u = u0; u < u1 && alive;) {
      // ---- an item: its queries, as the columns of the first product
      const Req r = at.r;
      const int64_t q0 = a.off[at.b];
      const int rows = r.n_q * group;  // n_q * group <= T * Hq fits the checks of the host
      uint32_t qf[NT][kSteps][2];
      float qs[NT][2];
      int32_t row_lo[NT][2], row_hi[NT][2];
      int32_t all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int R = at.rt * Sh::kRows + nt * 8 + g;
        float sum = 0.0f;
        if (R < rows) {
          const T *src = static_cast<const T *>(a.q) + (q0 + R / group) * a.q_row + (at.h * group + R % group) * a.q_head + t * (D / 4);
#pragma unroll
          for (int i = 0; i < kWords; ++i) {
            uint32_t x[4];
            if (a.wide) {
              *reinterpret_cast<uint4 *>(x) = *reinterpret_cast<const uint4 *>(src + 8 * i);
            } else {
              const uint16_t *p = reinterpret_cast<const uint16_t *>(src + 8 * i);
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = p[2 * e] | static_cast<uint32_t>(p[2 * e + 1]) << 16;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const T *y = reinterpret_cast<const T *>(&x[e]);
              sum += Cvt<T>::to(y[0]) + Cvt<T>::to(y[1]);
            }
            qf[nt][2 * i][0] = __byte_perm(x[0], x[2], 0x5410);
            qf[nt][2 * i][1] = __byte_perm(x[0], x[2], 0x7632);
            qf[nt][2 * i + 1][0] = __byte_perm(x[1], x[3], 0x5410);
            qf[nt][2 * i + 1][1] = __byte_perm(x[1], x[3], 0x7632);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kSteps; ++i) qf[nt][i][0] = qf[nt][i][1] = 0;
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          qs[nt][e] = __shfl_sync(0xffffffffu, sum, (2 * t + e) * 4);
          const int Rc = at.rt * Sh::kRows + nt * 8 + 2 * t + e;
          row_lo[nt][e] = 0;
          row_hi[nt][e] = r.n;  // a column that is no row sees everything; nobody reads it
          if (Rc < rows) {
            const int64_t pos = static_cast<int64_t>(r.n) - r.n_q + Rc / group;
            row_hi[nt][e] = pos < 0 ? 0 : a.causal ? static_cast<int32_t>(pos) + 1 : r.n;
            if (a.window > 0 && pos - a.window + 1 > 0) row_lo[nt][e] = static_cast<int32_t>(pos - a.window + 1);
          }
          all_lo = max(all_lo, row_lo[nt][e]);
          all_hi = min(all_hi, row_hi[nt][e]);
        }
      }
      all_lo = max(all_lo, __shfl_xor_sync(0xffffffffu, all_lo, 1));
      all_lo = max(all_lo, __shfl_xor_sync(0xffffffffu, all_lo, 2));
      all_hi = min(all_hi, __shfl_xor_sync(0xffffffffu, all_hi, 1));
      all_hi = min(all_hi, __shfl_xor_sync(0xffffffffu, all_hi, 2));

      float o[NT][kSteps][4], m[NT][2], l[NT][2], w[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[nt][j][e] = 0.0f;
#pragma unroll
        for (int e = 0; e < 2; ++e) m[nt][e] = -INFINITY, l[nt][e] = 0.0f, w[nt][e] = 0.0f;
      }

      const int64_t left = r.tiles - at.tile;
      const int64_t seg_end = u + (left < u1 - u ? left : u1 - u);
      const int32_t seg_first = at.tile;
      for (; u < seg_end; ++u, ++at.tile) {
        if (!bar_wait(bar32 + 8 * stage, parity)) {
          if (lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
          alive = false;
          break;
        }
        const uint8_t *buf = ring + stage * Sh::kBytes;
        const int32_t tok0 = r.lo + at.tile * Sh::kTok;
        const bool full = tok0 >= all_lo && tok0 + Sh::kTok <= all_hi;  // every row sees every token

        // ---- scores: 16 tokens x 8 rows, depth D
        float s[Sh::kGroups][NT][4];
#pragma unroll
        for (int gr = 0; gr < Sh::kGroups; ++gr) {
          const uint8_t *grp = buf + gr * kv4_group_bytes(D);
          uint32_t k0[kWords], k1[kWords];
          if (kWords == 2) {
            *reinterpret_cast<uint2 *>(k0) = *reinterpret_cast<const uint2 *>(grp + g * (D / 2) + t * (D / 8));
            *reinterpret_cast<uint2 *>(k1) = *reinterpret_cast<const uint2 *>(grp + (g + 8) * (D / 2) + t * (D / 8));
          } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
              *reinterpret_cast<uint4 *>(k0 + i) = *reinterpret_cast<const uint4 *>(grp + g * (D / 2) + t * (D / 8) + 4 * i);
              *reinterpret_cast<uint4 *>(k1 + i) = *reinterpret_cast<const uint4 *>(grp + (g + 8) * (D / 2) + t * (D / 8) + 4 * i);
            }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[gr][nt][e] = 0.0f;
#pragma unroll
          for (int st = 0; st < kSteps; ++st) {
            const int i = st / 2, rr = st % 2 * 2;
            const uint32_t a0 = Key<T>::two(k0[i], rr), a1 = Key<T>::two(k1[i], rr), a2 = Key<T>::two(k0[i], rr + 1), a3 = Key<T>::two(k1[i], rr + 1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) Key<T>::mma(s[gr][nt], a0, a1, a2, a3, qf[nt][st][0], qf[nt][st][1]);
          }
          const uint32_t *par = reinterpret_cast<const uint32_t *>(grp + 16 * D);
          const float sl2 = a.scale * 1.4426950408889634f;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const float2 p = kv4_param(par[g + 8 * half]);
            const float ks = p.x * (sl2 * Key<T>::kUnit), kz = fmaf(-Key<T>::kOffset, p.x, p.y) * sl2;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e) s[gr][nt][2 * half + e] = fmaf(ks, s[gr][nt][2 * half + e], kz * qs[nt][e]);
          }
          if (!full) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const int32_t tok = tok0 + gr * kGroup + g + 8 * half;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  if (tok < row_lo[nt][e] || tok >= row_hi[nt][e]) s[gr][nt][2 * half + e] = -INFINITY;
            }
          }
        }

        // ---- running maximum
        float ref[NT][2];
        bool grew = false;
        float mn[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = fmaxf(s[0][nt][e], s[0][nt][2 + e]);
#pragma unroll
            for (int gr = 1; gr < Sh::kGroups; ++gr) x = fmaxf(x, fmaxf(s[gr][nt][e], s[gr][nt][2 + e]));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            mn[nt][e] = fmaxf(m[nt][e], x);
            grew |= mn[nt][e] > m[nt][e];
          }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float c = mn[nt][e] == -INFINITY ? 1.0f : ex2(m[nt][e] - mn[nt][e]);
              m[nt][e] = mn[nt][e];
              l[nt][e] *= c;
              w[nt][e] *= c;
#pragma unroll
              for (int j = 0; j < kSteps; ++j) o[nt][j][e] *= c, o[nt][j][2 + e] *= c;
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) ref[nt][e] = m[nt][e] == -INFINITY ? 0.0f : m[nt][e];

        // ---- weights and sums over the values
#pragma unroll
        for (int gr = 0; gr < Sh::kGroups; ++gr) {
          const uint8_t *grp = buf + gr * kv4_group_bytes(D);
          const uint32_t *par = reinterpret_cast<const uint32_t *>(grp + 16 * D) + 16;
          constexpr int kParts = Key<T>::kParts;
          uint32_t pf[NT][kParts][2];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const float2 p = kv4_param(par[g + 8 * half]);
            const int32_t tok = tok0 + gr * kGroup + g + 8 * half;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float ps[2], pz[2];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float x = ex2(s[gr][nt][2 * half + e] - ref[nt][e]);
                l[nt][e] += x;
                ps[e] = x * p.x;
                pz[e] = x * p.y;
                // a token that the row does not see has weight 0, and whatever its scale is stays out
                if (!full && (tok < row_lo[nt][e] || tok >= row_hi[nt][e])) ps[e] = pz[e] = 0.0f;
              }
              const uint32_t hi = pack_bf16(ps[0], ps[1]);
              float r0 = lo_bf16(hi), r1 = hi_bf16(hi);
              pf[nt][0][half] = transpose8(hi);
              if (kParts == 2) {
                const uint32_t lo = pack_bf16(ps[0] - r0, ps[1] - r1);
                r0 += lo_bf16(lo);
                r1 += hi_bf16(lo);
                pf[nt][kParts - 1][half] = transpose8(lo);
              }
              w[nt][0] += fmaf(-128.0f, r0, pz[0]);
              w[nt][1] += fmaf(-128.0f, r1, pz[1]);
            }
          }
          uint32_t v0[kWords], v1[kWords];
          const uint8_t *vb = grp + 8 * D;
          if (kWords == 2) {
            *reinterpret_cast<uint2 *>(v0) = *reinterpret_cast<const uint2 *>(vb + lane * 8);
            *reinterpret_cast<uint2 *>(v1) = *reinterpret_cast<const uint2 *>(vb + 256 + lane * 8);
          } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
              *reinterpret_cast<uint4 *>(v0 + i) = *reinterpret_cast<const uint4 *>(vb + i / 4 * 512 + lane * 16);
              *reinterpret_cast<uint4 *>(v1 + i) = *reinterpret_cast<const uint4 *>(vb + (kWords + i) / 4 * 512 + lane * 16);
            }
          }
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            const int i = j / 2, rr = j % 2 * 2;
            const uint32_t a0 = two_values(v0[i], rr), a1 = two_values(v0[i], rr + 1), a2 = two_values(v1[i], rr), a3 = two_values(v1[i], rr + 1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int q = 0; q < kParts; ++q) Key<__nv_bfloat16>::mma(o[nt][j], a0, a1, a2, a3, pf[nt][q][0], pf[nt][q][1]);
          }
        }
        __syncwarp();  // the stage has been read
        issue(stage);
        if (++stage == Sh::kStages) stage = 0, parity ^= 1;
      }
      if (!alive) break;

      // ---- the item, or this warp's part of it
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) {
            l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], x);
            w[nt][e] += __shfl_xor_sync(0xffffffffu, w[nt][e], x);
          }
        }
      const bool whole = seg_first == 0 && at.tile == r.tiles;
      if (whole) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int R = at.rt * Sh::kRows + nt * 8 + 2 * t + e;
            if (R >= rows) continue;
            const int64_t i = q0 + R / group;
            const int hq = at.h * group + R % group;
            const float inv = l[nt][e] == 0.0f ? 0.0f : 1.0f / l[nt][e];
            const float add = l[nt][e] == 0.0f ? 0.0f : w[nt][e];
            T *dst = static_cast<T *>(a.out) + i * a.o_row + hq * a.o_head + g * kCh;
            T y[kCh];
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
              y[2 * j] = Cvt<T>::from((o[nt][j][e] + add) * inv);
              y[2 * j + 1] = Cvt<T>::from((o[nt][j][2 + e] + add) * inv);
            }
            if (a.wide) {
#pragma unroll
              for (int c = 0; c < kCh; c += 8) *reinterpret_cast<uint4 *>(dst + c) = *reinterpret_cast<const uint4 *>(y + c);
            } else {
#pragma unroll
              for (int c = 0; c < kCh; ++c) dst[c] = y[c];
            }
            if (a.lse && g == 0) a.lse[i * a.Hq + hq] = l[nt][e] == 0.0f ? -INFINITY : (m[nt][e] + log2f(l[nt][e])) * 0.6931471805599453f;
          }
      } else {
        // a run's first part goes to its own place, its last to the ring, which has been read to the end
        const bool is_first = u - (at.tile - seg_first) == u0;
        const int slot = 2 * warp + (is_first ? 0 : 1);
        float *part = is_first ? first_parts + warp * Sh::kPart : reinterpret_cast<float *>(ring);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int R = nt * 8 + 2 * t + e;
            float *dst = part + R * D + g * kCh;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
              dst[2 * j] = o[nt][j][e] + w[nt][e];
              dst[2 * j + 1] = o[nt][j][2 + e] + w[nt][e];
            }
            if (g == 0) {
              part[Sh::kRows * D + R] = m[nt][e];
              part[Sh::kRows * D + Sh::kRows + R] = l[nt][e];
            }
          }
        if (lane == 0) {
          s_id[slot] = u - at.tile;  // the item's first unit: at.tile units of it lie before u
          s_tiles[slot] = r.tiles;
          s_b[slot] = at.b;
          s_h[slot] = at.h;
          s_rt[slot] = at.rt;
        }
      }
      if (u < u1) at.next_item<Sh::kTok, Sh::kRows>(a);
    }
    if (!alive) {  // let what is under way land before the block ends
      for (int s = 0; s < Sh::kStages; ++s) (void)bar_wait(bar32 + 8 * s, s < stage ? parity ^ 1 : parity);
    }
  }
  __syncthreads();

  // ---- join the parts of the block's items, in the order of their keys
  const int64_t c0 = start(static_cast<int64_t>(blockIdx.x) * kWarps), c1 = start(static_cast<int64_t>(blockIdx.x + 1) * kWarps);
  auto part_of = [&](int slot) -> const float * {
    return slot % 2 == 0 ? first_parts + slot / 2 * Sh::kPart : reinterpret_cast<const float *>(ring_all + slot / 2 * Sh::kStages * Sh::kBytes);
  };
  auto write_row = [&](int b, int h, int rt, int R, int d, float num, float mm, float ll) {
    const Req r = request<Sh::kTok, Sh::kRows>(a, b);
    const int row = rt * Sh::kRows + R;
    if (row >= r.n_q * group) return;
    const int64_t i = a.off[b] + row / group;
    const int hq = h * group + row % group;
    static_cast<T *>(a.out)[i * a.o_row + hq * a.o_head + d] = Cvt<T>::from(ll == 0.0f ? 0.0f : num / ll);
    if (d == 0 && a.lse) a.lse[i * a.Hq + hq] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * 0.6931471805599453f;
  };
  for (int s0 = 0; s0 < 2 * kWarps;) {
    const int64_t id = s_id[s0];
    if (id < 0) {
      ++s0;
      continue;
    }
    int s1 = s0 + 1;
    while (s1 < 2 * kWarps && (s_id[s1] < 0 || s_id[s1] == id)) ++s1;
    const int tiles = s_tiles[s0], b = s_b[s0], h = s_h[s0], rt = s_rt[s0];
    const bool whole = id >= c0 && id + tiles <= c1;
    float *mine = a.parts + (static_cast<int64_t>(blockIdx.x) * 2 + (id < c0 ? 0 : 1)) * Sh::kPart;
    for (int x = tid; x < Sh::kRows * D; x += kThreads) {
      const int R = x / D, d = x - R * D;
      float M = -INFINITY;
      for (int s = s0; s < s1; ++s)
        if (s_id[s] == id) M = fmaxf(M, part_of(s)[Sh::kRows * D + R]);
      float num = 0.0f, den = 0.0f;
      for (int s = s0; s < s1; ++s) {
        if (s_id[s] != id) continue;
        const float *p = part_of(s);
        const float f = M == -INFINITY ? 1.0f : ex2(p[Sh::kRows * D + R] - M);
        num = fmaf(f, p[x], num);
        den = fmaf(f, p[Sh::kRows * D + Sh::kRows + R], den);
      }
      if (whole) {
        write_row(b, h, rt, R, d, num, M, den);
      } else {
        mine[x] = num;
        if (d == 0) mine[Sh::kRows * D + R] = M, mine[Sh::kRows * D + Sh::kRows + R] = den;
      }
    }
    if (!whole) {
      // blocks that hold a unit of the item: the first by its first unit, the last by its last
      auto block_of = [&](int64_t u) -> int64_t {
        const int64_t per = U / used, more = U % used;
        const int64_t w = u < more * (per + 1) ? u / (per + 1) : more + (u - more * (per + 1)) / per;
        return w / kWarps;
      };
      const int64_t f = block_of(id), e = block_of(id + tiles - 1);
      __threadfence();
      __syncthreads();
      const int shift = static_cast<int>(f & 3) * 8;
      if (tid == 0) s_last = (atom_add_acq_rel_u32(&a.arrived[f >> 2], 1u << shift) >> shift & 255u) == static_cast<uint32_t>(e - f) ? 1u : 0u;
      __syncthreads();
      if (s_last) {
        __threadfence();
        if (tid == 0) atomicSub(&a.arrived[f >> 2], static_cast<uint32_t>(e - f + 1) << shift);  // for the next call
        for (int x = tid; x < Sh::kRows * D; x += kThreads) {
          const int R = x / D, d = x - R * D;
          float M = -INFINITY, num = 0.0f, den = 0.0f;
          for (int64_t c = f; c <= e; ++c) M = fmaxf(M, __ldcg(a.parts + (c * 2 + (c == f)) * Sh::kPart + Sh::kRows * D + R));
          for (int64_t c = f; c <= e; ++c) {
            const float *p = a.parts + (c * 2 + (c == f)) * Sh::kPart;
            const float k = M == -INFINITY ? 1.0f : ex2(__ldcg(p + Sh::kRows * D + R) - M);
            num = fmaf(k, __ldcg(p + x), num);
            den = fmaf(k, __ldcg(p + Sh::kRows * D + Sh::kRows + R), den);
          }
          write_row(b, h, rt, R, d, num, M, den);
        }
      }
    }
    s0 = s1;
    __syncthreads();
  }
}

constexpr int kMaxParts = 16 * 128 + 32;  // floats of the largest part (two row tiles of 128 channels, or one of 256)
// The counters of arrivals lie in the control block, behind the status word: calls that share a
// workspace leave that zero, and so does this one.
constexpr int kArrivedAt = 64, kMaxGrid = kCtrlBytes - kArrivedAt;
int grid_size() { return sm_count() < kMaxGrid ? sm_count() : kMaxGrid; }

template <class T, int D, int NT>
int launch_few(const AttnArgs &a, cudaStream_t s) {
  using Sh = Shape<D, NT>;
  const size_t local = a.B <= kMaxLocalB ? static_cast<size_t>(a.B + 1) * 8 : 0;
  const size_t smem = static_cast<size_t>(kWarps) * Sh::kStages * Sh::kBytes + static_cast<size_t>(kWarps) * Sh::kPart * 4 + kWarps * Sh::kStages * 8 + local;
  auto kernel = attn_few_kernel<T, D, NT>;
  MAPS_TRY(cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem))));
  if (a.B > kMaxLocalB) launch_pdl(attn_plan_kernel<Sh::kTok, Sh::kRows>, 1, 1024, 0, s, a);
  launch_pdl(kernel, static_cast<unsigned>(grid_size()), kThreads, smem, s, a);
  return launch_ok();
}

template <class T>
int launch_dim(int D, const AttnArgs &a, cudaStream_t s) {
  // 8 rows to a tile where a request has at most 8 on average, else 16
  const bool one = a.T * (a.Hq / a.Hkv) <= static_cast<int64_t>(8) * a.B;
  if (D == 64) return one ? launch_few<T, 64, 1>(a, s) : launch_few<T, 64, 2>(a, s);
  if (D == 128) return one ? launch_few<T, 128, 1>(a, s) : launch_few<T, 128, 2>(a, s);
  return launch_few<T, 256, 1>(a, s);
}

}  // namespace
}  // namespace maps

extern "C" {

size_t maps_kv4_attention_workspace_size(int32_t B, int64_t T, int32_t Hq, int32_t Hkv, int32_t D) {
  using namespace maps;
  (void)T, (void)Hq, (void)Hkv, (void)D;
  Carve c(nullptr);
  c.take<float>(static_cast<size_t>(grid_size()) * 2 * kMaxParts);
  c.take<int64_t>(B > kMaxLocalB ? static_cast<size_t>(B) + 1 : 0);
  return c.bytes();
}

int maps_kv4_attention(int32_t dtype, int32_t B, int64_t T, int32_t Hq, int32_t Hkv, int32_t D,
                       int32_t S, const void *q, int64_t q_row, int64_t q_head,
                       const int64_t *qo_off, const int32_t *kv_len, const int32_t *table,
                       int64_t max_blocks, const void *cache, int64_t n_blocks, float sm_scale,
                       int32_t causal, int32_t window, void *out, int64_t o_row, int64_t o_head,
                       float *lse, void *ws, size_t ws_bytes, void *stream) {
  using namespace maps;
  if ((dtype != MAPS_BF16 && dtype != MAPS_F16) || !kv4_dim_ok(D) || !kv4_block_ok(S) || B < 0 ||
      T < 0 || T > (int64_t(1) << 30) || Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 || Hq > 65535 ||
      T > ((int64_t(1) << 31) - 64) / Hq || max_blocks < 0 || max_blocks > 0x7fffffff || n_blocks < 0 || window < 0 ||
      (causal != 0 && causal != 1) || !(sm_scale - sm_scale == 0.0f))
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, maps_kv4_attention_workspace_size(B, T, Hq, Hkv, D)));
  if (T == 0 || B == 0) return MAPS_OK;
  if (q == nullptr || out == nullptr || qo_off == nullptr || kv_len == nullptr ||
      (max_blocks > 0 && table == nullptr) || (n_blocks > 0 && cache == nullptr) || !aligned(cache, 16) || !aligned(q, 2) ||
      !aligned(lse, 4) || !aligned(out, 2))
    return MAPS_E_INVALID;
  const bool wide = aligned(q, 16) && aligned(out, 16) && q_row % 8 == 0 && q_head % 8 == 0 && o_row % 8 == 0 && o_head % 8 == 0;
  Carve c(ws);
  uint32_t *arrived = reinterpret_cast<uint32_t *>(static_cast<char *>(ws) + kArrivedAt);
  float *parts = c.take<float>(static_cast<size_t>(grid_size()) * 2 * kMaxParts);
  int64_t *prefix = c.take<int64_t>(B > kMaxLocalB ? static_cast<size_t>(B) + 1 : 0);
  const AttnArgs a = {B, Hq, Hkv, S, T, n_blocks, max_blocks, q, q_row, q_head, o_row, o_head, qo_off, kv_len, table,
                      static_cast<const uint8_t *>(cache), sm_scale, causal, window, wide, out, lse, prefix, arrived, parts, status_word(ws)};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MAPS_BF16) return launch_dim<__nv_bfloat16>(D, a, s);
  return launch_dim<__half>(D, a, s);
}

}  // extern "C"
