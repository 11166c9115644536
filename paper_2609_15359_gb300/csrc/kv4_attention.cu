// kv4_attention.cu -- attention over the paged 4-bit KV cache, form for few queries a request.
//
// out_i = sum_j softmax_j(sm_scale q_i . k_j) v_j over the keys j that query i sees, with the
// running maximum and sum of the softmax, so the cache is passed over once.
//
// Mathematics.  With k = s c + z (codes c), q . k = s (q . c) + z sum(q), and with weights p,
// sum p v = sum (p s) c + sum p z: the matrix products run on bare codes, and scales and zeros cost
// a few operations a token instead of D.  A code is a half number as it stands (codes_of), so eight
// codes take five operations.  q is scaled by a power of two to fill half's range; p s is held
// relative to the largest p s so far.
//
// Bound.  A key and value of D channels are D + 8 bytes and serve the few query rows (queries x
// heads of one KV head) of one request, so long calls are bound by the cache's bytes: 128 requests
// of 64 to 8,192 tokens, 8 KV heads of 128 channels, 566 MB, take 116 us (4.9 TB/s, 0.72 of the
// measured copy rate).  Within the passes it is 6.2 TB/s; the rest is a call's fixed part, about 11 us of
// dependent steps: the plan (2), first queries and records (2), a first unit (4), the joins (3).  Short calls take little
// else: one request of 2,048 tokens 12 us.
//
// Shape.  The products are transposed: 16 tokens (or 16 channels) are the 16 rows of an
// m16n8k16 step and 8 query rows its columns, so up to 8 rows waste nothing (as the columns of a
// tcgen05 product they would meet 128 rows and cross tensor memory twice), and K and V are the
// register operand, straight from the cache's bytes by 16-byte loads from shared memory.  P
// crosses from the first product's result to the second's operand by an 8 x 8 transpose between lanes.
//
// Split.  The call's work is cut into units of kTok tokens of one (request, KV head, tile of
// query rows).  Every warp of the grid takes an equal run of consecutive units, whatever
// the lengths, and streams its records of the cache through a ring of its own in shared
// memory with bulk copies, two or more stages ahead; nothing is waited for across warps until the end. What
// a run begins or ends inside of is joined afterwards: within the block through shared memory, across blocks
// by the last block to arrive, in the order of the keys, so results do not depend on timing.
#include "kv4_attention.cuh"

namespace maps {
namespace {

constexpr int kMaxWarps = 16;  // of a block
// Query rows of a request to a KV head up to which this form serves it where the other may.  Both grow with the rows, this
// one by tiles of 16: 32 requests of 4,096 random tokens, 128 channels: 64 rows 189 us here, 229 there; 96 rows 265, 229;
// 128 rows 343, 231.  With 64 channels 191, 181 at 96; with 4 requests 53, 57 at 96 and 100, 69 at 256.
constexpr int kFewRows = 96;

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Values for the second product.  Bare codes are all positive, so in sums over many tokens the products' sum and the sum
// of the zeros are far larger than their difference: by 1,000 at 100,000 tokens, where a half output shows what 32-bit
// sums then lose (6e-4 of the output's norm, 2e-4 its own rounding).  So for half the codes are taken about 8, at one
// packed addition more for two; the zeros follow.
template <class T>
struct Value {
  static constexpr float kEvenBy = kEven, kOddBy = kOdd, kCentre = 0.0f;
  static __device__ __forceinline__ Codes of(uint32_t w) { return codes_of(w); }
};
template <>
struct Value<__half> {
  static constexpr float kEvenBy = 1.0f, kOddBy = 0.0625f, kCentre = 8.0f;
  static __device__ __forceinline__ Codes of(uint32_t w) {
    Codes c = codes_of(w);
    const __half2 even = __float2half2_rn(-1032.0f), odd = __float2half2_rn(-1152.0f);  // 1024 + 8, 1024 + 16 * 8
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t x = c.x[r] | 0x64006400u;
      const __half2 y = __hadd2(*reinterpret_cast<const __half2 *>(&x), r % 2 ? odd : even);
      c.x[r] = *reinterpret_cast<const uint32_t *>(&y);
    }
    return c;
  }
};

// ---------------------------------------------------------------------------- the work, in units
template <int D, int NT>
struct Shape {
  static constexpr int kRows = 8 * NT;                       // query rows of a tile
  // As many warps as their registers allow: a unit is a chain of dependent steps, hidden by other warps alone.
  static constexpr int kWarps = NT == 2 || D == 256 ? 8 : 12, kThreads = 32 * kWarps;
  // Groups of 16 tokens in a unit: more of them share the row maxima and leave longer tails.  With 128 channels and 8 rows a
  // decode step of 64 requests takes 46 us with two, 42 with three, 44 with four; with 16 rows, 64 requests of 1,000 and 4,096
  // tokens take 38 and 106 us with two, 39 and 92 with three, 45 and 89 with four.
  static constexpr int kGroups = D == 256 ? 2 : D == 64 && NT == 1 ? 6 : 3;
  static constexpr int kTok = kGroups * kGroup;
  static constexpr int kBytes = kGroups * kv4_group_bytes(D);  // of a stage
  static constexpr int kStages = D == 64 && NT == 2 ? 4 : 2;
  static constexpr int kPart = kRows * D + 2 * kRows;        // floats of a part: sums, maxima, totals
};

// An item's first unit moves nothing: it stands for what an item costs besides its tokens, so that
// short requests, which have many items to a token, are dealt out evenly too.
//
// What one request is for the kernel: its first query row, tokens, queries, the first token any query sees (to 16), units of an item, row tiles.
struct Req {
  int64_t q0;
  int32_t n, n_q, lo, tiles, row_tiles, heads;  // a request without tokens is one item for all heads
};
template <int kTok, int kRows>
__device__ __forceinline__ Req request(const AttnArgs &a, int b, int32_t over) {
  Req r;
  const int64_t q0 = a.off[b], q1 = a.off[b + 1];
  int32_t n = a.len[b];
  int64_t m = q1 - q0;
  if (!length_ok(a, n)) {
    flag_error(a.status, MAPS_E_RANGE);
    n = 0;
  }
  if (q0 < 0 || m < 0 || q1 > a.T) {
    flag_error(a.status, MAPS_E_RANGE);
    m = 0;
  }
  r.q0 = q0;
  r.n = n;
  r.n_q = static_cast<int32_t>(m);
  int64_t lo = 0;
  if (a.window > 0) lo = static_cast<int64_t>(n) - m - a.window + 1;
  r.lo = lo > 0 ? static_cast<int32_t>(lo) / kGroup * kGroup : 0;
  const int32_t span = r.n - r.lo;
  r.tiles = (span + kTok - 1) / kTok + 1;
  r.row_tiles = static_cast<int32_t>((m * (a.Hq / a.Hkv) + kRows - 1) / kRows);
  r.heads = a.Hkv;
  if (n == 0) r.heads = 1, r.row_tiles = m > 0 ? 1 : 0;
  if (n > 0 && over > 0 && m * (a.Hq / a.Hkv) > over) r.row_tiles = 0;  // the other form's
  return r;
}

// A place in the list of units: unit `tile` of the item (request b, KV head h, row tile rt).
struct Cursor {
  int32_t b, h, rt, tile;
  Req r;
  template <int kTok, int kRows>
  __device__ __forceinline__ void next_item(const AttnArgs &a, int32_t over) {
    tile = 0;
    if (++rt < r.row_tiles) return;
    rt = 0;
    if (++h < r.heads) return;
    h = 0;
    do {
      if (++b >= a.B) return;
      r = request<kTok, kRows>(a, b, over);
    } while (r.row_tiles == 0);
  }
};

// A place as the request and the units of it that lie before.
struct Start {
  Req r;
  int32_t b;
  uint32_t rest;
  __device__ __forceinline__ Cursor cursor() const {
    Cursor c;
    const uint32_t item = rest / r.tiles;
    c.b = b;
    c.tile = static_cast<int32_t>(rest - item * r.tiles);
    c.h = static_cast<int32_t>(item / r.row_tiles);
    c.rt = static_cast<int32_t>(item - static_cast<uint32_t>(c.h) * r.row_tiles);
    c.r = r;
    return c;
  }
};

// Sums the units of all requests, kN threads a run of them each, and leaves where the workers
// w0 .. w1 - 1 start; returns the units.  put(w, start) keeps a worker's.
template <int kTok, int kRows, int kN, class Put>
__device__ __forceinline__ uint32_t plan(const AttnArgs &a, int32_t over, uint32_t workers, uint32_t w0, uint32_t w1, Put put) {
  __shared__ uint64_t s_warp[kN / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int run = (a.B + kN - 1) / kN, b0 = min(tid * run, a.B), b1 = min(b0 + run, a.B);
  auto units_of = [&](const Req &r) { return static_cast<uint64_t>(r.tiles) * r.row_tiles * r.heads; };
  Req r = {};
  uint64_t mine = 0;
  for (int b = b0; b < b1; ++b) {
    r = request<kTok, kRows>(a, b, over);
    mine += units_of(r);
  }
  uint64_t x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  uint64_t at = x - mine, U = 0;
#pragma unroll
  for (int w = 0; w < kN / 32; ++w) {
    const uint64_t y = s_warp[w];
    if (w < warp) at += y;
    U += y;
  }
  if (U >= 1ull << 31) {  // more than one call's worth of work
    if (tid == 0) flag_error(a.status, MAPS_E_RANGE);
    return 0;
  }
  const Deal deal(static_cast<uint32_t>(U), workers);
  for (int b = b0; b < b1; ++b) {
    if (run > 1) r = request<kTok, kRows>(a, b, over);
    const uint32_t lo = static_cast<uint32_t>(at), n = static_cast<uint32_t>(units_of(r));
    at += n;
    if (n == 0 || lo >= deal.start(w1) || lo + n <= deal.start(w0)) continue;
    uint32_t w = max(deal.worker(lo), w0);
    if (deal.start(w) < lo) ++w;
    for (; w < min(w1, deal.used) && deal.start(w) < lo + n; ++w) {
      put(w, Start{r, b, deal.start(w) - lo});
    }
  }
  return static_cast<uint32_t>(U);
}

template <int kTok, int kRows>
__global__ void __launch_bounds__(1024) attn_plan_kernel(const AttnArgs a, uint32_t workers) {
  pdl_prologue();
  const int32_t over = many_over<1024>(a);
  const uint32_t U = plan<kTok, kRows, 1024>(a, over, workers, 0, workers, [&](uint32_t w, const Start &c) { static_cast<Start *>(a.starts)[w] = c; });
  if (threadIdx.x == 0) a.units[0] = U, a.units[1] = static_cast<uint32_t>(over);
}

// Where four channels from d on of row R lie in a part: rows are turned by 16 bytes for every second of them, or the lanes that
// write a part, whose rows differ by two and whose channels by D/8, would meet in two banks.
template <int D>
__device__ __forceinline__ int in_part(int R, int d) { return R * D + ((d + 4 * (R >> 1)) & (D - 1)); }

// Parts joined so far, of kCh channels of a row.
template <int kCh>
struct Sum {
  alignas(16) float num[kCh];
  float top, den;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int c = 0; c < kCh; ++c) num[c] = 0.0f;
    top = -INFINITY, den = 0.0f;
  }
};

// Weights are held relative to the largest weight times value scale seen, so that what enters the
// second product has a largest size; scales count as at least 2^-60 there, so that a weight itself stays finite.
// The largest counts as 2^kBias, near half's end: what is 2^28 times smaller still has 11 bits.
constexpr float kMinLog = -60.0f, kBias = 14.0f;
// A row of one value has scale 0.  It counts with 2^-20 of its zero, or weight times zero would pass the 32-bit range from zeros of 2^54 on.
constexpr float kLeastScale = 9.5367431640625e-7f;

// ---------------------------------------------------------------------------- the kernel
template <class T, int D, int NT>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, 1) attn_few_kernel(const AttnArgs a) {
  using Sh = Shape<D, NT>;
  constexpr int kWarps = Sh::kWarps, kThreads = Sh::kThreads;
  constexpr int kSteps = D / 16, kWords = D / 32, kCh = D / 8;
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t *ring_all = smem;
  float *first_parts = reinterpret_cast<float *>(smem + kWarps * Sh::kStages * Sh::kBytes);
  uint64_t *bars = reinterpret_cast<uint64_t *>(first_parts + kWarps * Sh::kPart);
  __shared__ Part s_part[2 * kWarps];  // a warp's first and last part, where it has them
  __shared__ Start s_start[kWarps];
  __shared__ Part s_open[2];           // items that other blocks have parts of: begun before this block, and in it
  __shared__ uint64_t s_join;          // parts of those that have come to shared memory
  __shared__ int s_block[2][2];        // of those: the first block, and how many where all have brought their parts

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  uint8_t *ring = ring_all + warp * Sh::kStages * Sh::kBytes;
  const uint32_t ring32 = smem_u32(ring), bar32 = smem_u32(bars + warp * Sh::kStages);
  if (lane < Sh::kStages) bar_init(bar32 + 8 * lane, 1);
  if (lane < 2) s_part[2 * warp + lane].tiles = 0;
  if (tid < 2) s_open[tid].tiles = 0;
  if (tid == 0) bar_init(smem_u32(&s_join), 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  pdl_prologue();
  const uint32_t workers = gridDim.x * kWarps, w0 = blockIdx.x * kWarps, me = w0 + warp;
  uint32_t U;
  int32_t over;  // rows from which a request is the other form's
  Start from = {};
  if (a.B <= kMaxLocalB) {
    over = many_over<kThreads>(a);
    U = plan<Sh::kTok, Sh::kRows, kThreads>(a, over, workers, w0, w0 + kWarps, [&](uint32_t w, const Start &c) { s_start[w - w0] = c; });
    __syncthreads();
    from = s_start[warp];
  } else {
    __syncthreads();
    U = a.units[0];
    over = static_cast<int32_t>(a.units[1]);
    if (me < U) from = static_cast<const Start *>(a.starts)[me];
  }
  const Deal deal(U, workers);
  const uint32_t u0 = deal.start(me), u1 = deal.start(me + 1);
  const int group = a.Hq / a.Hkv;
  const float sl2 = a.scale * 1.4426950408889634f, k_sign = a.scale < 0.0f ? -1.0f : 1.0f, k_unit = k_sign * kEven;

  if (u0 < u1) {
    // The loads run ahead of the products by the ring's depth; lanes below kGroups move one group each.
    Cursor ahead = from.cursor(), at = ahead;
    uint32_t issued = u0;
    // the next unit's group of this lane: whether it holds tokens, its block (fetched one step early), its place there and head
    bool mine = false;
    int32_t block = -1, place = 0;
    auto fetch = [&]() {
      const int32_t tok = ahead.r.lo + (ahead.tile - 1) * Sh::kTok + lane * kGroup;
      mine = issued < u1 && lane < Sh::kGroups && tok < ahead.r.n;
      const int32_t grp = tok / kGroup, page = a.block_shift >= 0 ? grp >> a.block_shift : grp / a.block_groups;
      place = ahead.h * a.block_groups + grp - page * a.block_groups;
      if (mine) block = a.table[ahead.b * a.max_blocks + page];
    };
    auto step = [&]() {
      if (issued >= u1) return;
      do {
        ++issued;
        if (++ahead.tile == ahead.r.tiles && issued < u1) ahead.next_item<Sh::kTok, Sh::kRows>(a, over);
      } while (issued < u1 && ahead.tile == 0);
      fetch();
    };
    auto issue = [&](int stage) {
      const bool good = mine && block >= 0 && block < a.n_blocks;
      if (mine && !good) flag_error(a.status, MAPS_E_RANGE);
      const uint32_t n = __popc(__ballot_sync(0xffffffffu, good));
      if (lane == 0) bar_expect(bar32 + 8 * stage, n * kv4_group_bytes(D));
      __syncwarp();
      if (good)
        bulk_load(ring32 + stage * Sh::kBytes + lane * kv4_group_bytes(D), a.cache + (block * a.block_bytes + place * static_cast<int64_t>(kv4_group_bytes(D))),
                  kv4_group_bytes(D), bar32 + 8 * stage);
      step();
    };
    if (ahead.tile == 0)
      step();
    else
      fetch();
#pragma unroll
    for (int s = 0; s < Sh::kStages; ++s) issue(s);

    int stage = 0;
    uint32_t parity = 0;
    bool alive = true;
    for (uint32_t u = u0; u < u1 && alive;) {
      // ---- an item: its queries, as the columns of the first product
      const Req r = at.r;
      const int64_t q0 = r.q0;
      if (r.n == 0) {  // no token: no sums
        for (int i = 0; i < r.n_q; ++i) {
          for (int x = lane; x < a.Hq * (D / 8); x += 32) {
            T *dst = static_cast<T *>(a.out) + (q0 + i) * a.o_row + x / (D / 8) * a.o_head + x % (D / 8) * 8;
            if (a.wide) {
              *reinterpret_cast<uint4 *>(dst) = make_uint4(0, 0, 0, 0);
            } else {
#pragma unroll
              for (int c = 0; c < 8; ++c) dst[c] = Cvt<T>::from(0.0f);
            }
          }
          if (a.lse)
            for (int x = lane; x < a.Hq; x += 32) a.lse[(q0 + i) * a.Hq + x] = -INFINITY;
        }
        if (++u < u1) at.next_item<Sh::kTok, Sh::kRows>(a, over);
        continue;
      }
      const int rows = r.n_q * group;  // n_q * group <= T * Hq fits the checks of the host
      uint32_t qf[NT][kSteps][2];
      float qs[NT][2], qu[NT][2];  // a row's sum, and what a score of it is to be multiplied by
      int32_t row_lo[NT][2], row_hi[NT][2];
      int32_t all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int R = at.rt * Sh::kRows + nt * 8 + g;
        // A row is scaled by a power of two to fill half's range.  Only its smallest channels lose bits: below 2^-31 of the largest
        // (bfloat16) or 2^-28 (half), and the odd ones, which enter divided by 16, below 2^-27 and 2^-24.
        float x[kSteps * 4], top = 0.0f;
        const bool there = R < rows;
        const T *src = static_cast<const T *>(a.q) + (there ? (q0 + R / group) * a.q_row + (at.h * group + R % group) * a.q_head + t * (D / 4) : 0);
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
          uint4 y = make_uint4(0, 0, 0, 0);
          T *z = reinterpret_cast<T *>(&y);
          if (there) {
            if (a.wide) {
              y = *reinterpret_cast<const uint4 *>(src + 8 * i);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) z[e] = src[8 * i + e];
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[8 * i + e] = Cvt<T>::to(z[e]);
            top = fmaxf(top, fabsf(x[8 * i + e]));
          }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int ef = min(max(static_cast<int>(__float_as_uint(top) >> 23), 20), 254);  // top is 2^(ef - 127) or a little more
        const float up = __uint_as_float(static_cast<uint32_t>(268 - ef) << 23);             // makes it 2^14 or a little more
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[8 * i + e] *= up, sum += x[8 * i + e];
          qf[nt][2 * i][0] = pack_half(x[8 * i], x[8 * i + 4]);
          qf[nt][2 * i][1] = pack_half(x[8 * i + 1] * 0.0625f, x[8 * i + 5] * 0.0625f);
          qf[nt][2 * i + 1][0] = pack_half(x[8 * i + 2], x[8 * i + 6]);
          qf[nt][2 * i + 1][1] = pack_half(x[8 * i + 3] * 0.0625f, x[8 * i + 7] * 0.0625f);
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        const float unit = fmaxf(fabsf(sl2) * __uint_as_float(static_cast<uint32_t>(ef - 14) << 23), 1.17549435e-38f);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          qs[nt][e] = __shfl_sync(0xffffffffu, sum, (2 * t + e) * 4);
          qu[nt][e] = __shfl_sync(0xffffffffu, unit, (2 * t + e) * 4);
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

      const uint32_t seg_end = min(u1, u + static_cast<uint32_t>(r.tiles - at.tile));
      const int32_t seg_first = at.tile;
      for (; u < seg_end; ++u, ++at.tile) {
        if (at.tile == 0) continue;
        if (!warp_wait(bar32 + 8 * stage, parity)) {
          if (lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
          alive = false;
          break;
        }
        const uint8_t *buf = ring + stage * Sh::kBytes;
        const int32_t tok0 = r.lo + (at.tile - 1) * Sh::kTok;
        auto unit_sums = [&](auto every) {
          constexpr bool kEvery = decltype(every)::value;  // every row sees every token
          // ---- scores, up to a row's factor: 16 tokens x 8 rows, depth D
          float s[Sh::kGroups][NT][4];
          float vs[Sh::kGroups][2];
          float top[NT][2];  // of score + log2(value scale)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) top[nt][0] = top[nt][1] = -INFINITY;
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
            for (int i = 0; i < kWords; ++i) {
              const Codes x = codes_of(k0[i]), y = codes_of(k1[i]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma(s[gr][nt], x.x[0], y.x[0], x.x[1], y.x[1], qf[nt][2 * i][0], qf[nt][2 * i][1]);
                mma(s[gr][nt], x.x[2], y.x[2], x.x[3], y.x[3], qf[nt][2 * i + 1][0], qf[nt][2 * i + 1][1]);
              }
            }
            const uint32_t *par = reinterpret_cast<const uint32_t *>(grp + 16 * D);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const float2 p = kv4_param(par[g + 8 * half]);
              const float2 v = kv4_param(par[16 + g + 8 * half]);
              vs[gr][half] = v.x;
              const float ks = p.x * k_unit, kz = p.y * k_sign, ls = fmaxf(lg2(fmaxf(v.x, fabsf(v.y) * kLeastScale)), kMinLog);
              const int32_t tok = tok0 + gr * kGroup + g + 8 * half;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  float &x = s[gr][nt][2 * half + e];
                  x = fmaf(ks, x, kz * qs[nt][e]);
                  if (!kEvery && (tok < row_lo[nt][e] || tok >= row_hi[nt][e])) x = -INFINITY;
                  top[nt][e] = fmaxf(top[nt][e], fmaf(x, qu[nt][e], ls));
                }
            }
          }

          // ---- running maximum
          bool grew = false;
          float ref[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float x = top[nt][e];
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
              top[nt][e] = fmaxf(m[nt][e], x);
              grew |= top[nt][e] > m[nt][e];
            }
          if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float c = top[nt][e] == -INFINITY ? 1.0f : ex2(m[nt][e] - top[nt][e]);
                m[nt][e] = top[nt][e];
                l[nt][e] *= c;
                w[nt][e] *= c;
#pragma unroll
                for (int j = 0; j < kSteps; ++j) o[nt][j][e] *= c, o[nt][j][2 + e] *= c;
              }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) ref[nt][e] = kBias - (m[nt][e] == -INFINITY ? 0.0f : m[nt][e]);

          // ---- weights and sums over the values
#pragma unroll
          for (int gr = 0; gr < Sh::kGroups; ++gr) {
            const uint8_t *grp = buf + gr * kv4_group_bytes(D);
            const uint32_t *par = reinterpret_cast<const uint32_t *>(grp + 16 * D) + 16;
            uint32_t pf[NT][2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const float vz = fmaf(Value<T>::kCentre, vs[gr][half], kv4_param(par[g + 8 * half]).y);
              const int32_t tok = tok0 + gr * kGroup + g + 8 * half;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                float ps[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  const float x = ex2(fmaf(s[gr][nt][2 * half + e], qu[nt][e], ref[nt][e]));
                  l[nt][e] += x;
                  // a token that the row does not see has weight 0, and whatever its scale is stays out
                  const bool out = !kEvery && (tok < row_lo[nt][e] || tok >= row_hi[nt][e]);
                  ps[e] = out ? 0.0f : x * vs[gr][half];
                  w[nt][e] = out ? w[nt][e] : fmaf(x, vz, w[nt][e]);
                }
                pf[nt][half] = transpose8(pack_half(ps[0], ps[1]));
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
            for (int i = 0; i < kWords; ++i) {
              const Codes x = Value<T>::of(v0[i]), y = Value<T>::of(v1[i]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma(o[nt][2 * i], x.x[0], x.x[1], y.x[0], y.x[1], pf[nt][0], pf[nt][1]);
                mma(o[nt][2 * i + 1], x.x[2], x.x[3], y.x[2], y.x[3], pf[nt][0], pf[nt][1]);
              }
            }
          }
        };
        if (tok0 >= all_lo && tok0 + Sh::kTok <= all_hi)
          unit_sums(Yes{});
        else
          unit_sums(No{});
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
              y[2 * j] = Cvt<T>::from(fmaf(o[nt][j][e], Value<T>::kEvenBy, add) * inv);
              y[2 * j + 1] = Cvt<T>::from(fmaf(o[nt][j][2 + e], Value<T>::kOddBy, add) * inv);
            }
            if (a.wide) {
#pragma unroll
              for (int c = 0; c < kCh; c += 8) *reinterpret_cast<uint4 *>(dst + c) = *reinterpret_cast<const uint4 *>(y + c);
            } else {
#pragma unroll
              for (int c = 0; c < kCh; ++c) dst[c] = y[c];
            }
            if (a.lse && g == 0) a.lse[i * a.Hq + hq] = l[nt][e] == 0.0f ? -INFINITY : (m[nt][e] - kBias + log2f(l[nt][e])) * 0.6931471805599453f;
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
#pragma unroll
            for (int j = 0; j < kSteps; j += 2)
              *reinterpret_cast<float4 *>(part + in_part<D>(R, g * kCh + 2 * j)) =
                  make_float4(fmaf(o[nt][j][e], Value<T>::kEvenBy, w[nt][e]), fmaf(o[nt][j][2 + e], Value<T>::kOddBy, w[nt][e]),
                              fmaf(o[nt][j + 1][e], Value<T>::kEvenBy, w[nt][e]), fmaf(o[nt][j + 1][2 + e], Value<T>::kOddBy, w[nt][e]));
            if (g == 0) {
              part[Sh::kRows * D + R] = m[nt][e] - kBias;
              part[Sh::kRows * D + Sh::kRows + R] = l[nt][e];
            }
          }
        if (lane == 0) s_part[slot] = {q0, u - at.tile, static_cast<uint32_t>(r.tiles), rows, at.h, at.rt};  // at.tile units of the item lie before u
      }
      if (u < u1) at.next_item<Sh::kTok, Sh::kRows>(a, over);
    }
    if (!alive) {  // let what is under way land before the block ends
      for (int s = 0; s < Sh::kStages; ++s) (void)bar_wait(bar32 + 8 * s, s < stage ? parity ^ 1 : parity);
    }
  }
  __syncthreads();

  // ---- join the parts of the block's items, in the order of their keys
  const uint32_t c0 = deal.start(w0), c1 = deal.start(w0 + kWarps);
  auto write_row = [&](const Part &p, int R, int d, const auto &s) {
    constexpr int kN = sizeof(s.num) / 4;
    const int row = p.rt * Sh::kRows + R;
    if (row >= p.rows) return;
    const int64_t i = p.q0 + row / group;
    const int hq = p.h * group + row % group;
    const float inv = s.den == 0.0f ? 0.0f : 1.0f / s.den;
    T *dst = static_cast<T *>(a.out) + i * a.o_row + hq * a.o_head + d;
    alignas(16) T y[kN];
#pragma unroll
    for (int c = 0; c < kN; ++c) y[c] = Cvt<T>::from(s.num[c] * inv);
    if (a.wide) {
      if (kN == 8)
        *reinterpret_cast<uint4 *>(dst) = *reinterpret_cast<const uint4 *>(y);
      else
        *reinterpret_cast<uint2 *>(dst) = *reinterpret_cast<const uint2 *>(y);
    } else {
#pragma unroll
      for (int c = 0; c < kN; ++c) dst[c] = y[c];
    }
    if (d == 0 && a.lse) a.lse[i * a.Hq + hq] = s.den == 0.0f ? -INFINITY : (s.top + log2f(s.den)) * 0.6931471805599453f;
  };
  // Sums the parts lo .. hi - 1, which lie in shared memory, into `s`, four channels from x on, brought to their common maximum.
  auto add_parts = [&](auto &s, int x, int lo, int hi, auto part) {
    constexpr int kN = sizeof(s.num) / 4;
    const int R = x / D, d = x - R * D;
    for (int k = lo; k < hi; k += 2) {
      alignas(16) float v[2][kN];
      float mk[2], lk[2], top = s.top;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float *p = part(min(k + j, hi - 1));  // beyond the last: read again, and left out
#pragma unroll
        for (int c = 0; c < kN; c += 4) *reinterpret_cast<float4 *>(v[j] + c) = *reinterpret_cast<const float4 *>(p + in_part<D>(R, d + c));
        mk[j] = p[Sh::kRows * D + R];
        lk[j] = p[Sh::kRows * D + Sh::kRows + R];
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) top = fmaxf(top, mk[j]);
      const float c = top == -INFINITY ? 1.0f : ex2(s.top - top);
#pragma unroll
      for (int i = 0; i < kN; ++i) s.num[i] *= c;
      s.den *= c;
      s.top = top;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (k + j >= hi) break;
        const float f = top == -INFINITY ? 0.0f : ex2(mk[j] - top);
#pragma unroll
        for (int i = 0; i < kN; ++i) s.num[i] = fmaf(f, v[j][i], s.num[i]);
        s.den = fmaf(f, lk[j], s.den);
      }
    }
  };
  // within the block: the warps that have parts of an item share its channels
  for (int slot = 2 * warp; slot < 2 * warp + 2; ++slot) {
    const Part item = s_part[slot];
    if (item.tiles == 0) continue;
    const bool whole = item.id >= c0 && item.id + item.tiles <= c1;
    const int first = item.id < c0 ? 0 : static_cast<int>(deal.worker(item.id) - w0);
    const int last = item.id + item.tiles > c1 ? kWarps - 1 : static_cast<int>(deal.worker(item.id + item.tiles - 1) - w0);
    const float *head = item.id <= deal.start(w0 + first) ? first_parts + first * Sh::kPart : reinterpret_cast<const float *>(ring_all + first * Sh::kStages * Sh::kBytes);
    float *mine = a.parts + (static_cast<int64_t>(blockIdx.x) * 2 + (item.id < c0 ? 0 : 1)) * Sh::kPart;
    for (int x = 8 * (lane + 32 * (warp - first)); x < Sh::kRows * D; x += 8 * 32 * (last - first + 1)) {
      Sum<8> sum;
      sum.clear();
      add_parts(sum, x, 0, last - first + 1, [&](int k) { return k == 0 ? head : first_parts + (first + k) * Sh::kPart; });
      const int R = x / D, d = x - R * D;
      if (whole) {
        write_row(item, R, d, sum);
      } else {
#pragma unroll
        for (int c = 0; c < 8; c += 4) *reinterpret_cast<float4 *>(mine + in_part<D>(R, d + c)) = *reinterpret_cast<const float4 *>(sum.num + c);
        if (d == 0) mine[Sh::kRows * D + R] = sum.top, mine[Sh::kRows * D + Sh::kRows + R] = sum.den;
      }
    }
    if (!whole) {
      if (warp == first && lane == 0) s_open[item.id < c0 ? 0 : 1] = item;
      __threadfence();
    }
  }
  // across blocks: the last to bring its part joins them all
  __syncthreads();
  if (tid < 2 && s_open[tid].tiles) {
    const Part item = s_open[tid];
    const uint32_t f = deal.worker(item.id) / kWarps, e = deal.worker(item.id + item.tiles - 1) / kWarps;
    const int shift = static_cast<int>(f & 3) * 8;
    const uint32_t others = atom_add_acq_rel_u32(&a.arrived[f >> 2], 1u << shift) >> shift & 255u;
    const bool all = others == e - f;
    if (all) atomicSub(&a.arrived[f >> 2], (e - f + 1) << shift);  // zero again for the next call
    s_block[tid][0] = static_cast<int>(f);
    s_block[tid][1] = all ? static_cast<int>(e - f + 1) : 0;
  }
  __syncthreads();
  // Their parts come to shared memory, those of both items at once where they fit: a part then costs no round trip of its own.
  const int n0 = s_open[0].tiles ? s_block[0][1] : 0, n = n0 + (s_open[1].tiles ? s_block[1][1] : 0);
  if (n == 0) return;
  __threadfence();
  asm volatile("fence.proxy.async;" ::: "memory");  // what others wrote with plain stores, and this block in shared memory
  __syncthreads();
  constexpr int kRoom = Sh::kWarps * (Sh::kStages * Sh::kBytes / (Sh::kPart * 4) + 1), kTurns = (Sh::kRows * D / 4 + kThreads - 1) / kThreads;
  static_assert(kRoom <= kThreads, "a thread loads a part at most");
  const float *parts = reinterpret_cast<const float *>(smem);
  const uint32_t joined = smem_u32(&s_join);
  Sum<4> sum[kTurns];
  for (int p0 = 0; p0 < n; p0 += kRoom) {
    const int p1 = min(n, p0 + kRoom);
    if (tid == 0) bar_expect(joined, (p1 - p0) * Sh::kPart * 4);
    if (tid < p1 - p0) {
      const int k = p0 + tid >= n0 ? 1 : 0, c = p0 + tid - k * n0;
      bulk_load(smem_u32(parts + tid * Sh::kPart), a.parts + (static_cast<int64_t>(s_block[k][0] + c) * 2 + (c == 0)) * Sh::kPart, Sh::kPart * 4, joined);
    }
    if (!bar_wait(joined, p0 / kRoom & 1) && tid == 0) flag_error(a.status, MAPS_E_TIMEOUT);
    for (int k = 0; k < 2; ++k) {
      const int lo = k ? n0 : 0, hi = k ? n : n0, from = max(lo, p0), to = min(hi, p1);
      if (from >= to) continue;
      const Part item = s_open[k];
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int x = 4 * (tid + i * kThreads);
        if (x >= Sh::kRows * D) break;
        if (from == lo) sum[i].clear();
        add_parts(sum[i], x, from - p0, to - p0, [&](int c) { return parts + c * Sh::kPart; });
        if (to == hi) write_row(item, x / D, x % D, sum[i]);
      }
    }
    if (p1 < n) __syncthreads();  // the room is read before it is filled again
  }
}

constexpr int kMaxParts = 16 * 128 + 32;  // floats of the largest part (two row tiles of 128 channels, or one of 256)
// The counters of arrivals lie in the control block, behind the status word: calls that share a
// workspace leave that zero, and so does this one.
constexpr int kArrivedAt = 64;

template <class T, int D, int NT>
int launch_few(const AttnArgs &a, cudaStream_t s) {
  using Sh = Shape<D, NT>;
  constexpr int kWarps = Sh::kWarps, kThreads = Sh::kThreads;
  const size_t smem = static_cast<size_t>(kWarps) * Sh::kStages * Sh::kBytes + static_cast<size_t>(kWarps) * Sh::kPart * 4 + kWarps * Sh::kStages * 8;
  constexpr auto kernel = attn_few_kernel<T, D, NT>;
  MAPS_TRY(allow_smem<kernel>(smem));
  if (a.B > kMaxLocalB) launch_pdl(attn_plan_kernel<Sh::kTok, Sh::kRows>, 1, 1024, 0, s, a, static_cast<uint32_t>(attn_grid() * kWarps));
  launch_pdl(kernel, static_cast<unsigned>(attn_grid()), kThreads, smem, s, a);
  return launch_ok();
}

template <class T>
int launch_dim(int D, const AttnArgs &a, cudaStream_t s) {
  // 8 rows to a tile where a request has at most 8 on average, else 16: for 16 rows two tiles of 8 pass over the cache twice
  // (64 requests of 4,096 tokens, 128 channels: 112 us, 92 with one of 16; 1,000 tokens: 40, 39), for 8 a tile of 16 is half
  // empty (65, 89).  256 channels of 16 rows do not fit a warp's registers.
  const bool one = a.T * (a.Hq / a.Hkv) <= static_cast<int64_t>(8) * a.B;
  if (D == 64) return one ? launch_few<T, 64, 1>(a, s) : launch_few<T, 64, 2>(a, s);
  if (D == 128) return one ? launch_few<T, 128, 1>(a, s) : launch_few<T, 128, 2>(a, s);
  return launch_few<T, 256, 1>(a, s);
}

}  // namespace
}  // namespace maps

extern "C" {

static void carve(maps::Carve &c, maps::AttnArgs &a, int32_t B, int64_t T, int32_t Hq, int32_t Hkv, int32_t D) {
  using namespace maps;
  a.parts = c.take<float>(static_cast<size_t>(attn_grid()) * 2 * kMaxParts);
  a.starts = c.take<Start>(B > kMaxLocalB ? static_cast<size_t>(attn_grid()) * kMaxWarps : 0);
  a.units = c.take<uint32_t>(2);
  // A decode step has as many rows as requests and spends no launches on the other form; so has a batch of fewer rows than
  // requests, whose chunks, where it has any, are served here too.
  a.few_rows = Hkv > 0 && attn_many_dim(D) && T > B && T * (Hq / Hkv) > kFewRows ? kFewRows : 0;
  if (a.few_rows) attn_many_carve(c, a, B, D);
}

size_t maps_kv4_attention_workspace_size(int32_t B, int64_t T, int32_t Hq, int32_t Hkv, int32_t D) {
  maps::Carve c(nullptr);
  maps::AttnArgs a = {};
  carve(c, a, B, T, Hq, Hkv, D);
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
      T > ((int64_t(1) << 31) - 1024) / Hq || max_blocks < 0 || max_blocks > 0x7fffffff || n_blocks < 0 || window < 0 ||
      (causal != 0 && causal != 1) || !(sm_scale - sm_scale == 0.0f))
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, maps_kv4_attention_workspace_size(B, T, Hq, Hkv, D)));
  if (T == 0 || B == 0) return MAPS_OK;
  if (q == nullptr || out == nullptr || qo_off == nullptr || kv_len == nullptr ||
      (max_blocks > 0 && table == nullptr) || (n_blocks > 0 && cache == nullptr) || !aligned(cache, 16) || !aligned(q, 2) ||
      !aligned(lse, 4) || !aligned(out, 2))
    return MAPS_E_INVALID;
  const bool wide = aligned(q, 16) && aligned(out, 16) && q_row % 8 == 0 && q_head % 8 == 0 && o_row % 8 == 0 && o_head % 8 == 0;
  const int32_t groups = S / kGroup;
  int32_t shift = -1;
  for (int32_t i = 0; i < 16; ++i)
    if (groups == 1 << i) shift = i;
  AttnArgs a = {B, Hq, Hkv, S, T, n_blocks, max_blocks, q, q_row, q_head, o_row, o_head, qo_off, kv_len, table,
                static_cast<const uint8_t *>(cache), sm_scale, causal, window, wide,
                static_cast<int64_t>(Hkv) * groups * kv4_group_bytes(D), groups, shift, out, lse};
  a.arrived = reinterpret_cast<uint32_t *>(static_cast<char *>(ws) + kArrivedAt);
  a.status = status_word(ws);
  Carve c(ws);
  carve(c, a, B, T, Hq, Hkv, D);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  MAPS_TRY(dtype == MAPS_BF16 ? launch_dim<__nv_bfloat16>(D, a, s) : launch_dim<__half>(D, a, s));
  return a.few_rows ? attn_many(dtype, D, a, s) : MAPS_OK;
}

}  // extern "C"
