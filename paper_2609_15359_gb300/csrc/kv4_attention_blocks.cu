// kv4_attention_blocks.cu -- attention over the 4-bit cache where each query row and KV head has a list of blocks.
//
// The mathematics is that of the form for few queries (kv4_attention.cu): both products on bare codes in transposed m16n8k16
// steps, the running maximum and sum of the softmax, weights relative to the largest weight times scale.
//
// Split.  Lists have much the same length, so no run crosses from one to the next: four warps have an item, which is a row, KV head
// and tile of 8 or 16 of the head's query heads, and take its units of 32 to 64 tokens in turn; two to four items pass on a multiprocessor
// side by side.  Where items are few, and for the last ones that do not fill the device, a cluster of such blocks shares one.  Parts meet
// in shared memory, the block's and then the cluster's, in the order of the warps: no workspace, and results that depend on sizes and
// lengths alone.  (Equal runs of units over all lists, as behind block tables, cost a plan, parts in memory and joins across blocks: 66 us
// for 53 in the case below, 11.8 for 6.1 with one row.)
//
// Bound: 128 rows of 2,048 tokens, 8 KV heads of 128 channels, 285 MB, take 53.0 us (5.4 TB/s, 0.80 of the measured copy rate), the rest
// what a list costs before its first unit and after its last.  One row: 6.1 us, launch, three rounds of loads, a unit, two joins.  Lists of
// 64 channels and five query heads: issue slots, 210 instructions for 16 tokens.
#include "kv4_attention_products.cuh"

namespace maps {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kMaxCluster = 8;  // one row of 8 heads: 6.2 us, with 16 blocks 7.5, with four 7.2, with two 9.3

// Test aid (maps_test_attention_withhold), for a device: the block that never learns that its copies have landed, plus 1, and the
// tries after which a wait gives up (0: as by default).  They come with the call's arguments: in constant memory of their own the first
// look at them cost 0.2 us a block.
struct Withheld {
  std::atomic<int32_t> block{0};
  std::atomic<uint32_t> tries{0};
};
Withheld g_withheld[64];

struct ListArgs {
  int32_t Hq, H, group, tiles;  // query heads to a KV head, and tiles of them
  int32_t block_groups, block_shift;  // groups of a block, and their logarithm where they are a power of two, else -1
  int64_t n_list, n_blocks, block_bytes;
  int32_t S, wide;
  int32_t withheld;
  uint32_t tries;
  uint32_t single, cluster;  // items of one block each, the first; of a cluster's blocks, the rest
  const void *q;
  int64_t q_row, q_head, o_row, o_head;
  const int32_t *blocks, *tokens;
  const uint8_t *cache;
  float scale;
  void *out;
  float *lse;
  int32_t *status;
};

template <int D, int NT>
struct ListShape {
  static constexpr int kRows = 8 * NT;  // query rows of a tile
  // Groups of 16 tokens in a unit, which shares the row maxima: 128 rows of 128 channels with four 52.6 us, three 55.6, two 60; of 256
  // channels with two 19.7, one 33, three 21.
  static constexpr int kGroups = D == 256 ? 2 : NT == 1 ? 4 : 3;
  static constexpr int kTok = kGroups * kGroup;
  static constexpr int kBytes = kGroups * kv4_group_bytes(D);  // of a stage
  static constexpr int kStages = D == 64 && NT == 2 ? 4 : 2;
  static constexpr int kPart = kRows * D + 2 * kRows;  // floats of a part: sums, maxima, totals
  static constexpr int kBlocks = NT == 2 || D == 256 ? 2 : D == 64 ? 4 : 3;  // of a multiprocessor, as registers allow (64 channels: four 40.5 us, three 42.2)
  static constexpr size_t kSmem = static_cast<size_t>(kWarps) * kStages * kBytes + kPart * 4 + kWarps * kStages * 8;
  static_assert(kPart * 4 <= kStages * kBytes, "a warp's part lies in its ring");
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ const float *of_block(const float *p, int rank) {  // the same place in another block of the cluster
  uint64_t y;
  asm("mapa.u64 %0, %1, %2;" : "=l"(y) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
  return reinterpret_cast<const float *>(y);
}

template <class T, int D, int NT>
__global__ void __launch_bounds__(kThreads, ListShape<D, NT>::kBlocks) attn_lists_kernel(const ListArgs a) {
  using Sh = ListShape<D, NT>;
  constexpr int kSteps = D / 16, kWords = D / 32, kCh = D / 8;
  extern __shared__ __align__(128) uint8_t smem[];
  float *joined = reinterpret_cast<float *>(smem + kWarps * Sh::kStages * Sh::kBytes);  // the block's part
  uint64_t *bars = reinterpret_cast<uint64_t *>(joined + Sh::kPart);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  uint8_t *ring = smem + warp * Sh::kStages * Sh::kBytes;
  const uint32_t ring32 = smem_u32(ring), bar32 = smem_u32(bars + warp * Sh::kStages);
  if (lane < Sh::kStages) bar_init(bar32 + 8 * lane, static_cast<int>(blockIdx.x) == a.withheld ? 2 : 1);  // of two arrivals one never comes
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();
  pdl_prologue();

  const bool shared = blockIdx.x >= a.single;
  const uint32_t past = blockIdx.x - a.single, cluster = shared ? a.cluster : 1, rank = shared ? past % a.cluster : 0;
  const uint32_t item = shared ? a.single + past / a.cluster : blockIdx.x, list = item / a.tiles;
  const int tile = static_cast<int>(item - list * a.tiles), h = static_cast<int>(list % a.H);
  const int64_t i = list / a.H;
  const int head0 = h * a.group + tile * Sh::kRows, rows = min(Sh::kRows, a.group - tile * Sh::kRows);  // the tile's query heads
  // Worker w has the units w, w + workers, ...: so its first blocks are looked up, and the queries are under way, before the list's length is known.
  const int32_t workers = static_cast<int32_t>(cluster) * kWarps, me = static_cast<int32_t>(rank) * kWarps + warp;
  const int32_t *blocks = a.blocks + static_cast<int64_t>(list) * a.n_list;
  int32_t ahead = me * Sh::kGroups + lane;  // the group that this lane moves next
  int32_t block = -1, place = 0;
  auto fetch = [&]() {
    const int32_t page = a.block_shift >= 0 ? ahead >> a.block_shift : ahead / a.block_groups;
    place = ahead - page * a.block_groups;
    if (lane < Sh::kGroups && page < a.n_list) block = blocks[page];
  };
  fetch();
  uint4 raw[NT][kWords];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int R = nt * 8 + g;
    const T *src = static_cast<const T *>(a.q) + i * a.q_row + (head0 + min(R, rows - 1)) * a.q_head + t * (D / 4);
#pragma unroll
    for (int x = 0; x < kWords; ++x) {
      if (a.wide) {
        raw[nt][x] = *reinterpret_cast<const uint4 *>(src + 8 * x);
      } else {
        T *z = reinterpret_cast<T *>(&raw[nt][x]);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = src[8 * x + e];
      }
    }
  }
  int32_t n = a.tokens[list];
  if (n < 0) return;  // nobody's row
  if (n > a.n_list * a.S) {
    if (tid == 0) flag_error(a.status, MAPS_E_RANGE);
    n = 0;
  }
  T *out = static_cast<T *>(a.out) + i * a.o_row + head0 * a.o_head;
  float *lse = a.lse ? a.lse + i * a.Hq + head0 : nullptr;
  auto put = [&](T *dst, const auto &y) {
    constexpr int kN = sizeof(y) / sizeof(T);
    if (a.wide) {
      if (kN == 8)
        *reinterpret_cast<uint4 *>(dst) = *reinterpret_cast<const uint4 *>(&y);
      else
        *reinterpret_cast<uint2 *>(dst) = *reinterpret_cast<const uint2 *>(&y);
    } else {
#pragma unroll
      for (int c = 0; c < kN; ++c) dst[c] = y[c];
    }
  };
  if (n == 0) {  // no token: no sums
    if (rank > 0) return;
    alignas(16) T zero[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) zero[c] = Cvt<T>::from(0.0f);
    for (int x = tid; x < rows * (D / 8); x += kThreads) put(out + x / (D / 8) * a.o_head + x % (D / 8) * 8, zero);
    if (lse && tid < rows) lse[tid] = -INFINITY;
    return;
  }
  // ---- this warp's units
  const int32_t groups = (n + kGroup - 1) / kGroup, all = (groups + Sh::kGroups - 1) / Sh::kGroups, units = all > me ? (all - me + workers - 1) / workers : 0;
  const uint8_t *cache = a.cache + static_cast<int64_t>(h) * a.block_groups * kv4_group_bytes(D);
  auto issue = [&](int stage) {
    const bool mine = lane < Sh::kGroups && ahead < groups, good = mine && block >= 0 && block < a.n_blocks;
    if (mine && !good) flag_error(a.status, MAPS_E_RANGE);
    const uint32_t count = __popc(__ballot_sync(0xffffffffu, good));
    if (lane == 0) bar_expect(bar32 + 8 * stage, count * kv4_group_bytes(D));
    __syncwarp();
    if (good)
      bulk_load(ring32 + stage * Sh::kBytes + lane * kv4_group_bytes(D), cache + (block * a.block_bytes + place * static_cast<int64_t>(kv4_group_bytes(D))),
                kv4_group_bytes(D), bar32 + 8 * stage);
    ahead += workers * Sh::kGroups;
    if (ahead < groups) fetch();
  };

  // ---- the queries, as the columns of the first product
  const float sl2 = a.scale * 1.4426950408889634f, k_sign = a.scale < 0.0f ? -1.0f : 1.0f, k_unit = k_sign * kEven;
#pragma unroll
  for (int s = 0; s < Sh::kStages; ++s)
    if (s < units) issue(s);
  uint32_t qf[NT][kSteps][2];
  float qs[NT][2], qu[NT][2];  // a row's sum, and what a score of it is to be multiplied by
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    // A row is scaled by a power of two to fill half's range.  Only its smallest channels lose bits: below 2^-31 of the largest
    // (bfloat16) or 2^-28 (half), and the odd ones, which enter divided by 16, below 2^-27 and 2^-24.
    float x[kSteps * 4], top = 0.0f;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      const T *z = reinterpret_cast<const T *>(&raw[nt][k]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[8 * k + e] = nt * 8 + g < rows ? Cvt<T>::to(z[e]) : 0.0f;
        top = fmaxf(top, fabsf(x[8 * k + e]));
      }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int ef = min(max(static_cast<int>(__float_as_uint(top) >> 23), 20), 254);  // top is 2^(ef - 127) or a little more
    const float up = __uint_as_float(static_cast<uint32_t>(268 - ef) << 23);             // makes it 2^14 or a little more
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[8 * k + e] *= up, sum += x[8 * k + e];
      qf[nt][2 * k][0] = pack_half(x[8 * k], x[8 * k + 4]);
      qf[nt][2 * k][1] = pack_half(x[8 * k + 1] * 0.0625f, x[8 * k + 5] * 0.0625f);
      qf[nt][2 * k + 1][0] = pack_half(x[8 * k + 2], x[8 * k + 6]);
      qf[nt][2 * k + 1][1] = pack_half(x[8 * k + 3] * 0.0625f, x[8 * k + 7] * 0.0625f);
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    const float unit = fmaxf(fabsf(sl2) * __uint_as_float(static_cast<uint32_t>(ef - 14) << 23), 1.17549435e-38f);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      qs[nt][e] = __shfl_sync(0xffffffffu, sum, (2 * t + e) * 4);
      qu[nt][e] = __shfl_sync(0xffffffffu, unit, (2 * t + e) * 4);
    }
  }

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

  int stage = 0;
  uint32_t parity = 0;
  bool landed = true;  // nothing of this warp's is under way
  for (int32_t u = 0; u < units; ++u) {
    if (!warp_wait(bar32 + 8 * stage, parity, a.tries)) {
      if (lane == 0) flag_error(a.status, MAPS_E_TIMEOUT);
      // the copies of this unit and of the next ones that the ring holds land before the block ends; the others' stages wait for nothing
      for (int k = 0; k < Sh::kStages && u + k < units; ++k) {
        const bool wrapped = stage + k >= Sh::kStages;
        landed &= warp_wait(bar32 + 8 * (stage + k - (wrapped ? Sh::kStages : 0)), parity ^ (wrapped ? 1u : 0u), a.tries);
      }
      break;
    }
    const uint8_t *buf = ring + stage * Sh::kBytes;
    const int32_t tok0 = (me + u * workers) * Sh::kTok;
    auto unit_sums = [&](auto every) {
      constexpr bool kEvery = decltype(every)::value;  // every place holds a token
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
          for (int x = 0; x < kWords; x += 4) {
            *reinterpret_cast<uint4 *>(k0 + x) = *reinterpret_cast<const uint4 *>(grp + g * (D / 2) + t * (D / 8) + 4 * x);
            *reinterpret_cast<uint4 *>(k1 + x) = *reinterpret_cast<const uint4 *>(grp + (g + 8) * (D / 2) + t * (D / 8) + 4 * x);
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[gr][nt][e] = 0.0f;
#pragma unroll
        for (int x = 0; x < kWords; ++x) {
          const Codes c0 = codes_of(k0[x]), c1 = codes_of(k1[x]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma(s[gr][nt], c0.x[0], c1.x[0], c0.x[1], c1.x[1], qf[nt][2 * x][0], qf[nt][2 * x][1]);
            mma(s[gr][nt], c0.x[2], c1.x[2], c0.x[3], c1.x[3], qf[nt][2 * x + 1][0], qf[nt][2 * x + 1][1]);
          }
        }
        const uint32_t *par = reinterpret_cast<const uint32_t *>(grp + 16 * D);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const float2 p = kv4_param(par[g + 8 * half]);
          const float2 v = kv4_param(par[16 + g + 8 * half]);
          vs[gr][half] = v.x;
          const float ks = p.x * k_unit, kz = p.y * k_sign, ls = fmaxf(lg2(fmaxf(v.x, fabsf(v.y) * kLeastScale)), kMinLog);
          const bool out_of = !kEvery && tok0 + gr * kGroup + g + 8 * half >= n;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float &x = s[gr][nt][2 * half + e];
              x = fmaf(ks, x, kz * qs[nt][e]);
              if (out_of) x = -INFINITY;
              top[nt][e] = fmaxf(top[nt][e], out_of ? -INFINITY : fmaf(x, qu[nt][e], ls));
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
          const bool out_of = !kEvery && tok0 + gr * kGroup + g + 8 * half >= n;  // its weight is 0, and its scale, whatever it is, stays out
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float ps[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float x = ex2(fmaf(s[gr][nt][2 * half + e], qu[nt][e], ref[nt][e]));
              l[nt][e] += x;
              ps[e] = out_of ? 0.0f : x * vs[gr][half];
              w[nt][e] = out_of ? w[nt][e] : fmaf(x, vz, w[nt][e]);
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
          for (int x = 0; x < kWords; x += 4) {
            *reinterpret_cast<uint4 *>(v0 + x) = *reinterpret_cast<const uint4 *>(vb + x / 4 * 512 + lane * 16);
            *reinterpret_cast<uint4 *>(v1 + x) = *reinterpret_cast<const uint4 *>(vb + (kWords + x) / 4 * 512 + lane * 16);
          }
        }
#pragma unroll
        for (int x = 0; x < kWords; ++x) {
          const Codes c0 = Value<T>::of(v0[x]), c1 = Value<T>::of(v1[x]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma(o[nt][2 * x], c0.x[0], c0.x[1], c1.x[0], c1.x[1], pf[nt][0], pf[nt][1]);
            mma(o[nt][2 * x + 1], c0.x[2], c0.x[3], c1.x[2], c1.x[3], pf[nt][0], pf[nt][1]);
          }
        }
      }
    };
    if (tok0 + Sh::kTok <= n)
      unit_sums(Yes{});
    else
      unit_sums(No{});
    __syncwarp();  // the stage has been read
    if (u + Sh::kStages < units) issue(stage);
    if (++stage == Sh::kStages) stage = 0, parity ^= 1;
  }

  // ---- this warp's part, into its ring, which has been read to the end (and not where copies may still come: the row is lost anyway)
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
  __syncwarp();
  float *part = reinterpret_cast<float *>(ring);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int R = nt * 8 + 2 * t + e;
      if (!landed) continue;
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
  __syncthreads();

  // ---- joined over the block's warps, then over the cluster's blocks
  // The sums of kN parts of four channels from d on of row R, brought to their common maximum.
  auto join = [&](int R, int d, int count, auto part_of) {
    Sum<4> s;
    s.clear();
    for (int k = 0; k < count; ++k) s.top = fmaxf(s.top, part_of(k)[Sh::kRows * D + R]);
    for (int k = 0; k < count; ++k) {
      const float *p = part_of(k);
      const float4 v = *reinterpret_cast<const float4 *>(p + in_part<D>(R, d));
      const float f = s.top == -INFINITY ? 0.0f : ex2(p[Sh::kRows * D + R] - s.top);
      s.num[0] = fmaf(f, v.x, s.num[0]);
      s.num[1] = fmaf(f, v.y, s.num[1]);
      s.num[2] = fmaf(f, v.z, s.num[2]);
      s.num[3] = fmaf(f, v.w, s.num[3]);
      s.den = fmaf(f, p[Sh::kRows * D + Sh::kRows + R], s.den);
    }
    return s;
  };
  auto write = [&](int R, int d, const Sum<4> &s) {
    if (R >= rows) return;
    const float inv = s.den == 0.0f ? 0.0f : 1.0f / s.den;
    alignas(8) T y[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) y[c] = Cvt<T>::from(s.num[c] * inv);
    put(out + R * a.o_head + d, y);
    if (d == 0 && lse) lse[R] = s.den == 0.0f ? -INFINITY : (s.top + log2f(s.den)) * 0.6931471805599453f;
  };
  for (int x = 4 * tid; x < Sh::kRows * D; x += 4 * kThreads) {
    const int R = x / D, d = x % D;
    const Sum<4> s = join(R, d, kWarps, [&](int k) { return reinterpret_cast<const float *>(smem + k * Sh::kStages * Sh::kBytes); });
    if (cluster == 1) {
      write(R, d, s);
    } else {
      *reinterpret_cast<float4 *>(joined + in_part<D>(R, d)) = *reinterpret_cast<const float4 *>(s.num);
      if (d == 0) joined[Sh::kRows * D + R] = s.top, joined[Sh::kRows * D + Sh::kRows + R] = s.den;
    }
  }
  if (cluster == 1) return;
  cluster_arrive();
  cluster_wait();
  for (int x = 4 * static_cast<int>(tid * cluster + rank); x < Sh::kRows * D; x += 4 * kThreads * static_cast<int>(cluster))
    write(x / D, x % D, join(x / D, x % D, static_cast<int>(cluster), [&](int k) { return of_block(joined, k); }));
  cluster_arrive();  // nobody leaves before the others have read
  cluster_wait();
}

template <class T, int D, int NT>
int launch(ListArgs a, int64_t T_, cudaStream_t s) {
  using Sh = ListShape<D, NT>;
  constexpr auto kernel = attn_lists_kernel<T, D, NT>;
  int dev = 0;
  MAPS_TRY(allow_smem<kernel>(Sh::kSmem, &dev));
  a.withheld = dev < 64 ? g_withheld[dev].block.load(std::memory_order_relaxed) - 1 : -1;
  const uint32_t tries = dev < 64 ? g_withheld[dev].tries.load(std::memory_order_relaxed) : 0;
  a.tries = tries ? tries : kTries;
  a.tiles = (a.group + Sh::kRows - 1) / Sh::kRows;
  const int64_t items = T_ * a.H * a.tiles, room = static_cast<int64_t>(sm_count()) * Sh::kBlocks, groups = a.n_list * a.block_groups;
  // what does not fill the device once more is shared out
  int64_t single = items / room * room;
  uint32_t cluster = 1;
  while (cluster < kMaxCluster && 2 * cluster * (items - single) <= room && 2 * cluster * kWarps <= groups) cluster *= 2;
  single = cluster == 1 ? items : single / cluster * cluster;
  a.cluster = cluster;
  a.single = static_cast<uint32_t>(single);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(single + (items - single) * cluster));
  cfg.blockDim = kThreads;
  cfg.dynamicSmemBytes = Sh::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cuda_ok(cudaLaunchKernelEx(&cfg, kernel, static_cast<const ListArgs &>(a)));
}

template <class T>
int launch_dim(int D, const ListArgs &a, int64_t rows, cudaStream_t s) {
  const bool one = a.group <= 8;  // 8 rows to a tile, or 16; 256 channels of 16 rows do not fit a warp's registers
  if (D == 64) return one ? launch<T, 64, 1>(a, rows, s) : launch<T, 64, 2>(a, rows, s);
  if (D == 128) return one ? launch<T, 128, 1>(a, rows, s) : launch<T, 128, 2>(a, rows, s);
  return launch<T, 256, 1>(a, rows, s);
}

}  // namespace

int attn_lists_withhold(int32_t block, uint32_t tries) {
  int dev = 0;
  MAPS_TRY(cuda_ok(cudaGetDevice(&dev)));
  if (dev >= 64) return MAPS_E_INVALID;
  g_withheld[dev].block = block + 1;
  g_withheld[dev].tries = tries;
  return MAPS_OK;
}

}  // namespace maps

extern "C" {

int maps_kv4_attention_blocks(int32_t dtype, int64_t T, int32_t Hq, int32_t H, int32_t D, int32_t S, const void *q, int64_t q_row,
                              int64_t q_head, const int32_t *blocks, const int32_t *tokens, int64_t n_list, const void *cache,
                              int64_t n_blocks, float sm_scale, void *out, int64_t o_row, int64_t o_head, float *lse, void *ws,
                              size_t ws_bytes, void *stream) {
  using namespace maps;
  if ((dtype != MAPS_BF16 && dtype != MAPS_F16) || !kv4_dim_ok(D) || !kv4_block_ok(S) || T < 0 || T > (int64_t(1) << 30) || H < 1 || Hq < H ||
      Hq % H != 0 || Hq > 65535 || T > ((int64_t(1) << 31) - 1024) / Hq || n_list < 1 || n_list > (1 << 20) || n_list * S > kMaxLen ||
      n_blocks < 0 || !(sm_scale - sm_scale == 0.0f))
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, kCtrlBytes));
  if (T == 0) return MAPS_OK;
  if (q == nullptr || out == nullptr || blocks == nullptr || tokens == nullptr || (n_blocks > 0 && cache == nullptr) || !aligned(cache, 16) ||
      !aligned(q, 2) || !aligned(out, 2) || !aligned(lse, 4) || !aligned(blocks, 4) || !aligned(tokens, 4))
    return MAPS_E_INVALID;
  ListArgs a = {};
  a.Hq = Hq, a.H = H, a.group = Hq / H, a.S = S;
  a.block_groups = S / kGroup, a.block_shift = -1;
  for (int32_t i = 0; i < 16; ++i)
    if (a.block_groups == 1 << i) a.block_shift = i;
  a.n_list = n_list, a.n_blocks = n_blocks, a.block_bytes = static_cast<int64_t>(H) * a.block_groups * kv4_group_bytes(D);
  a.wide = aligned(q, 16) && aligned(out, 16) && q_row % 8 == 0 && q_head % 8 == 0 && o_row % 8 == 0 && o_head % 8 == 0;
  a.q = q, a.q_row = q_row, a.q_head = q_head, a.out = out, a.o_row = o_row, a.o_head = o_head, a.lse = lse;
  a.blocks = blocks, a.tokens = tokens, a.cache = static_cast<const uint8_t *>(cache), a.scale = sm_scale, a.status = status_word(ws);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return dtype == MAPS_BF16 ? launch_dim<__nv_bfloat16>(D, a, T, s) : launch_dim<__half>(D, a, T, s);
}

}  // extern "C"
