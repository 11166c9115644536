// kv4_ranges.cu -- the range of each channel over the keys of a cache block, 8 bits an end: what a block's score is made from.
//
// A warp takes a block and KV head.  The first block that each request's tokens went to is dealt out in turn, as a decode step has no
// others; where there are more, those are counted and dealt out evenly, whatever the requests' lengths.  A key is fl(scale * code + zero); least and greatest are taken of these 32-bit values, and the codes of the ends are
// exact: a code times the scale has 15 bits, so a comparison in 32 bits settles where a product's rounding may have crossed a
// whole number.
//
// Bound: neither the bytes nor one pipe.  A block and head of 16 x 128 keys takes 518 instructions, of which 230 take codes out of
// words, make keys and compare; 16 warps a multiprocessor, as many as 128 registers allow, issue 0.6 of what they could and wait for
// loads the rest.  48 prompts of 1,500 to 8,192 tokens, 8 heads of 128 channels, 162 MB: 86 us (1.9 TB/s, 0.28 of the measured copy
// rate).  One token each of 512 requests: 5.5 us, launch and three rounds of loads.  Four blocks a multiprocessor instead of two: 84 and
// 6.8 us.  (256 channels: 48 bytes a thread are spilled.)
#include "kv4_rows.cuh"

namespace maps {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kRequests = 1024;  // counted at a time
constexpr int kBlocksOfSm = 2;

struct Powers {
  uint64_t plus[4], minus[4];  // 2^(23 - 4k) and its negative, twice each, as the bits of floats
};

struct RangeArgs {
  int32_t B, H, S;
  const int32_t *held, *len, *table;
  int64_t max_blocks, n_blocks;
  const uint8_t *cache;
  int8_t *codes;
  float *scale;
  Powers powers;
  int32_t *status;
};

// The least bfloat16 number 127 times which is no less than `most`; 0 where that is below the normal numbers.
__device__ __forceinline__ float range_scale(float most) {
  uint32_t x = __float_as_uint(__fdiv_rn(most, 127.0f)) & 0xffff0000u;
  if (__fmul_rn(__uint_as_float(x), 127.0f) < most) x += 0x10000u;
  return x < 0x00800000u ? 0.0f : __uint_as_float(x);
}

__device__ __forceinline__ float least(float a, float b, float c) {  // NaN where one is
  float y;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float greatest(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// Eight keys fl(scale code + zero), codes 0 .. 7 from the low bits of w up.  Code k stays where it is, as the last bits of a number
// 2^(23 - 4k) + code, for k up to 3, beside code k + 4, which a shift by 16 brings to the same place.  The powers come with the
// call's arguments: as constants the compiler would spend two operations on what is one, (w & mask) | power.
__device__ __forceinline__ void keys_of(uint32_t w, float2 p, const Powers &k2, float (&y)[8]) {
  const Two scale(p.x, p.x), zero(p.y, p.y);
  const uint64_t both = static_cast<uint64_t>(w >> 16) << 32 | w;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    Two x = scale, c = scale;
    x.bits = k2.minus[k];
    c.bits = (both & 0x0000000f0000000full << 4 * k) | k2.plus[k];
    fused(c + x, scale, zero).get(y[k], y[k + 4]);
  }
}

// A block's keys of one head: all lanes of a warp.
template <int D>
__device__ __forceinline__ void unit(const RangeArgs &a, int32_t blk, int hd, int32_t places) {
  constexpr int kLanes = D / 8, kSub = 32 / kLanes, kTokens = kGroup / kSub;  // lanes of a token's key, tokens side by side, tokens of a lane
  const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
  if (blk < 0) return;
  const int64_t at = static_cast<int64_t>(blk) * a.H + hd;
  const uint8_t *group = a.cache + at * (a.S / kGroup) * kv4_group_bytes(D);
  float lo[8], hi[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) lo[c] = INFINITY, hi[c] = -INFINITY;
  for (int32_t g0 = 0; g0 < places; g0 += kGroup, group += kv4_group_bytes(D)) {
    uint32_t w[kTokens], p[kTokens];
    if (g0 + kGroup <= places) {
      const uint8_t *src = group + sub * kTokens * (D / 2) + 4 * l;
#pragma unroll
      for (int i = 0; i < kTokens; ++i) w[i] = *reinterpret_cast<const uint32_t *>(src + i * (D / 2));
#pragma unroll
      for (int i = 0; i < kTokens; i += 4) *reinterpret_cast<uint4 *>(p + i) = *reinterpret_cast<const uint4 *>(group + 16 * D + 4 * (sub * kTokens + i));
    } else {  // a token beyond the last is the last once more
#pragma unroll
      for (int i = 0; i < kTokens; ++i) {
        const int tau = min(sub * kTokens + i, places - 1 - g0);
        w[i] = *reinterpret_cast<const uint32_t *>(group + tau * (D / 2) + 4 * l);
        p[i] = *reinterpret_cast<const uint32_t *>(group + 16 * D + 4 * tau);
      }
    }
#pragma unroll
    for (int i = 0; i < kTokens; i += 2) {
      float x[8], y[8];
      keys_of(w[i], kv4_param(p[i]), a.powers, x);
      keys_of(w[i + 1], kv4_param(p[i + 1]), a.powers, y);
#pragma unroll
      for (int c = 0; c < 8; ++c) lo[c] = least(lo[c], x[c], y[c]), hi[c] = greatest(hi[c], x[c], y[c]);
    }
  }
  // joined over the tokens side by side, each lane keeping its share of the channels
  constexpr int kOwn = 8 / kSub;
#pragma unroll
  for (int o = kLanes, keep = 4; o < 32; o <<= 1, keep >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int c = 0; c < keep; ++c) {
      const float send_lo = up ? lo[c] : lo[c + keep], send_hi = up ? hi[c] : hi[c + keep];
      const float own_lo = up ? lo[c + keep] : lo[c], own_hi = up ? hi[c + keep] : hi[c];
      const float got_lo = __shfl_xor_sync(0xffffffffu, send_lo, o), got_hi = __shfl_xor_sync(0xffffffffu, send_hi, o);
      lo[c] = least(own_lo, got_lo, got_lo);
      hi[c] = greatest(own_hi, got_hi, got_hi);
    }
  }
  uint32_t top = 0;  // NaN's bits are above infinity's
#pragma unroll
  for (int c = 0; c < kOwn; ++c) top = max(top, max(__float_as_uint(lo[c]) & 0x7fffffffu, __float_as_uint(hi[c]) & 0x7fffffffu));
  top = __reduce_max_sync(0xffffffffu, top);
  const bool bad = top >= 0x7f800000u;
  const float sc = bad ? 0.0f : range_scale(__uint_as_float(top));
  const float inv = sc > 0.0f ? __fdividef(1.0f, sc) : 0.0f;
  uint32_t out[2][(kOwn + 3) / 4] = {};
  if (sc > 0.0f) {
#pragma unroll
    for (int c = 0; c < kOwn; ++c) {
      // rounded down and up to whole numbers in one step, right or one off, which exact products tell
      constexpr float kWhole = 12582912.0f;  // 1.5 * 2^23
      const float fx = __fmaf_rd(lo[c], inv, kWhole), fy = __fmaf_ru(hi[c], inv, kWhole), wx = fx - kWhole, wy = fy - kWhole;
      int x = __float_as_int(fx), y = __float_as_int(fy);
      if (__fmul_rn(wx, sc) > lo[c]) --x;
      if (__fmul_rn(wx + 1.0f, sc) <= lo[c]) ++x;
      if (__fmul_rn(wy, sc) < hi[c]) ++y;
      if (__fmul_rn(wy - 1.0f, sc) >= hi[c]) --y;
      out[0][c / 4] |= (static_cast<uint32_t>(x) & 255u) << (c % 4 * 8);
      out[1][c / 4] |= (static_cast<uint32_t>(y) & 255u) << (c % 4 * 8);
    }
  }
  // this lane's first channel: the highest bit of sub chose the halves of 8, the next of 4
  const int own = kSub == 1 ? 0 : kSub == 2 ? 4 * sub : 4 * (sub & 1) + 2 * (sub >> 1);
  int8_t *dst = a.codes + at * (2 * D) + 8 * l + own;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    if (kOwn == 8) *reinterpret_cast<uint2 *>(dst + x * D) = make_uint2(out[x][0], out[x][kOwn == 8]);
    if (kOwn == 4) *reinterpret_cast<uint32_t *>(dst + x * D) = out[x][0];
    if (kOwn == 2) *reinterpret_cast<uint16_t *>(dst + x * D) = static_cast<uint16_t>(out[x][0]);
  }
  if (lane == 0) a.scale[at] = bad ? __uint_as_float(0x7fffffffu) : sc;
}

template <int D>
__global__ void __launch_bounds__(kThreads, kBlocksOfSm) kv4_ranges_kernel(const RangeArgs a) {
  pdl_prologue();
  const int lane = threadIdx.x & 31;
  const int tid = threadIdx.x, warp = tid >> 5;
  __shared__ int64_t s_before[kRequests + 1];  // blocks of the requests ahead
  __shared__ int32_t s_first[kRequests], s_len[kRequests];
  __shared__ int64_t s_warp[kWarps];
  __shared__ int2 s_block[kThreads];  // a block of the cache, and its places that hold a token
  // The blocks of a request: its first, and the one behind its last.
  auto length = [&](int64_t b) { return b < a.B ? a.len[b] : 0; };
  auto before = [&](int64_t b) { return b < a.B && a.held ? a.held[b] : 0; };
  auto blocks_of = [&](int32_t &len, int32_t &first) -> int32_t {
    if (len < 0 || len > 0x7fffffff - 1023 || len > a.max_blocks * a.S || first < 0) {
      flag_error(a.status, MAPS_E_RANGE);
      len = first = 0;
    }
    first = min(first, len) / a.S;
    return static_cast<int32_t>(static_cast<uint32_t>(len + a.S - 1) / static_cast<uint32_t>(a.S));
  };
  // A request has blocks behind its first; one that is to be reported counts as such.
  auto has_more = [&](int32_t len, int32_t held) { return len < 0 || held < 0 || (len > held && static_cast<uint32_t>(len - 1) / a.S > static_cast<uint32_t>(held) / a.S); };
  constexpr int kOwn = kRequests / kThreads;
  int32_t some_len[kOwn], some_held[kOwn];  // all loads under way at once
#pragma unroll
  for (int k = 0; k < kOwn; ++k) some_len[k] = length(tid + k * kThreads), some_held[k] = before(tid + k * kThreads);
  const int64_t mine = blockIdx.x + static_cast<int64_t>(tid) * gridDim.x;
  int32_t my_len = length(mine), my_first = before(mine);
  const bool mine_there = blocks_of(my_len, my_first) > my_first;
  const int32_t my_block = mine_there ? a.table[mine * a.max_blocks + my_first] : -1;
  bool more = false;
#pragma unroll
  for (int k = 0; k < kOwn; ++k) more |= has_more(some_len[k], some_held[k]);
  for (int64_t b = tid + kRequests; b < a.B; b += kThreads) more |= has_more(length(b), before(b));
  const int step_x = kWarps / a.H, step_h = kWarps % a.H;
  // First every request's first block, dealt out in turn: a decode step has no others.  Then the others, in turns of kRequests.
  for (int32_t b0 = -kRequests; b0 < a.B; b0 += kRequests) {
    const bool others = b0 >= 0;
    int64_t from = 0, to = (a.B - static_cast<int64_t>(blockIdx.x) + gridDim.x - 1) / gridDim.x;
    if (others) {
      // ---- counted; this block of threads has an equal share of them, whatever the lengths
      int32_t count[kOwn];
      int64_t sum = 0;
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        int32_t len = length(b0 + tid * kOwn + k), first = before(b0 + tid * kOwn + k);
        count[k] = max(blocks_of(len, first) - first - 1, 0);
        s_first[tid * kOwn + k] = first + 1;
        s_len[tid * kOwn + k] = len;
        sum += count[k];
      }
      int64_t ahead = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, ahead, o);
        if (lane >= o) ahead += x;
      }
      if (lane == 31) s_warp[warp] = ahead;
      __syncthreads();
      ahead -= sum;
      int64_t total = 0;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) {
        if (k < warp) ahead += s_warp[k];
        total += s_warp[k];
      }
#pragma unroll
      for (int k = 0; k < kOwn; ++k) s_before[tid * kOwn + k] = ahead, ahead += count[k];
      if (tid == 0) s_before[kRequests] = total;
      __syncthreads();
      from = total * blockIdx.x / gridDim.x, to = total * (blockIdx.x + 1) / gridDim.x;
    }
    for (int64_t x0 = from; x0 < to; x0 += kThreads) {
      // ---- up to kThreads of them, looked up side by side
      const int here = static_cast<int>(min(to - x0, static_cast<int64_t>(kThreads)));
      if (tid < here) {
        int32_t j = my_first, len = my_len, block = my_block;
        bool there = mine_there;
        if (others) {
          int lo = 0;  // the last request with s_before <= x0 + tid
#pragma unroll
          for (int o = kRequests / 2; o > 0; o >>= 1)
            if (s_before[lo + o] <= x0 + tid) lo += o;
          j = s_first[lo] + static_cast<int32_t>(x0 + tid - s_before[lo]), len = s_len[lo], there = true;
          block = a.table[(b0 + lo) * a.max_blocks + j];
        } else if (x0 > 0) {
          const int64_t b = mine + x0 * gridDim.x;
          len = length(b), j = before(b);
          there = blocks_of(len, j) > j;
          block = there ? a.table[b * a.max_blocks + j] : -1;
        }
        if (there && (block < 0 || block >= a.n_blocks)) {
          flag_error(a.status, MAPS_E_RANGE);
          block = -1;
        }
        s_block[tid] = make_int2(block, min(a.S, len - j * a.S));
      }
      __syncthreads();
      for (int x = warp / a.H, h = warp % a.H; x < here; x += step_x) {
        unit<D>(a, s_block[x].x, h, s_block[x].y);
        h += step_h;
        if (h >= a.H) h -= a.H, ++x;
      }
      __syncthreads();
    }
    if (!__syncthreads_or(more)) return;
  }
}

}  // namespace
}  // namespace maps

extern "C" int maps_kv4_block_ranges(int32_t B, int32_t H, int32_t D, int32_t S, const int32_t *held, const int32_t *kv_len,
                                     const int32_t *table, int64_t max_blocks, const void *cache, int64_t n_blocks, int8_t *codes,
                                     float *scale, void *ws, size_t ws_bytes, void *stream) {
  using namespace maps;
  if (!kv4_dim_ok(D) || !kv4_block_ok(S) || B < 0 || B > (1 << 30) || H < 1 || H > 65535 || max_blocks < 0 || max_blocks > 0x7fffffff ||
      n_blocks < 0)
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, kCtrlBytes));
  if (B == 0) return MAPS_OK;
  if (kv_len == nullptr || (max_blocks > 0 && table == nullptr) || (n_blocks > 0 && (cache == nullptr || codes == nullptr || scale == nullptr)) ||
      !aligned(cache, 16) || !aligned(codes, 16) || !aligned(scale, 4) || !aligned(held, 4) || !aligned(kv_len, 4) || !aligned(table, 4))
    return MAPS_E_INVALID;
  const RangeArgs a = {B, H, S, held, kv_len, table, max_blocks, n_blocks, static_cast<const uint8_t *>(cache), codes, scale,
                       {{0x4b0000004b000000ull, 0x4900000049000000ull, 0x4700000047000000ull, 0x4500000045000000ull},
                        {0xcb000000cb000000ull, 0xc9000000c9000000ull, 0xc7000000c7000000ull, 0xc5000000c5000000ull}}, status_word(ws)};
  const unsigned grid = static_cast<unsigned>(sm_count() * kBlocksOfSm);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (D == 64) launch_pdl(kv4_ranges_kernel<64>, grid, kThreads, 0, s, a);
  if (D == 128) launch_pdl(kv4_ranges_kernel<128>, grid, kThreads, 0, s, a);
  if (D == 256) launch_pdl(kv4_ranges_kernel<256>, grid, kThreads, 0, s, a);
  return launch_ok();
}
