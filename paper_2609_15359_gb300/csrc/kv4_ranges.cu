// kv4_ranges.cu -- the range of each channel over the keys of a cache block, 8 bits an end: what a block's score is made from.
//
// A warp takes a block and KV head.  A key is fl(scale * code + zero); least and greatest are taken of these 32-bit values, and
// the codes of the ends are exact: a code times the scale has 15 bits, so a comparison in 32 bits settles where a division's
// rounding may have crossed a whole number.
#include "kv4_rows.cuh"

namespace maps {
namespace {

constexpr int kWarps = 8;

struct RangeArgs {
  int32_t B, H, S;
  const int32_t *held, *len, *table;
  int64_t max_blocks, n_blocks;
  const uint8_t *cache;
  int8_t *codes;
  float *scale;
  uint64_t power[4];  // 2^(23 - 4k) twice, as the bits of floats
  float minus[4];     // the same, negative
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
__device__ __forceinline__ void keys_of(uint32_t w, float2 p, const uint64_t (&power)[4], const float (&minus)[4], float (&y)[8]) {
  const Two scale(p.x, p.x), zero(p.y, p.y);
  const uint64_t both = static_cast<uint64_t>(w >> 16) << 32 | w;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    Two x(minus[k], minus[k]), c = x;
    c.bits = (both & 0x0000000f0000000full << 4 * k) | power[k];
    fused(c + x, scale, zero).get(y[k], y[k + 4]);
  }
}

template <int D>
__global__ void __launch_bounds__(32 * kWarps, 4) kv4_ranges_kernel(const RangeArgs a) {
  pdl_prologue();
  constexpr int kLanes = D / 8, kSub = 32 / kLanes, kTokens = kGroup / kSub;  // lanes of a token's key, tokens side by side, tokens of a lane
  const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
  const int b = blockIdx.x;
  const int32_t n = a.len[b];
  const int32_t held = a.held ? a.held[b] : 0;
  if (n < 0 || n > 0x7fffffff - 1023 || n > a.max_blocks * a.S || held < 0) {
    if (threadIdx.x == 0) flag_error(a.status, MAPS_E_RANGE);
    return;
  }
  // the warp's units: blocks j and heads h, a stride of both apart
  const int32_t end = (n + a.S - 1) / a.S;
  int32_t j, h, block = -1, step_j, step_h;
  {
    const int64_t u = static_cast<int64_t>(blockIdx.y) * kWarps + (threadIdx.x >> 5), stride = static_cast<int64_t>(gridDim.y) * kWarps;
    const int64_t at = min(held, n) / a.S + u / a.H;
    if (at >= end) return;
    j = static_cast<int32_t>(at);
    h = static_cast<int32_t>(u % a.H);
    step_j = static_cast<int32_t>(min(stride / a.H, static_cast<int64_t>(1) << 28));
    step_h = static_cast<int32_t>(stride % a.H);
  }
  const int32_t *table = a.table + b * a.max_blocks;
  auto next = [&]() {  // the next unit, its block looked up
    j += step_j;
    h += step_h;
    if (h >= a.H) h -= a.H, ++j;
    block = j < end ? table[j] : -1;
  };
  block = table[j];
  while (j < end) {
    const int32_t blk = block, hd = h, places = min(a.S, n - j * a.S);
    next();
    if (blk < 0 || blk >= a.n_blocks) {
      if (lane == 0) flag_error(a.status, MAPS_E_RANGE);
      continue;
    }
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
        keys_of(w[i], kv4_param(p[i]), a.power, a.minus, x);
        keys_of(w[i + 1], kv4_param(p[i + 1]), a.power, a.minus, y);
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
                       {0x4b0000004b000000ull, 0x4900000049000000ull, 0x4700000047000000ull, 0x4500000045000000ull},
                       {-8388608.0f, -524288.0f, -32768.0f, -2048.0f}, status_word(ws)};
  // enough blocks a request to fill the device, no more than its table's blocks need
  const int64_t most = (max_blocks * H + kWarps - 1) / kWarps, fill = (static_cast<int64_t>(sm_count()) * 8 + B - 1) / B;
  const unsigned y = static_cast<unsigned>(most < 1 ? 1 : most < fill ? most : fill);
  const dim3 grid(static_cast<unsigned>(B), y);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (D == 64) launch_pdl(kv4_ranges_kernel<64>, grid, 32 * kWarps, 0, s, a);
  if (D == 128) launch_pdl(kv4_ranges_kernel<128>, grid, 32 * kWarps, 0, s, a);
  if (D == 256) launch_pdl(kv4_ranges_kernel<256>, grid, 32 * kWarps, 0, s, a);
  return launch_ok();
}
