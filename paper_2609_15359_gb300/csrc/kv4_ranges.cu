// kv4_ranges.cu -- the range of each channel over the keys of a cache block, 8 bits an end: what a block's score is made from.
//
// A warp takes a block and KV head.  A key is fl(scale * code + zero); least and greatest are taken of these 32-bit values, and
// the codes of the ends are exact: a code times the scale has 15 bits, so a comparison in 32 bits settles where a division's
// rounding may have crossed a whole number.
#include "kv4.cuh"

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
  int32_t *status;
};

// The least bfloat16 number 127 times which is no less than `most`; 0 where that is below the normal numbers.
__device__ __forceinline__ float range_scale(float most) {
  uint32_t x = __float_as_uint(__fdiv_rn(most, 127.0f)) & 0xffff0000u;
  if (__fmul_rn(__uint_as_float(x), 127.0f) < most) x += 0x10000u;
  return x < 0x00800000u ? 0.0f : __uint_as_float(x);
}

template <int D>
__global__ void __launch_bounds__(32 * kWarps) kv4_ranges_kernel(const RangeArgs a) {
  pdl_prologue();
  constexpr int kLanes = D / 8, kSub = 32 / kLanes, kTokens = kGroup / kSub;
  const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
  const int b = blockIdx.x;
  const int32_t n = a.len[b];
  int32_t held = a.held ? a.held[b] : 0;
  if (n < 0 || n > 0x7fffffff - 1023 || n > a.max_blocks * a.S || held < 0) {
    if (threadIdx.x == 0) flag_error(a.status, MAPS_E_RANGE);
    return;
  }
  const int32_t first = min(held, n) / a.S, end = (n + a.S - 1) / a.S;
  const int64_t units = static_cast<int64_t>(end - first) * a.H;
  for (int64_t u = static_cast<int64_t>(blockIdx.y) * kWarps + (threadIdx.x >> 5); u < units; u += static_cast<int64_t>(gridDim.y) * kWarps) {
    const int32_t j = first + static_cast<int32_t>(u / a.H);
    const int h = static_cast<int>(u % a.H);
    const int32_t block = a.table[b * a.max_blocks + j];
    if (block < 0 || block >= a.n_blocks) {
      if (lane == 0) flag_error(a.status, MAPS_E_RANGE);
      continue;
    }
    const int32_t places = min(a.S, n - j * a.S);
    const int64_t at = static_cast<int64_t>(block) * a.H + h;
    const uint8_t *group = a.cache + at * (a.S / kGroup) * kv4_group_bytes(D);
    float lo[8], hi[8];
    bool bad = false;
#pragma unroll
    for (int c = 0; c < 8; ++c) lo[c] = INFINITY, hi[c] = -INFINITY;
    for (int g0 = 0; g0 < places; g0 += kGroup, group += kv4_group_bytes(D)) {
#pragma unroll
      for (int i = 0; i < kTokens; ++i) {
        const int tau = sub * kTokens + i;
        if (g0 + tau >= places) break;
        const uint32_t w = *reinterpret_cast<const uint32_t *>(group + tau * (D / 2) + 4 * l);
        const float2 p = kv4_param(*reinterpret_cast<const uint32_t *>(group + 16 * D + 4 * tau));
        bad |= !isfinite(p.x) || !isfinite(p.y);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const float y = fmaf(p.x, __uint_as_float(0x4b000000u | (w >> (4 * c) & 15u)) - 8388608.0f, p.y);
          lo[c] = fminf(lo[c], y);
          hi[c] = fmaxf(hi[c], y);
        }
      }
    }
    float most = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
#pragma unroll
      for (int o = kLanes; o < 32; o <<= 1) {
        lo[c] = fminf(lo[c], __shfl_xor_sync(0xffffffffu, lo[c], o));
        hi[c] = fmaxf(hi[c], __shfl_xor_sync(0xffffffffu, hi[c], o));
      }
      most = fmaxf(most, fmaxf(fabsf(lo[c]), fabsf(hi[c])));
    }
    most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
    bad = __any_sync(0xffffffffu, bad) || !isfinite(most);
    const float sc = bad ? 0.0f : range_scale(most);
    uint32_t out[2][2] = {};
    if (sc > 0.0f) {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        float x = floorf(__fdiv_rn(lo[c], sc)), y = ceilf(__fdiv_rn(hi[c], sc));
        if (x * sc > lo[c]) x -= 1.0f;
        if (y * sc < hi[c]) y += 1.0f;
        out[0][c / 4] |= (static_cast<uint32_t>(static_cast<int>(x)) & 255u) << (c % 4 * 8);
        out[1][c / 4] |= (static_cast<uint32_t>(static_cast<int>(y)) & 255u) << (c % 4 * 8);
      }
    }
    int8_t *dst = a.codes + at * (2 * D) + 8 * l;
    if (sub == 0) *reinterpret_cast<uint2 *>(dst) = make_uint2(out[0][0], out[0][1]);
    if (sub == kSub - 1) *reinterpret_cast<uint2 *>(dst + D) = make_uint2(out[1][0], out[1][1]);
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
  const RangeArgs a = {B, H, S, held, kv_len, table, max_blocks, n_blocks, static_cast<const uint8_t *>(cache), codes, scale, status_word(ws)};
  // enough blocks a request to fill the device, no more than its table's blocks need
  const int64_t most = (max_blocks * H + kWarps - 1) / kWarps, fill = (static_cast<int64_t>(sm_count()) * 16 + B - 1) / B;
  const unsigned y = static_cast<unsigned>(most < 1 ? 1 : most < fill ? most : fill);
  const dim3 grid(static_cast<unsigned>(B), y);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (D == 64) launch_pdl(kv4_ranges_kernel<64>, grid, 32 * kWarps, 0, s, a);
  if (D == 128) launch_pdl(kv4_ranges_kernel<128>, grid, 32 * kWarps, 0, s, a);
  if (D == 256) launch_pdl(kv4_ranges_kernel<256>, grid, 32 * kWarps, 0, s, a);
  return launch_ok();
}
