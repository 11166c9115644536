// kv4_cache.cu -- writing keys and values to the 4-bit cache, and reading them back.
//
// A row is one token's K or V of one KV head, D channels.  It is held as 16 evenly spaced
// levels: zero = bf16(min), scale = bf16((max - min) * (1/15)), code = round((x - zero) / scale)
// with the reciprocal taken once per row, value = scale * code + zero.  scale * code has at
// most 12 significant bits, so a value is rounded once.  D/8 lanes share a row, 8 channels
// (16 bytes) each; extremes are joined by shuffles.
#include "kv4.cuh"

namespace maps {
namespace {

struct KVArgs {
  int64_t T, n_blocks;
  int32_t H, S;
  const void *k, *v;
  void *ko, *vo;
  int64_t k_row, k_head, v_row, v_head;  // elements
  const int64_t *slots;
  uint8_t *cache;
  int32_t *status;
};

// Where a slot's token lies: its group's first byte and its place there; false for a slot that is none.
__device__ __forceinline__ bool locate(const KVArgs &a, int64_t slot, int h, int group_bytes, uint8_t *&group, int &tau) {
  if (slot < 0) return false;
  const int64_t block = slot / a.S;
  if (block >= a.n_blocks) {
    flag_error(a.status, MAPS_E_RANGE);
    return false;
  }
  const int within = static_cast<int>(slot - block * a.S);
  tau = within % kGroup;
  group = a.cache + ((block * a.H + h) * (a.S / kGroup) + within / kGroup) * group_bytes;
  return true;
}

template <class T, int D, bool kWide>
__global__ void __launch_bounds__(256) kv4_append_kernel(const KVArgs a) {
  pdl_prologue();
  constexpr int kLanes = D / 8;
  const int64_t row = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / kLanes;  // (token, K or V, head)
  const int l = threadIdx.x % kLanes;
  if (row >= a.T * 2 * a.H) return;  // whole rows leave together, and kLanes divides 32
  const unsigned mask = __activemask();
  const int64_t tok = row / (2 * a.H);
  const int rest = static_cast<int>(row - tok * 2 * a.H);
  const bool is_v = rest >= a.H;
  const int h = is_v ? rest - a.H : rest;
  const T *src = is_v ? static_cast<const T *>(a.v) + tok * a.v_row + h * a.v_head
                      : static_cast<const T *>(a.k) + tok * a.k_row + h * a.k_head;
  T raw[8];
  if (kWide) {
    *reinterpret_cast<uint4 *>(raw) = *reinterpret_cast<const uint4 *>(src + 8 * l);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = src[8 * l + i];
  }
  float x[8], lo, hi;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = Cvt<T>::to(raw[i]);
    bad |= !isfinite(x[i]);
    lo = i ? fminf(lo, x[i]) : x[i];
    hi = i ? fmaxf(hi, x[i]) : x[i];
  }
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(mask, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(mask, hi, o));
    bad |= __shfl_xor_sync(mask, static_cast<int>(bad), o) != 0;
  }
  const float spread = __fsub_rn(hi, lo);
  bad |= !isfinite(spread);
  const float scale = __bfloat162float(__float2bfloat16_rn(__fmul_rn(spread, 1.0f / 15.0f)));
  const float zero = __bfloat162float(__float2bfloat16_rn(lo));
  const float inv = scale >= 1.17549435e-38f ? __fdiv_rn(1.0f, scale) : 0.0f;  // smallest normal number
  uint32_t codes = 0;  // channel 8l + i in bits 4i
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = fminf(fmaxf(rintf(__fmul_rn(__fsub_rn(x[i], zero), inv)), 0.0f), 15.0f);
    codes |= static_cast<uint32_t>(static_cast<int>(c)) << (4 * i);
  }
  uint32_t param = __float_as_uint(scale) >> 16 | (__float_as_uint(zero) & 0xffff0000u);
  if (bad) codes = 0, param = 0x7fff7fffu;
  uint8_t *group;
  int tau;
  if (!locate(a, a.slots[tok], h, kv4_group_bytes(D), group, tau)) return;
  if (is_v) {
    *reinterpret_cast<uint16_t *>(group + 8 * D + kv4_v_unit<D>(tau, 2 * l)) = static_cast<uint16_t>(codes);
    *reinterpret_cast<uint16_t *>(group + 8 * D + kv4_v_unit<D>(tau, 2 * l + 1)) = static_cast<uint16_t>(codes >> 16);
  } else {
    *reinterpret_cast<uint32_t *>(group + tau * (D / 2) + 4 * l) = codes;
  }
  if (l == 0) reinterpret_cast<uint32_t *>(group + 16 * D)[(is_v ? 16 : 0) + tau] = param;
}

template <class T, int D, bool kWide>
__global__ void __launch_bounds__(256) kv4_read_kernel(const KVArgs a) {
  pdl_prologue();
  constexpr int kLanes = D / 8;
  const int64_t row = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / kLanes;
  const int l = threadIdx.x % kLanes;
  if (row >= a.T * 2 * a.H) return;
  const int64_t tok = row / (2 * a.H);
  const int rest = static_cast<int>(row - tok * 2 * a.H);
  const bool is_v = rest >= a.H;
  const int h = is_v ? rest - a.H : rest;
  uint8_t *group;
  int tau;
  T y[8];
  if (locate(a, a.slots[tok], h, kv4_group_bytes(D), group, tau)) {
    uint32_t codes;
    if (is_v)
      codes = *reinterpret_cast<const uint16_t *>(group + 8 * D + kv4_v_unit<D>(tau, 2 * l)) |
              static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(group + 8 * D + kv4_v_unit<D>(tau, 2 * l + 1))) << 16;
    else
      codes = *reinterpret_cast<const uint32_t *>(group + tau * (D / 2) + 4 * l);
    const float2 p = kv4_param(reinterpret_cast<const uint32_t *>(group + 16 * D)[(is_v ? 16 : 0) + tau]);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = Cvt<T>::from(fmaf(p.x, static_cast<float>(codes >> (4 * i) & 15u), p.y));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = Cvt<T>::from(0.0f);
  }
  T *dst = is_v ? static_cast<T *>(a.vo) + tok * a.v_row + h * a.v_head : static_cast<T *>(a.ko) + tok * a.k_row + h * a.k_head;
  if (kWide) {
    *reinterpret_cast<uint4 *>(dst + 8 * l) = *reinterpret_cast<const uint4 *>(y);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[8 * l + i] = y[i];
  }
}

bool wide(const void *p, int64_t row, int64_t head) { return aligned(p, 16) && row % 8 == 0 && head % 8 == 0; }

template <class T, int D>
void launch_rows(bool append, bool w, const KVArgs &a, cudaStream_t s) {
  const int64_t threads = a.T * 2 * a.H * (D / 8);
  const unsigned grid = static_cast<unsigned>((threads + 255) / 256);
  if (append)
    w ? launch_pdl(kv4_append_kernel<T, D, true>, grid, 256, 0, s, a) : launch_pdl(kv4_append_kernel<T, D, false>, grid, 256, 0, s, a);
  else
    w ? launch_pdl(kv4_read_kernel<T, D, true>, grid, 256, 0, s, a) : launch_pdl(kv4_read_kernel<T, D, false>, grid, 256, 0, s, a);
}

template <class T>
void launch_dim(int D, bool append, bool w, const KVArgs &a, cudaStream_t s) {
  if (D == 64) launch_rows<T, 64>(append, w, a, s);
  if (D == 128) launch_rows<T, 128>(append, w, a, s);
  if (D == 256) launch_rows<T, 256>(append, w, a, s);
}

int run(bool append, int32_t dtype, int32_t D, KVArgs &a, void *ws, size_t ws_bytes, void *stream) {
  const void *k = append ? a.k : a.ko, *v = append ? a.v : a.vo;
  if ((dtype != MAPS_BF16 && dtype != MAPS_F16) || !kv4_dim_ok(D) || !kv4_block_ok(a.S) || a.H < 1 || a.H > 65535 || a.T < 0 ||
      a.T > (int64_t(1) << 30) / a.H || a.n_blocks < 0)
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, kCtrlBytes));
  if (a.T == 0) return MAPS_OK;
  if (k == nullptr || v == nullptr || a.slots == nullptr || (a.n_blocks > 0 && a.cache == nullptr) || !aligned(a.cache, 16) ||
      !aligned(k, 2) || !aligned(v, 2))
    return MAPS_E_INVALID;
  a.status = status_word(ws);
  const bool w = wide(k, a.k_row, a.k_head) && wide(v, a.v_row, a.v_head);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MAPS_BF16)
    launch_dim<__nv_bfloat16>(D, append, w, a, s);
  else
    launch_dim<__half>(D, append, w, a, s);
  return launch_ok();
}

}  // namespace
}  // namespace maps

extern "C" {

size_t maps_kv4_record_bytes(int32_t S, int32_t D) {
  if (!maps::kv4_dim_ok(D) || !maps::kv4_block_ok(S)) return 0;
  return static_cast<size_t>(S / maps::kGroup) * maps::kv4_group_bytes(D);
}

size_t maps_kv4_workspace_size(void) { return maps::kCtrlBytes; }

int maps_kv4_append(int32_t dtype, int64_t T, int32_t H, int32_t D, int32_t S, const void *k,
                    int64_t k_row, int64_t k_head, const void *v, int64_t v_row, int64_t v_head,
                    const int64_t *slots, void *cache, int64_t n_blocks, void *ws,
                    size_t ws_bytes, void *stream) {
  maps::KVArgs a = {T, n_blocks, H, S, k, v, nullptr, nullptr, k_row, k_head, v_row, v_head, slots,
                    static_cast<uint8_t *>(cache), nullptr};
  return maps::run(true, dtype, D, a, ws, ws_bytes, stream);
}

int maps_kv4_read(int32_t dtype, int64_t T, int32_t H, int32_t D, int32_t S, const int64_t *slots,
                  const void *cache, int64_t n_blocks, void *k_out, int64_t k_row, int64_t k_head,
                  void *v_out, int64_t v_row, int64_t v_head, void *ws, size_t ws_bytes,
                  void *stream) {
  maps::KVArgs a = {T, n_blocks, H, S, nullptr, nullptr, k_out, v_out, k_row, k_head, v_row, v_head,
                    slots, static_cast<uint8_t *>(const_cast<void *>(cache)), nullptr};
  return maps::run(false, dtype, D, a, ws, ws_bytes, stream);
}

}  // extern "C"
