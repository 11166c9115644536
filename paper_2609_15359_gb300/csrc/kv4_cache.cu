// kv4_cache.cu -- writing keys and values to the 4-bit cache, and reading them back.
//
// A row is one token's K or V of one KV head, D channels.  It is held as 16 evenly spaced
// levels: zero = bf16(min), scale = bf16((max - min) * (1/15)), code = round((x - zero) / scale)
// with the reciprocal taken once per row, value = scale * code + zero.  scale * code has at
// most 12 significant bits, so a value is rounded once.  D/8 lanes share a row, 8 channels
// (16 bytes) each; extremes are joined by shuffles.
//
// Bound: the bytes of the 16-bit rows and the records.  65,536 tokens of 8 heads and 128 channels, 340 MB a call,
// take 84 us to append (4.1 TB/s, 0.60 of the measured copy rate; a row's minimum, maximum and
// codes cost about as many issue slots) and 52 us to read (6.5 TB/s).  A decode step's rows take 2-5 us,
// which is launch and latency.
#include "kv4.cuh"

namespace maps {
namespace {

// Warps of a multiprocessor from which on a warp takes 16 tokens of a head: shared loads of slots and whole groups moved at
// once, but fewer and longer threads.  8 heads of 128 channels, append / read, rows side by side and 16 to a warp:
// 1,024 tokens (3 warps) 3.8 / 3.3 and 5.2 / 3.4 us; 4,096 (13) 9.7 / 7.9 and 9.4 / 4.7; 16,384 34.6 / 28.0 and 20.2 / 12.8.
constexpr int kManyWarps = 8;

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

// 16-bit pairs of either type, with NaN in either argument kept.
template <class T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
  using V = __nv_bfloat162;
};
template <>
struct Pair<__half> {
  using V = __half2;
};

// A row's 8 channels of this lane: codes (channel i in bits 4i) and {scale, zero} of the row, whose
// kLanes lanes have it between them.
template <class T, int kLanes>
__device__ __forceinline__ void quantise(const uint4 raw, unsigned mask, uint32_t &codes, uint32_t &param) {
  using V = typename Pair<T>::V;
  const V *x = reinterpret_cast<const V *>(&raw);
  V lo = __hmin2_nan(__hmin2_nan(x[0], x[1]), __hmin2_nan(x[2], x[3]));
  V hi = __hmax2_nan(__hmax2_nan(x[0], x[1]), __hmax2_nan(x[2], x[3]));
  // {min, -max} in one word, so a step of the join is one shuffle and one minimum
  V ends;
  ends.x = __hmin_nan(lo.x, lo.y);
  ends.y = __hneg(__hmax_nan(hi.x, hi.y));
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    const uint32_t u = __shfl_xor_sync(mask, *reinterpret_cast<const uint32_t *>(&ends), o);
    ends = __hmin2_nan(ends, *reinterpret_cast<const V *>(&u));
  }
  const float low = Cvt<T>::to(ends.x), high = -Cvt<T>::to(ends.y), spread = __fsub_rn(high, low);
  const bool bad = !isfinite(low) || !isfinite(high) || !isfinite(spread);
  const float scale = __bfloat162float(__float2bfloat16_rn(__fmul_rn(spread, 1.0f / 15.0f)));
  const float zero = __bfloat162float(__float2bfloat16_rn(low));
  const float inv = scale >= 1.17549435e-38f ? __fdiv_rn(1.0f, scale) : 0.0f;  // smallest normal number
  // adding 1.5 * 2^23 rounds to an integer in the low bits; the sum of those times 16^i then has 8 known offsets to take off
  uint32_t sum = 0;
#pragma unroll
  for (int i = 7; i >= 0; --i) {
    const float y = Cvt<T>::to(i % 2 ? x[i / 2].y : x[i / 2].x);
    const float c = fminf(fmaxf(__fmul_rn(__fsub_rn(y, zero), inv), 0.0f), 15.0f);
    sum = sum * 16u + __float_as_uint(__fadd_rn(c, 12582912.0f));
  }
  codes = bad ? 0u : sum - 0x4b400000u * 0x11111111u;
  param = bad ? 0x7fff7fffu : __float_as_uint(scale) >> 16 | (__float_as_uint(zero) & 0xffff0000u);
}

// The values of 8 codes.
template <class T>
__device__ __forceinline__ uint4 values(uint32_t codes, uint32_t param) {
  const float2 p = kv4_param(param);
  uint4 y;
  T *z = reinterpret_cast<T *>(&y);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = __uint_as_float(0x4b000000u | (codes >> (4 * i) & 15u)) - 8388608.0f;
    z[i] = Cvt<T>::from(fmaf(p.x, c, p.y));
  }
  return y;
}

template <class T, bool kWide>
__device__ __forceinline__ uint4 load8(const T *src) {
  if (kWide) return *reinterpret_cast<const uint4 *>(src);
  uint4 raw;
  T *x = reinterpret_cast<T *>(&raw);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = src[i];
  return raw;
}
template <class T, bool kWide>
__device__ __forceinline__ void store8(T *dst, uint4 y) {
  if (kWide) {
    *reinterpret_cast<uint4 *>(dst) = y;
  } else {
    const T *x = reinterpret_cast<const T *>(&y);
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[i] = x[i];
  }
}

template <int D>
__device__ __forceinline__ void put_row(uint8_t *group, int tau, bool is_v, int l, uint32_t codes, uint32_t param) {
  if (is_v) {
    *reinterpret_cast<uint16_t *>(group + 8 * D + kv4_v_unit<D>(tau, 2 * l)) = static_cast<uint16_t>(codes);
    *reinterpret_cast<uint16_t *>(group + 8 * D + kv4_v_unit<D>(tau, 2 * l + 1)) = static_cast<uint16_t>(codes >> 16);
  } else {
    *reinterpret_cast<uint32_t *>(group + tau * (D / 2) + 4 * l) = codes;
  }
  if (l == 0) reinterpret_cast<uint32_t *>(group + 16 * D)[(is_v ? 16 : 0) + tau] = param;
}
template <int D>
__device__ __forceinline__ void get_row(const uint8_t *group, int tau, bool is_v, int l, uint32_t &codes, uint32_t &param) {
  if (is_v)
    codes = *reinterpret_cast<const uint16_t *>(group + 8 * D + kv4_v_unit<D>(tau, 2 * l)) |
            static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(group + 8 * D + kv4_v_unit<D>(tau, 2 * l + 1))) << 16;
  else
    codes = *reinterpret_cast<const uint32_t *>(group + tau * (D / 2) + 4 * l);
  param = reinterpret_cast<const uint32_t *>(group + 16 * D)[(is_v ? 16 : 0) + tau];
}

// ---- few rows: D/8 lanes a row and nothing else, for the shortest chain of loads
template <class T, int D, bool kWide, bool kAppend>
__global__ void __launch_bounds__(256) kv4_few_kernel(const KVArgs a) {
  pdl_prologue();
  constexpr int kLanes = D / 8;
  const int64_t row = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / kLanes;  // (token, K or V, head)
  const int l = threadIdx.x % kLanes;
  const unsigned mask = __ballot_sync(0xffffffffu, row < a.T * 2 * a.H);
  if (row >= a.T * 2 * a.H) return;  // whole rows leave together: kLanes divides 32
  const int64_t tok = row / (2 * a.H);
  const int rest = static_cast<int>(row - tok * 2 * a.H);
  const bool is_v = rest >= a.H;
  const int h = is_v ? rest - a.H : rest;
  const int64_t at = (is_v ? tok * a.v_row + h * a.v_head : tok * a.k_row + h * a.k_head) + 8 * l;
  const int64_t slot = a.slots[tok];
  uint8_t *group;
  int tau;
  if (kAppend) {
    uint32_t codes, param;
    quantise<T, kLanes>(load8<T, kWide>(static_cast<const T *>(is_v ? a.v : a.k) + at), mask, codes, param);
    if (locate(a, slot, h, kv4_group_bytes(D), group, tau)) put_row<D>(group, tau, is_v, l, codes, param);
  } else {
    uint32_t codes = 0, param = 0;  // no slot: zeros
    if (locate(a, slot, h, kv4_group_bytes(D), group, tau)) get_row<D>(group, tau, is_v, l, codes, param);
    store8<T, kWide>(static_cast<T *>(is_v ? a.vo : a.ko) + at, values<T>(codes, param));
  }
}

// ---- many rows: a warp takes 16 consecutive tokens of a head, keys and values.  Prompts fill the cache in
// runs, and the bytes are what counts there, so a group of 16 tokens that the batch holds whole and in order is moved as a
// whole: its V units pass through shared memory, because a token's lie 2 bytes in every 4, and reach memory as full lines.  The
// warp whose tokens a group starts in takes it; the tokens of no whole group go one by one as above.
template <class T, int D, bool kWide, bool kAppend>
__global__ void __launch_bounds__(256) kv4_many_kernel(const KVArgs a) {
  pdl_prologue();
  constexpr int kLanes = D / 8, kRows = 32 / kLanes, kPasses = kGroup / kRows;
  constexpr int kBatch = kPasses < 8 ? kPasses : 8;  // rows' loads under way at once
  constexpr int kStage = 8 * D + 128;                // V codes and parameters of a group
  __shared__ __align__(16) uint8_t s_stage[8][kStage];
  const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
  uint8_t *stage = s_stage[threadIdx.x >> 5];
  const int64_t w = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int64_t i0 = w / a.H * kGroup;
  const int h = static_cast<int>(w % a.H);
  if (i0 >= a.T) return;

  // slots of the tokens i0 - 16 .. i0 + 31: bit q of `next` says that token i0 - 16 + q follows its predecessor's
  auto slot_of = [&](int64_t i) -> int64_t { return i >= 0 && i < a.T ? a.slots[i] : -1; };
  const int64_t s0 = slot_of(i0 - kGroup + lane), s1 = slot_of(i0 + kGroup + lane);
  const int64_t p0 = __shfl_up_sync(0xffffffffu, s0, 1), last = __shfl_sync(0xffffffffu, s0, 31);
  int64_t p1 = __shfl_up_sync(0xffffffffu, s1, 1);
  if (lane == 0) p1 = last;
  const unsigned n0 = __ballot_sync(0xffffffffu, lane > 0 && p0 >= 0 && s0 == p0 + 1), n1 = __ballot_sync(0xffffffffu, p1 >= 0 && s1 == p1 + 1);
  const uint64_t next = n0 | static_cast<uint64_t>(n1) << 32;
  const bool starts = s0 >= 0 && s0 % kGroup == 0 && s0 / a.S < a.n_blocks && ((next >> (lane + 1)) & 0x7fffu) == 0x7fffu;
  const unsigned whole = __ballot_sync(0xffffffffu, starts);  // at most one in each half
  const int before = __ffs(whole & 0xffffu) - 1, here = __ffs(whole >> 16) - 1;
  const int from = before > 0 ? before : 0, to = here >= 0 ? here : kGroup;  // tokens of no whole group

  if (here >= 0) {
    const int64_t i = i0 + here, slot = __shfl_sync(0xffffffffu, s0, kGroup + here);
    uint8_t *group;
    int tau0;
    (void)locate(a, slot, h, kv4_group_bytes(D), group, tau0);
    uint32_t *par = reinterpret_cast<uint32_t *>(stage + 8 * D);
    if (!kAppend) {
#pragma unroll
      for (int x = lane; x < kStage / 16; x += 32) reinterpret_cast<uint4 *>(stage)[x] = reinterpret_cast<const uint4 *>(group + 8 * D)[x];
      __syncwarp();
    }
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const int64_t row = kind ? a.v_row : a.k_row;
      const int64_t at = i * row + h * (kind ? a.v_head : a.k_head) + 8 * l;
#pragma unroll
      for (int b = 0; b < kPasses; b += kBatch) {
        if (kAppend) {
          uint4 raw[kBatch];
#pragma unroll
          for (int p = 0; p < kBatch; ++p) raw[p] = load8<T, kWide>(static_cast<const T *>(kind ? a.v : a.k) + at + ((b + p) * kRows + sub) * row);
#pragma unroll
          for (int p = 0; p < kBatch; ++p) {
            const int tau = (b + p) * kRows + sub;
            uint32_t codes, param;
            quantise<T, kLanes>(raw[p], 0xffffffffu, codes, param);
            if (kind == 0) {
              *reinterpret_cast<uint32_t *>(group + tau * (D / 2) + 4 * l) = codes;
            } else {
              *reinterpret_cast<uint16_t *>(stage + kv4_v_unit<D>(tau, 2 * l)) = static_cast<uint16_t>(codes);
              *reinterpret_cast<uint16_t *>(stage + kv4_v_unit<D>(tau, 2 * l + 1)) = static_cast<uint16_t>(codes >> 16);
            }
            if (l == 0) par[16 * kind + tau] = param;
          }
        } else {
          uint32_t codes[kBatch];
#pragma unroll
          for (int p = 0; p < kBatch; ++p) {
            const int tau = (b + p) * kRows + sub;
            if (kind == 0)
              codes[p] = *reinterpret_cast<const uint32_t *>(group + tau * (D / 2) + 4 * l);
            else
              codes[p] = *reinterpret_cast<const uint16_t *>(stage + kv4_v_unit<D>(tau, 2 * l)) |
                         static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(stage + kv4_v_unit<D>(tau, 2 * l + 1))) << 16;
          }
#pragma unroll
          for (int p = 0; p < kBatch; ++p) {
            const int tau = (b + p) * kRows + sub;
            store8<T, kWide>(static_cast<T *>(kind ? a.vo : a.ko) + at + tau * row, values<T>(codes[p], par[16 * kind + tau]));
          }
        }
      }
    }
    if (kAppend) {
      __syncwarp();
#pragma unroll
      for (int x = lane; x < kStage / 16; x += 32) reinterpret_cast<uint4 *>(group + 8 * D)[x] = reinterpret_cast<const uint4 *>(stage)[x];
    }
  }
  for (int j0 = from / kRows * kRows; j0 < to; j0 += kRows) {
    const int j = j0 + sub;
    const int64_t i = i0 + j;
    const bool mine = j >= from && j < to && i < a.T;
    const int64_t slot = mine ? a.slots[i] : -1;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const int64_t at = i * (kind ? a.v_row : a.k_row) + h * (kind ? a.v_head : a.k_head) + 8 * l;
      uint8_t *group;
      int tau;
      uint32_t codes = 0, param = 0;
      if (kAppend) {
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (mine) raw = load8<T, kWide>(static_cast<const T *>(kind ? a.v : a.k) + at);
        quantise<T, kLanes>(raw, 0xffffffffu, codes, param);
        if (locate(a, slot, h, kv4_group_bytes(D), group, tau)) put_row<D>(group, tau, kind, l, codes, param);
      } else {
        if (locate(a, slot, h, kv4_group_bytes(D), group, tau)) get_row<D>(group, tau, kind, l, codes, param);
        if (mine) store8<T, kWide>(static_cast<T *>(kind ? a.vo : a.ko) + at, values<T>(codes, param));
      }
    }
  }
}

bool wide(const void *p, int64_t row, int64_t head) { return aligned(p, 16) && row % 8 == 0 && head % 8 == 0; }

template <class T, int D, bool kWide, bool kAppend>
void launch_rows(const KVArgs &a, cudaStream_t s) {
  // 16 tokens to a warp once that is a full load of the multiprocessors; below, a token's rows side by side end sooner
  const int64_t warps = (a.T + kGroup - 1) / kGroup * a.H;
  if (warps >= static_cast<int64_t>(kManyWarps) * sm_count())
    launch_pdl(kv4_many_kernel<T, D, kWide, kAppend>, static_cast<unsigned>((warps + 7) / 8), 256, 0, s, a);
  else
    launch_pdl(kv4_few_kernel<T, D, kWide, kAppend>, static_cast<unsigned>((a.T * 2 * a.H * (D / 8) + 255) / 256), 256, 0, s, a);
}

template <class T, int D>
void launch_wide(bool append, bool w, const KVArgs &a, cudaStream_t s) {
  if (append)
    w ? launch_rows<T, D, true, true>(a, s) : launch_rows<T, D, false, true>(a, s);
  else
    w ? launch_rows<T, D, true, false>(a, s) : launch_rows<T, D, false, false>(a, s);
}

template <class T>
void launch_dim(int D, bool append, bool w, const KVArgs &a, cudaStream_t s) {
  if (D == 64) launch_wide<T, 64>(append, w, a, s);
  if (D == 128) launch_wide<T, 128>(append, w, a, s);
  if (D == 256) launch_wide<T, 256>(append, w, a, s);
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
