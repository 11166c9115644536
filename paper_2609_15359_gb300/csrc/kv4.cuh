// kv4.cuh -- the 4-bit KV cache's layout and value types, shared by the kernels
// that write, read back and attend over it.
//
// cache[block][kv head] is one record: S/16 groups of 16 tokens, each
//   8D bytes  K codes, row-major: token tau's row is D/2 bytes, channel 2i in the low half of byte i;
//   8D bytes  V codes, in units of 16 bits that hold 4 neighbouring channels of one token (below);
//   128 bytes 16 x {K scale, K zero}, 16 x {V scale, V zero}, bfloat16.
// A value is scale * code + zero.  Everything that one KV head of one block holds lies
// together, so a reader moves it with one bulk copy.
//
// V order.  In out = P V the 16 tokens of a group are the depth of a tensor-core step whose
// A operand is V transposed: lane (g, t) of a warp (g = lane / 4, t = lane % 4) holds the
// token pairs 2t, 2t+1 and 8+2t, 8+2t+1 of channel rows.  Channels go to lanes in runs of
// D/8, four to a 32-bit word with the even token in its low half, so a lane's words are
// consecutive and (word & 0x000f000f) is the pair of one channel:
//   token = 8h + 2t + parity, channel = g * (D/8) + 4 * (a * B + b) + r,  B = min(D/32, 4),
//   unit index = ((((h * A + a) * 8 + g) * 4 + t) * B + b) * 2 + parity,  A = D/32/B.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "maps_internal.cuh"

namespace maps {

constexpr int kGroup = 16;  // tokens of a group

__host__ __device__ constexpr int kv4_group_bytes(int D) { return 16 * D + 128; }
inline bool kv4_dim_ok(int D) { return D == 64 || D == 128 || D == 256; }
inline bool kv4_block_ok(int S) { return S >= kGroup && S % kGroup == 0 && S <= 4096; }

// Byte offset within a group's V codes of the unit of token tau (0..15) that holds channels 4c4 .. 4c4+3.
template <int D>
__host__ __device__ __forceinline__ int kv4_v_unit(int tau, int c4) {
  constexpr int B = D / 32 < 4 ? D / 32 : 4, A = D / 32 / B;
  const int g = c4 / (D / 32), w = c4 % (D / 32);
  const int h = tau >> 3, t = (tau & 7) >> 1, parity = tau & 1;
  return (((((h * A + w / B) * 8 + g) * 4 + t) * B + w % B) * 2 + parity) * 2;
}

template <class T>
struct Cvt;
template <>
struct Cvt<__nv_bfloat16> {
  static __device__ __forceinline__ float to(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 from(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Cvt<__half> {
  static __device__ __forceinline__ float to(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half from(float x) { return __float2half_rn(x); }
};

__device__ __forceinline__ float2 kv4_param(uint32_t w) {  // {scale, zero}
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

}  // namespace maps
