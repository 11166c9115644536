// kv4_attention_products.cuh -- what the kernels of attention for few query rows share: the two products on codes, the scale that
// weights are held at, and parts of sums that are joined.
#pragma once

#include "kv4_attention.cuh"

namespace maps {
namespace {

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

}  // namespace
}  // namespace maps
