// kv4_rotate.cu -- new tokens' keys and values into the 4-bit cache, keys and queries turned by their tokens' positions.
//
// A pair (a, b) of channels turns by its angle: (a c - b s, b c + a s), products and sums rounded one by one in 32 bits (no
// fused product and sum, so that any program that follows the definition gets the same codes).  A turned key never becomes
// 16 bits: its extremes and codes come from the 32.
//
// D/8 lanes share a row, 8 channels (16 bytes) each; a channel's partner is rot/16 lanes away, or beside it.
#include "kv4_rows.cuh"

namespace maps {
namespace {

struct RotArgs {
  KVArgs kv;
  int32_t Hq, axes, rot;
  const void *q;
  void *qo;
  int64_t q_row, q_head, qo_row, qo_head;
  const int32_t *pos, *axis;
  const float *cos_sin;
  int64_t n_pos;
};

// The angles of this lane's channels 8l .. 8l + 7 at a token: of their 8 pairs, or, where pairs are neighbours, 4.
template <bool kInter>
struct Turn {
  static constexpr int kN = kInter ? 4 : 8;
  float c[kN], s[kN];  // the sine with the sign that it has for this half of the pairs
  bool on;
  int partner;  // lanes from here
  __device__ __forceinline__ void load(const RotArgs &a, int64_t tok, int l) {
    const int F = a.rot / 2;
    on = 8 * l < a.rot;
    const bool second = !kInter && 8 * l >= F;
    partner = kInter || !on ? 0 : second ? -(F / 8) : F / 8;
    if (!on) return;
    const int f0 = kInter ? 4 * l : second ? 8 * l - F : 8 * l;
    int64_t at[kN];
    bool same = true;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int32_t x = a.axis ? a.axis[f0 + i] : 0;
      const bool good = x >= 0 && x < a.axes;
      const int32_t p = good ? a.pos[x * a.kv.T + tok] : -1;
      at[i] = p >= 0 && p < a.n_pos ? static_cast<int64_t>(p) * a.rot : -1;
      if (at[i] < 0) flag_error(a.kv.status, MAPS_E_RANGE);
      same &= at[i] == at[0];
    }
    if (same && at[0] >= 0) {
      const float4 *src = reinterpret_cast<const float4 *>(a.cos_sin + at[0] + f0);
      const float4 *sin = reinterpret_cast<const float4 *>(a.cos_sin + at[0] + F + f0);
#pragma unroll
      for (int i = 0; i < kN; i += 4) {
        *reinterpret_cast<float4 *>(c + i) = src[i / 4];
        *reinterpret_cast<float4 *>(s + i) = sin[i / 4];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        c[i] = at[i] >= 0 ? a.cos_sin[at[i] + f0 + i] : 1.0f;
        s[i] = at[i] >= 0 ? a.cos_sin[at[i] + F + f0 + i] : 0.0f;
      }
    }
    if (!kInter && !second) {
#pragma unroll
      for (int i = 0; i < kN; ++i) s[i] = -s[i];
    }
  }
  // A row's 8 channels, turned.  `mask`: the lanes that call this, whole rows.
  template <class T>
  __device__ __forceinline__ void apply(const uint4 raw, unsigned mask, float (&y)[8]) const {
    const T *x = reinterpret_cast<const T *>(&raw);
    if (kInter) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = Cvt<T>::to(x[2 * i]), q = Cvt<T>::to(x[2 * i + 1]);
        y[2 * i] = on ? __fsub_rn(__fmul_rn(p, c[i]), __fmul_rn(q, s[i])) : p;
        y[2 * i + 1] = on ? __fadd_rn(__fmul_rn(q, c[i]), __fmul_rn(p, s[i])) : q;
      }
    } else {
      uint4 other;
      const int from = (threadIdx.x & 31) + partner;
      other.x = __shfl_sync(mask, raw.x, from);
      other.y = __shfl_sync(mask, raw.y, from);
      other.z = __shfl_sync(mask, raw.z, from);
      other.w = __shfl_sync(mask, raw.w, from);
      const T *z = reinterpret_cast<const T *>(&other);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = Cvt<T>::to(x[i]);
        y[i] = on ? __fadd_rn(__fmul_rn(p, c[i % kN]), __fmul_rn(Cvt<T>::to(z[i]), s[i % kN])) : p;
      }
    }
  }
};

template <class T>
__device__ __forceinline__ uint4 rounded(const float (&y)[8]) {
  uint4 out;
  T *z = reinterpret_cast<T *>(&out);
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] = Cvt<T>::from(y[i]);
  return out;
}

// ---- few rows: D/8 lanes a row and nothing else, for the shortest chain of loads
template <class T, int D, bool kWide, bool kInter>
__global__ void __launch_bounds__(256) kv4_rotate_few_kernel(const RotArgs a) {
  pdl_prologue();
  constexpr int kLanes = D / 8;
  const int64_t row = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / kLanes;
  const int l = threadIdx.x % kLanes, per = a.Hq + 2 * a.kv.H;
  const bool there = row < a.kv.T * per;
  const int64_t tok = row / per;
  const int rest = static_cast<int>(row - tok * per);
  const bool is_q = rest < a.Hq, is_v = rest >= a.Hq + a.kv.H;
  const unsigned turned = __ballot_sync(0xffffffffu, there && !is_v);
  const unsigned values = __ballot_sync(0xffffffffu, there && is_v);
  if (!there) return;  // whole rows leave together: kLanes divides 32
  if (is_v) {
    const int h = rest - a.Hq - a.kv.H;
    const uint4 raw = load8<T, kWide>(static_cast<const T *>(a.kv.v) + tok * a.kv.v_row + h * a.kv.v_head + 8 * l);
    uint32_t codes, param;
    quantise<T, kLanes>(raw, values, codes, param);
    uint8_t *group;
    int tau;
    if (locate(a.kv, a.kv.slots[tok], h, kv4_group_bytes(D), group, tau)) put_row<D>(group, tau, true, l, codes, param);
    return;
  }
  const int h = is_q ? rest : rest - a.Hq;
  const T *src = is_q ? static_cast<const T *>(a.q) + tok * a.q_row + h * a.q_head : static_cast<const T *>(a.kv.k) + tok * a.kv.k_row + h * a.kv.k_head;
  const uint4 raw = load8<T, kWide>(src + 8 * l);
  const int64_t slot = is_q ? -1 : a.kv.slots[tok];
  Turn<kInter> turn;
  turn.load(a, tok, l);
  float y[8];
  turn.template apply<T>(raw, turned, y);
  const unsigned keys = __ballot_sync(turned, !is_q);
  if (is_q) {
    store8<T, kWide>(static_cast<T *>(a.qo) + tok * a.qo_row + h * a.qo_head + 8 * l, rounded<T>(y));
  } else {
    uint32_t codes, param;
    quantise32<kLanes>(y, keys, codes, param);
    uint8_t *group;
    int tau;
    if (locate(a.kv, slot, h, kv4_group_bytes(D), group, tau)) put_row<D>(group, tau, false, l, codes, param);
  }
}

template <class T, int D, bool kWide, bool kInter>
void launch_rows(const RotArgs &a, cudaStream_t s) {
  launch_pdl(kv4_rotate_few_kernel<T, D, kWide, kInter>, static_cast<unsigned>((a.kv.T * (a.Hq + 2 * a.kv.H) * (D / 8) + 255) / 256), 256, 0, s, a);
}
template <class T, int D>
void launch_form(bool w, bool inter, const RotArgs &a, cudaStream_t s) {
  if (inter)
    w ? launch_rows<T, D, true, true>(a, s) : launch_rows<T, D, false, true>(a, s);
  else
    w ? launch_rows<T, D, true, false>(a, s) : launch_rows<T, D, false, false>(a, s);
}
template <class T>
void launch_dim(int D, bool w, bool inter, const RotArgs &a, cudaStream_t s) {
  if (D == 64) launch_form<T, 64>(w, inter, a, s);
  if (D == 128) launch_form<T, 128>(w, inter, a, s);
  if (D == 256) launch_form<T, 256>(w, inter, a, s);
}

}  // namespace
}  // namespace maps

extern "C" int maps_kv4_append_rotated(int32_t dtype, int64_t T, int32_t Hq, int32_t H, int32_t D, int32_t S, const void *q, int64_t q_row,
                                       int64_t q_head, const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                                       int64_t v_head, int32_t axes, const int32_t *pos, const int32_t *axis, int32_t rot,
                                       int32_t interleaved, const float *cos_sin, int64_t n_pos, const int64_t *slots, void *cache,
                                       int64_t n_blocks, void *q_out, int64_t qo_row, int64_t qo_head, void *ws, size_t ws_bytes,
                                       void *stream) {
  using namespace maps;
  if ((dtype != MAPS_BF16 && dtype != MAPS_F16) || !kv4_dim_ok(D) || !kv4_block_ok(S) || H < 1 || H > 65535 || Hq < 0 || Hq > 65535 || T < 0 ||
      T > (int64_t(1) << 30) / (static_cast<int64_t>(Hq) + H) || n_blocks < 0 || rot < 0 || rot > D || rot % 16 != 0 || axes < 1 || axes > 8 ||
      n_pos < 0 || (interleaved != 0 && interleaved != 1))
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, kCtrlBytes));
  if (T == 0) return MAPS_OK;
  if (k == nullptr || v == nullptr || slots == nullptr || (n_blocks > 0 && cache == nullptr) || !aligned(cache, 16) || !aligned(k, 2) ||
      !aligned(v, 2) || (Hq > 0 && (q == nullptr || q_out == nullptr || !aligned(q, 2) || !aligned(q_out, 2))) ||
      (rot > 0 && (pos == nullptr || (n_pos > 0 && cos_sin == nullptr) || !aligned(pos, 4) || !aligned(axis, 4) || !aligned(cos_sin, 16))))
    return MAPS_E_INVALID;
  RotArgs a = {{T, n_blocks, H, S, k, v, nullptr, nullptr, k_row, k_head, v_row, v_head, slots, static_cast<uint8_t *>(cache), status_word(ws)},
               Hq, axes, rot, q, q_out, q_row, q_head, qo_row, qo_head, pos, axis, cos_sin, n_pos};
  const bool w = wide(k, k_row, k_head) && wide(v, v_row, v_head) && (Hq == 0 || (wide(q, q_row, q_head) && wide(q_out, qo_row, qo_head)));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MAPS_BF16)
    launch_dim<__nv_bfloat16>(D, w, interleaved, a, s);
  else
    launch_dim<__half>(D, w, interleaved, a, s);
  return launch_ok();
}
