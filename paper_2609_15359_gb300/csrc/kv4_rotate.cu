// kv4_rotate.cu -- new tokens' keys and values into the 4-bit cache, keys and queries turned by their tokens' positions.
//
// A pair (a, b) of channels turns by its angle: (a c - b s, b c + a s), products and sums rounded one by one in 32 bits (no
// fused product and sum, so that any program that follows the definition gets the same codes).  A turned key never becomes
// 16 bits: its extremes and codes come from the 32.
//
// D/8 lanes share a row, 8 channels (16 bytes) each; a channel's partner is rot/16 lanes away, or beside it.
//
// Bound: long batches by the bytes, of which queries are most, with issue slots close behind.  65,536 tokens of 32 query heads and 8 KV
// heads of 128 channels on three axes, 1.42 GB, take 261 us (5.4 TB/s, 0.81 of the measured copy rate).  Short ones by launch and
// three rounds of loads (position, angles, rows): 512 tokens 5.4 us.
#include "kv4_rows.cuh"

namespace maps {
namespace {

// Warps of a multiprocessor up to which a token's heads are shared out among several.  512 tokens of 40 heads: 8 or 16 warps 6.1 us, 32 6.8,
// 64 6.7.
constexpr int kUnitWarps = 16;
// Warps of a multiprocessor from which on values pass in groups of 16 tokens: 3,001 tokens of 5 heads of 64 channels (6 warps) 8.6 us, row by
// row 9.1; 512 tokens of 8 heads (2 warps) 5.4 either way.
constexpr int kGroupWarps = 4;

struct RotArgs {
  KVArgs kv;
  int32_t Hq, axes, rot;
  bool wide_axis;
  const void *q;
  void *qo;
  int64_t q_row, q_head, qo_row, qo_head;
  const int32_t *pos, *axis;
  const float *cos_sin;
  int64_t n_pos;
  float minus_zero;
};

// The angles of this lane's channels 8l .. 8l + 7 at a token: channel i becomes x_i c_i + z_i s_i, z its partner, the sine with
// the sign that it has there (a c - b s is a c + b (-s), rounded alike).
template <bool kInter>
struct Turn {
  float c[8], s[8];
  // Of two channels each: 16 bits set, or none for a channel that does not turn, which is x 1 + 0 (-0), x itself whatever it and its
  // partner are.  (One mask for all eight, and channels without a position apart by a branch: 65,536 tokens 263.5 us for 260.7.)
  uint32_t on[4];
  int partner;  // lanes from here
  __device__ __forceinline__ void load(const RotArgs &a, int64_t tok, int l) {
    constexpr int kN = kInter ? 4 : 8;  // pairs
    const int F = a.rot / 2;
    const bool turns = 8 * l < a.rot;
#pragma unroll
    for (int i = 0; i < 4; ++i) on[i] = turns ? 0xffffffffu : 0u;
    const bool second = !kInter && 8 * l >= F;
    partner = !turns ? 0 : second ? -(F / 8) : F / 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = 1.0f, s[i] = -0.0f;
    if (!turns) return;
    const int f0 = kInter ? 4 * l : second ? 8 * l - F : 8 * l;
    int32_t ax[kN] = {};
    if (a.axis) {
#pragma unroll
      for (int i = 0; i < kN; i += 4) {
        if (a.wide_axis) {
          *reinterpret_cast<int4 *>(ax + i) = *reinterpret_cast<const int4 *>(a.axis + f0 + i);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) ax[i + k] = a.axis[f0 + i + k];
        }
      }
    }
    // a position once for each run of pairs on one axis
    auto row_of = [&](int32_t x) -> int64_t {
      const int32_t p = x >= 0 && x < a.axes ? a.pos[x * a.kv.T + tok] : -1;
      if (p < 0 || p >= a.n_pos) {
        flag_error(a.kv.status, MAPS_E_RANGE);
        return -1;
      }
      return static_cast<int64_t>(p) * a.rot;
    };
    int64_t at = row_of(ax[0]);
    uint32_t lost = 0;  // pairs
    bool same = true;
#pragma unroll
    for (int i = 1; i < kN; ++i) same &= ax[i] == ax[0];
    if (same) {
      if (at >= 0) {
        const float *src = a.cos_sin + at + f0;
#pragma unroll
        for (int i = 0; i < kN; i += 4) {
          *reinterpret_cast<float4 *>(c + i) = *reinterpret_cast<const float4 *>(src + i);
          *reinterpret_cast<float4 *>(s + i) = *reinterpret_cast<const float4 *>(src + F + i);
        }
      } else {
        lost = (1u << kN) - 1u;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        if (i > 0 && ax[i] != ax[i - 1]) at = row_of(ax[i]);
        if (at >= 0)
          c[i] = a.cos_sin[at + f0 + i], s[i] = a.cos_sin[at + F + f0 + i];
        else
          lost |= 1u << i;
      }
    }
    if (kInter) {
#pragma unroll
      for (int i = 3; i >= 0; --i) c[2 * i + 1] = c[2 * i] = c[i], s[2 * i + 1] = s[i], s[2 * i] = -s[i];
    } else if (!second) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = -s[i];
    }
    if (lost) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (lost >> (kInter ? i / 2 : i) & 1u) s[i] = -0.0f, on[i / 2] &= i % 2 ? 0x0000ffffu : 0xffff0000u;
      }
    }
  }
  // A row's 8 channels, turned.  All lanes of the warp call it.  A product of two is a fused one with minus_zero, which
  // only the host knows to be -0: the compiler joins a product and a sum of two to one operation, rounded once.
  template <class T>
  __device__ __forceinline__ void apply(const uint4 raw, float minus_zero, float (&y)[8]) const {
    uint4 other;
    if (kInter) {
      other = make_uint4(__funnelshift_l(raw.x, raw.x, 16), __funnelshift_l(raw.y, raw.y, 16), __funnelshift_l(raw.z, raw.z, 16), __funnelshift_l(raw.w, raw.w, 16));
    } else {
      const int from = (threadIdx.x & 31) + partner;
      other.x = __shfl_sync(0xffffffffu, raw.x, from);
      other.y = __shfl_sync(0xffffffffu, raw.y, from);
      other.z = __shfl_sync(0xffffffffu, raw.z, from);
      other.w = __shfl_sync(0xffffffffu, raw.w, from);
    }
    other.x &= on[0], other.y &= on[1], other.z &= on[2], other.w &= on[3];
    const T *x = reinterpret_cast<const T *>(&raw), *z = reinterpret_cast<const T *>(&other);
    const Two none(minus_zero, minus_zero);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const Two own = fused(Two(Cvt<T>::to(x[i]), Cvt<T>::to(x[i + 1])), Two(c[i], c[i + 1]), none);
      (own + fused(Two(Cvt<T>::to(z[i]), Cvt<T>::to(z[i + 1])), Two(s[i], s[i + 1]), none)).get(y[i], y[i + 1]);
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

// A unit is a token and `per` of its query and key heads (queries first); a warp takes one and keeps the angles in registers for
// all its rows, of which 32 / (D/8) pass side by side and kAhead more are under way.  Values, which do not turn, are
// other blocks' of the same launch: row by row, or (kGroups) 16 tokens of a head to a warp, as in maps_kv4_append.
// Four: 65,536 tokens take 261 us, with two 275 (512 tokens 5.2 for 5.4), with eight (registers) 313.  Four blocks a multiprocessor: 261,
// three 277.  Four leave 64 registers a thread, of which all these kernels spill some: 48 bytes in that case, 44 to 240 in the others,
// most where channels do not lie on 16 bytes.
constexpr int kAhead = 4;

template <class T, int D, bool kWide, bool kInter, bool kGroups>
__global__ void __launch_bounds__(256, 4) kv4_rotate_kernel(const RotArgs a, const int64_t value_blocks, const int32_t units, const int32_t per) {
  pdl_prologue();
  constexpr int kLanes = D / 8, kRows = 32 / kLanes;
  __shared__ __align__(16) uint8_t s_stage[kGroups ? 8 : 1][kGroups ? kStageBytes<D> : 16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % kLanes, sub = lane / kLanes;
  uint8_t *group;
  int tau;
  if (blockIdx.x < value_blocks) {
    const int64_t w = static_cast<int64_t>(blockIdx.x) * 8 + warp;
    if (kGroups) {
      move_groups<T, D, kWide, true, 1>(a.kv, w, s_stage[warp]);
    } else {
      const int64_t row = w * kRows + sub, tok = row / a.kv.H;
      const int h = static_cast<int>(row - tok * a.kv.H);
      const bool there = tok < a.kv.T;
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (there) raw = load8<T, kWide>(static_cast<const T *>(a.kv.v) + tok * a.kv.v_row + h * a.kv.v_head + 8 * l);
      const int64_t slot = there ? a.kv.slots[tok] : -1;
      uint32_t codes, param;
      quantise<T, kLanes>(raw, 0xffffffffu, codes, param);
      if (locate(a.kv, slot, h, kv4_group_bytes(D), group, tau)) put_row<D>(group, tau, true, l, codes, param);
    }
    return;
  }
  const int64_t u = (static_cast<int64_t>(blockIdx.x) - value_blocks) * 8 + warp, tok = u / units;
  if (tok >= a.kv.T) return;
  const int first = static_cast<int>(u - tok * units) * per, end = min(first + per, a.Hq + a.kv.H);
  const int64_t slot = end > a.Hq ? a.kv.slots[tok] : -1;
  Turn<kInter> turn;
  bool ready = false;
  // Rows r .. r_end - 1 of the token's rows at `base`.  All lanes of the warp call put(row, y, whether this lane has the row).
  auto pass = [&](const T *base, int64_t stride, int r, int r_end, auto put) {
    const T *src = base + (r + sub) * stride;
    for (; r < r_end; r += kAhead * kRows, src += kAhead * kRows * stride) {
      uint4 raw[kAhead];
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        raw[x] = make_uint4(0, 0, 0, 0);
        if (r + x * kRows + sub < r_end) raw[x] = load8<T, kWide>(src + x * kRows * stride);
      }
      if (!ready) turn.load(a, tok, l), ready = true;
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        if (r + x * kRows >= r_end) break;
        float y[8];
        turn.template apply<T>(raw[x], a.minus_zero, y);
        put(r + x * kRows + sub, y, r + x * kRows + sub < r_end);
      }
    }
  };
  if (first < a.Hq) {
    T *out = static_cast<T *>(a.qo) + tok * a.qo_row + 8 * l;
    pass(static_cast<const T *>(a.q) + tok * a.q_row + 8 * l, a.q_head, first, min(a.Hq, end), [&](int r, const float (&y)[8], bool mine) {
      if (mine) store8<T, kWide>(out + r * a.qo_head, rounded<T>(y));
    });
  }
  if (end > a.Hq) {
    const bool held = locate(a.kv, slot, 0, kv4_group_bytes(D), group, tau);
    const int64_t head = static_cast<int64_t>(a.kv.S / kGroup) * kv4_group_bytes(D);
    pass(static_cast<const T *>(a.kv.k) + tok * a.kv.k_row + 8 * l, a.kv.k_head, max(first - a.Hq, 0), end - a.Hq, [&](int r, const float (&y)[8], bool mine) {
      uint32_t codes, param;
      quantise32<kLanes>(y, 0xffffffffu, codes, param);
      if (mine && held) put_row<D>(group + r * head, tau, false, l, codes, param);
    });
  }
}

template <class T, int D, bool kWide, bool kInter>
void launch_rows(const RotArgs &a, cudaStream_t s) {
  constexpr int kRows = 256 / D;
  const int64_t T_ = a.kv.T, passes = (a.Hq + a.kv.H + kRows - 1) / kRows, want = static_cast<int64_t>(sm_count()) * kUnitWarps;
  const int64_t cut = T_ >= want ? 1 : (want + T_ - 1) / T_;  // units of a token
  const int32_t per = static_cast<int32_t>((passes + (cut < passes ? cut : passes) - 1) / (cut < passes ? cut : passes)) * kRows;
  const int32_t units = (a.Hq + a.kv.H + per - 1) / per;
  const int64_t warps = T_ * units, groups = (T_ + kGroup - 1) / kGroup * a.kv.H;
  const bool many = groups >= static_cast<int64_t>(kGroupWarps) * sm_count();
  const int64_t values = many ? (groups + 7) / 8 : (T_ * a.kv.H + 8 * kRows - 1) / (8 * kRows);
  const unsigned grid = static_cast<unsigned>(values + (warps + 7) / 8);
  if (many)
    launch_pdl(kv4_rotate_kernel<T, D, kWide, kInter, true>, grid, 256, 0, s, a, values, units, per);
  else
    launch_pdl(kv4_rotate_kernel<T, D, kWide, kInter, false>, grid, 256, 0, s, a, values, units, per);
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
               Hq, axes, rot, aligned(axis, 16), q, q_out, q_row, q_head, qo_row, qo_head, pos, axis, cos_sin, n_pos, -0.0f};
  const bool w = wide(k, k_row, k_head) && wide(v, v_row, v_head) && (Hq == 0 || (wide(q, q_row, q_head) && wide(q_out, qo_row, qo_head)));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MAPS_BF16)
    launch_dim<__nv_bfloat16>(D, w, interleaved, a, s);
  else
    launch_dim<__half>(D, w, interleaved, a, s);
  return launch_ok();
}
