// kv4_attention.cu -- attention over the paged 4-bit KV cache.
//
// out_i = sum_j softmax_j(sm_scale q_i . k_j) v_j over the keys j that query i sees, with the
// running maximum and sum of the softmax, so the keys are passed over once.
#include "kv4.cuh"

namespace maps {
namespace {

constexpr int kTile = 128;  // keys of a step, one per thread

struct AttnArgs {
  int32_t B, Hq, Hkv, S;
  int64_t T, n_blocks, max_blocks;
  const void *q;
  int64_t q_row, q_head, o_row, o_head;
  const int64_t *off;
  const int32_t *len, *table;
  const uint8_t *cache;
  float scale;
  int32_t causal, window;
  void *out;
  float *lse;
  int32_t *status;
};

template <class T, int D>
__global__ void __launch_bounds__(kTile) attn_simple_kernel(const AttnArgs a) {
  pdl_prologue();
  __shared__ float s_q[D], s_p[kTile], s_red[8];
  const int tid = threadIdx.x;
  const int64_t i = blockIdx.x;
  const int hq = blockIdx.y, h = hq / (a.Hq / a.Hkv);
  T *out = static_cast<T *>(a.out) + i * a.o_row + hq * a.o_head;
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.off[mid] <= i)
      lo = mid;
    else
      hi = mid;
  }
  const int b = lo;
  const int64_t n_q = a.off[b + 1] - a.off[b];
  int32_t n = a.len[b];
  if (i < a.off[b] || i >= a.off[b + 1]) return;
  if (n < 0 || n > a.max_blocks * a.S) {
    if (tid == 0) flag_error(a.status, MAPS_E_RANGE);
    n = 0;
  }
  const int64_t pos = n - n_q + (i - a.off[b]);
  const int64_t last = pos < 0 ? -1 : a.causal ? pos : n - 1;
  const int64_t first = a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
  for (int d = tid; d < D; d += kTile) s_q[d] = Cvt<T>::to(static_cast<const T *>(a.q)[i * a.q_row + hq * a.q_head + d]);
  __syncthreads();
  float m = -INFINITY, l = 0.0f, acc[2] = {0.0f, 0.0f};
  auto group_of = [&](int64_t j) -> const uint8_t * {
    const int64_t page = j / a.S;
    const int32_t block = a.table[b * a.max_blocks + page];
    if (block < 0 || block >= a.n_blocks) {
      flag_error(a.status, MAPS_E_RANGE);
      return nullptr;
    }
    return a.cache + ((static_cast<int64_t>(block) * a.Hkv + h) * (a.S / kGroup) + (j - page * a.S) / kGroup) * kv4_group_bytes(D);
  };
  for (int64_t j0 = first; j0 <= last; j0 += kTile) {
    const int64_t j = j0 + tid;
    float x = -INFINITY;
    if (j <= last) {
      if (const uint8_t *grp = group_of(j)) {
        const float2 p = kv4_param(reinterpret_cast<const uint32_t *>(grp + 16 * D)[j % kGroup]);
        const uint32_t *row = reinterpret_cast<const uint32_t *>(grp + (j % kGroup) * (D / 2));
        float dot = 0.0f;
        for (int w = 0; w < D / 8; ++w) {
          const uint32_t c = row[w];
#pragma unroll
          for (int e = 0; e < 8; ++e) dot = fmaf(s_q[8 * w + e], fmaf(p.x, static_cast<float>(c >> (4 * e) & 15u), p.y), dot);
        }
        x = dot * a.scale;
      }
    }
    float mx = x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if (tid % 32 == 0) s_red[tid / 32] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    const float mn = fmaxf(m, mx);
    const float ref = mn == -INFINITY ? 0.0f : mn;
    const float p = x == -INFINITY ? 0.0f : __expf(x - ref), corr = __expf(m - ref);
    s_p[tid] = p;
    float sum = p;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (tid % 32 == 0) s_red[4 + tid / 32] = sum;
    __syncthreads();
    l = l * corr + (s_red[4] + s_red[5] + s_red[6] + s_red[7]);
    m = mn;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int d = tid + e * kTile;
      if (d >= D) break;
      acc[e] *= corr;
      for (int64_t jj = j0; jj <= last && jj < j0 + kTile; ++jj) {
        const float w = s_p[jj - j0];
        if (w == 0.0f) continue;
        const uint8_t *grp = group_of(jj);
        const int tau = static_cast<int>(jj % kGroup);
        const float2 vp = kv4_param(reinterpret_cast<const uint32_t *>(grp + 16 * D)[16 + tau]);
        const uint16_t unit = *reinterpret_cast<const uint16_t *>(grp + 8 * D + kv4_v_unit<D>(tau, d / 4));
        acc[e] = fmaf(w, fmaf(vp.x, static_cast<float>(unit >> (4 * (d % 4)) & 15), vp.y), acc[e]);
      }
    }
    __syncthreads();
  }
  for (int e = 0; e < 2; ++e) {
    const int d = tid + e * kTile;
    if (d < D) out[d] = Cvt<T>::from(l == 0.0f ? 0.0f : acc[e] / l);
  }
  if (a.lse && tid == 0) a.lse[i * a.Hq + hq] = l == 0.0f ? -INFINITY : m + logf(l);
}

template <class T>
void launch_simple(int D, const AttnArgs &a, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.T), static_cast<unsigned>(a.Hq));
  if (D == 64) launch_pdl(attn_simple_kernel<T, 64>, grid, kTile, 0, s, a);
  if (D == 128) launch_pdl(attn_simple_kernel<T, 128>, grid, kTile, 0, s, a);
  if (D == 256) launch_pdl(attn_simple_kernel<T, 256>, grid, kTile, 0, s, a);
}

}  // namespace
}  // namespace maps

extern "C" {

size_t maps_kv4_attention_workspace_size(int32_t B, int64_t T, int32_t Hq, int32_t Hkv, int32_t D) {
  (void)B, (void)T, (void)Hq, (void)Hkv, (void)D;
  return maps::kCtrlBytes;
}

int maps_kv4_attention(int32_t dtype, int32_t B, int64_t T, int32_t Hq, int32_t Hkv, int32_t D,
                       int32_t S, const void *q, int64_t q_row, int64_t q_head,
                       const int64_t *qo_off, const int32_t *kv_len, const int32_t *table,
                       int64_t max_blocks, const void *cache, int64_t n_blocks, float sm_scale,
                       int32_t causal, int32_t window, void *out, int64_t o_row, int64_t o_head,
                       float *lse, void *ws, size_t ws_bytes, void *stream) {
  using namespace maps;
  if ((dtype != MAPS_BF16 && dtype != MAPS_F16) || !kv4_dim_ok(D) || !kv4_block_ok(S) || B < 0 ||
      T < 0 || T > (int64_t(1) << 30) || Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 || Hq > 65535 ||
      max_blocks < 0 || max_blocks > 0x7fffffff || n_blocks < 0 || window < 0 || (causal != 0 && causal != 1) || !(sm_scale - sm_scale == 0.0f))
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, maps_kv4_attention_workspace_size(B, T, Hq, Hkv, D)));
  if (T == 0 || B == 0) return MAPS_OK;
  if (q == nullptr || out == nullptr || qo_off == nullptr || kv_len == nullptr ||
      (max_blocks > 0 && table == nullptr) || (n_blocks > 0 && cache == nullptr) || !aligned(cache, 16) || !aligned(q, 2) || !aligned(lse, 4) ||
      !aligned(out, 2))
    return MAPS_E_INVALID;
  const AttnArgs a = {B, Hq, Hkv, S, T, n_blocks, max_blocks, q, q_row, q_head, o_row, o_head, qo_off, kv_len, table,
                      static_cast<const uint8_t *>(cache), sm_scale, causal, window, out, lse, status_word(ws)};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MAPS_BF16)
    launch_simple<__nv_bfloat16>(D, a, s);
  else
    launch_simple<__half>(D, a, s);
  return launch_ok();
}

}  // extern "C"
