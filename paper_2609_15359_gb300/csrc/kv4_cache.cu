// kv4_cache.cu -- writing keys and values to the 4-bit cache, and reading them back.
//
// A row is one token's K or V of one KV head, D channels.  It is held as 16 evenly spaced
// levels: zero = bf16(min), scale = bf16((max - min) * (1/15)), code = round((x - zero) / scale)
// with the reciprocal taken once per row, value = scale * code + zero.  scale * code has at
// most 12 significant bits, so a value is rounded once.  D/8 lanes share a row, 8 channels
// (16 bytes) each; extremes are joined by shuffles.
//
// Bound: the bytes of the 16-bit rows and the records.  65,536 tokens of 8 heads and 128 channels, 340 MB a call,
// take 79 us to append (4.3 TB/s, 0.64 of the measured copy rate; a row's minimum, maximum and
// codes cost about as many issue slots) and 54 us to read (6.3 TB/s).  A decode step's rows take 2-5 us,
// which is launch and latency.
#include "kv4_rows.cuh"

namespace maps {
namespace {

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

template <class T, int D, bool kWide, bool kAppend>
__global__ void __launch_bounds__(256) kv4_many_kernel(const KVArgs a) {
  pdl_prologue();
  __shared__ __align__(16) uint8_t s_stage[8][kStageBytes<D>];
  const int warp = threadIdx.x >> 5;
  move_groups<T, D, kWide, kAppend, 0>(a, static_cast<int64_t>(blockIdx.x) * 8 + warp, s_stage[warp]);
}

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
