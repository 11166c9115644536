// kv4_attention_blocks.cu -- attention over the 4-bit cache where each query row and KV head has a list of blocks.
//
// The mathematics, the work's cut into units and the kernel are those of the form for few queries (kv4_attention.cu); a row
// and KV head stands for a request with one query, its list for the block table.  Lists differ between heads, so a unit's
// records are those of one head, and nothing is shared between rows but what the L2 holds.
#include "kv4_attention_few.cuh"

namespace maps {
namespace {

template <class T>
int launch_lists(int D, const AttnArgs &a, cudaStream_t s) {
  const bool one = a.Hq / a.Hkv <= 8;  // 8 rows to a tile, or 16
  if (D == 64) return one ? launch_few<T, 64, 1, true>(a, s) : launch_few<T, 64, 2, true>(a, s);
  if (D == 128) return one ? launch_few<T, 128, 1, true>(a, s) : launch_few<T, 128, 2, true>(a, s);
  return launch_few<T, 256, 1, true>(a, s);
}

void carve_lists(Carve &c, AttnArgs &a, int64_t items) {
  a.parts = c.take<float>(static_cast<size_t>(attn_grid()) * 2 * kMaxParts);
  a.starts = c.take<Start>(items > kMaxLocalB ? static_cast<size_t>(attn_grid()) * kMaxWarps : 0);
  a.units = c.take<uint32_t>(2);
}

}  // namespace
}  // namespace maps

extern "C" {

size_t maps_kv4_attention_blocks_workspace_size(int64_t T, int32_t Hq, int32_t H, int32_t D) {
  (void)Hq, (void)D;
  maps::Carve c(nullptr);
  maps::AttnArgs a = {};
  maps::carve_lists(c, a, T > 0 && H > 0 ? T * H : 0);
  return c.bytes();
}

int maps_kv4_attention_blocks(int32_t dtype, int64_t T, int32_t Hq, int32_t H, int32_t D, int32_t S, const void *q, int64_t q_row,
                              int64_t q_head, const int32_t *blocks, const int32_t *tokens, int64_t n_list, const void *cache,
                              int64_t n_blocks, float sm_scale, void *out, int64_t o_row, int64_t o_head, float *lse, void *ws,
                              size_t ws_bytes, void *stream) {
  using namespace maps;
  if ((dtype != MAPS_BF16 && dtype != MAPS_F16) || !kv4_dim_ok(D) || !kv4_block_ok(S) || T < 0 || T > (int64_t(1) << 30) || H < 1 || Hq < H ||
      Hq % H != 0 || Hq > 65535 || T > ((int64_t(1) << 31) - 1024) / Hq || n_list < 1 || n_list > (1 << 20) || n_list * S > kMaxLen ||
      n_blocks < 0 || !(sm_scale - sm_scale == 0.0f))
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, maps_kv4_attention_blocks_workspace_size(T, Hq, H, D)));
  if (T == 0) return MAPS_OK;
  if (q == nullptr || out == nullptr || blocks == nullptr || tokens == nullptr || (n_blocks > 0 && cache == nullptr) || !aligned(cache, 16) ||
      !aligned(q, 2) || !aligned(out, 2) || !aligned(lse, 4) || !aligned(blocks, 4) || !aligned(tokens, 4))
    return MAPS_E_INVALID;
  const bool wide = aligned(q, 16) && aligned(out, 16) && q_row % 8 == 0 && q_head % 8 == 0 && o_row % 8 == 0 && o_head % 8 == 0;
  const int32_t groups = S / kGroup;
  int32_t shift = -1;
  for (int32_t i = 0; i < 16; ++i)
    if (groups == 1 << i) shift = i;
  AttnArgs a = {static_cast<int32_t>(T * H), Hq, H, S, T, n_blocks, n_list, q, q_row, q_head, o_row, o_head, nullptr, tokens, blocks,
                static_cast<const uint8_t *>(cache), sm_scale, 0, 0, wide,
                static_cast<int64_t>(H) * groups * kv4_group_bytes(D), groups, shift, out, lse};
  a.arrived = reinterpret_cast<uint32_t *>(static_cast<char *>(ws) + kArrivedAt);
  a.status = status_word(ws);
  Carve c(ws);
  carve_lists(c, a, T * H);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return dtype == MAPS_BF16 ? launch_lists<__nv_bfloat16>(D, a, s) : launch_lists<__half>(D, a, s);
}

}  // extern "C"
