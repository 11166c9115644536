// kv4_attention.cu -- attention over the paged 4-bit KV cache, form for few queries a request.
//
// out_i = sum_j softmax_j(sm_scale q_i . k_j) v_j over the keys j that query i sees, with the
// running maximum and sum of the softmax, so the cache is passed over once.
//
// Mathematics.  With k = s c + z (codes c), q . k = s (q . c) + z sum(q), and with weights p,
// sum p v = sum (p s) c + sum p z: the matrix products run on bare codes, and scales and zeros cost
// a few operations a token instead of D.  A code is a half number as it stands (codes_of), so eight
// codes take five operations.  q is scaled by a power of two to fill half's range; p s is held
// relative to the largest p s so far.
//
// Bound.  A key and value of D channels are D + 8 bytes and serve the few query rows (queries x
// heads of one KV head) of one request, so long calls are bound by the cache's bytes: 128 requests
// of 64 to 8,192 tokens, 8 KV heads of 128 channels, 566 MB, take 116 us (4.9 TB/s, 0.72 of the
// measured copy rate).  Within the passes it is 6.2 TB/s; the rest is a call's fixed part, about 11 us of
// dependent steps: the plan (2), first queries and records (2), a first unit (4), the joins (3).  Short calls take little
// else: one request of 2,048 tokens 12 us.
//
// Shape.  The products are transposed: 16 tokens (or 16 channels) are the 16 rows of an
// m16n8k16 step and 8 query rows its columns, so up to 8 rows waste nothing (as the columns of a
// tcgen05 product they would meet 128 rows and cross tensor memory twice), and K and V are the
// register operand, straight from the cache's bytes by 16-byte loads from shared memory.  P
// crosses from the first product's result to the second's operand by an 8 x 8 transpose between lanes.
//
// Split.  The call's work is cut into units of kTok tokens of one (request, KV head, tile of
// query rows).  Every warp of the grid takes an equal run of consecutive units, whatever
// the lengths, and streams its records of the cache through a ring of its own in shared
// memory with bulk copies, two or more stages ahead; nothing is waited for across warps until the end. What
// a run begins or ends inside of is joined afterwards: within the block through shared memory, across blocks
// by the last block to arrive, in the order of the keys, so results do not depend on timing.
#include "kv4_attention_few.cuh"

namespace maps {
namespace {

// Query rows of a request to a KV head up to which this form serves it where the other may.  Both grow with the rows, this
// one by tiles of 16: 32 requests of 4,096 random tokens, 128 channels: 64 rows 189 us here, 229 there; 96 rows 265, 229;
// 128 rows 343, 231.  With 64 channels 191, 181 at 96; with 4 requests 53, 57 at 96 and 100, 69 at 256.
constexpr int kFewRows = 96;

template <class T>
int launch_dim(int D, const AttnArgs &a, cudaStream_t s) {
  // 8 rows to a tile where a request has at most 8 on average, else 16: for 16 rows two tiles of 8 pass over the cache twice
  // (64 requests of 4,096 tokens, 128 channels: 112 us, 92 with one of 16; 1,000 tokens: 40, 39), for 8 a tile of 16 is half
  // empty (65, 89).  256 channels of 16 rows do not fit a warp's registers.
  const bool one = a.T * (a.Hq / a.Hkv) <= static_cast<int64_t>(8) * a.B;
  if (D == 64) return one ? launch_few<T, 64, 1, false>(a, s) : launch_few<T, 64, 2, false>(a, s);
  if (D == 128) return one ? launch_few<T, 128, 1, false>(a, s) : launch_few<T, 128, 2, false>(a, s);
  return launch_few<T, 256, 1, false>(a, s);
}

}  // namespace
}  // namespace maps

extern "C" {

static void carve(maps::Carve &c, maps::AttnArgs &a, int32_t B, int64_t T, int32_t Hq, int32_t Hkv, int32_t D) {
  using namespace maps;
  a.parts = c.take<float>(static_cast<size_t>(attn_grid()) * 2 * kMaxParts);
  a.starts = c.take<Start>(B > kMaxLocalB ? static_cast<size_t>(attn_grid()) * kMaxWarps : 0);
  a.units = c.take<uint32_t>(2);
  // A decode step has as many rows as requests and spends no launches on the other form; so has a batch of fewer rows than
  // requests, whose chunks, where it has any, are served here too.
  a.few_rows = Hkv > 0 && attn_many_dim(D) && T > B && T * (Hq / Hkv) > kFewRows ? kFewRows : 0;
  if (a.few_rows) attn_many_carve(c, a, B, D);
}

size_t maps_kv4_attention_workspace_size(int32_t B, int64_t T, int32_t Hq, int32_t Hkv, int32_t D) {
  maps::Carve c(nullptr);
  maps::AttnArgs a = {};
  carve(c, a, B, T, Hq, Hkv, D);
  return c.bytes();
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
      T > ((int64_t(1) << 31) - 1024) / Hq || max_blocks < 0 || max_blocks > 0x7fffffff || n_blocks < 0 || window < 0 ||
      (causal != 0 && causal != 1) || !(sm_scale - sm_scale == 0.0f))
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, maps_kv4_attention_workspace_size(B, T, Hq, Hkv, D)));
  if (T == 0 || B == 0) return MAPS_OK;
  if (q == nullptr || out == nullptr || qo_off == nullptr || kv_len == nullptr ||
      (max_blocks > 0 && table == nullptr) || (n_blocks > 0 && cache == nullptr) || !aligned(cache, 16) || !aligned(q, 2) ||
      !aligned(lse, 4) || !aligned(out, 2))
    return MAPS_E_INVALID;
  const bool wide = aligned(q, 16) && aligned(out, 16) && q_row % 8 == 0 && q_head % 8 == 0 && o_row % 8 == 0 && o_head % 8 == 0;
  const int32_t groups = S / kGroup;
  int32_t shift = -1;
  for (int32_t i = 0; i < 16; ++i)
    if (groups == 1 << i) shift = i;
  AttnArgs a = {B, Hq, Hkv, S, T, n_blocks, max_blocks, q, q_row, q_head, o_row, o_head, qo_off, kv_len, table,
                static_cast<const uint8_t *>(cache), sm_scale, causal, window, wide,
                static_cast<int64_t>(Hkv) * groups * kv4_group_bytes(D), groups, shift, out, lse};
  a.arrived = reinterpret_cast<uint32_t *>(static_cast<char *>(ws) + kArrivedAt);
  a.status = status_word(ws);
  Carve c(ws);
  carve(c, a, B, T, Hq, Hkv, D);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  MAPS_TRY(dtype == MAPS_BF16 ? launch_dim<__nv_bfloat16>(D, a, s) : launch_dim<__half>(D, a, s));
  return a.few_rows ? attn_many(dtype, D, a, s) : MAPS_OK;
}

}  // extern "C"
