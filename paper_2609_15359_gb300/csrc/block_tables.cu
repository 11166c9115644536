// block_tables.cu -- block tables and slot maps from request lengths.
//
// A decoder holds its KV tokens in blocks of S tokens (Sec. 3.3: capacity is
// counted in blocks).  Given each request's tokens now (held) and wanted, the
// call gives back the blocks of requests that shrink, takes blocks for those
// that grow, in the scheduler's order while the pool lasts, and writes for
// every new token the cache slot it goes to.  All of it is integer.
//
// Everything follows from three exclusive sums over the requests: blocks given
// back and new tokens in index order, blocks needed in the scheduler's order.
// They are taken by one block (bt_scan_kernel), which also puts the returned
// blocks on the stack; then every new token finds its request by bisection of
// the token offsets and its block from the stack (bt_fill_kernel).  A new
// block's first token always is a new token, so that token writes the table.
#include "maps_internal.cuh"

namespace maps {
namespace {

constexpr int kScanThreads = 1024;

struct BTArgs {
  int32_t R, S, max_blocks, pool;
  const int32_t *held, *want, *order;
  int32_t *table, *free_blocks;
  const int32_t *n_free;
  int32_t *n_free_out, *got;
  int64_t *off;
  int64_t *slots;
  int64_t slots_cap;
  int32_t *pos;
  int64_t *before;  // [R] blocks granted ahead of each request's first, -1 where it is refused
  int64_t *top;     // stack height after the returned blocks
  int32_t *status;
};

struct Need {
  int32_t held, want, hb, wb;
};

// A request's lengths and block counts; both zero (nothing to do) where a length is out of its domain.
__device__ __forceinline__ Need need_of(const BTArgs &a, int r, bool report) {
  Need n;
  n.held = a.held[r];
  n.want = a.want[r];
  const int64_t most = static_cast<int64_t>(a.max_blocks) * a.S;
  if (n.held < 0 || n.want < 0 || n.held > most || n.want > most) {
    if (report) flag_error(a.status, MAPS_E_RANGE);
    n.held = n.want = 0;
  }
  n.hb = static_cast<int32_t>((static_cast<uint32_t>(n.held) + a.S - 1u) / static_cast<uint32_t>(a.S));
  n.wb = static_cast<int32_t>((static_cast<uint32_t>(n.want) + a.S - 1u) / static_cast<uint32_t>(a.S));
  return n;
}

// Exclusive sums of two values over the block, and their totals.
__device__ __forceinline__ void block_scan2(int64_t &x, int64_t &y, int64_t &tx, int64_t &ty) {
  __shared__ int64_t sx[32], sy[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t ix = x, iy = y;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t ux = __shfl_up_sync(0xffffffffu, ix, o), uy = __shfl_up_sync(0xffffffffu, iy, o);
    if (lane >= o) ix += ux, iy += uy;
  }
  if (lane == 31) sx[warp] = ix, sy[warp] = iy;
  __syncthreads();
  if (warp == 0) {
    int64_t wx = sx[lane], wy = sy[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t ux = __shfl_up_sync(0xffffffffu, wx, o), uy = __shfl_up_sync(0xffffffffu, wy, o);
      if (lane >= o) wx += ux, wy += uy;
    }
    sx[lane] = wx;
    sy[lane] = wy;
  }
  __syncthreads();
  x = ix - x + (warp ? sx[warp - 1] : 0);
  y = iy - y + (warp ? sy[warp - 1] : 0);
  tx = sx[31];
  ty = sy[31];
  __syncthreads();
}

__global__ void __launch_bounds__(kScanThreads) bt_scan_kernel(const BTArgs a) {
  pdl_prologue();
  int32_t nf = *a.n_free;
  if (nf < 0 || nf > a.pool) {
    if (threadIdx.x == 0) flag_error(a.status, MAPS_E_RANGE);
    nf = 0;
  }
  // index order: blocks given back (written to the stack as their place is known) and new tokens
  int64_t back = 0, toks = 0;
  for (int base = 0; base < a.R; base += kScanThreads) {
    const int r = base + threadIdx.x;
    Need n = {0, 0, 0, 0};
    if (r < a.R) n = need_of(a, r, true);
    const int64_t mine = n.hb > n.wb ? n.hb - n.wb : 0;
    int64_t x = mine, y = n.want > n.held ? n.want - n.held : 0, tx, ty;
    block_scan2(x, y, tx, ty);
    if (r < a.R) {
      a.off[r] = toks + y;
      for (int64_t i = 0, at = nf + back + x; i < mine; ++i, ++at) {
        if (at >= a.pool) {
          flag_error(a.status, MAPS_E_RANGE);
          break;
        }
        a.free_blocks[at] = a.table[static_cast<int64_t>(r) * a.max_blocks + n.wb + i];
      }
    }
    back += tx;
    toks += ty;
  }
  const int64_t N = min(static_cast<int64_t>(nf) + back, static_cast<int64_t>(a.pool));
  // the scheduler's order: blocks needed, granted while the stack lasts
  int64_t need = 0;
  __shared__ unsigned long long s_granted;
  if (threadIdx.x == 0) s_granted = 0;
  __syncthreads();
  for (int base = 0; base < a.R; base += kScanThreads) {
    const int i = base + threadIdx.x;
    int r = -1;
    Need n = {0, 0, 0, 0};
    if (i < a.R) {
      r = a.order ? a.order[i] : i;
      if (r < 0 || r >= a.R) {
        flag_error(a.status, MAPS_E_RANGE);
        r = -1;
      } else {
        n = need_of(a, r, false);
      }
    }
    const int64_t mine = n.wb > n.hb ? n.wb - n.hb : 0;
    int64_t x = mine, y = 0, tx, ty;
    block_scan2(x, y, tx, ty);
    if (r >= 0) {
      const bool ok = mine == 0 || need + x + mine <= N;
      a.before[r] = ok ? need + x : -1;
      a.got[r] = n.want < n.held || ok ? n.want : n.held;
      if (ok && mine) atomicMax(&s_granted, static_cast<unsigned long long>(need + x + mine));
    }
    need += tx;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    a.off[a.R] = toks;
    *a.top = N;
    *a.n_free_out = static_cast<int32_t>(N - static_cast<int64_t>(s_granted));
    if (toks > a.slots_cap) flag_error(a.status, MAPS_E_RANGE);
  }
}

__global__ void __launch_bounds__(256) bt_fill_kernel(const BTArgs a) {
  pdl_prologue();
  const int64_t j = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t total = a.off[a.R];
  if (j >= total || j >= a.slots_cap) return;
  int lo = 0, hi = a.R;  // off[lo] <= j < off[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.off[mid] <= j)
      lo = mid;
    else
      hi = mid;
  }
  const Need n = need_of(a, lo, false);
  const int32_t p = n.held + static_cast<int32_t>(j - a.off[lo]);
  const int32_t bi = p / a.S, within = p - bi * a.S;
  const int64_t before = a.before[lo];
  int64_t slot = -1;
  if (before >= 0) {
    int32_t *row = a.table + static_cast<int64_t>(lo) * a.max_blocks;
    int32_t block;
    if (bi >= n.hb) {
      const int64_t at = *a.top - 1 - (before + (bi - n.hb));
      block = at >= 0 ? a.free_blocks[at] : -1;
      if (within == 0) row[bi] = block;
    } else {
      block = row[bi];
    }
    slot = static_cast<int64_t>(block) * a.S + within;
  }
  a.slots[j] = slot;
  if (a.pos) a.pos[j] = p;
}

}  // namespace
}  // namespace maps

extern "C" {

size_t maps_block_tables_workspace_size(int32_t R) {
  maps::Carve c(nullptr);
  c.take<int64_t>(1);
  c.take<int64_t>(R > 0 ? static_cast<size_t>(R) : 0);
  return c.bytes();
}

int maps_block_tables(int32_t R, int32_t S, const int32_t *held, const int32_t *want,
                      const int32_t *order, int32_t *table, int32_t max_blocks,
                      int32_t *free_blocks, int32_t pool, const int32_t *n_free,
                      int32_t *n_free_out, int32_t *got_out, int64_t *slot_off_out,
                      int64_t *slots_out, int64_t slots_cap, int32_t *pos_out, void *ws,
                      size_t ws_bytes, void *stream) {
  using namespace maps;
  if (R < 0 || S < 1 || max_blocks < 0 || pool < 0 || slots_cap < 0 ||
      slots_cap > (int64_t(1) << 38))
    return MAPS_E_INVALID;
  if (n_free == nullptr || n_free_out == nullptr || slot_off_out == nullptr) return MAPS_E_INVALID;
  if (R > 0 && (held == nullptr || want == nullptr || got_out == nullptr ||
                (max_blocks > 0 && table == nullptr)))
    return MAPS_E_INVALID;
  if ((pool > 0 && free_blocks == nullptr) || (slots_cap > 0 && slots_out == nullptr))
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, maps_block_tables_workspace_size(R)));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Carve c(ws);
  BTArgs a = {R, S, max_blocks, pool, held, want, order, table, free_blocks, n_free, n_free_out,
              got_out, slot_off_out, slots_out, slots_cap, pos_out, nullptr, nullptr,
              status_word(ws)};
  a.top = c.take<int64_t>(1);
  a.before = c.take<int64_t>(static_cast<size_t>(R));
  launch_pdl(bt_scan_kernel, 1, kScanThreads, 0, s, a);
  if (R > 0 && slots_cap > 0)
    launch_pdl(bt_fill_kernel, static_cast<unsigned>((slots_cap + 255) / 256), 256, 0, s, a);
  return launch_ok();
}

}  // extern "C"
