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
// bt_scan_kernel takes them, one block for up to 1,024 requests, else a cluster
// of eight blocks; its time is the latency of two rounds of loads and sums.
// Then the sums are expanded, one thread a token: a coarse index and a short
// bisection of the token offsets give the request, a record of it the rest.  A
// new block's first token always is a new token, so that token writes the
// table.  With few tokens one kernel does it all, and takes a block that was
// just returned from its old row, so that returning and taking need not wait
// for one another; with many, which the writes bound, the returned blocks go
// onto the stack first and a token costs one load of it.
//
// Bound: a decode step (64 requests) by latency, 4.5 us for a launch and three rounds of dependent loads;
// 4,096 requests with prompts up to 8,192 tokens, 32 MB mostly written, 27 us: 16 of them are sums and
// launches, in the rest slots and positions are written at about 3 TB/s.
#include <cooperative_groups.h>

#include <algorithm>

#include "maps_internal.cuh"

namespace maps {
namespace {

namespace cg = cooperative_groups;

constexpr int kScanThreads = 1024;
constexpr int kCluster = 8;
constexpr int kFillThreads = 256;
// Up to here a token is a thread's, beyond a thread has eight: 2,048 requests with 131,072 new tokens take 11.4 us in the first
// form and 14.7 in the second, with 1,048,576 of them 15.7 and 14.6.
constexpr int kFewTokens = 1 << 19;
constexpr int kManyEach = 8;
constexpr int kCoarse = 2048;      // marks of a coarse index

// What the tokens of a request need to know of it.
struct alignas(32) Request {
  int64_t begin;   // its first new token
  int64_t before;  // blocks granted ahead of its first, -1 where it is refused
  int32_t held, last;  // tokens held, and the block of the last of them (where it is not full)
  uint32_t named;      // whether the order has named it (where several blocks take the sums)
};
// The sums over all, for the kernels that expand them.
struct alignas(32) Totals {
  int64_t returned, tokens, stack;  // stack: entries once the returned blocks are on it
  int32_t free, token_shift, returned_shift;
};

struct BTArgs {
  int32_t R, S, max_blocks, pool;
  int32_t s_shift;  // log2 S where S is a power of two, else -1
  const int32_t *held, *want, *order;
  int32_t *table, *free_blocks;
  const int32_t *n_free;
  int32_t *n_free_out, *got;
  int64_t *off;
  int64_t *slots;
  int64_t slots_cap;
  int32_t *pos;
  Totals *totals;
  Request *requests;  // [R]
  int64_t *back;      // [R + 1] blocks given back ahead of each request's
  int32_t *coarse;    // [2][kCoarse + 2] the requests of every 2^shift-th new token and returned block
  int32_t *status;
};

__device__ __forceinline__ uint32_t block_of(const BTArgs &a, uint32_t position) {
  return a.s_shift >= 0 ? position >> a.s_shift : position / static_cast<uint32_t>(a.S);
}

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
  n.hb = static_cast<int32_t>(block_of(a, static_cast<uint32_t>(n.held) + a.S - 1u));
  n.wb = static_cast<int32_t>(block_of(a, static_cast<uint32_t>(n.want) + a.S - 1u));
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

// Sums of x and y ahead of this block over the cluster, and over all of it.
template <int kBlocks>
__device__ __forceinline__ void cluster_sums(int64_t x, int64_t y, int64_t &bx, int64_t &by, int64_t &tx, int64_t &ty) {
  bx = by = 0;
  tx = x;
  ty = y;
  if (kBlocks == 1) return;
  __shared__ int64_t s_sum[2], s_all[4];
  cg::cluster_group cl = cg::this_cluster();
  if (threadIdx.x == 0) s_sum[0] = x, s_sum[1] = y;
  cl.sync();
  if (threadIdx.x < 32) {
    const int k = threadIdx.x;
    int64_t ux = 0, uy = 0;
    if (k < kBlocks) {
      const int64_t *p = cl.map_shared_rank(s_sum, k);
      ux = p[0], uy = p[1];
    }
    const bool ahead = k < static_cast<int>(cl.block_rank());
    int64_t v[4] = {ahead ? ux : 0, ahead ? uy : 0, ux, uy};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
      if (k == 0) s_all[i] = v[i];
    }
  }
  cl.sync();  // nobody goes on to write its sums, or leaves, while they are being read
  bx = s_all[0], by = s_all[1], tx = s_all[2], ty = s_all[3];
}

// The coarse index over sums: mark c is the request that element c << shift belongs to, so an
// element's request lies between two neighbouring marks.
__device__ __forceinline__ int mark_shift(int64_t total) {
  const int bits = 64 - __clzll(total > kCoarse ? (total - 1) / kCoarse : 0);
  return bits;
}
__device__ __forceinline__ void set_marks(int32_t *marks, int r, int64_t begin, int64_t n, int shift) {
  for (int64_t c = (begin + (int64_t(1) << shift) - 1) >> shift; c << shift < begin + n; ++c) marks[c] = r;
}
__device__ __forceinline__ void end_marks(int32_t *marks, int R, int64_t total, int shift) { marks[(total + (int64_t(1) << shift) - 1) >> shift] = R - 1; }

// The request that element x belongs to: the last r with sums[r] <= x, for 0 <= x < sums[R].
__device__ __forceinline__ int owner(const int64_t *sums, const int32_t *marks, int shift, int64_t x) {
  int lo = marks[x >> shift], hi = marks[(x >> shift) + 1] + 1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// The block that entry k of the returned ones is: still in its old row, which nothing overwrites.
__device__ __forceinline__ int32_t returned(const BTArgs &a, int64_t k, int shift) {
  const int r = owner(a.back, a.coarse + kCoarse + 2, shift, k);
  return a.table[static_cast<int64_t>(r) * a.max_blocks + need_of(a, r, false).wb + (k - a.back[r])];
}

// The returned blocks onto the stack, by `blocks` blocks of which this is number b.
__device__ __forceinline__ void push(const BTArgs &a, const Totals &t, int b, int blocks) {
  for (int64_t k = static_cast<int64_t>(b) * blockDim.x + threadIdx.x; k < t.returned; k += static_cast<int64_t>(blocks) * blockDim.x)
    a.free_blocks[t.free + k] = returned(a, k, t.returned_shift);
}

// The slot of new token j, and its block into the table where it is the block's first.
__device__ __forceinline__ void fill_token(const BTArgs &a, const Totals &t, int64_t j) {
  if (j >= t.tokens) return;
  const int r = owner(a.off, a.coarse, t.token_shift, j);
  const Request q = a.requests[r];
  const uint32_t p = static_cast<uint32_t>(q.held) + static_cast<uint32_t>(j - q.begin);
  const uint32_t hb = block_of(a, static_cast<uint32_t>(q.held) + a.S - 1u), bi = block_of(a, p), within = p - bi * static_cast<uint32_t>(a.S);
  int64_t slot = -1;
  if (q.before >= 0) {
    int32_t block = q.last;
    if (bi >= hb) {
      const int64_t at = t.stack - 1 - (q.before + (bi - hb));
      block = at < 0 ? -1 : at < t.free ? a.free_blocks[at] : returned(a, at - t.free, t.returned_shift);
      if (within == 0) a.table[static_cast<int64_t>(r) * a.max_blocks + bi] = block;
    }
    slot = static_cast<int64_t>(block) * a.S + within;
  }
  a.slots[j] = slot;
  if (a.pos) a.pos[j] = static_cast<int32_t>(p);
}

template <int kBlocks, bool kAll>  // kAll: and expands the sums too
__global__ void __launch_bounds__(kScanThreads) bt_scan_kernel(const BTArgs a) {
  __shared__ uint32_t s_named[kBlocks == 1 ? kScanThreads / 32 : 1];  // one block: the requests that the order has named
  const int tid = threadIdx.x;
  if (kBlocks == 1 && tid < kScanThreads / 32) s_named[tid] = 0;
  pdl_prologue();
  // the block's tiles of 1,024 requests; where it has more than one, a first pass sums them up
  const int tiles = (a.R + kScanThreads - 1) / kScanThreads, each = (tiles + kBlocks - 1) / kBlocks;
  const int r0 = static_cast<int>(min(static_cast<int64_t>(blockIdx.x) * each * kScanThreads, static_cast<int64_t>(a.R)));
  const int r1 = static_cast<int>(min(r0 + static_cast<int64_t>(each) * kScanThreads, static_cast<int64_t>(a.R)));
  const bool twice = kBlocks > 1 && each > 1;
  const int ordered = a.order && r0 + tid < r1 ? a.order[r0 + tid] : r0 + tid;  // needed later, fetched now
  int32_t nf = *a.n_free;
  if (nf < 0 || nf > a.pool) {
    if (tid == 0) flag_error(a.status, MAPS_E_RANGE);
    nf = 0;
  }

  // index order: blocks given back and new tokens
  auto index_values = [&](int r, bool report, int64_t &x, int64_t &y, Need &n) {
    x = y = 0;
    n = {0, 0, 0, 0};
    if (r >= r1) return;
    n = need_of(a, r, report);
    if (n.hb > n.wb) x = n.hb - n.wb;
    if (n.want > n.held) y = n.want - n.held;
  };
  int64_t bx = 0, by = 0, back = 0, toks = 0, unused = 0;
  Need n;
  if (twice) {
    int64_t sx = 0, sy = 0, tx, ty;
    for (int r = r0 + tid; r < r1; r += kScanThreads) {
      int64_t x, y;
      index_values(r, false, x, y, n);
      sx += x, sy += y;
    }
    block_scan2(sx, sy, tx, ty);
    cluster_sums<kBlocks>(tx, ty, bx, by, back, toks);
  }
  for (int base = r0, k = 0; k < each; base += kScanThreads, ++k) {
    const int r = base + tid;
    int64_t x, y, tx, ty;
    index_values(r, true, x, y, n);
    int32_t last = -1;
    if (y && n.hb > 0) last = a.table[static_cast<int64_t>(r) * a.max_blocks + n.hb - 1];
    int64_t sx = x, sy = y;
    block_scan2(sx, sy, tx, ty);
    if (!twice) cluster_sums<kBlocks>(tx, ty, bx, by, back, toks);
    sx += bx, sy += by;
    if (r < r1) {
      a.off[r] = sy, a.back[r] = sx;
      Request &q = a.requests[r];
      q.begin = sy, q.held = n.held, q.last = last;
      if (a.order) q.before = -1, q.named = 0u;  // one that the order leaves out gets nothing
      set_marks(a.coarse, r, sy, y, mark_shift(toks));
      set_marks(a.coarse + kCoarse + 2, r, sx, x, mark_shift(back));
    }
    bx += tx, by += ty;
  }
  const int64_t N = min(static_cast<int64_t>(nf) + back, static_cast<int64_t>(a.pool));

  // the scheduler's order: blocks needed, granted while the stack lasts
  auto place = [&](int i, int &r, Need &n) -> int64_t {
    r = -1;
    n = {0, 0, 0, 0};
    if (i >= r1) return 0;
    r = i == r0 + tid ? ordered : a.order ? a.order[i] : i;
    if (r < 0 || r >= a.R) {
      flag_error(a.status, MAPS_E_RANGE);
      r = -1;
      return 0;
    }
    n = need_of(a, r, false);
    return n.wb > n.hb ? n.wb - n.hb : 0;
  };
  int64_t ahead = 0, all = 0;
  if (twice) {
    int64_t sx = 0, sy = 0, tx, ty;
    for (int i = r0 + tid; i < r1; i += kScanThreads) {
      int r;
      sx += place(i, r, n);
    }
    block_scan2(sx, sy, tx, ty);
    cluster_sums<kBlocks>(tx, 0, ahead, unused, all, unused);
  }
  int64_t granted = 0;  // the needs up to the last one granted
  uint32_t twice_named = 0;
  for (int base = r0, k = 0; k < each; base += kScanThreads, ++k) {
    int r;
    const int64_t x = place(base + tid, r, n);
    int64_t sx = x, sy = 0, tx, ty;
    block_scan2(sx, sy, tx, ty);
    if (!twice) cluster_sums<kBlocks>(tx, 0, ahead, unused, all, unused);
    sx += ahead;
    if (r >= 0) {
      const bool ok = x == 0 || sx + x <= N;
      if (a.order) {
        if (kBlocks == 1)
          twice_named |= atomicOr(&s_named[r >> 5], 1u << (r & 31)) >> (r & 31) & 1u;
        else
          twice_named |= atomicExch(&a.requests[r].named, 1u);
      }
      a.requests[r].before = ok ? sx : -1;
      a.got[r] = n.want < n.held || ok ? n.want : n.held;
      if (ok && x) granted = sx + x;
    }
    ahead += tx;
  }
  // the stack left: what the last one granted leaves
  __shared__ unsigned long long s_granted;
  if (tid == 0) s_granted = 0;
  __syncthreads();
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) granted = max(granted, static_cast<int64_t>(__shfl_xor_sync(0xffffffffu, granted, o)));
  if ((tid & 31) == 0 && granted) atomicMax(&s_granted, static_cast<unsigned long long>(granted));
  __syncthreads();
  if (twice_named) flag_error(a.status, MAPS_E_RANGE);
  int64_t most = static_cast<int64_t>(s_granted);
  if (kBlocks > 1) {
    cg::cluster_group cl = cg::this_cluster();
    cl.sync();
    if (blockIdx.x == 0 && tid == 0)
      for (int k = 1; k < kBlocks; ++k) most = max(most, static_cast<int64_t>(*cl.map_shared_rank(&s_granted, k)));
    cl.sync();
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.off[a.R] = toks;
    a.back[a.R] = back;
    *a.totals = {N - nf, min(toks, a.slots_cap), N, nf, mark_shift(toks), mark_shift(back)};
    end_marks(a.coarse, a.R, toks, mark_shift(toks));
    end_marks(a.coarse + kCoarse + 2, a.R, back, mark_shift(back));
    *a.n_free_out = static_cast<int32_t>(N - most);
    if (toks > a.slots_cap || nf + back > a.pool) flag_error(a.status, MAPS_E_RANGE);
  }
  if (kAll) {
    __syncthreads();  // the requests' records and the marks
    const Totals t = *a.totals;
    push(a, t, 0, 1);
    for (int64_t j = tid; j < t.tokens; j += kScanThreads) fill_token(a, t, j);
  }
}

__global__ void __launch_bounds__(kFillThreads) bt_push_kernel(const BTArgs a) {
  pdl_prologue();
  push(a, *a.totals, blockIdx.x, gridDim.x);
}

// Few tokens: one a thread, since each is a chain of loads; further blocks put the returned ones onto the stack.
__global__ void __launch_bounds__(kFillThreads) bt_fill_kernel(const BTArgs a, int token_blocks) {
  pdl_prologue();
  const Totals t = *a.totals;
  if (static_cast<int>(blockIdx.x) >= token_blocks)
    push(a, t, blockIdx.x - token_blocks, gridDim.x - token_blocks);
  else
    fill_token(a, t, static_cast<int64_t>(blockIdx.x) * kFillThreads + threadIdx.x);
}

// Many tokens: a warp maps 256 consecutive ones, lane by lane so that writes are whole lines, and all
// eight loads of a lane's blocks are under way at once.
__global__ void __launch_bounds__(kFillThreads) bt_fill_many_kernel(const BTArgs a) {
  pdl_prologue();
  const Totals t = *a.totals;
  const int64_t j0 = (static_cast<int64_t>(blockIdx.x) * (kFillThreads / 32) + threadIdx.x / 32) * (32 * kManyEach) + threadIdx.x % 32;
  int32_t at[kManyEach], owner_of[kManyEach], block[kManyEach];  // at: the stack's entry, -1: the block is known
  uint32_t pos[kManyEach];
  int64_t end = 0;
  int r = -1;
  uint32_t hb = 0;
  Request q = {0, -1, 0, -1, 0};
#pragma unroll
  for (int i = 0; i < kManyEach; ++i) {
    const int64_t j = j0 + 32 * i;
    at[i] = -1;
    block[i] = -1;
    pos[i] = 0;
    if (j < t.tokens) {
      if (j >= end) {
        r = owner(a.off, a.coarse, t.token_shift, j);
        q = a.requests[r];
        end = a.off[r + 1];
        hb = block_of(a, static_cast<uint32_t>(q.held) + a.S - 1u);
      }
      pos[i] = static_cast<uint32_t>(q.held) + static_cast<uint32_t>(j - q.begin);
      const uint32_t bi = block_of(a, pos[i]);
      if (q.before >= 0) {
        if (bi >= hb)
          at[i] = static_cast<int32_t>(max(t.stack - 1 - (q.before + (bi - hb)), int64_t(-1)));
        else
          block[i] = q.last;
      }
    }
    owner_of[i] = r;
  }
#pragma unroll
  for (int i = 0; i < kManyEach; ++i)
    if (at[i] >= 0) block[i] = a.free_blocks[at[i]];
#pragma unroll
  for (int i = 0; i < kManyEach; ++i) {
    const int64_t j = j0 + 32 * i;
    if (j >= t.tokens) return;
    const uint32_t bi = block_of(a, pos[i]), within = pos[i] - bi * static_cast<uint32_t>(a.S);
    if (at[i] >= 0 && within == 0) a.table[static_cast<int64_t>(owner_of[i]) * a.max_blocks + bi] = block[i];
    a.slots[j] = block[i] >= 0 ? static_cast<int64_t>(block[i]) * a.S + within : -1;
    if (a.pos) a.pos[j] = static_cast<int32_t>(pos[i]);
  }
}

// A launch of one cluster, programmatically serialised as launch_pdl's.
void launch_cluster(void (*kernel)(BTArgs), int blocks, int threads, cudaStream_t s, const BTArgs &a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(blocks);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace
}  // namespace maps

extern "C" {

static void carve(maps::Carve &c, maps::BTArgs &a) {
  a.totals = c.take<maps::Totals>(1);
  a.requests = c.take<maps::Request>(static_cast<size_t>(a.R));
  a.back = c.take<int64_t>(static_cast<size_t>(a.R) + 1);
  a.coarse = c.take<int32_t>(2 * (maps::kCoarse + 2));
}

size_t maps_block_tables_workspace_size(int32_t R) {
  maps::Carve c(nullptr);
  maps::BTArgs a = {};
  a.R = R > 0 ? R : 0;
  carve(c, a);
  return c.bytes();
}

int maps_block_tables(int32_t R, int32_t S, const int32_t *held, const int32_t *want,
                      const int32_t *order, int32_t *table, int32_t max_blocks,
                      int32_t *free_blocks, int32_t pool, const int32_t *n_free,
                      int32_t *n_free_out, int32_t *got_out, int64_t *slot_off_out,
                      int64_t *slots_out, int64_t slots_cap, int32_t *pos_out, void *ws,
                      size_t ws_bytes, void *stream) {
  using namespace maps;
  // R: a thread's place in the last tile of 1,024 requests stays a 32-bit number
  if (R < 0 || R > 1 << 30 || S < 1 || max_blocks < 0 || pool < 0 || slots_cap < 0 ||
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
  int32_t s_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (S == 1 << i) s_shift = i;
  BTArgs a = {R, S, max_blocks, pool, s_shift, held, want, order, table, free_blocks, n_free, n_free_out,
              got_out, slot_off_out, slots_out, slots_cap, pos_out, nullptr, nullptr, nullptr, nullptr,
              status_word(ws)};
  carve(c, a);
  // A decode step's worth in one kernel: what one block has to expand besides costs less than a launch (64 requests, a token
  // each: 3.9 us, 4.7 with two kernels; 256 with 8 tokens 5.4, 5.9; with 16 tokens 7.1, 6.3).  The sums are one block's up to
  // its threads, then a cluster's of eight (1,024 requests: 7.8, 11.1 us; 2,048: 16.0, 15.6; 4,096: 24.2, 16.0).
  // The pool bounds the blocks that one block may have to put back (256 requests of 32 blocks, one kernel and two: none finish
  // 4.5, 5.3 us; 32 do 5.8, 6.8; 128 do 7.4, 7.1; all do 8.7, 7.0); from a larger pool they could be more.
  const bool all = R <= kScanThreads && slots_cap <= 2 * kScanThreads && pool <= 16 * kScanThreads;
  if (all)
    launch_pdl(bt_scan_kernel<1, true>, 1, kScanThreads, 0, s, a);
  else if (R <= kScanThreads)
    launch_pdl(bt_scan_kernel<1, false>, 1, kScanThreads, 0, s, a);
  else
    launch_cluster(bt_scan_kernel<kCluster, false>, kCluster, kScanThreads, s, a);
  if (R > 0 && !all) {
    const int64_t rows = (static_cast<int64_t>(R) * max_blocks + 4 * kFillThreads - 1) / (4 * kFillThreads);
    const int64_t back = std::min(std::min((static_cast<int64_t>(pool) + 4 * kFillThreads - 1) / (4 * kFillThreads), rows), static_cast<int64_t>(4 * sm_count()));
    if (slots_cap <= kFewTokens) {
      const int64_t tokens = (slots_cap + kFillThreads - 1) / kFillThreads;
      if (tokens + back > 0) launch_pdl(bt_fill_kernel, static_cast<unsigned>(tokens + back), kFillThreads, 0, s, a, static_cast<int>(tokens));
    } else {
      const int64_t per = kFillThreads * kManyEach;
      if (back > 0) launch_pdl(bt_push_kernel, static_cast<unsigned>(back), kFillThreads, 0, s, a);
      launch_pdl(bt_fill_many_kernel, static_cast<unsigned>((slots_cap + per - 1) / per), kFillThreads, 0, s, a);
    }
  }
  return launch_ok();
}

}  // extern "C"
