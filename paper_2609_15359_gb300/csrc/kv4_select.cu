// kv4_select.cu -- the blocks of the cache that a cheap score ranks highest, for each query row and KV head.
//
// Score.  With lo <= k <= hi in every channel, q . k <= sum_d max(q_d lo_d, q_d hi_d); summed over the query heads x of a KV head
// that is sum_d N_d lo_d + P_d hi_d, N and P the sums of the heads' negative and positive parts.  So a group of heads costs one
// row of 2 D products, in 8 bits on both sides: whole numbers below 2^23, exact in any order, and one rounding with the scale.
// The same list comes out whatever the split.
//
// A block takes a row and KV head, or a cluster of them where there are few: 256 cache blocks each in turn.  Scores become keys, whole
// numbers in the scores' order, in the shared memory of the cluster's first block, which goes on alone (in the workspace where they
// are too many).  The least key that is taken is found by bisection, up to 16 keys a thread in registers, or for longer rows by
// histograms of the keys that are still in question, ten bits at a time; then the list is written in order.
//
// Bound: chains of dependent steps.  Where rows are many, enough of them side by side hide these: 128 requests of 64 to 8,192 tokens, 8
// heads of 128 channels, 68 MB of ranges, 19.3 us (floor 10.6).  One request of 100,000 to 131,072 tokens: 15 us where its ranges lie in
// L2, 19 from memory; of 17.6 between look-ups and first codes took 3, its 8,192 blocks' codes 1.5, the cluster's barrier 1.5, bisection
// 5, the list 2.  Many long rows: 64 requests of 131,072 tokens, 1.1 GB, 186 us (5.9 TB/s), 128 of 65,536 255 (4.3 TB/s).
#include <atomic>

#include "kv4.cuh"

namespace maps {
namespace {

constexpr int kBinBits = 10, kBins = 1 << kBinBits;
constexpr int kSmemKeys = 8192;   // of shared memory; longer rows of keys stay in the workspace
// Threads of a multiprocessor up to which a row and head is shared out.  35 rows of 4 heads and up to 1,024 blocks: 512 8.4 us, 2,048 9.6.
constexpr int kThreadsOfSm = 512;
// Rows and heads for each multiprocessor from which on 128 threads take one, six a multiprocessor: 1,024 of them 19.2 us, by 256
// threads 23.2.  Below, 256 threads end a row sooner.  So they do where rows have more blocks than kNarrowBlocks, which 128 threads sift
// slowly: 128 requests x 8 heads of 131,072 tokens (8,192 blocks) by 128 threads 656 us, by 256 361, of 64 to 131,072 tokens 368 and 230;
// up to 65,536 tokens 121 and 124, of 65,536 each 253 and 194.
constexpr int kNarrowRows = 4;
constexpr int kNarrowBlocks = 4096;
// Blocks of a row from which on 512 threads take it, where rows are few: 8 rows of 8,192 blocks 17.7 us, by 256 threads 20.7.  Clusters of 16
// 17.7, of 8 26, of 4 39.
constexpr int kWideRow = 2048;
constexpr int kMaxCluster = 16;
constexpr size_t kMostKeys = size_t(1) << 26;  // in the workspace: more rows take their turns

template <int kValue>
struct Int { static constexpr int value = kValue; };

struct SelectArgs {
  int32_t B, Hq, H, S;
  int64_t T, max_blocks, n_blocks;
  const void *q;
  int64_t q_row, q_head;
  const int64_t *off;
  const int32_t *len, *table;
  const int8_t *codes;
  const float *scale;
  int32_t first, last, n_list;
  int32_t *blocks, *tokens;
  int64_t row0;      // the launch's first row
  int32_t cluster;
  int32_t smem_keys;
  uint32_t *keys;    // [rows of a launch * H][stride], or NULL: in shared memory
  int64_t stride;
  int32_t *status;
};

// Whole numbers in the order of the scores, NaN above all.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);  // one zero
  return x != x ? 0xfffffffeu : u >> 31 ? ~u : u | 0x80000000u;
}

// Adds x to the running sum s + e, of which e holds what s's roundings lost: 48 bits.
__device__ __forceinline__ void add_twice(float &s, float &e, float x) {
  const float t = __fadd_rn(s, x), y = __fsub_rn(t, s);
  e = __fadd_rn(e, __fadd_rn(__fsub_rn(s, __fsub_rn(t, y)), __fsub_rn(x, y)));
  s = t;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t *of_first_block(uint32_t *p) {  // the same place in the shared memory of the cluster's first block
  uint64_t y;
  asm("mapa.u64 %0, %1, 0;" : "=l"(y) : "l"(reinterpret_cast<uint64_t>(p)));
  return reinterpret_cast<uint32_t *>(y);
}

// The greatest b with off[b] <= i of b in [0, B], -1 where there is none.  All threads call it.
template <int kThreads>
__device__ __forceinline__ int request_of(const int64_t *off, int B, int64_t i) {
  int64_t lo = 0, n = static_cast<int64_t>(B) + 1;
  for (;;) {
    const int64_t step = (n + kThreads - 1) / kThreads, at = threadIdx.x * step;
    const int count = __syncthreads_count(at < n && off[lo + at] <= i);
    if (count == 0) return -1;
    lo += (count - 1) * step;
    if (step == 1) return static_cast<int>(lo);
    n = min(step, n - (count - 1) * step);
  }
}

// Sums of acc[k] over the 2 kHalf lanes that differ in their low bits, lane x keeping that of acc[x].
template <int kHalf>
__device__ __forceinline__ void join(int (&acc)[8], int lane) {
#pragma unroll
  for (int o = kHalf; o > 0; o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int k = 0; k < o; ++k) {
      const int send = up ? acc[k] : acc[k + o], keep = up ? acc[k + o] : acc[k];
      acc[k] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
  }
}

// 256 threads four times a multiprocessor leave 64 registers a thread, of which the branch of 16 keys a thread spills 208 to 296 bytes;
// 128 threads spill 20 to 32.
template <class T, int D, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 1 : kThreads == 256 ? 4 : 6) kv4_select_kernel(const SelectArgs a) {
  constexpr int kWarps = kThreads / 32;
  constexpr int kLanes = D / 8, kSub = 32 / kLanes;  // lanes of a block's 2 D codes, and blocks of a warp's load
  constexpr int kBatch = 4;                          // loads under way at once; D/8 of them make a step of 32 blocks
  extern __shared__ __align__(16) uint32_t s_keys[];
  __shared__ __align__(16) int8_t s_w[2 * D];
  __shared__ uint32_t s_hist[kBins];
  __shared__ uint32_t s_warp[kWarps][2];
  __shared__ uint32_t s_found[3];
  __shared__ uint32_t s_count[2][kWarps];
  __shared__ struct { int32_t b, n; int64_t q1; } s_request;
  pdl_prologue();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = static_cast<int>(blockIdx.x) & (a.cluster - 1);
  const int64_t here = blockIdx.x / a.cluster, item = a.row0 * a.H + here, i = a.row0 + here / a.H;
  const int h = static_cast<int>(here % a.H);
  // the first queries are under way before anything is known of the request
  constexpr int kHeads = 4, kOwnCh = (D + kThreads - 1) / kThreads;  // channels of a thread
  const int group = a.Hq / a.H;
  const T *q = static_cast<const T *>(a.q) + i * a.q_row + static_cast<int64_t>(h) * group * a.q_head;
  T y[kOwnCh][kHeads];
#pragma unroll
  for (int c = 0; c < kOwnCh; ++c)
#pragma unroll
    for (int x = 0; x < kHeads; ++x)
      if (tid + c * kThreads < D && x < group) y[c][x] = q[x * a.q_head + tid + c * kThreads];
  // the row's request: the one of its number, where each has one row, else searched for; so the first blocks are looked up at once
  const int l = lane % kLanes, sub = lane / kLanes, mine = l * kSub + sub;  // of a step's 32 blocks, that whose score this lane ends up with
  const int start = (rank * kWarps + warp) * 32;
  int32_t raw = i < a.B && a.first + start + mine < a.max_blocks ? a.table[i * a.max_blocks + a.first + start + mine] : -1;
  int64_t b = i, q1 = 0;
  int32_t n = 0;
  bool found = false;
  if (i < a.B) {
    const int64_t q0 = a.off[i];
    q1 = a.off[i + 1];
    n = a.len[i];
    found = q0 >= 0 && q0 <= i && i < q1;
  }
  if (!found && a.B <= kThreads) {  // every thread looks at one, so that its length comes with it
    bool this_one = false;
    if (tid < a.B) {
      const int64_t next = a.off[tid + 1];
      const int32_t length = a.len[tid];
      this_one = a.off[tid] <= i && i < next;
      if (this_one) s_request.b = tid, s_request.n = length, s_request.q1 = next;
    }
    if (!__syncthreads_or(this_one)) return;  // no request's
    b = s_request.b, n = s_request.n, q1 = s_request.q1;
  } else if (!found) {
    b = request_of<kThreads>(a.off, a.B, i);
    if (b < 0 || b == a.B) return;
    q1 = a.off[b + 1];
    n = a.len[b];
  }
  int32_t *out = a.blocks + item * a.n_list;
  if (q1 > a.T || i >= q1 || n < 0 || n > 0x7fffffff - 1023 || n > a.max_blocks * a.S || (n > 0 && a.n_blocks == 0)) {
    if (tid == 0) flag_error(a.status, MAPS_E_RANGE);
    n = 0;
  }
  const int64_t seen = n - (q1 - i) + 1;  // keys
  const int32_t nb = n == 0 || seen <= 0 ? 0 : static_cast<int32_t>(static_cast<uint32_t>(seen + a.S - 1) / static_cast<uint32_t>(a.S)), count = min(nb, a.n_list);
  const int32_t N = nb - a.first - a.last;           // blocks in question
  uint32_t need = a.n_list - a.first - a.last;       // of which so many are taken
  const bool all = nb <= a.n_list;
  const int sharers = all || need == 0 ? 1 : min(a.cluster, (N + kThreads - 1) / kThreads);
  if (rank >= sharers) return;  // the cluster's barriers count those that are left
  const int32_t *table = a.table + b * a.max_blocks;
  auto checked = [&](int32_t block) {  // an entry that goes into the list without a score
    if (block < 0 || block >= a.n_blocks) flag_error(a.status, MAPS_E_RANGE);
    return block;
  };
  // what needs no scores: the ends of the list, and its tokens
  auto write_ends = [&]() {
    if (tid == 0) a.tokens[item] = nb == 0 ? 0 : static_cast<int32_t>((count - 1) * static_cast<int64_t>(a.S) + seen - (nb - 1) * static_cast<int64_t>(a.S));
    for (int x = tid; x < a.first + a.last; x += kThreads) {
      const bool front = x < a.first;
      out[front ? x : x - a.first + count - a.last] = checked(table[front ? x : x - a.first + nb - a.last]);
    }
  };
  if (all || need == 0) {
    if (!all) {
      write_ends();
      return;
    }
    if (tid == 0) a.tokens[item] = static_cast<int32_t>(nb == 0 ? 0 : seen);
    for (int x = tid; x < a.n_list; x += kThreads) out[x] = x < nb ? checked(table[x]) : -1;
    return;
  }
  if (sharers > 1) cluster_arrive();  // this block runs, so its shared memory may be written
  const int32_t *inner = table + a.first;  // the blocks in question

  // ---- the first blocks' codes are under way while the queries' weights are made
  const int stride = sharers * kThreads;
  int32_t block = 0;
  float sc = 0.0f;
  auto ask = [&](int j) { raw = j < N ? inner[j] : -1; };
  auto settle = [&](int j) {  // places past the end stand for block 0, whose score nobody wants
    const bool good = raw >= 0 && raw < a.n_blocks;
    block = good ? raw : 0;
    sc = NAN;
    if (j < N && !good) flag_error(a.status, MAPS_E_RANGE);
    if (good) sc = a.scale[static_cast<int64_t>(block) * a.H + h];
  };
  int4 c[kBatch];
  const int8_t *codes = a.codes + static_cast<int64_t>(h) * (2 * D) + 16 * l;
  const uint32_t block_bytes = static_cast<uint32_t>(a.H) * (2 * D);
  auto fetch = [&](int k0) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      c[k] = *reinterpret_cast<const int4 *>(codes + static_cast<uint64_t>(block_bytes) * static_cast<uint32_t>(__shfl_sync(0xffffffffu, block, sub * kLanes + k0 + k)));
  };
  if (!found) ask(start + mine);
  if (start + mine >= N) raw = -1;
  settle(start + mine);
  fetch(0);
  ask(start + stride + mine);
  float P[kOwnCh], M[kOwnCh];
  uint32_t most = 0;  // NaN's bits are above infinity's
#pragma unroll
  for (int c = 0; c < kOwnCh; ++c) {
    float Pe = 0.0f, Me = 0.0f;
    P[c] = M[c] = 0.0f;
    auto add = [&](float x) {
      add_twice(P[c], Pe, x > 0.0f || x != x ? x : 0.0f);
      add_twice(M[c], Me, x < 0.0f || x != x ? x : 0.0f);
    };
    if (tid + c * kThreads < D) {
#pragma unroll
      for (int x = 0; x < kHeads; ++x)
        if (x < group) add(Cvt<T>::to(y[c][x]));
#pragma unroll 4
      for (int x = kHeads; x < group; ++x) add(Cvt<T>::to(q[x * a.q_head + tid + c * kThreads]));
      P[c] = __fadd_rn(P[c], Pe);
      M[c] = __fadd_rn(M[c], Me);
    }
    most = max(most, max(__float_as_uint(P[c]) & 0x7fffffffu, __float_as_uint(M[c]) & 0x7fffffffu));
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if (lane == 0) s_warp[warp][0] = most;
  __syncthreads();
  uint32_t top = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) top = max(top, s_warp[w][0]);
  const float step = __fmul_rn(__uint_as_float(top), 1.0f / 127.0f);
  const bool no_number = !(step < INFINITY);
  const float inv = step >= 1.17549435e-38f ? __fdiv_rn(1.0f, step) : 0.0f;
#pragma unroll
  for (int c = 0; c < kOwnCh; ++c) {
    const int d = tid + c * kThreads;
    if (d < D && !no_number) {
      s_w[d] = static_cast<int8_t>(fminf(fmaxf(rintf(__fmul_rn(M[c], inv)), -127.0f), 127.0f));
      s_w[D + d] = static_cast<int8_t>(fminf(fmaxf(rintf(__fmul_rn(P[c], inv)), -127.0f), 127.0f));
    }
  }
  __syncthreads();

  // ---- keys
  const bool fits = N <= a.smem_keys;
  uint32_t *keys = !fits ? a.keys + here * a.stride : sharers > 1 ? of_first_block(s_keys) : s_keys;
  uint32_t lo = 0xffffffffu, hi = 0;
  const int4 w = *reinterpret_cast<const int4 *>(s_w + 16 * l);
  if (sharers > 1) cluster_wait();
  for (int j0 = start; j0 < N; j0 += stride) {
    // a step's D/8 loads, their sums eight at a time joined over 8 lanes, lane x keeping that of load x; then over the rest of a block's lanes
    int part[kLanes / 8];
#pragma unroll
    for (int k0 = 0; k0 < kLanes; k0 += 8) {
      int acc[8];
#pragma unroll
      for (int k1 = 0; k1 < 8; k1 += kBatch) {
        if (k0 + k1 > 0) fetch(k0 + k1);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) acc[k1 + k] = __dp4a(c[k].x, w.x, __dp4a(c[k].y, w.y, __dp4a(c[k].z, w.z, __dp4a(c[k].w, w.w, 0))));
      }
      join<4>(acc, lane);
      part[k0 / 8] = acc[0];
    }
    const float scale = sc;
    const int j = j0 + mine;
    if (j0 + stride < N) {
      settle(j + stride);
      fetch(0);
      ask(j + 2 * stride);
    }
#pragma unroll
    for (int o = kLanes / 2; o >= 8; o >>= 1) {
#pragma unroll
      for (int k = 0; k < o / 8; ++k) {
        const int send = l & o ? part[k] : part[k + o / 8], keep = l & o ? part[k + o / 8] : part[k];
        part[k] = keep + __shfl_xor_sync(0xffffffffu, send, o);
      }
    }
    if (j < N) keys[j] = no_number ? 0xfffffffeu : key_of(__fmul_rn(static_cast<float>(part[0]), scale));
  }
  if (sharers > 1) {
    cluster_arrive();
    if (rank > 0) return;
    cluster_wait();
    keys = fits ? s_keys : keys;
  } else {
    __syncthreads();
  }
  const uint32_t wanted = need;
  int32_t *inner_out = out + a.first;

  // ---- the least key that is taken, where a thread's keys fit its registers: by bisection, until the right number are above
  const unsigned below = (1u << lane) - 1u;
  auto in_registers = [&](auto per) {
    constexpr int kPer = decltype(per)::value;
    const int j0 = warp * 32 * kPer + lane;
    uint32_t key[kPer];
    int32_t name[kPer];
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
      const int j = j0 + 32 * x;
      key[x] = j < N ? keys[j] : 0u;  // less than any score's
      name[x] = j < N ? inner[j] : -1;
    }
    uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
    for (int x = 0; x < kPer; ++x) lo = key[x] ? min(lo, key[x]) : lo, hi = max(hi, key[x]);
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) s_warp[warp][0] = lo, s_warp[warp][1] = hi;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kWarps; ++x) lo = min(lo, s_warp[x][0]), hi = max(hi, s_warp[x][1]);
    // Keys >= lo: `wanted` or more; keys >= hi: `above`, fewer.  (A place between them guessed from the counts took more turns, and
    // longer ones: 128 requests 27 us for 23.)
    ++hi;
    uint32_t above = 0, ties = 0;
    int turn = 0;
    for (;; turn ^= 1) {
      if (hi - lo == 1) {
        ties = wanted - above;
        lo = hi;
        break;
      }
      const uint32_t mid = lo + (hi - lo) / 2;
      uint32_t c = 0;
      if (kPer == 1) {
        c = __syncthreads_count(key[0] >= mid);
      } else {
#pragma unroll
        for (int x = 0; x < kPer; ++x) c += key[x] >= mid;
        c = __reduce_add_sync(0xffffffffu, c);
        if (lane == 0) s_count[turn][warp] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int x = 0; x < kWarps; ++x) c += s_count[turn][x];
      }
      if (c >= wanted) lo = mid;
      if (c < wanted) hi = mid, above = c;
      if (c == wanted) break;
    }
    // taken: the keys from lo on, and of those one below the first `ties`
    uint32_t over = 0, same = 0;
    unsigned overs[kPer], sames[kPer];
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
      overs[x] = __ballot_sync(0xffffffffu, key[x] >= lo);
      sames[x] = __ballot_sync(0xffffffffu, ties > 0 && key[x] == lo - 1);
      over += __popc(overs[x]);
      same += __popc(sames[x]);
    }
    __syncthreads();  // everybody has read the last turn's
    if (lane == 0) s_warp[warp][0] = over, s_warp[warp][1] = same;
    __syncthreads();
    over = same = 0;
#pragma unroll
    for (int x = 0; x < kWarps; ++x)
      if (x < warp) over += s_warp[x][0], same += s_warp[x][1];
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
      const uint32_t rank_same = same + __popc(sames[x] & below);
      const bool tie = sames[x] >> lane & 1u && rank_same < ties;
      if (overs[x] >> lane & 1u || tie) inner_out[over + __popc(overs[x] & below) + min(rank_same, ties)] = name[x];
      over += __popc(overs[x]);
      same += __popc(sames[x]);
    }
    write_ends();
  };
  if (fits && N <= kThreads) return in_registers(Int<1>{});
  if (fits && N <= 2 * kThreads) return in_registers(Int<2>{});
  if (fits && N <= 4 * kThreads) return in_registers(Int<4>{});
  if (fits && N <= 16 * kThreads) return in_registers(Int<16>{});

  // ---- more keys: by histograms
  lo = 0xffffffffu, hi = 0;
  for (int j = tid; j < N; j += kThreads) {
    const uint32_t key = fits ? keys[j] : __ldcg(keys + j);
    lo = min(lo, key);
    hi = max(hi, key);
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) s_warp[warp][0] = lo, s_warp[warp][1] = hi;
  for (int x = tid; x < kBins; x += kThreads) s_hist[x] = 0;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kWarps; ++x) lo = min(lo, s_warp[x][0]), hi = max(hi, s_warp[x][1]);
  __syncthreads();
  // the keys in question are those of [lo, hi], of which `need` are wanted, the greatest first
  while (lo < hi) {
    const int shift = max(0, 32 - __clz(hi - lo) - kBinBits);
    for (int j = tid; j < N; j += kThreads) {
      const uint32_t key = keys[j];
      if (key >= lo && key <= hi) atomicAdd(&s_hist[(key - lo) >> shift], 1u);
    }
    __syncthreads();
    constexpr int kOwn = kBins / kThreads;  // bins of a thread, from the top down
    uint32_t own[kOwn], own_sum = 0;
#pragma unroll
    for (int x = 0; x < kOwn; ++x) {
      uint32_t &bin = s_hist[kBins - 1 - (tid * kOwn + x)];
      own[x] = bin;
      own_sum += own[x];
      bin = 0;  // for the next turn
    }
    uint32_t sum = own_sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    if (lane == 31) s_warp[warp][0] = sum;
    __syncthreads();
    uint32_t above = sum - own_sum;
    for (int x = 0; x < warp; ++x) above += s_warp[x][0];
#pragma unroll
    for (int x = 0; x < kOwn; ++x) {
      if (above < need && need <= above + own[x]) s_found[0] = kBins - 1 - (tid * kOwn + x), s_found[1] = above, s_found[2] = own[x];
      above += own[x];
    }
    __syncthreads();
    lo += s_found[0] << shift;
    need -= s_found[1];
    const bool whole = s_found[2] == need;
    hi = lo + min(hi - lo, (1u << shift) - 1u);
    __syncthreads();
    if (whole) {
      need = 0;
      break;
    }
  }
  // taken: keys above hi, with need == 0 those from lo on, else the first `need` of those that are lo
  const uint32_t from = need == 0 ? lo : lo + 1;

  // ---- the list, in the order of the blocks: first their numbers, in shared memory where there is room
  uint32_t *pick = s_hist;
  const bool room = wanted <= kBins;
  const int span = (N + kThreads - 1) / kThreads * 32;  // of a warp
  const int j0 = min(warp * span, N), j1 = min(j0 + span, N);
  uint32_t over = 0, same = 0;
  for (int j = j0 + lane; j - lane < j1; j += 32) {
    const uint32_t key = j < j1 ? keys[j] : 0;
    over += __popc(__ballot_sync(0xffffffffu, j < j1 && key >= from));
    same += __popc(__ballot_sync(0xffffffffu, j < j1 && key == lo));
  }
  if (lane == 0) s_warp[warp][0] = over, s_warp[warp][1] = same;
  write_ends();
  __syncthreads();
  over = same = 0;
  for (int x = 0; x < warp; ++x) over += s_warp[x][0], same += s_warp[x][1];
  for (int j = j0 + lane; j - lane < j1; j += 32) {
    const uint32_t key = j < j1 ? keys[j] : 0;
    const bool is_over = j < j1 && key >= from, is_same = j < j1 && key == lo && need > 0;
    const unsigned overs = __ballot_sync(0xffffffffu, is_over), sames = __ballot_sync(0xffffffffu, is_same);
    const uint32_t rank_same = same + __popc(sames & below);
    if (is_over || (is_same && rank_same < need)) {
      const uint32_t at = over + __popc(overs & below) + min(rank_same, need);
      if (room)
        pick[at] = j;
      else
        inner_out[at] = inner[j];
    }
    over += __popc(overs);
    same += __popc(sames);
  }
  if (room) {
    __syncthreads();
    for (uint32_t x = tid; x < wanted; x += kThreads) inner_out[x] = inner[pick[x]];
  }
}

// How a call is split: blocks that share a row and head, a power of two, and rows of a launch where their keys lie in the workspace.
struct Split {
  int32_t cluster = 1;
  int64_t rows, stride;
  bool in_ws;
  int32_t threads;
  Split(int64_t T, int32_t H, int64_t max_blocks) {
    threads = max_blocks > kWideRow && T * H <= sm_count() ? 512 : T * H >= static_cast<int64_t>(kNarrowRows) * sm_count() && max_blocks <= kNarrowBlocks ? 128 : 256;
    const int64_t steps = (max_blocks + threads - 1) / threads, most = static_cast<int64_t>(sm_count()) * kThreadsOfSm / threads;
    while (cluster < kMaxCluster && cluster < steps && 2 * cluster * T * H <= most) cluster *= 2;
    in_ws = max_blocks > kSmemKeys;
    stride = max_blocks;
    rows = T;
    const size_t row = static_cast<size_t>(stride) * static_cast<size_t>(H);
    if (in_ws && row * T > kMostKeys) rows = static_cast<int64_t>(kMostKeys / row);
    if (rows < 1) rows = 1;
  }
};

void carve_keys(Carve &c, SelectArgs &a, const Split &p, int32_t H) {
  a.stride = p.stride;
  if (p.in_ws) a.keys = c.take<uint32_t>(static_cast<size_t>(p.rows) * H * p.stride);
}

template <class T, int D, int kThreads>
int launch(SelectArgs a, const Split &p, cudaStream_t s) {
  constexpr auto kernel = kv4_select_kernel<T, D, kThreads>;
  a.smem_keys = static_cast<int32_t>(a.max_blocks < kSmemKeys ? a.max_blocks : kSmemKeys);
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = kThreads;
  cfg.dynamicSmemBytes = static_cast<size_t>(a.smem_keys) * 4;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.cluster > 1 ? 2 : 1;
  a.cluster = p.cluster;
  if (a.cluster > 8) {  // more than every device takes: asked for once, and 8 where it is not to be had
    static std::atomic<uint64_t> asked, had;
    int dev = 0;
    MAPS_TRY(cuda_ok(cudaGetDevice(&dev)));
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (!(asked.load(std::memory_order_acquire) & bit)) {
      int clusters = 0;
      cfg.gridDim = dim3(static_cast<unsigned>(a.cluster));
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
          cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters > 0)
        had.fetch_or(bit, std::memory_order_relaxed);
      else
        (void)cudaGetLastError();
      asked.fetch_or(bit, std::memory_order_release);
    }
    if (!(had.load(std::memory_order_relaxed) & bit)) a.cluster = 8;
    attr[1].val.clusterDim.x = a.cluster;
  }
  for (a.row0 = 0; a.row0 < a.T; a.row0 += p.rows) {
    const int64_t rows = a.T - a.row0 < p.rows ? a.T - a.row0 : p.rows;
    cfg.gridDim = dim3(static_cast<unsigned>(rows * a.H * a.cluster));
    MAPS_TRY(cuda_ok(cudaLaunchKernelEx(&cfg, kernel, static_cast<const SelectArgs &>(a))));
  }
  return launch_ok();
}
template <class T, int kThreads>
int launch_dim(int D, const SelectArgs &a, const Split &p, cudaStream_t s) {
  return D == 64 ? launch<T, 64, kThreads>(a, p, s) : D == 128 ? launch<T, 128, kThreads>(a, p, s) : launch<T, 256, kThreads>(a, p, s);
}

template <class T>
int launch_threads(int D, const SelectArgs &a, const Split &p, cudaStream_t s) {
  return p.threads == 512 ? launch_dim<T, 512>(D, a, p, s) : p.threads == 256 ? launch_dim<T, 256>(D, a, p, s) : launch_dim<T, 128>(D, a, p, s);
}

}  // namespace
}  // namespace maps

extern "C" {

size_t maps_kv4_select_blocks_workspace_size(int64_t T, int32_t H, int64_t max_blocks) {
  using namespace maps;
  Carve c(nullptr);
  SelectArgs a = {};
  if (T > 0 && H > 0 && max_blocks > 0) carve_keys(c, a, Split(T, H, max_blocks), H);
  return c.bytes();
}

int maps_kv4_select_blocks(int32_t dtype, int32_t B, int64_t T, int32_t Hq, int32_t H, int32_t D, int32_t S, const void *q, int64_t q_row,
                           int64_t q_head, const int64_t *qo_off, const int32_t *kv_len, const int32_t *table, int64_t max_blocks,
                           const int8_t *codes, const float *scale, int64_t n_blocks, int32_t first, int32_t last, int32_t n_list,
                           int32_t *blocks, int32_t *tokens, void *ws, size_t ws_bytes, void *stream) {
  using namespace maps;
  if ((dtype != MAPS_BF16 && dtype != MAPS_F16) || !kv4_dim_ok(D) || !kv4_block_ok(S) || B < 0 || T < 0 || T > (int64_t(1) << 30) || H < 1 ||
      Hq < H || Hq % H != 0 || Hq > 65535 || T > 0x7fffffff / H || max_blocks < 0 || max_blocks > 0x7fffffff || n_blocks < 0 || first < 0 ||
      last < 1 || n_list < 1 || n_list > (1 << 20) || first > n_list - last || static_cast<int64_t>(n_list) * S > 0x7fffffff - 1023)
    return MAPS_E_INVALID;
  MAPS_TRY(check_ws(ws, ws_bytes, maps_kv4_select_blocks_workspace_size(T, H, max_blocks)));
  if (T == 0 || B == 0) return MAPS_OK;
  if (q == nullptr || qo_off == nullptr || kv_len == nullptr || (max_blocks > 0 && table == nullptr) || blocks == nullptr || tokens == nullptr ||
      (n_blocks > 0 && (codes == nullptr || scale == nullptr)) || !aligned(q, 2) || !aligned(codes, 16) || !aligned(scale, 4) ||
      !aligned(qo_off, 8) || !aligned(kv_len, 4) || !aligned(table, 4) || !aligned(blocks, 4) || !aligned(tokens, 4))
    return MAPS_E_INVALID;
  SelectArgs a = {B, Hq, H, S, T, max_blocks, n_blocks, q, q_row, q_head, qo_off, kv_len, table, codes, scale, first, last, n_list, blocks, tokens};
  a.status = status_word(ws);
  const Split p(T, H, max_blocks < 1 ? 1 : max_blocks);
  Carve c(ws);
  carve_keys(c, a, p, H);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return dtype == MAPS_BF16 ? launch_threads<__nv_bfloat16>(D, a, p, s) : launch_threads<__half>(D, a, p, s);
}

}  // extern "C"
