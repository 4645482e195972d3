// What the two kernels of diffqkv_extend share (extend.cu: chunks of many rows; extend_thin.cu: a few rows a sequence).
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace diffqkv {

constexpr int kRows = 128;  // matrix rows of a tile
constexpr int kKT = 128;    // cached tokens of a K/V tile
constexpr int kTmemCols = 512;
constexpr int kDMax = 128;
constexpr int kRingBytes = 5 * kKT * kDMax * 2;  // K and V tiles in shared memory
constexpr int kThinCols = 64;  // columns (rows of the chunk times heads) of a thin sequence
constexpr float kRescaleThreshold = 8.f;  // log2 domain
constexpr int kMaxBlocks = 256;

struct ExtendMeta {  // an item that is cut, left by the block that has its first tile
  int rows;          // 0: no such item; of the item, and of a head group of it (thin), else all
  int part_rows;
  int row_lo, head0; // first row in q, first head
  int parts;         // the teams from this block's on that have some of its tiles each
};

// One of the two flat lists of work, and where its cut items go.
struct ExtendList {
  float* part_o;       // [2 blocks][slot_rows][d_v] normalised partial rows
  float* part_lse;     // [2 blocks][slot_rows] base-2 log-sum-exp
  ExtendMeta* meta;    // [blocks]
  int slot_rows;
  int team;            // blocks that share an item's K or V head, next to each other
};

struct ExtendParams {
  const int* cu_q;
  const int* seqlens;
  const int* page_table;
  int page_size, max_pages_per_seq, num_blocks, max_seqlen;
  int batch, total_q, n_q;
  int G, T, t_log2;    // heads per group, tokens per row tile and its logarithm (-1: no power of two)
  int n_units, parts;  // head groups = n_units * parts: the groups of a unit share their K head or their V head
  int thin_max;        // sequences of at most this many rows are thin
  int region;          // columns of a head group of a thin sequence
  // SMs; teams of the list of long chunks and blocks in one; cost of a tile of a thin sequence in that list's units
  int blocks, n_teams, team;
  float thin_weight;
  int k_parts, v_parts;  // K heads and V heads of a unit: (1, parts), (parts, 1) or (1, 1)
  int heads_per_k, heads_per_v;
  // the thin kernel's K and V tiles: ring lengths; whether a TMA box brings whole rows, and then the groups of eight
  // tokens from one head of a page to the next
  int k_ring, v_ring, k_rows, v_rows, head_groups;
  int box_tok;         // tokens per TMA box of the cache maps
  int first;           // this kernel comes before the other one
  float scale_log2;
  void* out;
  int out_is_f32;
  float* lse;
  int* dev_status;
  ExtendList list;     // of the kernel that gets these parameters
};

// Rows of sequence b: first row, number, tokens cached before; false when they do not fit.
__device__ __forceinline__ bool load_rows(const ExtendParams& p, int b, int& lo, int& n, int& past) {
  return ragged_rows(p.cu_q, p.seqlens, b, p.total_q, p.max_seqlen, lo, n, past);
}

// Shares are at least as long as the longest way between the starts of two tiles of an item (see item_tile), so that of
// the teams between the first and the last tile of an item every one has some; a short list leaves teams without work.
__device__ __forceinline__ int shares(long long total, int n, int least) {
  return total >= (long long)n * least ? n : max(1, (int)total / least);
}
__device__ __forceinline__ long long quotient(long long x, long long y) {  // x >= 0, y > 0
  return x < (1ll << 31) && y < (1ll << 31) ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}
// The share that a place of the list belongs to.
__device__ __forceinline__ int share_of(long long at, long long total, int n) {
  return (int)quotient((at + 1) * n - 1, total);
}
// Start of share k of n equal shares of a list, floor(total k / n); in 32-bit arithmetic where that is enough (a 64-bit
// quotient costs most of a microsecond at the start of every block).
__device__ __forceinline__ long long share_start(long long total, int k, int n) {
  if (total < (1ll << 22)) return (long long)((uint32_t)total * (uint32_t)k / (uint32_t)n);  // k <= kMaxBlocks
  return total * k / n;
}

// The first of an item's nt tiles that begins `at` or more behind the item's start: tile 0 begins with the item, tile j
// at extra + cost j.
__device__ __forceinline__ int item_tile(long long at, int cost, int nt, int extra) {
  if (at <= 0) return 0;
  if (at >= (long long)cost * nt + extra) return nt;
  const int x = (int)at - extra;
  return max(1, (x + cost - 1) / cost);
}

// Start of an item's last tile, from the item's start.
__device__ __forceinline__ long long last_tile(int cost, int nt, int extra) {
  return nt == 1 ? 0 : extra + (long long)cost * (nt - 1);
}
// In the division of the work: a K/V tile of a wide and of a narrow item, and what an item costs next to its tiles (its
// rows are written out and the pipeline fills again).  Measured on prompts of 1.5k-2k rows over 0-6k tokens: 1.85 us a
// tile, 4-5 us an item; without the last, blocks with many short items ended 13 % late, 4 to 7 makes 1 %.
constexpr int kWideCost = 2, kNarrowCost = 1, kItemCost = 5;
// Likewise for thin items, in tiles: a block's second item costs it about as much as five more tiles.
constexpr int kThinItemCost = 5;

// sum of floor((a x + b) / m) for x = 0 .. n - 1 with a, b >= 0, m > 0: the Euclid-like recursion on (m, a).  Not inlined:
// the code that a block runs once at its start is fetched from the second-level cache line by line, which is what it
// costs (with every quotient inlined a block began its first loads 16 us after its start).
static __device__ __noinline__ long long floor_sum(long long n, long long m, long long a, long long b) {
  long long ans = 0;
  while (n > 0) {
    if (a >= m) { ans += (n - 1) * n / 2 * (a / m); a %= m; }
    if (b >= m) { ans += n * (b / m); b %= m; }
    const long long y = a * n + b;
    if (y < m) break;
    n = y / m;
    b = y % m;
    const long long t = m; m = a; a = t;
  }
  return ans;
}
// The same with m = 128 and a = 2^s: for a >= 128 every term is floor(b / 128) + x a / 128, else with r = 128 / a terms in
// a turn and e = floor(b / a) the sum of floor((e + x) / r), a difference of sums from 0.
__device__ __forceinline__ long long floor_sum_128(int n, int s, int b) {
  if (s >= 7) return (long long)n * (b >> 7) + (((long long)n * (n - 1) / 2) << (s - 7));
  const int h = 7 - s, e = b >> s;
  auto upto = [&](int t) -> long long {  // sum of y >> h for y < t
    const int q = t >> h;
    return ((long long)q * (q - 1) / 2 << h) + (long long)q * (t - (q << h));
  };
  return upto(e + n) - upto(e);
}
// Inclusive sum over the lanes.  Not inlined either.
static __device__ __noinline__ long long warp_scan(long long x) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// Sum over the threads before this one, and over all, of a block of at most 32 warps; a word per warp in s, which a
// barrier of the caller's separates from the call before.  Holds a barrier.
template <int kWarps>
__device__ __forceinline__ long long block_scan(long long mine, long long* s, long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long incl = warp_scan(mine);
  if (lane == 31) s[warp] = incl;
  __syncthreads();
  const long long x = lane < kWarps ? s[lane] : 0, all = warp_scan(x);
  total = __shfl_sync(0xffffffffu, all, 31);
  return incl - mine + __shfl_sync(0xffffffffu, all - x, warp);
}
// One sequence of the step as the list of long chunks has it.
struct Seq {
  int lo, n, past, items;  // first row, rows (0: not in this list), tokens cached before, items per head group
  int rows, thin_tiles;    // rows in either list; tiles of one unit of the other list (0: not in that one)
  bool bad;                // does not fit
  __device__ void load(const ExtendParams& p, int b) {
    bad = !load_rows(p, b, lo, n, past);
    thin_tiles = items = 0;
    rows = n;
    if (n > p.thin_max) {
      items = (n + 2 * p.T - 1) / (2 * p.T);
    } else {
      thin_tiles = n > 0 ? (past + n + kKT - 1) / kKT : 0;
      n = 0;
    }
  }
  // cost of the first i items, i < items
  __device__ long long cost_before(const ExtendParams& p, int i) const {
    const int b = past + 2 * p.T + kKT - 1;
    const long long tiles = p.t_log2 >= 0 ? floor_sum_128(i, p.t_log2 + 1, b) : floor_sum(i, kKT, 2 * p.T, b);
    return kWideCost * tiles + (long long)kItemCost * i;
  }
  __device__ bool wide(const ExtendParams& p, int i) const { return n - i * 2 * p.T > p.T; }
  __device__ int tiles(const ExtendParams& p, int i) const {  // K/V tiles of item i
    return (past + min(n, (i + 1) * 2 * p.T) + kKT - 1) / kKT;
  }
  __device__ long long cost(const ExtendParams& p) const {  // of one head group
    if (n == 0) return 0;
    return cost_before(p, items - 1) + kItemCost + (wide(p, items - 1) ? kWideCost : kNarrowCost) * (long long)tiles(p, items - 1);
  }
};

// Teams that the list of long chunks is divided over; the thin sequences have the other SMs, so that neither kernel waits
// for the other (one thread block of either fits an SM): what a step of both kinds saves is one start, one end and one
// uneven finish (a chunk of 512 rows next to 15 single ones over 0.5k-4k tokens, 16/2/4 heads: 72 -> 64 us).  The weight
// of a thin tile, 0.3 + 0.48 units for each of its K and V tiles, is the middle of what was fastest for seven mixtures of
// 64 and 128 channels; a third more or less costs up to a tenth, far too little or too much twice the time.
// (The two kernels need not agree to the last block: each divides its own list, whatever the other takes.)
__device__ __forceinline__ int wide_teams(const ExtendParams& p, long long wide, long long thin) {
  if (wide == 0) return 0;
  int n = p.n_teams;
  if (thin > 0 && n > 1) {
    const float w = (float)wide * p.team, t = (float)thin * p.thin_weight;
    n = min(max((int)(n * (w / (w + t)) + 0.5f), 1), n - 1);
  }
  return shares(wide, n, kItemCost + kWideCost);
}
__device__ __forceinline__ int thin_blocks_left(const ExtendParams& p, int wide_teams) {
  const int left = p.blocks - wide_teams * p.team;
  return left > 0 ? left : p.blocks;  // one team alone: the lists one after the other
}
constexpr int kExtendThinThreads = 576;
cudaError_t launch_extend_thin(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const ExtendParams& p,
                               int d_qk, int d_v, int blocks, bool second, cudaStream_t stream);

}  // namespace diffqkv
