// What the two kernels of diffqkv_extend share (extend.cu: chunks of many rows; extend_thin.cu: a few rows a sequence), and
// those of its ranged forms (diffqkv_extend_window, diffqkv_extend_shared), in which a row does not see all tokens before it
// (extend.cu again, and extend_few.cu).
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

constexpr int kNoWindow = 0x7fffffff;
// Where the rows of an entry of a ranged step go: to the result, or, where a row has two entries (the prefix of its group and
// its own tokens), to a buffer for each.
constexpr int kDstOut = 0, kDstPrefix = 1, kDstOwn = 2;
struct RowBuffer {
  float* o;    // [total_q n_q][d_v]
  float* lse;  // [total_q n_q] base 2
};
// Of a step with groups, where the parts of an item are, for extend_merge_kernel: left by the block that has its first tile,
// at [kind of entry][first row of the item][unit].
struct ItemRef {
  int first;  // that block, or its team
  int parts;  // negative in the list of long chunks; 1: the whole item, in its buffer or the result
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
  // ranged: row i of a sequence sees, of its tokens from `start` on, those before `sinks` and those less than `window` before
  // its own position.  The first `groups` entries of the list are the prefixes of groups of sequences, the others, up to
  // `entries`, the sequences, whose own tokens begin behind their group's prefix.
  int window, sinks, sink_tiles, sink_few;  // the sinks in tiles of this kernel and of extend_few.cu
  int few_stages, few_cost[3], mid_most;
  int alone;  // the kernel of few rows comes without the other one: too few rows in all for a long chunk
  int groups, entries;
  const int* cu_groups;
  const int* prefix_lens;
  int share;            // see ExtendRange
  RowBuffer buffer[2];  // kDstPrefix - 1, kDstOwn - 1
  ItemRef* refs;        // [2][total_q][n_units], and one that says whether the step is left out, and whether its rows are all few
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
// Ranged, an item costs more next to its tiles: the masks of its first and last tile, and the rows of a step with groups are
// written in fp32.  5, 7 and 9: chunks of 150-600 rows of two groups (32/4/16 heads, 64 and 128 channels) 289, 284 and 284 us,
// 16 chunks of 30-60 rows behind 4k tokens 97, 96 and 101, windows of 2k tokens 296, 296 and 299.
constexpr int kRangedItemCost = 7;
template <bool kRanged>
constexpr int item_cost = kRanged ? kRangedItemCost : kItemCost;
// Likewise for thin items, in tiles: a block's second item costs it about as much as five more tiles.
constexpr int kThinItemCost = 5;
// The ranged steps' few rows go by tiles of 64 tokens, whose cost is a quarter of what one of three 128-channel heads takes
// when memory bounds it (see few_cost); an item costs about two such more.
constexpr int kFewT = 64, kFewItemCost = 8, kFewMostCost = 16;
constexpr int kFewCols = 128;  // as kThinCols
// A step whose long chunks are short in all goes to the kernel of few rows too, in blocks of rows that each read the chunk's
// tokens: the kernel of long chunks takes 20 us for its start and its first tiles alone, this one three or four times as long
// for what comes behind them.  Up to this many units of cost for an SM; a chunk of more blocks, or of more cost than
// kMidLong, is too long by itself.  64 rows in three groups behind 30-60 tokens 31 -> 20 us, 143 rows behind 320-960 tokens
// 41 -> 30, 540 rows in a window of 33 tokens 35 -> 24; with 24 units the last two stay as they were, with 84 nothing changes.
constexpr int kMidMost = 44, kMidLong = 8192, kMidBlocks = 16;

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
// The rows of group g and the tokens that its sequences share; false when they do not fit.
__device__ __forceinline__ bool group_rows(const ExtendParams& p, int g, int& lo, int& hi, int& first, int& prefix) {
  first = p.cu_groups[g];
  const int end = p.cu_groups[g + 1];
  prefix = p.prefix_lens[g];
  if (first < 0 || end < first || end > p.batch || prefix < 0 || prefix > p.max_seqlen) return false;
  lo = p.cu_q[first];
  hi = p.cu_q[end];
  return lo >= 0 && hi >= lo && hi <= p.total_q && prefix <= 0x7ffffe00 - (hi - lo);  // positions stay within 32 bits
}
// Whether the prefix of a group, sequences first .. end - 1 with the rows lo .. hi - 1, is worth an entry of its own next to its
// sequences', which read it each otherwise.  It costs items more, and two parts to every row that are joined, and saves the
// reading of all sequences with rows but one.  With few rows to a sequence the cost is as much as reading some hundred tokens
// more; long chunks are bound by their products, of which sharing saves the empty rows of their tiles alone.
// Shared and not, in us, 32/4/8 heads of 128 channels with 100 tokens of their own: 3 chunks of 100-140 rows behind 8k tokens
// 84, 96; 2 of 150 behind 8k 75, 81; 4 of 500 behind 4k 202, 190; 8 of 260 behind 4k 203, 195; 16 of 40 behind 8k 121, 172; two
// single rows behind 400 tokens 22, 19, behind 1k 23, 25.  Over 604 steps (2-16 chunks of 20-600 rows behind 1k-32k tokens, four
// head layouts) what the rule takes is 1.1 % slower in the mean than the better of the two; with 500 or 1000 for 700 1.2 and
// 1.3 %.  To find out costs a step up to 1.5 us.
// Never where the first sequence, from which a shared prefix is read, does not hold it (it may have no rows and be given up).
constexpr int kShareTokens = 512, kShareLeast = 1024;
constexpr float kShareLong = 700.f;
constexpr int kShareLook = 64;  // sequences that are looked at, until enough have rows; those behind them are taken to have some
__device__ __forceinline__ bool sharing_saves(const ExtendParams& p, int rows, int prefix, int readers) {  // stays true with more of them
  if (rows <= readers * p.thin_max) return (float)prefix * (readers - 1) >= (float)kShareTokens;
  return (float)(prefix - kShareLeast) * p.T * (readers - 1) >= kShareLong * rows;
}
__device__ __forceinline__ bool worth_sharing(const ExtendParams& p, int first, int end, int lo, int hi, int prefix) {
  const int rows = hi - lo;
  if (rows == 0 || prefix == 0 || p.seqlens[first] < prefix) return false;
  if (p.share != 0) return p.share == 1;
  const int look = min(end, first + kShareLook);
  int readers = min(end - first, rows), b = first - 1, at = lo;  // at first as many as there can be
#pragma unroll 1
  for (;;) {
    const bool saves = sharing_saves(p, rows, prefix, readers);
    if (b < first) {
      if (!saves) return false;
      b = first;
      readers = 0;
    } else if (saves || b == look) {
      return saves;
    }
    while (b < look) {  // up to the next one with rows
      const int next = p.cu_q[++b];
      if (next <= at) continue;
      at = next;
      ++readers;
      break;
    }
    if (b == look) readers += min(end - b, hi - at);
  }
}
// The group that sequence b is in, -1: none.
__device__ __forceinline__ int group_of(const ExtendParams& p, int b) {
  int g = 0, z = p.groups;  // the last group that begins at or before b
  if (z == 0) return -1;
  while (z - g > 1) {
    const int mid = (g + z) >> 1;
    if (p.cu_groups[mid] <= b) g = mid; else z = mid;
  }
  return b < p.cu_groups[g] || b >= p.cu_groups[g + 1] ? -1 : g;
}
// Tokens of sequence b, whose rows are lo .. lo + n - 1 behind `past` tokens, that its group has for it (0 outside of all
// groups, and where they are not shared); -1 when the group's rows or tokens do not hold those of the sequence.  The group's rows are g_lo .. g_hi - 1.
__device__ __forceinline__ int group_prefix(const ExtendParams& p, int b, int lo, int n, int past, int& g_lo, int& g_hi) {
  const int g = group_of(p, b);
  if (g < 0) return 0;
  int first, prefix;
  if (!group_rows(p, g, g_lo, g_hi, first, prefix) || prefix > past || lo < g_lo || lo + n > g_hi) return -1;
  return worth_sharing(p, first, p.cu_groups[g + 1], g_lo, g_hi, prefix) ? prefix : 0;
}

// Blocks that the kernel of few rows would cut n > thin_max rows into; one more than it takes, for more, and where a single
// token's heads are too many for it (thin_max 0).
__device__ __forceinline__ int few_blocks(const ExtendParams& p, int n) {
  return p.thin_max == 0 ? kMidBlocks + 1 : min((n + p.thin_max - 1) / p.thin_max, kMidBlocks + 1);
}

// One sequence of the step as the list of long chunks has it.
template <bool kRanged>
struct SeqOf;
using Seq = SeqOf<false>;
template <>
struct SeqOf<false> {
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

// An entry of a ranged step.  Its K/V tiles are numbered without those that no row of the item sees: tile v of an item is the
// tile v of the cache in front of `sink_tiles`, and `skip` tiles further on behind them.
template <>
struct SeqOf<true> {
  int lo, n, past, items;
  int rows, thin_tiles;
  int blocks, block_rows;  // of rows, for the kernel of few rows
  int end, start;  // its tokens: from start (or the first) on, below end
  int tab, dst;    // row of the page table, kDst...
  bool bad, back;  // does not fit; ends in front of its beginning
  __device__ void load(const ExtendParams& p, int x) {
    start = 0;
    dst = kDstOut;
    int g = x, g_lo = 0, g_hi = 0, first = 0, prefix = 0;
    bad = back = false;
    if (x >= p.groups) {
      tab = x - p.groups;
      bad = !load_rows(p, tab, lo, n, past);
      back = bad && p.cu_q[tab + 1] < lo;
      g = n > 0 ? group_of(p, tab) : -1;
    }
    bool fits = true, shared = false;
    if (g >= 0) {  // the same code for prefixes and sequences
      fits = group_rows(p, g, g_lo, g_hi, first, prefix);
      shared = fits && worth_sharing(p, first, p.cu_groups[g + 1], g_lo, g_hi, prefix);
    }
    if (x < p.groups) {  // every row of the group sees the whole prefix: as if it were cached before any of them
      back = p.cu_groups[x + 1] < p.cu_groups[x];  // (of a group that does not fit every sequence with rows says so)
      tab = first;
      lo = g_lo;
      n = shared ? g_hi - g_lo : 0;
      past = end = shared ? prefix : 0;
      dst = kDstPrefix;
    } else {
      if (g >= 0 && (!fits || prefix > past || lo < g_lo || lo + n > g_hi)) {
        bad = true;
        shared = false;
        n = past = 0;
      }
      if (shared) {
        start = prefix;
        dst = kDstOwn;
      }
      end = past + n;
    }
    items = 0;
    rows = block_rows = n;
    blocks = 1;
    thin_tiles = n > 0 ? (end + kFewT - 1) / kFewT - skip_few(p) : 0;
    if (n > p.thin_max) {
      items = (n + 2 * p.T - 1) / (2 * p.T);
      blocks = few_blocks(p, n);
      block_rows = (n + blocks - 1) / blocks;
    } else {
      n = 0;
    }
  }
  // the list that it is in, which the step's length decides
  __device__ void choose(bool all_few) {
    if (all_few) n = 0;
    else if (n > 0) thin_tiles = 0;
  }
  // the other kernel's cost of a long chunk
  __device__ int mid(const ExtendParams& p) const {
    if (n == 0) return 0;
    if (blocks > kMidBlocks || thin_tiles > kMidLong / kFewItemCost) return kMidLong;
    return min(min(p.n_units, kMidLong) * min(few_unit(p), kMidLong), kMidLong);  // (a unit alone may be 2^18)
  }
  // cost of one of extend_few.cu's tiles, by its groups of 16 rows: up to two, up to four, more
  __device__ int few_cost(const ExtendParams& p) const {
    const int groups = p.parts * ((block_rows * p.G + 15) >> 4);
    return p.few_cost[groups <= 2 ? 0 : groups <= 4 ? 1 : 2];
  }
  // and of a unit of it, all blocks of rows
  __device__ int few_unit(const ExtendParams& p) const {
    return thin_tiles > 0 ? blocks * (thin_tiles * few_cost(p) + kFewItemCost) : 0;
  }
  // of extend_few.cu's tiles, behind the sinks, those that no row sees
  __device__ int skip_few(const ExtendParams& p) const { return max(low(p, 0) / kFewT - p.sink_few, 0); }
  // first token behind the sinks that the chunk's row `tok` sees
  __device__ int low(const ExtendParams& p, int tok) const { return max(start, past + tok + 1 - p.window); }
  // tiles behind the sinks that no row from `tok` on sees
  __device__ int skip(const ExtendParams& p, int tok) const { return max(low(p, tok) / kKT - p.sink_tiles, 0); }
  // tiles of the cache up to the last one that rows before `tok` see
  __device__ int reach(const ExtendParams& p, int tok) const { return (min(past + tok, end) + kKT - 1) / kKT; }
  // sum over x < count of floor((b + 2 T x) / 128), b >= 0
  __device__ static int steps(const ExtendParams& p, int count, int b) {
    const int whole = count * (b >> 7);
    b &= kKT - 1;
    if (p.t_log2 >= 0) return whole + (int)floor_sum_128(count, p.t_log2 + 1, b);
    return whole + (int)floor_sum(count, kKT, 2 * p.T, b);
  }
  // cost of the first i items, i < items
  __device__ int cost_before(const ExtendParams& p, int i) const {
    if (i == 0) return 0;
    int tiles = dst == kDstPrefix ? i * ((end + kKT - 1) / kKT) : steps(p, i, past + 2 * p.T + kKT - 1);
    if (p.window == kNoWindow) {
      tiles -= i * (start / kKT);
    } else {  // item x skips max(0, floor((c + 2 T x) / 128)) tiles
      int c = past + 1 - p.window - p.sink_tiles * kKT, x0 = 0;
      if (c < 0) {
        x0 = (2 * p.T - 1 - c) / (2 * p.T);
        c += x0 * 2 * p.T;
      }
      if (i > x0) tiles -= steps(p, i - x0, c);
    }
    return kWideCost * tiles + item_cost<true> * i;
  }
  __device__ bool wide(const ExtendParams& p, int i) const { return n - i * 2 * p.T > p.T; }
  __device__ int tiles(const ExtendParams& p, int i) const {  // K/V tiles of item i
    return reach(p, min(n, (i + 1) * 2 * p.T)) - skip(p, i * 2 * p.T);
  }
  __device__ int cost(const ExtendParams& p) const {  // of one head group
    if (n == 0) return 0;
    return cost_before(p, items - 1) + item_cost<true> + (wide(p, items - 1) ? kWideCost : kNarrowCost) * tiles(p, items - 1);
  }
};
template <bool kRanged>
__device__ __forceinline__ int entries_of(const ExtendParams& p) { return kRanged ? p.entries : p.batch; }

// Whether an entry of a ranged step may be for the kernel of long chunks, if it fits.
__device__ __forceinline__ bool long_entry(const ExtendParams& p, int x) {
  int lo, hi;
  if (x < p.groups) {
    int first, prefix;
    return group_rows(p, x, lo, hi, first, prefix) && hi - lo > p.thin_max && p.share != 2 &&
           (p.share == 1 || sharing_saves(p, hi - lo, prefix, min(p.cu_groups[x + 1] - first, hi - lo)));
  }
  return p.cu_q[x - p.groups + 1] - p.cu_q[x - p.groups] > p.thin_max;
}

// Where a block of a ranged step begins.  What a block runs once at its start is fetched line by line, some 25 cycles an
// instruction, so this is one short piece of code for both kernels, in 32-bit arithmetic (the host sees to it that both lists
// stay below 2^31): with the plain steps' code a block of long chunks made its first request 16 us after its start.
__device__ __forceinline__ uint32_t ranged_share_start(uint32_t total, uint32_t k, uint32_t n) {  // floor(total k / n)
  const uint32_t q = total / n, r = total - q * n;
  return q * k + r * k / n;
}
__device__ __forceinline__ int ranged_shares(uint32_t total, int n, int least) {  // see shares
  return total >= (uint32_t)(n * least) ? n : max(1, (int)(total / (uint32_t)least));
}
__device__ __forceinline__ int ranged_wide_teams(const ExtendParams& p, uint32_t wide, uint32_t few) {  // see wide_teams
  if (wide == 0) return 0;
  int n = p.n_teams;
  if (few > 0 && n > 1) {
    const float w = (float)wide * p.team, f = (float)few * p.thin_weight;
    n = min(max((int)(n * __fdividef(w, w + f) + 0.5f), 1), n - 1);
  }
  return ranged_shares(wide, n, item_cost<true> + kWideCost);
}
struct RangedStart {
  uint32_t wide, few;        // lengths of the two lists
  int first, busy;           // the thread's first entry; blocks of few rows, where no thread has more than one entry
  bool single;               // no thread has more than one entry
  bool all_few;              // long chunks are in the list of few rows too
  uint32_t before_wide, before_few;  // of the lists, in front of the thread's entries
};
template <int kWarps>
struct RangedScan {
  unsigned long long sum[kWarps];
  uint32_t mid[kWarps], busy[kWarps];
  SeqOf<true> seq;  // of the block's first item: its entry, the entry's start in the list
  int e;
  uint32_t lo;
};
// Sums up both lists, which are empty where ends are out of order: rows may then be several entries' own, and the lists longer
// than the host has counted.  `my` is the thread's first entry.  Holds a barrier, and report's that an entry does not fit.
template <int kWarps>
__device__ __forceinline__ RangedStart ranged_start(const ExtendParams& p, RangedScan<kWarps>& sc, SeqOf<true>& my, bool reports) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per_thread = (p.entries + kWarps * 32 - 1) / (kWarps * 32);
  RangedStart r;
  r.single = per_thread == 1;
  r.first = tid * per_thread;
  uint32_t wide = 0, few = 0, mid = 0;
  bool back = false;
  my.n = my.thin_tiles = 0;
#pragma unroll 1
  for (int i = per_thread - 1; i >= 0; --i) {
    if (r.first + i >= p.entries) continue;
    my.load(p, r.first + i);
    if ((my.bad || my.back) && reports) report(p.dev_status, DIFFQKV_ERR_INDEX);
    back |= my.back;
    if (my.n > 0) {
      wide += p.n_units * (uint32_t)my.cost(p);
      mid += my.mid(p);
    } else {
      few += p.n_units * my.few_unit(p);
    }
  }
  const unsigned long long mine = (unsigned long long)wide << 32 | few;
  unsigned long long x = mine;
  uint32_t z = mid;
#pragma unroll 1
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long y = __shfl_up_sync(0xffffffffu, x, o);
    const uint32_t v = __shfl_up_sync(0xffffffffu, z, o);
    if (lane >= o) {
      x += y;
      z += v;
    }
  }
  const uint32_t busy = __reduce_add_sync(0xffffffffu, few > 0 ? 1 : mid > 0 ? my.blocks << 16 : 0);
  if (lane == 31) {
    sc.sum[warp] = x;
    sc.mid[warp] = z;
    sc.busy[warp] = busy;
  }
  back = __syncthreads_or(back);
  unsigned long long before = x - mine, all = 0;
  uint32_t before_mid = z - mid, all_mid = 0, all_busy = 0;
#pragma unroll 1
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) {
      before += sc.sum[w];
      before_mid += sc.mid[w];
    }
    all += sc.sum[w];
    all_mid += sc.mid[w];
    all_busy += sc.busy[w];
  }
  if (back) all = all_mid = 0;
  r.wide = (uint32_t)(all >> 32);
  r.few = (uint32_t)all;
  r.before_wide = (uint32_t)(before >> 32);
  r.before_few = (uint32_t)before;
  r.busy = all_busy & 0xffff;
  r.all_few = all_mid <= (uint32_t)p.mid_most;
  if (r.all_few) {
    r.wide = 0;
    r.few += all_mid;
    r.before_few += before_mid;
    r.busy += all_busy >> 16;
  }
  my.choose(r.all_few);
  if (reports && p.groups > 0 && tid == 0) p.refs[2LL * p.total_q * p.n_units] = {back, r.all_few};
  return r;
}
// The thread that has place w0 of a list among its entries, which begin at `before`, leaves the entry there.  cost: an entry's
// length in the list.
template <int kWarps, typename F>
__device__ __forceinline__ void ranged_seek(const ExtendParams& p, RangedScan<kWarps>& sc, const RangedStart& r, SeqOf<true>& my,
                                            uint32_t w0, uint32_t before, F cost) {
  const int per_thread = (p.entries + kWarps * 32 - 1) / (kWarps * 32);
#pragma unroll 1
  for (int i = 0; i < per_thread && r.first + i < p.entries; ++i) {
    if (before > w0) break;
    if (!r.single) {
      my.load(p, r.first + i);
      my.choose(r.all_few);
    }
    const uint32_t c = cost(my);
    if (before <= w0 && w0 - before < c) {
      sc.seq = my;
      sc.e = r.first + i;
      sc.lo = before;
      break;
    }
    before += c;
  }
}

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
// The K and V boxes bring box_tok (at most 64) tokens, all channels of one head.
cudaError_t launch_extend_few(const CUtensorMap& mk, const CUtensorMap& mv, const void* q, ExtendParams p, int d_qk, int d_v,
                              int blocks, cudaStream_t stream);

}  // namespace diffqkv
