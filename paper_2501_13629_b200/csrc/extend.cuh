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
  int member;        // place of the block in its team
  int parts;         // the teams from this block's on that have some of its tiles each
};

// One of the two flat lists of work, and where its cut items go.
struct ExtendList {
  float* part_o;       // [2 blocks][slot_rows][d_v] normalised partial rows
  float* part_lse;     // [2 blocks][slot_rows] base-2 log-sum-exp
  ExtendMeta* meta;    // [blocks]
  int slot_rows;
  int team, n_teams;   // blocks = n_teams * team
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
  lo = p.cu_q[b];
  const int hi = p.cu_q[b + 1];
  past = p.seqlens[b];
  n = hi - lo;
  if (lo < 0 || n < 0 || hi > p.total_q || past < 0 || (long long)past + n > p.max_seqlen) {
    n = 0;
    past = 0;
    return false;
  }
  return true;
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
// Likewise for thin items, in tiles: a block's second item costs it about as much as five more tiles.
constexpr int kThinItemCost = 5;
constexpr int kExtendThinThreads = 576;
cudaError_t launch_extend_thin(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const ExtendParams& p,
                               int d_qk, int d_v, int blocks, bool second, cudaStream_t stream);

}  // namespace diffqkv
