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
  int valid, row_lo, rows, head0, cost, nt, member, part_rows;  // part_rows: rows of a head group (thin), else all
  long long lo;  // place of the item in the flat list
  int chunks;    // (thin) 0, or the blocks from the first on that have a chunk of the item each
};

// One of the two flat lists of work, and where its cut items go.
struct ExtendList {
  float* part_o;       // [2 blocks][slot_rows][d_v] normalised partial rows
  float* part_lse;     // [2 blocks][slot_rows] base-2 log-sum-exp
  ExtendMeta* meta;    // [blocks]
  long long* total;    // of the list
  int slot_rows;
  int team, n_teams;   // blocks = n_teams * team
};

struct ExtendParams {
  const int* cu_q;
  const int* seqlens;
  const int* page_table;
  int page_size, max_pages_per_seq, num_blocks, max_seqlen;
  int batch, total_q, n_q;
  int G, T;            // heads per group, tokens per row tile
  int n_units, parts;  // head groups = n_units * parts: the groups of a unit share their K head or their V head
  int thin_max;        // sequences of at most this many rows are thin
  int region;          // columns of a head group of a thin sequence
  int k_parts, v_parts;  // K heads and V heads of a unit: (1, parts), (parts, 1) or (1, 1)
  int heads_per_k, heads_per_v;
  // the thin kernel's K and V tiles: ring lengths; whether a TMA box brings whole rows, and then the groups of eight
  // tokens from one head of a page to the next
  int k_ring, v_ring, k_rows, v_rows, head_groups;
  int box_tok;         // tokens per TMA box of the cache maps
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

// Start of share k of n equal shares of a list, floor(total k / n); in 32-bit arithmetic where that is enough (a 64-bit
// quotient costs most of a microsecond at the start of every block).
__device__ __forceinline__ long long share_start(long long total, int k, int n) {
  if (total < (1ll << 22)) return (long long)((uint32_t)total * (uint32_t)k / (uint32_t)n);  // k <= kMaxBlocks
  return total * k / n;
}

constexpr int kExtendThinThreads = 576;
cudaError_t launch_extend_thin(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const ExtendParams& p,
                               int d_qk, int d_v, int blocks, cudaStream_t stream);

}  // namespace diffqkv
