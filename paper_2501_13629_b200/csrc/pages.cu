// Upkeep of a paged cache: pages with reference counts, handed out, shared, given back, copied and compacted on the
// device (diffqkv_pages_*), so that a serving loop needs no trip to the host between steps.
//
// State: page_table [num_seqs, row] (-1 = no page), seqlens, ref_counts [num_pages] (0 = free).  There is no free list:
// "the i-th lowest id whose count is 0" is found by a prefix sum over the counts, which keeps every call deterministic
// and leaves nothing to get out of step with the counts.
//
// The searches (reserve, compact) need the whole pool's counts before the first decision, that is two or three passes
// with a barrier between them.  One thread-block cluster of eight blocks does them in one launch: 8 x 1024 threads read
// a megabyte of counts (262 144 pages, 12.9 GB of 16-token pages) in about a microsecond, and barrier.cluster costs less
// than a second launch.  Pages themselves are moved by a second kernel over all SMs, from a list the first one leaves
// in the workspace; it is bound by memory (each moved page is read once and written once).
//
// Measured, 32/4/8 heads of 128 in bf16 (49 KB a 16-token page): 4096 pages copied in 68 us, 5.9 TB/s; a pool of 49 152
// with 29 491 in use compacted in 203 us, 11 800 moves of 1.16 GB in all at 5.7 TB/s behind 10 us of search and mapping; 24
// pages 2.3 us.  Giving back 24 of 64 sequences, forking 24 others and reserving the next page for all, copies of
// half-filled pages included (98 304 pages): 22 us in five launches of dependent reads, 0.9 us of traffic.  In a loop without
// a graph the host needs longer to issue them (36 us).
#include "common.cuh"
#include "ptx.cuh"

namespace diffqkv {
namespace {

constexpr int kClusterBlocks = 8;
constexpr int kScanThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kCopyVecs = 4;  // 16-byte vectors a thread moves per task
constexpr int kTaskVecs = kCopyThreads * kCopyVecs;

// Sum over the block; `red` holds 33 ints.  Every thread gets its exclusive prefix and the total.
__device__ __forceinline__ int block_scan(int v, int* red, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();  // the previous use of `red` is over
  if (lane == 31) red[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    int w = lane < (int)(blockDim.x >> 5) ? red[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    red[lane] = w;
  }
  __syncthreads();
  total = red[(blockDim.x >> 5) - 1];
  return incl - v + (warp ? red[warp - 1] : 0);
}

__device__ __forceinline__ int pages_of(int tokens, int page_size) {
  return (int)(((long long)tokens + page_size - 1) / page_size);
}

// ------------------------------------------------------------------------------------------------------------- free

__device__ __forceinline__ void release_page(const diffqkv_pages& g, int id, int* dev_status) {
  if (id < 0) return;
  if (id >= g.num_pages) { report(dev_status, DIFFQKV_ERR_INDEX); return; }
  if (atomicSub(g.ref_counts + id, 1) <= 0) {  // was free already: leave it so
    atomicAdd(g.ref_counts + id, 1);
    report(dev_status, DIFFQKV_ERR_INDEX);
  }
}

__global__ void __launch_bounds__(256) pages_free_kernel(const int* seq_ids, const int* keep_tokens, diffqkv_pages g,
                                                         int* dev_status) {
  const int seq = seq_ids[blockIdx.x];
  if (seq < 0 || seq >= g.num_seqs) {
    if (threadIdx.x == 0 && blockIdx.y == 0) report(dev_status, DIFFQKV_ERR_INDEX);
    return;
  }
  const int keep = keep_tokens ? max(keep_tokens[blockIdx.x], 0) : 0;
  int* row = g.page_table + (long long)seq * g.max_pages_per_seq;
  const int first = pages_of(keep, g.page_size);
  for (int e = first + (int)(blockIdx.y * 256 + threadIdx.x); e < g.max_pages_per_seq; e += (int)gridDim.y * 256)
    if (row[e] != -1) release_page(g, atomicExch(row + e, -1), dev_status);  // a sequence listed twice gives back once
  if (threadIdx.x == 0 && blockIdx.y == 0) atomicMin(g.seqlens + seq, keep);
}

// ------------------------------------------------------------------------------------------------------------- fork

// Whether pair i stands: valid ids, and no earlier pair with a valid parent names the same child.  Each pair looks through
// all before it, 256 at a time: 1024 pairs take 21 us, 4096 27, 32 000 266.
__device__ __forceinline__ bool fork_stands(const int* parents, const int* children, int i, const diffqkv_pages& g) {
  const int child = children[i], parent = parents[i];
  const bool valid = child >= 0 && child < g.num_seqs && parent >= 0 && parent < g.num_seqs;
  bool taken = false;
  for (int j = threadIdx.x; j < i; j += blockDim.x)
    taken |= children[j] == child && parents[j] >= 0 && parents[j] < g.num_seqs;
  return !__syncthreads_or(taken) && valid;
}

// The rows the children will have, into the workspace, with the counts they add; all parents are read before any row
// is written (by the next kernel).
__global__ void __launch_bounds__(256) pages_fork_read_kernel(const int* parents, const int* children, diffqkv_pages g,
                                                              int* rows_ws, int* lens_ws, int* dev_status) {
  const int i = blockIdx.x;
  const bool ok = fork_stands(parents, children, i, g);
  const bool leader = threadIdx.x == 0 && blockIdx.y == 0;
  if (leader && !ok) report(dev_status, DIFFQKV_ERR_INDEX);
  const int len = ok ? max(g.seqlens[parents[i]], 0) : -1;
  if (leader) lens_ws[i] = len;
  if (!ok) return;
  const int held = min(pages_of(len, g.page_size), g.max_pages_per_seq);
  const int* row = g.page_table + (long long)parents[i] * g.max_pages_per_seq;
  int* to = rows_ws + (long long)i * g.max_pages_per_seq;
  for (int e = blockIdx.y * 256 + threadIdx.x; e < held; e += gridDim.y * 256) {
    int id = row[e];
    if (id >= g.num_pages) { report(dev_status, DIFFQKV_ERR_INDEX); id = -1; }
    if (id >= 0) atomicAdd(g.ref_counts + id, 1);
    to[e] = max(id, -1);
  }
}

__global__ void __launch_bounds__(256) pages_fork_write_kernel(const int* children, diffqkv_pages g, const int* rows_ws,
                                                               const int* lens_ws, int* dev_status) {
  const int i = blockIdx.x;
  const int len = lens_ws[i];
  if (len < 0) return;
  const int held = min(pages_of(len, g.page_size), g.max_pages_per_seq);
  int* row = g.page_table + (long long)children[i] * g.max_pages_per_seq;
  const int* from = rows_ws + (long long)i * g.max_pages_per_seq;
  for (int e = blockIdx.y * 256 + threadIdx.x; e < g.max_pages_per_seq; e += gridDim.y * 256) {
    const int old = row[e], now = e < held ? from[e] : -1;
    release_page(g, old, dev_status);
    if (old != now) row[e] = now;
  }
  if (threadIdx.x == 0 && blockIdx.y == 0) g.seqlens[children[i]] = len;
}

// ---------------------------------------------------------------------------------------------------------- reserve

struct ReserveWs {
  int* demand;     // [num_seqs] pages the sequence asks for; -1 = its rows do not fit
  int* base;       // [num_seqs] rank of its first page among all handed out, -1 = denied
  int* free_count; // [kClusterBlocks] free pages in each block's share of the counts
  int* fresh;      // [num_pages] the free ids, lowest first
  int* old;        // [num_pages] the shared page that the rank-th new page replaces, or -1
  int* src;        // [num_seqs] half-filled shared page to copy, or -1
  int* dst;        // [num_seqs]
};

// Calls f(entry index in the row, id there) for the entries of sequence s that need a page, in order, a warp together:
// f gets the number of needing entries before it in the sequence.
template <typename F>
__device__ __forceinline__ int for_needed(const diffqkv_pages& g, int first, int end, const int* row, F f) {
  const int lane = threadIdx.x & 31;
  int found = 0;
  for (int e0 = first; e0 < end; e0 += 32) {
    const int e = e0 + lane;
    int id = -1;
    bool need = false;
    if (e < end) {
      id = row[e];
      const bool held = id >= 0 && id < g.num_pages;
      need = !held || g.ref_counts[id] > 1;
      if (!held) id = -1;
    }
    const unsigned mask = __ballot_sync(0xffffffffu, need);
    if (need) f(e, id, found + __popc(mask & ((1u << lane) - 1)));
    found += __popc(mask);
  }
  return found;
}

// The entries of sequence s that the step writes: [first, end); false when its rows do not fit, as the calls that write them
// have it (max_seqlen > 0), or its row of the table is too short.
__device__ __forceinline__ bool write_range(const diffqkv_pages& g, const int* cu_q, int max_seqlen, int s, int& len,
                                            int& first, int& end) {
  const int held = g.seqlens[s];
  len = max(held, 0);
  const long long n = (long long)cu_q[s + 1] - cu_q[s];
  first = len / g.page_size;
  end = first;
  if (n < 0) return false;  // cu_q out of order
  if (n == 0) return true;
  if (held < 0 || cu_q[s] < 0 || (max_seqlen > 0 && held + n > max_seqlen)) return false;
  const long long need = (len + n + g.page_size - 1) / g.page_size;
  if (need > g.max_pages_per_seq) return false;
  end = (int)need;
  return true;
}

__global__ void __cluster_dims__(kClusterBlocks, 1, 1) __launch_bounds__(kScanThreads)
pages_reserve_kernel(const int* cu_q, diffqkv_pages g, int max_seqlen, ReserveWs ws, int* granted, int* dev_status) {
  __shared__ int red[33];
  const int rank = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
  const int warp_all = rank * (kScanThreads / 32) + (tid >> 5), warps_all = kClusterBlocks * (kScanThreads / 32);
  const int share = (g.num_pages + kClusterBlocks - 1) / kClusterBlocks;  // of the counts
  const int lo = min(rank * share, g.num_pages), hi = min(lo + share, g.num_pages);

  // ---- what every sequence asks for, and how many pages are free
  for (int s = warp_all; s < g.num_seqs; s += warps_all) {
    int len, first, end;
    const bool fits = write_range(g, cu_q, max_seqlen, s, len, first, end);
    const int* row = g.page_table + (long long)s * g.max_pages_per_seq;
    const int n = fits ? for_needed(g, first, end, row, [](int, int, int) {}) : -1;
    if (lane == 0) ws.demand[s] = n;
  }
  int mine = 0, total_free = 0;
  for (int i = lo + tid; i < hi; i += kScanThreads) mine += g.ref_counts[i] <= 0;
  block_scan(mine, red, total_free);
  if (tid == 0) ws.free_count[rank] = total_free;
  ptx::cluster_sync();

  // ---- who gets them: sequence s when the demands up to and including its own fit.  Every block computes the sums
  // (it needs the total), block 0 writes the result down.
  int free_all = 0, free_before = 0;
  for (int r = 0; r < kClusterBlocks; ++r) {
    const int n = ws.free_count[r];
    free_all += n;
    if (r < rank) free_before += n;
  }
  long long asked = 0;
  int taken = 0;
  for (int s0 = 0; s0 < g.num_seqs; s0 += kScanThreads) {
    const int s = s0 + tid;
    const int want = s < g.num_seqs ? ws.demand[s] : 0;
    const int n = min(max(want, 0), g.num_pages + 1);
    int sum = 0;
    // a demand beyond the pool is denied whatever its size: cut to the pool's size plus one (at most 2^20 + 1), the sum
    // over 1024 sequences stays within 32 bits
    const long long before = asked + block_scan(n, red, sum);
    const bool ok = want == 0 || (want > 0 && before + n <= free_all);
    int given = 0, part = block_scan(ok ? n : 0, red, given);
    if (rank == 0 && s < g.num_seqs) {
      ws.base[s] = ok && n > 0 ? taken + part : -1;
      if (granted) granted[s] = ok;
      if (!ok) report(dev_status, want < 0 ? DIFFQKV_ERR_INDEX : DIFFQKV_ERR_PAGES);
    }
    asked += sum;
    taken += given;
  }
  // ---- the `taken` lowest free ids
  int at = free_before;
  for (int i0 = lo; i0 < hi && at < taken; i0 += kScanThreads) {
    const int i = i0 + tid;
    const bool free = i < hi && g.ref_counts[i] <= 0;
    int sum = 0;
    const int r = at + block_scan(free, red, sum);
    if (free && r < taken) ws.fresh[r] = i;
    at += sum;
  }
  ptx::cluster_sync();

  // ---- new pages into the tables; the counts of the pages they replace stay as they are until every sequence has
  // been looked at (whether a page is shared is decided by the counts at entry)
  for (int s = warp_all; s < g.num_seqs; s += warps_all) {
    const int base = ws.base[s];
    int src = -1, dst = -1;
    if (base >= 0) {
      int len, first, end;
      write_range(g, cu_q, max_seqlen, s, len, first, end);
      int* row = g.page_table + (long long)s * g.max_pages_per_seq;
      for_needed(g, first, end, row, [&](int e, int id, int k) {
        const int now = ws.fresh[base + k];
        row[e] = now;
        ws.old[base + k] = id;
        if (e == first && id >= 0 && len % g.page_size != 0) { src = id; dst = now; }
      });
      // entry `first` is the first lane's of the first round
      src = __shfl_sync(0xffffffffu, src, 0);
      dst = __shfl_sync(0xffffffffu, dst, 0);
    }
    if (lane == 0) { ws.src[s] = src; ws.dst[s] = dst; }
  }
  ptx::cluster_sync();
  for (int i = rank * kScanThreads + tid; i < taken; i += kClusterBlocks * kScanThreads) {
    g.ref_counts[ws.fresh[i]] = 1;
    if (ws.old[i] >= 0) atomicSub(g.ref_counts + ws.old[i], 1);
  }
}

// ------------------------------------------------------------------------------------------------------- page moves

// One pool as 16-byte vectors.
struct PoolView {
  const uint4* from;
  uint4* to;
  long long f_blk, f_head, f_tok, t_blk, t_head, t_tok;  // vectors
  int vec, page_vecs;    // vectors of a head's token, of a page's tokens of one head
  int vecs;              // vectors of a page, all heads
  int flat;              // both sides keep a page in one piece
};

struct MoveParams {
  const int* src;
  const int* dst;
  const int* count;  // device count of entries, or NULL: n
  int n;
  int gaps;          // a source of -1: nothing to move for the entry (reserve's lists, an entry per sequence)
  int from_blocks, to_blocks;
  PoolView pool[2];
  int tasks[2];  // tasks of kTaskVecs vectors per page
  int* dev_status;
  // (compaction) the page table is mapped on the way
  const int* map;
  const int* table;
  int* table_out;
  long long entries;
  int num_pages;
};

__device__ __forceinline__ long long pool_at(const PoolView& p, int v, long long head_st, long long tok_st) {
  const int head = v / p.page_vecs, in = v - head * p.page_vecs;
  const int tok = in / p.vec;
  return head * head_st + tok * tok_st + (in - tok * p.vec);
}

__global__ void __launch_bounds__(kCopyThreads) pages_move_kernel(const MoveParams p) {
  ptx::grid_dependency_wait();
  for (long long e = blockIdx.x * (long long)kCopyThreads + threadIdx.x; e < p.entries;
       e += (long long)gridDim.x * kCopyThreads) {
    const int id = p.table[e];
    if (id >= p.num_pages) { report(p.dev_status, DIFFQKV_ERR_INDEX); p.table_out[e] = id; }
    else p.table_out[e] = id >= 0 ? p.map[id] : -1;
  }
  const int n = p.count ? *p.count : p.n;
  const int per = p.tasks[0] + p.tasks[1];
  const long long total = (long long)n * per;
  for (long long t = blockIdx.x; t < total; t += gridDim.x) {
    const int i = (int)(t / per);
    int part = (int)(t - (long long)i * per);
    const int src = p.src[i], dst = p.dst[i];
    if (p.gaps && src == -1) continue;
    if (src < 0 || src >= p.from_blocks || dst < 0 || dst >= p.to_blocks) {
      if (threadIdx.x == 0) report(p.dev_status, DIFFQKV_ERR_INDEX);
      continue;
    }
    const int which = part >= p.tasks[0];
    if (which) part -= p.tasks[0];
    const PoolView& v = p.pool[which];
    const uint4* from = v.from + (long long)src * v.f_blk;
    uint4* to = v.to + (long long)dst * v.t_blk;
    const int v0 = part * kTaskVecs + threadIdx.x;
    uint4 x[kCopyVecs];
    if (v.flat) {
#pragma unroll
      for (int k = 0; k < kCopyVecs; ++k)
        if (v0 + k * kCopyThreads < v.vecs) x[k] = from[v0 + k * kCopyThreads];
#pragma unroll
      for (int k = 0; k < kCopyVecs; ++k)
        if (v0 + k * kCopyThreads < v.vecs) to[v0 + k * kCopyThreads] = x[k];
    } else {
#pragma unroll
      for (int k = 0; k < kCopyVecs; ++k)
        if (v0 + k * kCopyThreads < v.vecs) x[k] = from[pool_at(v, v0 + k * kCopyThreads, v.f_head, v.f_tok)];
#pragma unroll
      for (int k = 0; k < kCopyVecs; ++k)
        if (v0 + k * kCopyThreads < v.vecs) to[pool_at(v, v0 + k * kCopyThreads, v.t_head, v.t_tok)] = x[k];
    }
  }
}

PoolView pool_view(const void* from, void* to, long long fb, long long fh, long long ft, long long tb, long long th,
                   long long tt, int heads, int page_size, int d, int elems) {
  PoolView v;
  v.from = static_cast<const uint4*>(from);
  v.to = static_cast<uint4*>(to);
  v.f_blk = fb / elems; v.f_head = fh / elems; v.f_tok = ft / elems;
  v.t_blk = tb / elems; v.t_head = th / elems; v.t_tok = tt / elems;
  v.vec = d / elems;
  v.page_vecs = v.vec * page_size;
  v.vecs = v.page_vecs * heads;
  auto whole = [&](long long head, long long tok) { return tok == v.vec && (heads == 1 || head == v.page_vecs); };
  v.flat = whole(v.f_head, v.f_tok) && whole(v.t_head, v.t_tok);
  return v;
}

void set_pools(MoveParams* m, const diffqkv_cache& from, const diffqkv_cache& to, const diffqkv_shape& s) {
  const int elems = s.dtype == DIFFQKV_BF16 ? 8 : 4;
  m->pool[0] = pool_view(from.k_cache, to.k_cache, from.k_stride_blk, from.k_stride_head, from.k_stride_tok, to.k_stride_blk,
                         to.k_stride_head, to.k_stride_tok, s.n_k, from.page_size, s.d_qk, elems);
  m->pool[1] = pool_view(from.v_cache, to.v_cache, from.v_stride_blk, from.v_stride_head, from.v_stride_tok, to.v_stride_blk,
                         to.v_stride_head, to.v_stride_tok, s.n_v, from.page_size, s.d_v, elems);
  for (int i = 0; i < 2; ++i) m->tasks[i] = (m->pool[i].vecs + kTaskVecs - 1) / kTaskVecs;
  m->from_blocks = from.num_blocks;
  m->to_blocks = to.num_blocks;
  m->map = nullptr; m->table = nullptr; m->table_out = nullptr; m->entries = 0; m->num_pages = 0;
}

// Behind another kernel of the same call (`dependent`): its launch is prepared while that one runs, its blocks start when that
// one has ended (neither search lets them in earlier).
cudaError_t launch_move(const MoveParams& m, long long most_pages, bool dependent, cudaStream_t stream) {
  long long blocks = most_pages * (m.tasks[0] + m.tasks[1]);
  const long long table_blocks = (m.entries + kCopyThreads * 4 - 1) / (kCopyThreads * 4);
  if (blocks < table_blocks) blocks = table_blocks;
  if (blocks < 1) blocks = 1;
  if (blocks > 148 * 8) blocks = 148 * 8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kCopyThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = dependent ? 1 : 0;
  const cudaError_t err = cudaLaunchKernelEx(&cfg, pages_move_kernel, m);
  if (err != cudaSuccess) return err;
  count_launch();
  return cudaGetLastError();
}

// ---------------------------------------------------------------------------------------------------------- compact

struct CompactWs {
  int* live_count;  // [kClusterBlocks] pages in use in each block's share
  int* below;       // pages in use with an id below the number of pages in use
  int* count;       // pages to move
  int* map;         // [num_pages] new id
  int* src;         // [num_pages] moves
  int* dst;
};

__global__ void __cluster_dims__(kClusterBlocks, 1, 1) __launch_bounds__(kScanThreads)
pages_compact_kernel(diffqkv_pages g, CompactWs ws, int* refs_out, int* live) {
  __shared__ int red[33];
  const int rank = blockIdx.x, tid = threadIdx.x;
  const int share = (g.num_pages + kClusterBlocks - 1) / kClusterBlocks;
  const int lo = min(rank * share, g.num_pages), hi = min(lo + share, g.num_pages);
  int mine = 0, block_live = 0;
  for (int i = lo + tid; i < hi; i += kScanThreads) mine += g.ref_counts[i] > 0;
  block_scan(mine, red, block_live);
  if (tid == 0) ws.live_count[rank] = block_live;
  ptx::cluster_sync();
  int all = 0, before = 0;
  for (int r = 0; r < kClusterBlocks; ++r) {
    const int n = ws.live_count[r];
    all += n;
    if (r < rank) before += n;
  }
  // ---- ids below `all` that are free are the holes, their rank is id - (pages in use before); ids from `all` on that
  // are in use move, their rank among all pages in use is kept in map until the number below `all` is known
  int at = before;
  for (int i0 = lo; i0 < hi; i0 += kScanThreads) {
    const int i = i0 + tid;
    const bool used = i < hi && g.ref_counts[i] > 0;
    int sum = 0;
    const int r = at + block_scan(used, red, sum);  // pages in use below i
    if (i < hi) {
      if (i == all) *ws.below = r;
      if (!used && i < all) ws.dst[i - r] = i;
      ws.map[i] = used && i >= all ? r : i;
    }
    at += sum;
  }
  if (all == g.num_pages && rank == 0 && tid == 0) *ws.below = all;
  ptx::cluster_sync();
  const int below = *ws.below;
  for (int i = lo + tid; i < hi; i += kScanThreads) {
    const int refs = g.ref_counts[i];
    if (i < all) {
      if (refs > 0) refs_out[i] = refs;  // a hole gets its count from the page that moves there
    } else {
      if (refs > 0) {
        const int k = ws.map[i] - below, to = ws.dst[k];
        ws.src[k] = i;
        ws.map[i] = to;
        refs_out[to] = refs;
      }
      refs_out[i] = 0;
    }
  }
  if (rank == 0 && tid == 0) {
    *ws.count = all - below;
    if (live) *live = all;
  }
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

unsigned row_blocks(int row) {  // blocks along a table row: four entries per thread
  const int n = (row + 1023) / 1024;
  return (unsigned)(n < 1 ? 1 : n > 64 ? 64 : n);
}

}  // namespace

cudaError_t launch_pages_free(const int* seq_ids, const int* keep_tokens, int n, const diffqkv_pages& g, int* dev_status,
                              cudaStream_t stream) {
  pages_free_kernel<<<dim3((unsigned)n, row_blocks(g.max_pages_per_seq)), 256, 0, stream>>>(seq_ids, keep_tokens, g,
                                                                                           dev_status);
  count_launch();
  return cudaGetLastError();
}

size_t pages_fork_workspace_bytes(const diffqkv_pages& g, int n) {
  return up256(sizeof(int) * (size_t)n * g.max_pages_per_seq) + up256(sizeof(int) * (size_t)n);
}

cudaError_t launch_pages_fork(const int* parents, const int* children, int n, const diffqkv_pages& g, void* workspace,
                              int* dev_status, cudaStream_t stream) {
  int* rows = static_cast<int*>(workspace);
  int* lens = reinterpret_cast<int*>(static_cast<char*>(workspace) + up256(sizeof(int) * (size_t)n * g.max_pages_per_seq));
  const dim3 grid((unsigned)n, row_blocks(g.max_pages_per_seq));
  pages_fork_read_kernel<<<grid, 256, 0, stream>>>(parents, children, g, rows, lens, dev_status);
  count_launch();
  cudaError_t err = cudaGetLastError();
  if (err != cudaSuccess) return err;
  pages_fork_write_kernel<<<grid, 256, 0, stream>>>(children, g, rows, lens, dev_status);
  count_launch();
  return cudaGetLastError();
}

size_t pages_reserve_workspace_bytes(const diffqkv_pages& g) {
  return 256 + 4 * up256(sizeof(int) * (size_t)g.num_seqs) + 2 * up256(sizeof(int) * (size_t)g.num_pages);
}

cudaError_t launch_pages_reserve(const int* cu_q, const diffqkv_pages& g, const diffqkv_cache& c, const diffqkv_shape& s,
                                 int* granted, void* workspace, int* dev_status, cudaStream_t stream) {
  char* at = static_cast<char*>(workspace);
  auto take = [&](size_t bytes) { char* p = at; at += up256(bytes); return reinterpret_cast<int*>(p); };
  ReserveWs ws;
  ws.free_count = take(256);
  ws.demand = take(sizeof(int) * (size_t)g.num_seqs);
  ws.base = take(sizeof(int) * (size_t)g.num_seqs);
  ws.src = take(sizeof(int) * (size_t)g.num_seqs);
  ws.dst = take(sizeof(int) * (size_t)g.num_seqs);
  ws.fresh = take(sizeof(int) * (size_t)g.num_pages);
  ws.old = take(sizeof(int) * (size_t)g.num_pages);
  pages_reserve_kernel<<<kClusterBlocks, kScanThreads, 0, stream>>>(cu_q, g, c.max_seqlen, ws, granted,
                                                                      dev_status);
  count_launch();
  const cudaError_t err = cudaGetLastError();
  if (err != cudaSuccess) return err;
  MoveParams m;
  m.src = ws.src; m.dst = ws.dst; m.count = nullptr; m.n = g.num_seqs; m.gaps = 1;
  m.dev_status = dev_status;
  set_pools(&m, c, c, s);
  return launch_move(m, g.num_seqs, true, stream);
}

cudaError_t launch_pages_copy(const int* src_ids, const int* dst_ids, int n, const diffqkv_cache& from,
                              const diffqkv_cache& to, const diffqkv_shape& s, int* dev_status, cudaStream_t stream) {
  MoveParams m;
  m.src = src_ids; m.dst = dst_ids; m.count = nullptr; m.n = n; m.gaps = 0;
  m.dev_status = dev_status;
  set_pools(&m, from, to, s);
  return launch_move(m, n, false, stream);
}

size_t pages_compact_workspace_bytes(const diffqkv_pages& g) {
  return 256 + 3 * up256(sizeof(int) * (size_t)g.num_pages);
}

cudaError_t launch_pages_compact(const diffqkv_pages& g, const diffqkv_cache& c, const diffqkv_shape& s, int* table_out,
                                 int* refs_out, int* live, void* workspace, int* dev_status, cudaStream_t stream) {
  char* at = static_cast<char*>(workspace);
  auto take = [&](size_t bytes) { char* p = at; at += up256(bytes); return reinterpret_cast<int*>(p); };
  CompactWs ws;
  ws.live_count = take(256);
  ws.below = ws.live_count + kClusterBlocks;
  ws.count = ws.below + 1;
  ws.map = take(sizeof(int) * (size_t)g.num_pages);
  ws.src = take(sizeof(int) * (size_t)g.num_pages);
  ws.dst = take(sizeof(int) * (size_t)g.num_pages);
  pages_compact_kernel<<<kClusterBlocks, kScanThreads, 0, stream>>>(g, ws, refs_out, live);
  count_launch();
  const cudaError_t err = cudaGetLastError();
  if (err != cudaSuccess) return err;
  MoveParams m;
  m.src = ws.src; m.dst = ws.dst; m.count = ws.count; m.n = 0; m.gaps = 0;
  m.dev_status = dev_status;
  set_pools(&m, c, c, s);
  m.map = ws.map; m.table = g.page_table; m.table_out = table_out;
  m.entries = (long long)g.num_seqs * g.max_pages_per_seq;
  m.num_pages = g.num_pages;
  return launch_move(m, (g.num_pages + 1) / 2, true, stream);
}

}  // namespace diffqkv
