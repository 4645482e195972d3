// Causal attention of ragged chunks of new tokens over the cache on the sm_100a tensor cores (diffqkv_extend; paper
// Section 2 formulation, head map of Eq. (idx)).
//
// Mathematics: row i of sequence b sits at position past_b + i and sees cached tokens 0 .. past_b + i:
//     s_j = scale <q, k_j>,  out = sum_j 2^(s_j log2 e - m) v_j / sum_j 2^(s_j log2 e - m),  one pass over the tokens
// with a running reference m per row (raised only when exceeded by 2^8, the accumulator is then rescaled).  Scores,
// statistics and the accumulator are fp32; the weights are rounded to bf16 for the second product (the tensor core
// takes 16-bit operands), their sum is of the unrounded values.
//
// Rows.  The G query heads that share both their K head and their V head read the same tokens, so a tile of 128 matrix
// rows holds T = 128 / G tokens of the chunk times G heads (row = token * G + head): one token of 32/4/8 heads already
// fills four rows, and K and V are staged once for all of them.
//
// Work.  Sequences of a few rows are left to extend_thin.cu.  A longer chunk is cut into items of 2 T tokens.  An item of
// more than T tokens ("wide") has two row tiles that share every 128-token K/V tile; one of at most T tokens ("narrow":
// the end of a chunk) has a single row tile, which is given to both softmax groups: one takes the even K/V tiles, the
// other the odd ones, and the first joins the two results at the end (softmax does not care which tokens it has seen).
// All (sequence, head group, item, K/V tile) form one flat list, in which an item costs something next to its tiles, that
// is divided evenly over the persistent blocks, so that one long chunk and a hundred short ones both fill the SMs.  A
// block's run inside an item is a segment; an item that is cut leaves normalised partial rows in the workspace, which
// extend_combine_kernel joins in a fixed order.  Lengths are known on the device alone: each block finds its place by a
// closed-form sum (floor_sum) and walks from there.
// Head groups that differ only in their V head (or only in their K head) are given to a team of neighbouring blocks
// that walk the same tiles at the same time, so that the shared K (V) tiles come out of the second-level cache.
//
// Roles of the twelve warps, as in prefill.cu: warp 0 TMA producer, one thread of warp 1 issues the products, warps 4-7
// and 8-11 are the two softmax groups (one thread per row).  The producer walks the segments and hands them to the other
// roles through a small ring; the roles meet only at mbarriers, so the next segment's K, V and Q are on their way while
// the last one is being written out.  Every wait is bounded; on expiry the block reports DIFFQKV_ERR_TIMEOUT, drains and
// frees its tensor memory.
//
// Bound by the chain score product -> softmax -> value product of each of the two row tiles, one of which computes while
// the other's products run.  Chunks of 1.5k-2k rows over 0-6k cached tokens, four sequences, 32/4/8 heads of 128: 430 us
// while the SMs run at 1965 MHz, 1065 TFLOP/s of causal work (0.62 of a large matrix product in a burst); calls without a
// pause run into the power limit and settle at 1730 MHz and 490 us, the same number of cycles.  A pair of row tiles takes
// 3460 cycles: 2200 of softmax, of which 1024 are exponentials at the rate of the special-function unit when both groups
// are at it, and 1260 from the last weight to the next score, 768 of them products.  The tensor pipe is active 55 % of the
// time, the special-function unit 55 %.  What did not help: announcing 96 or 112 instead of 64 tokens' weights first
// (436 us), waiting for the next K before the last weights (450-470).  Not settled: exponentials by polynomial for a part
// of the scores.  Earlier forms of this kernel took 415 to 850 us with them for an eighth to a half of the scores.
// Heads of 64 channels (32/4/16), the same chunks: 396 us without a pause, 580 TFLOP/s; 64-channel keys with 128-channel
// values 471 us, 730 TFLOP/s (half the products, as many exponentials).
//
// Ranged steps (diffqkv_extend_window, diffqkv_extend_shared), whose sequences of a few rows are extend_few.cu's: the tiles
// that no row of an item sees are left out of its list, so that an item's tiles are those of its first tokens and, `skip`
// tiles further on, those of its window; a group's prefix is an entry in front of the sequences', whose own tokens begin
// behind it, and extend_merge_kernel joins the two.  A step begins in one short piece of code in 32-bit arithmetic (see
// ranged_start); a block's first request still goes out 16 thousand cycles, 9 us, after its start, nearly all of it code that
// is fetched once, and an item costs 7-8 thousand cycles next to its tiles (2.5 of them the masks of its first and last tile).
// The same four chunks in windows of 2k tokens: 285 us in a graph, 298 call by call, 750 TFLOP/s of what is seen; tensor pipe
// 44 % active, special-function unit 45 %.  3k rows behind two prefixes of 3k-5k tokens, 64 and 128 channels: 274 us (power
// keeps the SMs at 1.4-1.6 GHz); with the prefixes shared 284, some 36 of them the join of 98 MB of parts; the plain kernel 245.
// Tried and not kept: rows written 32 bytes a lane without the exchange of four lanes (329 -> 343 us: the same lines, and
// none of it was instructions), a thread a barrier at the start (283 -> 289), two rows at a time in the join (36 -> 37), a way
// of its own there for rows of whole items (36), four blocks of it an SM (34, but 4 x 4 single rows 24.2 -> 25.1), rows with
// something to join listed first (24 -> 20, but small steps 0.4 us longer).
#include <algorithm>
#include <atomic>
#include <numeric>
#include <type_traits>

#include "attn_math.cuh"
#include "common.cuh"
#include "extend.cuh"
#include "ptx.cuh"
#include "tcgen05.cuh"
#include "tmap.cuh"

namespace diffqkv {
namespace {

constexpr int kExtendThreads = 384;
constexpr int kSoftmaxWarp0 = 4;
// Shared memory: two Q tiles, the rings of K and V tiles, the exchange of the two softmax groups, barriers.
constexpr int kExtendSmem = 1024 + 2 * (kRows * kDMax * 2) + kRingBytes + 1024 + 320;
// A segment as the producer hands it to the other roles, through a ring in shared memory.
struct Segment {
  int row_lo, n, past;  // the sequence: first row, rows, tokens cached before
  int tok0, head0;      // first token of the item within the chunk, first head of the group
  int ta, tb;           // K/V tiles
  int nst0;             // tiles of the first softmax group
  int v0;               // V tiles requested before the segment (the ring's position)
  int flags;
};
struct RangedSegment : Segment {
  int end, start;  // the entry's tokens
  int low, skip;   // first token behind the sinks that some row of the item sees; tiles skipped
  int dst;
};
constexpr int kSegRing = 4;
constexpr int kSegEnd = 1, kSegWide = 2, kSegWhole = 4, kSegFirst = 8;  // first: holds the item's first tile

// The segments of one block, in order.
template <bool kRanged>
struct Walk {
  int b, u, item;
  long long item_lo, end, begin;
  SeqOf<kRanged> seq;
  // of the current segment
  bool wide;
  int nt, ta, tb, nst0;

  // ranged: likewise, the sequence is loaded already
  __device__ void start(const ExtendParams& p, uint32_t w0, uint32_t w1, int b0, uint32_t lo, const SeqOf<true>& s0) {
    begin = w0; end = w1;
    b = b0;
    seq = s0;
    const uint32_t per = seq.cost(p);
    u = (int)((w0 - lo) / per);
    const int r = (int)(w0 - lo - u * per);
    int a = 0, z = seq.items;  // largest item whose start is not behind r
    while (z - a > 1) {
      const int mid = (a + z) >> 1;
      if (seq.cost_before(p, mid) <= r) a = mid; else z = mid;
    }
    item = a;
    item_lo = (long long)lo + u * per + seq.cost_before(p, item);
  }
  // from the sequence b0 in which the block's range begins, whose flat place is lo
  __device__ void start(const ExtendParams& p, long long w0, long long w1, int b0, long long lo) {
    begin = w0; end = w1;
    b = b0;
    if (w0 >= w1) { item_lo = w1; b = entries_of<kRanged>(p); return; }
    seq.load(p, b);
    const long long per = seq.cost(p);
    u = (int)quotient(w0 - lo, per);
    const long long r = (w0 - lo) - u * per;
    int a = 0, z = seq.items;  // largest item whose start is not behind r
    while (z - a > 1) {
      const int mid = (a + z) >> 1;
      if (seq.cost_before(p, mid) <= r) a = mid; else z = mid;
    }
    item = a;
    item_lo = lo + u * per + seq.cost_before(p, item);
  }
  __device__ bool next(const ExtendParams& p) {  // false: no more segments
    while (b < entries_of<kRanged>(p) && item_lo < end) {
      wide = seq.wide(p, item);
      nt = seq.tiles(p, item);
      const int cost = wide ? kWideCost : kNarrowCost;
      ta = item_tile(begin - item_lo, cost, nt, item_cost<kRanged>);
      tb = item_tile(end - item_lo, cost, nt, item_cost<kRanged>);
      if (ta < tb) {
        if (wide) {
          int nt0;  // tiles that the first row tile sees
          if constexpr (kRanged) nt0 = seq.reach(p, item * 2 * p.T + p.T) - seq.skip(p, item * 2 * p.T);
          else nt0 = (seq.past + item * 2 * p.T + p.T + kKT - 1) / kKT;
          nst0 = max(0, min(tb, nt0) - ta);
        } else {
          nst0 = (tb - ta + 1) / 2;
        }
        return true;
      }
      advance(p);
    }
    return false;
  }
  __device__ void advance(const ExtendParams& p) {
    item_lo += item_cost<kRanged> + (long long)(seq.wide(p, item) ? kWideCost : kNarrowCost) * seq.tiles(p, item);
    if (kRanged && item_lo >= end) return;  // no reading on through entries of a few rows, 800 cycles each
    if (++item < seq.items) return;
    item = 0;
    if (++u < p.n_units) return;
    u = 0;
    do {
      if (++b >= entries_of<kRanged>(p)) return;
      seq.load(p, b);
    } while (seq.n == 0);
  }
  __device__ int tok0(const ExtendParams& p) const { return item * 2 * p.T; }
};

// The 4 x 4 matrix of 16-byte pieces that four neighbouring lanes hold, a row each, transposed: piece y of a lane becomes
// its own piece of lane y.
__device__ __forceinline__ void transpose4(uint4 (&v)[4], int lane) {
  auto swap = [](uint4& a, uint4& b, bool yes) {
    const uint4 x = a;
    a = yes ? b : a;
    b = yes ? x : b;
  };
  auto pass = [](uint4& a, int by) {
    a.x = __shfl_xor_sync(0xffffffffu, a.x, by);
    a.y = __shfl_xor_sync(0xffffffffu, a.y, by);
    a.z = __shfl_xor_sync(0xffffffffu, a.z, by);
    a.w = __shfl_xor_sync(0xffffffffu, a.w, by);
  };
  swap(v[0], v[1], lane & 1); swap(v[2], v[3], lane & 1);
  pass(v[1], 1); pass(v[3], 1);
  swap(v[0], v[1], lane & 1); swap(v[2], v[3], lane & 1);
  swap(v[0], v[2], lane & 2); swap(v[1], v[3], lane & 2);
  pass(v[2], 2); pass(v[3], 2);
  swap(v[0], v[2], lane & 2); swap(v[1], v[3], lane & 2);
}

// kDQK, kD: channels per head of Q/K and of V: (128, 128), (64, 64) or (64, 128).  kRanged: rows do not see all tokens before
// them; the tiles that no row of an item sees are left out of the list, boxes of pages that none sees are not read.
template <int kDQK, int kD, bool kRanged>
__global__ void __launch_bounds__(kExtendThreads, 1)
extend_attn_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                   const __grid_constant__ CUtensorMap tmap_v, const ExtendParams p) {
  constexpr int kHalvesK = kDQK / 64, kHalves = kD / 64;  // 64-channel halves of a Q/K row and of a V row
  constexpr int kHalvesMax = kHalvesK > kHalves ? kHalvesK : kHalves;
  constexpr int kQBytes = kRows * kDQK * 2;
  constexpr int kKBytes = kKT * kDQK * 2;
  constexpr int kTBytes = kKT * kD * 2;
  constexpr int kKSlots = 3 * kDMax / kDQK, kVSlots = 2 * kDMax / kD;
  // With 64-channel values P has tensor-memory columns of its own: [S0 128][S1 128][O0 64][O1 64][P0 64][P1 64], and the
  // next tile's scores are issued once the current ones are in registers; otherwise P lies over its scores' columns.
  constexpr bool kSepP = kD == 64;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char* q_s = smem;                      // 2 row tiles
  unsigned char* k_s = q_s + 2 * kQBytes;         // ring of K tiles
  unsigned char* v_s = k_s + kKSlots * kKBytes;   // ring of V tiles
  float2* xch_s = reinterpret_cast<float2*>(v_s + kVSlots * kTBytes);  // [128] (m, l) of the second softmax group
  uint64_t* bars = reinterpret_cast<uint64_t*>(xch_s + kRows);
  const uint32_t q_full = ptx::smem_u32(bars), q_empty = q_full + 8;
  const uint32_t k_full0 = q_empty + 8, k_empty0 = k_full0 + 8 * kKSlots;
  const uint32_t v_full0 = k_empty0 + 8 * kKSlots, v_empty0 = v_full0 + 8 * kVSlots;
  const uint32_t s_full0 = v_empty0 + 8 * kVSlots, p_half0 = s_full0 + 16, p_full0 = p_half0 + 16;
  const uint32_t o_done0 = p_full0 + 16, o_free0 = o_done0 + 16, s_free0 = o_free0 + 16;
  const uint32_t x_full = s_free0 + 16, drain = x_full + 8;
  const uint32_t seg_full0 = drain + 8, seg_empty0 = seg_full0 + 8 * kSegRing;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 + 2 * kKSlots + 2 * kVSlots + 14 + 2 * kSegRing);
  volatile int* abort_flag = reinterpret_cast<int*>(tmem_slot + 1);
  using Seg = typename std::conditional<kRanged, RangedSegment, Segment>::type;
  __shared__ Seg seg_s[kSegRing];
  __shared__ long long scan_s[kExtendThreads / 32], others_s[kExtendThreads / 32];
  __shared__ RangedScan<kExtendThreads / 32> ranged_s;
  __shared__ long long seek_lo_s;
  __shared__ int seek_b_s;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // The kernel for thin sequences works on other rows; whichever of the two comes second may take the SMs that the
  // first one's blocks leave.  The joining kernel depends on the second alone, which therefore ends behind the first.
  // Ranged, the first of the two is launched before the work in front of it has ended, for which it waits here.
  if (kRanged && p.first) ptx::grid_dependency_wait();
  if (p.first) ptx::grid_launch_dependents();
  const int team = (int)blockIdx.x / p.list.team, member = (int)blockIdx.x - team * p.list.team;
  long long total, w0, w1;  // of the flat list; this block's range of it
  int n_teams;              // that take part
  uint32_t tmem_base;
  auto init = [&] {
    if (tid == 0) {
      *abort_flag = 0;
      if constexpr (!kRanged) {
        seek_b_s = p.batch;
        seek_lo_s = 0;
      }
      ptx::mbar_init(q_full, 1);
      ptx::mbar_init(q_empty, 1);
      for (int s = 0; s < kKSlots; ++s) {
        ptx::mbar_init(k_full0 + 8 * s, 1);
        ptx::mbar_init(k_empty0 + 8 * s, 1);
      }
      for (int s = 0; s < kVSlots; ++s) {
        ptx::mbar_init(v_full0 + 8 * s, 1);
        ptx::mbar_init(v_empty0 + 8 * s, 1);
      }
      for (int t = 0; t < 2; ++t) {
        ptx::mbar_init(s_full0 + 8 * t, 1);
        ptx::mbar_init(p_half0 + 8 * t, 4);
        ptx::mbar_init(p_full0 + 8 * t, 4);
        ptx::mbar_init(o_done0 + 8 * t, 1);
        ptx::mbar_init(o_free0 + 8 * t, 4);
        ptx::mbar_init(s_free0 + 8 * t, 4);
      }
      ptx::mbar_init(x_full, 4);
      for (int s = 0; s < kSegRing; ++s) {
        ptx::mbar_init(seg_full0 + 8 * s, 1);
        ptx::mbar_init(seg_empty0 + 8 * s, 9);  // the MMA thread and eight softmax warps
      }
      ptx::mbar_init(drain, 1);
      ptx::fence_barrier_init();
      ptx::prefetch_tmap(&tmap_q);
      ptx::prefetch_tmap(&tmap_k);
      ptx::prefetch_tmap(&tmap_v);
    }
    if (warp == 1) {
      tc::tmem_alloc(ptx::smem_u32(tmem_slot), kTmemCols);
      tc::tmem_relinquish();
    }
  };
  if constexpr (kRanged) {
    // a step of a few rows each (decode): most blocks leave here, in a third of the time that the sums below take
    bool any = blockIdx.x == 0;  // which reports the entries that do not fit
    for (int e = tid; e < p.entries; e += kExtendThreads) any |= long_entry(p, e);
    if (!__syncthreads_or(any)) {
      if (tid == 0) p.list.meta[blockIdx.x].rows = 0;
      ptx::grid_dependency_wait();
      return;
    }
    init();
    tc::fence_before_sync();
    SeqOf<true> my;
    const RangedStart at = ranged_start(p, ranged_s, my, blockIdx.x == 0);
    tc::fence_after_sync();
    tmem_base = *tmem_slot;
    total = at.wide;
    n_teams = ranged_wide_teams(p, at.wide, at.few);
    if (team >= n_teams) {  // no long chunks (decode), or fewer than blocks
      if (tid == 0) p.list.meta[blockIdx.x].rows = 0;
      if (warp == 1) tc::tmem_dealloc(tmem_base, kTmemCols);
      ptx::grid_dependency_wait();
      return;
    }
    w0 = ranged_share_start(at.wide, team, n_teams);
    w1 = ranged_share_start(at.wide, team + 1, n_teams);
    ranged_seek(p, ranged_s, at, my, (uint32_t)w0, at.before_wide,
                [&](const SeqOf<true>& s) -> uint32_t { return s.n > 0 ? p.n_units * (uint32_t)s.cost(p) : 0u; });
  } else {
    const int per_thread = (p.batch + kExtendThreads - 1) / kExtendThreads;
    const int b_lo = min(tid * per_thread, p.batch), b_hi = min(b_lo + per_thread, p.batch);
    SeqOf<false> my = {};  // the thread's first sequence: there is seldom another
    if (b_lo < b_hi) my.load(p, b_lo);
    {  // a step of thin sequences alone (decode): nothing to do here
      bool any = my.n > 0 || my.bad;
      for (int b = b_lo + 1; b < b_hi; ++b) {
        SeqOf<false> x;
        x.load(p, b);
        any |= x.n > 0 || x.bad;
      }
      if (!__syncthreads_or(any)) {
        if (tid == 0) p.list.meta[blockIdx.x].rows = 0;
        ptx::grid_dependency_wait();
        return;
      }
    }
    init();
    // ---- this block's range of the flat list: every thread sums the cost of its share of the sequences
    long long mine = 0, others = 0;
    bool any_thin = false;
    SeqOf<false> s = my;
    for (int b = b_lo; b < b_hi;) {
      if (s.bad && blockIdx.x == 0) report(p.dev_status, DIFFQKV_ERR_INDEX);
      if (s.n > 0) mine += p.n_units * s.cost(p);
      if (s.thin_tiles > 0) {
        others += (long long)p.n_units * (s.thin_tiles + kThinItemCost);
        any_thin = true;
      }
      if (++b < b_hi) s.load(p, b);
    }
    tc::fence_before_sync();
    any_thin = __syncthreads_or(any_thin);
    long long before = block_scan<kExtendThreads / 32>(mine, scan_s, total);
    tc::fence_after_sync();
    tmem_base = *tmem_slot;
    if (any_thin) block_scan<kExtendThreads / 32>(others, others_s, others);
    n_teams = wide_teams(p, total, others);  // that take part
    if (team >= n_teams) {
      if (tid == 0) p.list.meta[blockIdx.x].rows = 0;
      if (warp == 1) tc::tmem_dealloc(tmem_base, kTmemCols);
      ptx::grid_dependency_wait();
      return;
    }
    w0 = share_start(total, team, n_teams);
    w1 = share_start(total, team + 1, n_teams);
    if (w0 < w1 && before <= w0 && w0 < before + mine) {
      s = my;
      for (int b = b_lo;;) {
        const long long c = p.n_units * s.cost(p);
        if (w0 < before + c) {
          seek_b_s = b;
          seek_lo_s = before;
          break;
        }
        before += c;
        if (++b >= b_hi) break;
        s.load(p, b);
      }
    }
  }
  __syncthreads();
  const uint32_t q_u32 = ptx::smem_u32(q_s), k_u32 = ptx::smem_u32(k_s), v_u32 = ptx::smem_u32(v_s);

  if (warp < kSoftmaxWarp0) {
  // 12 x 168 = 4 x 72 + 8 x 216: the producer walks the segments in 64-bit arithmetic (56 spilled it)
  asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    // One box per (token part, channel half) of a tile: lane x owns box x of every K tile and of every V tile.
    const int parts = kKT / p.box_tok;
    // Ranged: where the cache allows (see make_row_map) a box brings whole rows, half as many boxes: tiles of 16-token pages
    // come at the rate of boxes (7.2 thousand cycles for a K and a V tile of 128 channels, not 3.5).
    int box_halves = kHalvesMax;
    if constexpr (kRanged) box_halves = (kHalvesK == 2 && !p.k_rows) || (kHalves == 2 && !p.v_rows) ? 2 : 1;
    const int boxes = box_halves * parts;
    const int my_part = lane / box_halves, my_half = lane % box_halves;
    const uint32_t my_off = my_half * (kKT * 128) + my_part * (p.box_tok * 128);
    const bool k_here = kRanged && p.k_rows ? my_half == 0 : my_half < kHalvesK;
    const bool v_here = kRanged && p.v_rows ? my_half == 0 : my_half < kHalves;
    int kc = 0, vc = 0, segs = 0;  // K tiles, V tiles, Q loads requested so far
    bool ok = true;
    ExtendMeta m = {};
    Walk<kRanged> w;
    if constexpr (kRanged) w.start(p, (uint32_t)w0, (uint32_t)w1, ranged_s.e, ranged_s.lo, ranged_s.seq);
    else w.start(p, w0, w1, seek_b_s, seek_lo_s);
    auto hand_out = [&](const Seg& d) -> bool {
      const int s = segs % kSegRing;
      if (!wait_warp(seg_empty0 + 8 * s, ((segs / kSegRing) & 1) ^ 1, abort_flag)) return false;
      if (lane == 0) {
        seg_s[s] = d;
        ptx::mbar_arrive(seg_full0 + 8 * s);  // releases the stores above
      }
      __syncwarp();
      return true;
    };
    for (; ok && w.next(p); w.advance(p), ++segs) {
      int kv_len = w.seq.past + w.seq.n, tab = w.b, low = 0, skip = 0;
      if constexpr (kRanged) {
        kv_len = w.seq.end;
        tab = w.seq.tab;
        low = w.seq.low(p, w.tok0(p));
        skip = w.seq.skip(p, w.tok0(p));
      }
      const int g = w.u * p.list.team + member;
      const int head0 = g * p.G;
      const int hk = head0 / p.heads_per_k, hv = head0 / p.heads_per_v;  // Eq. (idx)
      const int tok0 = w.tok0(p);
      if (w.ta == 0 && w.tb < w.nt) {
        m.rows = m.part_rows = min(w.seq.n - tok0, 2 * p.T) * p.G; m.row_lo = w.seq.lo + tok0; m.head0 = head0;
        m.parts = share_of(w.item_lo + last_tile(w.wide ? kWideCost : kNarrowCost, w.nt, item_cost<kRanged>), total, n_teams) - team + 1;
      }
      if constexpr (kRanged) {
        if (w.ta == 0 && member == 0 && p.groups > 0 && lane == 0)
          p.refs[((w.seq.dst == kDstPrefix ? 0LL : p.total_q) + w.seq.lo + tok0) * p.n_units + w.u] = {team, w.tb < w.nt ? -m.parts : -1};
      }
      Seg seg;
      static_cast<Segment&>(seg) = {w.seq.lo, w.seq.n, w.seq.past, tok0, head0, w.ta, w.tb, w.nst0, vc,
                                    (w.wide ? kSegWide : 0) | (w.ta == 0 ? kSegFirst : 0) |
                                        (w.ta == 0 && w.tb == w.nt ? kSegWhole : 0)};
      if constexpr (kRanged) {
        seg.end = kv_len; seg.start = w.seq.start; seg.low = low; seg.skip = skip; seg.dst = w.seq.dst;
      }
      if (!hand_out(seg)) {
        ok = false;
        break;
      }
      // first token of tile `tile`, and whether this lane's box of it has a token that is wanted
      auto token_of = [&](int tile) -> int {
        return (kRanged && tile >= p.sink_tiles ? tile + skip : tile) * kKT;
      };
      auto wanted = [&](int tok) -> bool { return !kRanged || tok < p.sinks || tok + p.box_tok > low; };
      const int per_step = w.wide ? 1 : 2;
      // page of this lane's box of a tile (fetched a step ahead)
      auto fetch = [&](int tile) -> int {
        if (!p.page_table) return tab;
        const int tok = token_of(tile) + my_part * p.box_tok;
        if (tile >= w.tb || lane >= boxes || tok >= kv_len || !wanted(tok)) return 0;
        return p.page_table[(long long)tab * p.max_pages_per_seq + tok / p.page_size];
      };
      int blk[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) blk[x] = x < per_step ? fetch(w.ta + x) : 0;
      for (int tile = w.ta; tile < w.tb && ok; tile += per_step) {
        const int count = min(per_step, w.tb - tile);
        int now[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          now[x] = blk[x];
          if (x < count && lane < boxes && token_of(tile + x) + my_part * p.box_tok < kv_len &&
              (now[x] < 0 || now[x] >= p.num_blocks)) {  // never read outside the pool: flag it, read block 0 instead
            report(p.dev_status, DIFFQKV_ERR_INDEX);
            now[x] = 0;
          }
          blk[x] = x < per_step ? fetch(tile + per_step + x) : 0;
        }
        for (int kv = 0; kv < 2 && ok; ++kv) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (x >= count || !ok) continue;
            const int tok = token_of(tile + x);
            int parts_valid = min(parts, (kv_len - tok + p.box_tok - 1) / p.box_tok);
            const int first = tok + my_part * p.box_tok;
            const int slot_tok = p.page_table ? first % p.page_size : first;
            const bool here = lane < boxes && my_part < parts_valid && wanted(first);
            if constexpr (kRanged) parts_valid = __popc(__ballot_sync(0xffffffffu, here && my_half == 0));
            if (kv == 0) {
              const int s = kc % kKSlots;
              if (!wait_warp(k_empty0 + 8 * s, ((kc / kKSlots) & 1) ^ 1, abort_flag)) { ok = false; continue; }
              if (lane == 0) ptx::mbar_arrive_expect_tx(k_full0 + 8 * s, (uint32_t)parts_valid * p.box_tok * 128u * kHalvesK);
              __syncwarp();
              if (here && k_here) {
                if (kRanged && p.k_rows)
                  ptx::tma_load_5d(k_u32 + s * kKBytes + my_part * (p.box_tok * 256), &tmap_k, k_full0 + 8 * s, 0, 0, 0,
                                   hk * p.head_groups + slot_tok / 8, now[x]);
                else
                  ptx::tma_load_5d(k_u32 + s * kKBytes + my_off, &tmap_k, k_full0 + 8 * s, 0, slot_tok, my_half, hk, now[x]);
              }
              ++kc;
            } else {
              const int s = vc % kVSlots;
              if (!wait_warp(v_empty0 + 8 * s, ((vc / kVSlots) & 1) ^ 1, abort_flag)) { ok = false; continue; }
              if (lane == 0) ptx::mbar_arrive_expect_tx(v_full0 + 8 * s, (uint32_t)parts_valid * p.box_tok * 128u * kHalves);
              __syncwarp();
              if (here && v_here) {
                if (kRanged && p.v_rows)
                  ptx::tma_load_5d(v_u32 + s * kTBytes + my_part * (p.box_tok * 256), &tmap_v, v_full0 + 8 * s, 0, 0, 0,
                                   hv * p.head_groups + slot_tok / 8, now[x]);
                else
                  ptx::tma_load_5d(v_u32 + s * kTBytes + my_off, &tmap_v, v_full0 + 8 * s, 0, slot_tok, my_half, hv, now[x]);
              }
              ++vc;
            }
          }
          if (kv == 0 && tile == w.ta && ok) {  // the segment's Q behind its first K tiles
            if (!wait_warp(q_empty, (segs & 1) ^ 1, abort_flag)) { ok = false; continue; }
            if (lane == 0) {
              const int tiles = w.wide ? 2 : 1;
              ptx::mbar_arrive_expect_tx(q_full, (uint32_t)(tiles * kHalvesK * p.G * p.T) * 128u);
              for (int t = 0; t < tiles; ++t)
#pragma unroll
                for (int h = 0; h < kHalvesK; ++h)
                  ptx::tma_load_4d(q_u32 + t * kQBytes + h * (kRows * 128), &tmap_q, q_full, 0, head0, w.seq.lo + tok0 + t * p.T, h);
            }
            __syncwarp();
          }
        }
      }
      if (!ok) break;
    }
    // Ranged: the joining kernel, which waits for the end of both, may take its place once the second one's last tiles are on
    // their way (a launch and the search for a row's items are then no longer in its time).
    if (kRanged && !p.first) ptx::grid_launch_dependents();
    Seg last = {};
    last.flags = kSegEnd;
    if (ok) ok = hand_out(last);
    if (lane == 0) p.list.meta[blockIdx.x] = m;
    if (!ok) {
      report(p.dev_status, DIFFQKV_ERR_TIMEOUT);
      // give copies in flight a bounded chance to land before the block's shared memory is released (a Q request is
      // counted once its segment is over, so the last one may be one more)
      if (segs > 0) ptx::mbar_wait(q_full, (uint32_t)(segs - 1) & 1u, nullptr);
      ptx::mbar_wait(q_full, (uint32_t)segs & 1u, nullptr);
      for (int s = 0; s < min(kc, kKSlots); ++s)
        ptx::mbar_wait(k_full0 + 8 * s, (uint32_t)((kc - s + kKSlots - 1) / kKSlots - 1) & 1u, nullptr);
      for (int s = 0; s < min(vc, kVSlots); ++s)
        ptx::mbar_wait(v_full0 + 8 * s, (uint32_t)((vc - s + kVSlots - 1) / kVSlots - 1) & 1u, nullptr);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (one thread)
    constexpr uint32_t idesc = tc::idesc_bf16_f32(kRows, kKT, 0, 0);    // S: Q and K both K-major, N = 128 tokens
    constexpr uint32_t idesc_pv = tc::idesc_bf16_f32(kRows, kD, 0, 1);  // O: V is N-major, N = kD channels
    constexpr uint32_t hi = tc::smem_desc_hi_sw128(1024);
    if (ptx::elect_one()) {
      bool ok = true;
      const uint32_t q_lo = tc::smem_desc_lo(q_u32, 16), k_lo = tc::smem_desc_lo(k_u32, 16);
      // 64-channel chunks of V are one half tile apart; or, where boxes bring whole rows, a tile is [16 groups of 8
      // tokens][half][8][128 B]
      const bool k_rows = kRanged && p.k_rows, v_rows = kRanged && p.v_rows;
      const uint32_t v_lo = tc::smem_desc_lo(v_u32, v_rows ? 1024 : kKT * 128);
      const uint32_t k_hi = k_rows ? tc::smem_desc_hi_sw128(2048) : hi, v_hi = v_rows ? tc::smem_desc_hi_sw128(2048) : hi;
      const uint32_t k_half = (k_rows ? 1024 : 128 * 128) >> 4, v_16 = (v_rows ? 4096 : 16 * 128) >> 4;  // 16 tokens of V
      auto issue_s = [&](int t, int qt, int slot) {  // S_t = Q_qt . K^T
        const uint32_t qa = q_lo + qt * (kQBytes >> 4), ka = k_lo + slot * (kKBytes >> 4);
        const uint32_t d = tmem_base + t * 128;
        tc::mma_ss_halves<false>(d, qa, hi, ka, k_hi, idesc);
#pragma unroll
        for (int ks = 1; ks < kDQK / 16; ++ks) {
          const uint32_t step = ((ks / 4) * (128 * 128) + (ks % 4) * 32) >> 4;
          const uint32_t k_step = (ks / 4) * k_half + (((ks % 4) * 32) >> 4);
          tc::mma_ss_halves<true>(d, qa + step, hi, ka + k_step, k_hi, idesc);
        }
        tc::commit(s_full0 + 8 * t);
      };
      auto issue_pv = [&](int t, int slot, bool first, int half) {  // O_t += P_t . V, 64 tokens at a time
        const uint32_t va = v_lo + slot * (kTBytes >> 4);
        const uint32_t d = tmem_base + 256 + t * kD, pa = kSepP ? tmem_base + 384 + t * 64 : tmem_base + t * 128;
        constexpr int kSteps = kKT / 32;
        if (half == 0) {
          if (first) tc::mma_ts_halves<false>(d, pa, va, v_hi, idesc_pv);
          else tc::mma_ts_halves<true>(d, pa, va, v_hi, idesc_pv);
#pragma unroll
          for (int k = 1; k < kSteps; ++k) tc::mma_ts_halves<true>(d, pa + k * 8, va + k * v_16, v_hi, idesc_pv);
        } else {
#pragma unroll
          for (int k = kSteps; k < 2 * kSteps; ++k)
            tc::mma_ts_halves<true>(d, pa + k * 8, va + k * v_16, v_hi, idesc_pv);
          tc::commit(o_done0 + 8 * t);
        }
      };
      // Ring positions of the next K tile to score and the next V tile to use, with the parities of their passes; the
      // parity of the next tile of either group; and the parity of the last release of O_t (none for the first use).
      int ks = 0, vs = 0, segs = 0;
      uint32_t kph = 0, vph = 0, tp0 = 0, tp1 = 0, of0 = 1, of1 = 1;
      for (;; ++segs) {
        const int slot = segs % kSegRing;
        if (!ptx::mbar_wait(seg_full0 + 8 * slot, (segs / kSegRing) & 1, abort_flag)) { ok = false; break; }
        const int flags = seg_s[slot].flags, tiles = seg_s[slot].tb - seg_s[slot].ta, n0 = seg_s[slot].nst0;
        ptx::mbar_arrive(seg_empty0 + 8 * slot);
        if (flags & kSegEnd) break;
        const bool wide = flags & kSegWide;
        const int n1 = wide ? tiles : tiles - n0, steps = wide ? tiles : n0;
        if (!ptx::mbar_wait(q_full, segs & 1, abort_flag)) { ok = false; break; }
        // step -1 scores the first tiles; step i uses tile i's weights and scores tile i + 1.  Wide: both groups take the
        // same K and V tile, the rings move on behind the second group; narrow: a tile each, in turn.
        for (int i = -1; i < steps && ok; ++i) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int n = t == 0 ? n0 : n1;
            const bool last = t == 1 || !wide;  // the ring moves on
            auto scores = [&](uint32_t tile) __attribute__((always_inline)) {  // parity of the tile whose scores they replace
              if (i + 1 < n) {
                if (!ptx::mbar_wait(k_full0 + 8 * ks, kph, abort_flag)) { ok = false; return; }
                // (kSepP) the last scores have been read; otherwise P_t lies there and has been issued to the same pipe
                if (kSepP && !ptx::mbar_wait(s_free0 + 8 * t, tile, abort_flag)) { ok = false; return; }
                tc::fence_after_sync();
                issue_s(t, wide ? t : 0, ks);
                if (last) {
                  tc::commit(k_empty0 + 8 * ks);
                  if (++ks == kKSlots) { ks = 0; kph ^= 1; }
                }
              }
            };
            if (kSepP) scores((t == 0 ? tp0 : tp1) ^ (i < 0));
            if (ok && i >= 0 && i < n) {
              if (i == 0) {  // the accumulator of the segment before has been read out
                if (!ptx::mbar_wait(o_free0 + 8 * t, t == 0 ? of0 : of1, abort_flag)) { ok = false; break; }
                if (t == 0) of0 ^= 1; else of1 ^= 1;
              }
              if (!ptx::mbar_wait(p_half0 + 8 * t, t == 0 ? tp0 : tp1, abort_flag) ||
                  !ptx::mbar_wait(v_full0 + 8 * vs, vph, abort_flag)) { ok = false; break; }
              tc::fence_after_sync();
              issue_pv(t, vs, i == 0, 0);
              if (!ptx::mbar_wait(p_full0 + 8 * t, t == 0 ? tp0 : tp1, abort_flag)) { ok = false; break; }
              tc::fence_after_sync();
              issue_pv(t, vs, i == 0, 1);
              if (t == 0) tp0 ^= 1; else tp1 ^= 1;
              if (last) {
                tc::commit(v_empty0 + 8 * vs);
                if (++vs == kVSlots) { vs = 0; vph ^= 1; }
              }
            }
            if (!kSepP && ok) scores(0);
          }
          if (ok && i + 2 == steps) tc::commit(q_empty);  // the segment's last scores have been issued
        }
        if (!ok) break;
      }
      if (!ok) report(p.dev_status, DIFFQKV_ERR_TIMEOUT);
      tc::commit(drain);
    }
    __syncwarp();
  }
  } else {
    // ------------------------------------------------------------------ softmax warps
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int t = (warp - kSoftmaxWarp0) >> 2;  // softmax group
    const int quarter = warp & 3;               // tensor-memory lanes this warp may touch
    const int r = quarter * 32 + lane;          // row
    // What a row needs next to its 128 scores has to fit 216 registers: one word for this group's barriers, one for its
    // tensor memory, a parity bit, the tile; the rest is read from the segment's words when it is wanted.
    const uint32_t gbar = s_full0 + 8 * t;
    const uint32_t s_taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + t * 128;
    const uint32_t p_taddr = kSepP ? s_taddr + 384 - t * 64 : s_taddr;
    const uint32_t o_taddr = s_taddr + 256 - t * (128 - kD);
    constexpr uint32_t kPHalf = 16, kPFull = 32, kODone = 48, kOFree = 64, kSFree = 80;  // from gbar
    uint32_t par = 0;  // parity of the next tile's barriers
    uint32_t joins = 0;  // narrow segments in which both groups had tiles
    bool ok = true;
    // first token of this group's rows within the chunk, and the rows in use
    auto tok0_of = [&](const Seg& w) { return w.tok0 + ((w.flags & kSegWide) ? t * p.T : 0); };
    auto rows_of = [&](const Seg& w) { return min(p.T, w.n - tok0_of(w)) * p.G; };
    for (uint32_t segs = 0;; ++segs) {
      const Seg& w = seg_s[segs % kSegRing];  // released at the end of the segment
      if (!wait_warp(seg_full0 + 8 * (segs % kSegRing), (segs / kSegRing) & 1, abort_flag)) { ok = false; break; }
      if (w.flags & kSegEnd) break;
      const bool wide = w.flags & kSegWide;
      const int n = t == 0 ? w.nst0 : (wide ? w.tb - w.ta : w.tb - w.ta - w.nst0);  // tiles of this group
      const bool busy = quarter * 32 < rows_of(w);                                 // some row of this warp is in use
      // tiles from here on reach past some row's position (a ragged last tile is one of them)
      int j_diag = (w.past + tok0_of(w) + 1) / kKT;
      // ranged: first token of tile j; the first token behind the sinks that the last of the group's rows sees
      auto token_of = [&](int j) -> int {
        if constexpr (kRanged) return (j >= p.sink_tiles ? j + w.skip : j) * kKT;
        else return j * kKT;
      };
      int low_last = 0;
      if constexpr (kRanged) {
        j_diag = min(w.past + tok0_of(w) + 1, w.end) / kKT;
        low_last = max(w.start, w.past + tok0_of(w) + p.T - p.window);
      }
      float m_ref = -INFINITY, l = 0.f;
      int j = w.ta + (wide ? 0 : t);
      const int j_end = j + (wide ? n : 2 * n);
      bool later = false;  // not the segment's first tile
#pragma unroll 1
      for (; j < j_end; j += wide ? 1 : 2, par ^= 1, later = true) {
        if (!wait_warp(gbar, par, abort_flag)) { ok = false; break; }
        tc::fence_after_sync();
        bool clear;
        if constexpr (kRanged) {
          const int k0 = token_of(j);
          clear = k0 + kKT > w.end || (k0 < w.low && k0 + kKT > p.sinks);
        } else {
          clear = j >= j_diag && j * kKT + kKT > w.past + w.n;
        }
        if (clear) {
          // ragged last tile: V rows past the sequence end hold whatever followed in memory; zero them before any
          // product reads the tile (0 * NaN would poison it).  Both groups may do this; they write the same zeros.  Ranged:
          // likewise tokens that no row of the item sees, whose boxes may not have been read.
          const int idx = w.v0 + j - w.ta, vslot = idx % kVSlots;
          if (!wait_warp(v_full0 + 8 * vslot, (idx / kVSlots) & 1, abort_flag)) { ok = false; break; }
          bool zero;
          if constexpr (kRanged) {
            const int token = token_of(j) + r;
            zero = token >= w.end || (token < w.low && token >= p.sinks);
          } else {
            zero = r >= w.past + w.n - j * kKT;
          }
          if (zero) {
#pragma unroll
            for (int half = 0; half < kHalves; ++half) {
              const int at = kRanged && p.v_rows ? (r / 8) * 2048 + half * 1024 + (r % 8) * 128 : half * (kKT * 128) + r * 128;
              uint4* dst = reinterpret_cast<uint4*>(v_s + vslot * kTBytes + at);
#pragma unroll
              for (int e = 0; e < 8; ++e) dst[e ^ (lane & 7)] = make_uint4(0, 0, 0, 0);  // every bank at once
            }
          }
          ptx::fence_proxy_async();
        }
        if (!busy) {  // nothing to compute, but the barriers count this warp
          if (kSepP) {
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(gbar + kSFree);
            if (later && !wait_warp(gbar + kODone, par ^ 1, abort_flag)) { ok = false; break; }
          }
          __syncwarp();
          if (lane == 0) {
            ptx::mbar_arrive(gbar + kPHalf);
            ptx::mbar_arrive(gbar + kPFull);
          }
          continue;
        }
        // ---- all 128 scores of the row into registers; row maximum of the raw scores (scale > 0 keeps the order)
        uint32_t s[128];
#pragma unroll
        for (int x = 0; x < 4; ++x) tc::ld_32x32b_x32(s_taddr + x * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[x * 32]));
        tc::wait_ld();
        if (kSepP) {  // the score columns may take the next tile's scores from here on
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(gbar + kSFree);
        }
        if constexpr (kRanged) {
          const int k0 = token_of(j);
          if (k0 / kKT >= j_diag || (k0 < low_last && k0 + kKT > p.sinks)) {
            // a word of 32 columns at a time, most of which every row of the warp sees or none does
            const int pos = w.past + tok0_of(w) + r / p.G;
            const int sees = min(pos, w.end - 1) - k0, low = max(w.start, pos + 1 - p.window) - k0, sinks = p.sinks - k0;
            auto below = [](int x) -> uint32_t { return x >= 32 ? ~0u : x <= 0 ? 0u : (1u << x) - 1; };  // columns before x
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
              const uint32_t seen = below(sees + 1 - c) & (~below(low - c) | below(sinks - c));
              if (__any_sync(0xffffffffu, seen != ~0u)) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (!(seen >> e & 1)) s[c + e] = 0xff800000u;  // -inf
              }
            }
          }
        } else if (j >= j_diag) {
          const int sees = min(w.past + tok0_of(w) + r / p.G, w.past + w.n - 1) - j * kKT;  // last column the row sees
#pragma unroll
          for (int e = 0; e < 128; ++e)
            if (e > sees) s[e] = 0xff800000u;  // -inf
        }
        float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
        for (int e = 0; e < 128; e += 8) {
          mx0 = max3(mx0, __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
          mx1 = max3(mx1, __uint_as_float(s[e + 2]), __uint_as_float(s[e + 3]));
          mx2 = max3(mx2, __uint_as_float(s[e + 4]), __uint_as_float(s[e + 5]));
          mx3 = max3(mx3, __uint_as_float(s[e + 6]), __uint_as_float(s[e + 7]));
        }
        const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * p.scale_log2;
        float alpha = 1.f;
        const bool bump = mx > m_ref + kRescaleThreshold;  // true on the first tile that the row sees (m_ref = -inf)
        if (bump) {
          alpha = exp2f(m_ref - mx);
          m_ref = mx;
        }
        if (later && __any_sync(0xffffffffu, bump)) {  // rescale this warp's rows of O in tensor memory
          if (!wait_warp(gbar + kODone, par ^ 1, abort_flag)) { ok = false; break; }
          tc::fence_after_sync();
#pragma unroll 1
          for (int x = 0; x < kD / 32; ++x) {
            uint32_t o[32];
            tc::ld_32x32b_x32(o_taddr + x * 32, o);
            tc::wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            tc::st_32x32b_x32(o_taddr + x * 32, o);
          }
          tc::wait_st();
        }
        l *= alpha;
        const float neg_m = m_ref == -INFINITY ? 0.f : -m_ref;  // a segment may begin behind a row's position
        if (kSepP && later) {  // P's own columns still hold the previous tile's P until its product is done
          if (!wait_warp(gbar + kODone, par ^ 1, abort_flag)) { ok = false; break; }
          tc::fence_after_sync();
        }
        // ---- P = 2^(S scale - m_ref) as packed bf16; fp32 row sum.  The first 64 tokens are announced on their own,
        // so that their half of the product runs during the second half's work.
        uint64_t l2 = 0;
        const uint64_t scale2 = pair(p.scale_log2, p.scale_log2), negm2 = pair(neg_m, neg_m);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          uint32_t pw[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            float x0, x1;
            unpair(fma2(pair(s[x * 64 + 2 * e], s[x * 64 + 2 * e + 1]), scale2, negm2), x0, x1);
            const float p0 = ex2(x0), p1 = ex2(x1);
            pw[e] = pack2(p0, p1);
            l2 = add2(l2, pair(p0, p1));
          }
          tc::st_32x32b_x32(p_taddr + x * 32, pw);
          if (x == 0) {
            tc::wait_st();
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(gbar + kPHalf);
          }
        }
        float l0, l1;
        unpair(l2, l0, l1);
        l += l0 + l1;
        tc::wait_st();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(gbar + kPFull);
      }
      if (!ok) break;
      // ---- the segment's result
      if (n > 0) {
        if (!wait_warp(gbar + kODone, par ^ 1, abort_flag)) { ok = false; break; }
        tc::fence_after_sync();
      }
      // a sum of zero: the row sees no token of the segment; a NaN stays one
      float weight = l != 0.f ? 1.f / l : 0.f, weight1 = 0.f, lse2 = l != 0.f ? m_ref + log2f(l) : -INFINITY;
      const bool join = !wide && w.tb - w.ta > 1;
      if (join && t == 1) {  // hand over to the first group, which reads both accumulators
        xch_s[r] = make_float2(m_ref, l);
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(x_full);
          ptx::mbar_arrive(seg_empty0 + 8 * (segs % kSegRing));
        }
        continue;
      }
      if (!wide && t == 1) {
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(seg_empty0 + 8 * (segs % kSegRing));
        continue;
      }
      if (join) {
        if (!wait_warp(x_full, joins & 1, abort_flag)) { ok = false; break; }
        ++joins;
        tc::fence_after_sync();
        const float2 o = xch_s[r];
        const float top = fmaxf(l != 0.f ? m_ref : -INFINITY, o.y != 0.f ? o.x : -INFINITY);
        const float e0 = l != 0.f ? exp2f(m_ref - top) : 0.f, e1 = o.y != 0.f ? exp2f(o.x - top) : 0.f;
        const float sum = l * e0 + o.y * e1;
        weight = sum != 0.f ? e0 / sum : 0.f;
        weight1 = sum != 0.f ? e1 / sum : 0.f;
        lse2 = sum != 0.f ? top + log2f(sum) : -INFINITY;
      }
      if (busy) {
        const bool store = r < rows_of(w);
        const bool whole = w.flags & kSegWhole;
        auto out_row = [&](int y) -> long long {  // row y of this tile in q and out
          const int tok = y / p.G;
          return (long long)(w.row_lo + tok0_of(w) + tok) * p.n_q + w.head0 + (y - tok * p.G);
        };
        const long long row = out_row(r);
        const long long prow0 = (2LL * blockIdx.x + ((w.flags & kSegFirst) ? 1 : 0)) * p.list.slot_rows + (wide ? t * p.T * p.G : 0);
        const long long prow = prow0 + r;
        if (n > 0) {
          // Four lanes exchange their rows' 16-byte pieces, so that a store covers 64 consecutive bytes of eight rows and
          // not 16 of 32 (which took 4 of the 7 thousand cycles between an item's last product and the next one's).
          const int r4 = quarter * 32 + (lane & ~3), piece = lane & 3;
          long long at[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) at[y] = (whole ? out_row(r4 + y) : prow0 + r4 + y) * kD;
          const int rows = rows_of(w);
          bool as_f32 = !whole || p.out_is_f32;
          float* dst32 = whole ? reinterpret_cast<float*>(p.out) : p.list.part_o;
          if constexpr (kRanged) {
            if (whole && w.dst != kDstOut) {
              as_f32 = true;
              dst32 = p.buffer[w.dst - 1].o;
            }
          }
          __nv_bfloat16* dst16 = reinterpret_cast<__nv_bfloat16*>(p.out);
#pragma unroll 1
          for (int x = 0; x < kD / 32; ++x) {
            uint32_t o[32], o1[32];
            tc::ld_32x32b_x32(o_taddr + x * 32, o);
            if (join) tc::ld_32x32b_x32(o_taddr + kD + x * 32, o1);
            tc::wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              float y = __uint_as_float(o[e]) * weight;
              if (join) y = fmaf(__uint_as_float(o1[e]), weight1, y);
              o[e] = __float_as_uint(y);
            }
            if (as_f32) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint4 v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int z = h * 16 + e * 4;
                  v[e] = make_uint4(o[z], o[z + 1], o[z + 2], o[z + 3]);
                }
                transpose4(v, lane);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                  if (r4 + y < rows) *reinterpret_cast<uint4*>(dst32 + at[y] + x * 32 + h * 16 + piece * 4) = v[y];
              }
            } else {
              uint4 v[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                uint32_t y[4];
#pragma unroll
                for (int z = 0; z < 4; ++z)
                  y[z] = pack2(__uint_as_float(o[8 * e + 2 * z]), __uint_as_float(o[8 * e + 2 * z + 1]));
                v[e] = make_uint4(y[0], y[1], y[2], y[3]);
              }
              transpose4(v, lane);
#pragma unroll
              for (int y = 0; y < 4; ++y)
                if (r4 + y < rows) *reinterpret_cast<uint4*>(dst16 + at[y] + x * 32 + piece * 8) = v[y];
            }
          }
        }
        if (store) {
          bool done = false;
          if constexpr (kRanged) {
            done = whole && w.dst != kDstOut;
            if (done) p.buffer[w.dst - 1].lse[row] = lse2;
          }
          if (!whole) p.list.part_lse[prow] = lse2;
          else if (!done && p.lse) p.lse[row] = lse2 * kLn2;
        }
      }
      // the accumulators may be overwritten
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        if (n > 0) ptx::mbar_arrive(gbar + kOFree);
        if (join) ptx::mbar_arrive(o_free0 + 8);
        ptx::mbar_arrive(seg_empty0 + 8 * (segs % kSegRing));
      }
    }
    if (!ok) report(p.dev_status, DIFFQKV_ERR_TIMEOUT);
  }

  // ---- teardown: all MMAs this block issued must be done before its tensor memory is released
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    ptx::mbar_wait(drain, 0, nullptr);
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem_base, kTmemCols);
  }
  ptx::grid_dependency_wait();
}

// Joins the partial rows of the items that were cut, left by the blocks of both kernels: all rows of all such items in one
// list, dealt to the groups of kD / 4 lanes (four channels each) of as many blocks as are resident at once.  Bound by the
// latency of its few dependent loads: a group takes up to four rows of an item, two at a time with four parts
// each in flight.
constexpr int kCombineThreads = 256, kCombineBlocks = 3;  // per SM

template <int kD>
__global__ void __launch_bounds__(kCombineThreads, kCombineBlocks)
extend_combine_kernel(const ExtendParams p, const ExtendList thin, const int thin_blocks, const int wide_blocks) {
  constexpr int kLanes = kD / 8, kGroups = kCombineThreads / kLanes, kItems = 2 * kMaxBlocks;
  __shared__ int start_s[kItems + 1];  // bundles of rows in the items before this one
  __shared__ uint64_t scan_s[kCombineThreads / 32];
  const int lane = threadIdx.x % kLanes;
  ptx::grid_dependency_wait();
  const int items = thin_blocks + wide_blocks;
  auto meta_of = [&](int x) { return x < thin_blocks ? thin.meta + x : p.list.meta + (x - thin_blocks); };
  // Rows go in bundles: one each while that keeps no group waiting, two (read together) up to twice as many, else four (one
  // search for all).  The three counts, at most 2^17 each, in one scan.
  static_assert(kItems == 2 * kCombineThreads, "two items a thread");
  uint64_t sum = 0;
  int rows[2];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int x = 2 * threadIdx.x + y;
    rows[y] = x < items ? meta_of(x)->rows : 0;
    sum += (uint64_t)rows[y] | (uint64_t)((rows[y] + 1) >> 1) << 21 | (uint64_t)((rows[y] + 3) >> 2) << 42;
  }
  const uint64_t mine = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t y = __shfl_up_sync(0xffffffffu, sum, o);
    if ((int)(threadIdx.x % 32) >= o) sum += y;
  }
  if (threadIdx.x % 32 == 31) scan_s[threadIdx.x / 32] = sum;
  __syncthreads();
  uint64_t total = 0;
  sum -= mine;
#pragma unroll
  for (int w = 0; w < kCombineThreads / 32; ++w) {
    if (w < (int)threadIdx.x / 32) sum += scan_s[w];
    total += scan_s[w];
  }
  const int all = (int)total & 0x1fffff, at_once = (int)gridDim.x * kGroups;
  const int log = all > 2 * at_once ? 2 : all > at_once ? 1 : 0, bundle = 1 << log;
  auto count = [&](uint64_t x) {
    const int c0 = (int)x & 0x1fffff, c1 = (int)(x >> 21) & 0x1fffff, c2 = (int)(x >> 42);
    return log == 0 ? c0 : log == 1 ? c1 : c2;
  };
  const int mine0 = count(sum);
  start_s[2 * threadIdx.x] = mine0;
  start_s[2 * threadIdx.x + 1] = mine0 + ((rows[0] + bundle - 1) >> log);
  if (threadIdx.x == 0) start_s[kItems] = count(total);
  __syncthreads();
  const int bundles = start_s[kItems];
  for (int g = blockIdx.x * kGroups + threadIdx.x / kLanes; g < bundles; g += gridDim.x * kGroups) {
    int x = 0, z = kItems;  // the item: the last that begins at or before bundle g
    while (z - x > 1) {
      const int mid = (x + z) >> 1;
      if (start_s[mid] <= g) x = mid; else z = mid;
    }
    const bool first_list = x < thin_blocks;
    const ExtendList& list = first_list ? thin : p.list;
    const ExtendMeta m = *meta_of(x);
    // the parts lie one team apart, the first in its block's second slot, the others in the first: in order, so that sums
    // do not depend on timing.  A slot's number, and any row's, fits 32 bits: 2 kMaxBlocks slots of at most 2 kRows rows.
    const uint32_t slot0 = 2 * (first_list ? x : x - thin_blocks), step = 2 * list.team * list.slot_rows;
    const int r0 = bundle * (g - start_s[x]), end = min(r0 + bundle, m.rows);
    int part = r0 / m.part_rows, lr = r0 - part * m.part_rows, tok = lr / p.G, head = lr - tok * p.G;
#pragma unroll 1
    for (int r = r0; r < end; r += 2) {  // two rows at a time
      const int second = r + 1 < end;
      const uint32_t at1 = slot0 * list.slot_rows + r, at0 = at1 + list.slot_rows;  // first part's, and before the others'
      float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
      float4 acc[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) acc[h][0] = acc[h][1] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
      for (int i = 0; i < m.parts; i += 2) {
        float ls[2][2];
        float4 o[2][2][2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          ls[y][0] = ls[y][1] = -INFINITY;
          if (i + y < m.parts) {
            const uint32_t at = i + y == 0 ? at0 : at1 + (i + y) * step;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t row = at + (h == 0 ? 0 : second);
              ls[y][h] = list.part_lse[row];
              const float4* src = reinterpret_cast<const float4*>(list.part_o + (size_t)row * kD) + lane * 2;
              o[y][h][0] = src[0];
              o[y][h][1] = src[1];
            }
          }
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (ls[y][h] == -INFINITY) continue;  // the part saw no token of this row (and may have left no values)
            const float up = fmaxf(top[h], ls[y][h]);
            const float was = ex2(top[h] - up), f = ex2(ls[y][h] - up);
            top[h] = up;
            sum[h] = fmaf(sum[h], was, f);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              acc[h][e].x = fmaf(f, o[y][h][e].x, acc[h][e].x * was);
              acc[h][e].y = fmaf(f, o[y][h][e].y, acc[h][e].y * was);
              acc[h][e].z = fmaf(f, o[y][h][e].z, acc[h][e].z * was);
              acc[h][e].w = fmaf(f, o[y][h][e].w, acc[h][e].w * was);
            }
          }
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (h == 1 && !second) break;
        const float inv = sum[h] != 0.f ? 1.f / sum[h] : 0.f;
        const long long row = (long long)(m.row_lo + tok) * p.n_q + m.head0 + part * p.G + head;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          acc[h][e].x *= inv;
          acc[h][e].y *= inv;
          acc[h][e].z *= inv;
          acc[h][e].w *= inv;
        }
        if (p.out_is_f32) {
          float4* dst = reinterpret_cast<float4*>(reinterpret_cast<float*>(p.out) + row * kD) + lane * 2;
          dst[0] = acc[h][0];
          dst[1] = acc[h][1];
        } else {
          reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) + row * kD)[lane] =
              make_uint4(pack2(acc[h][0].x, acc[h][0].y), pack2(acc[h][0].z, acc[h][0].w), pack2(acc[h][1].x, acc[h][1].y),
                         pack2(acc[h][1].z, acc[h][1].w));
        }
        if (p.lse && lane == 0) p.lse[row] = sum[h] != 0.f ? (top[h] + log2f(sum[h])) * kLn2 : -INFINITY;
        if (++head == p.G) {
          head = 0;
          ++tok;
        }
        if (++lr == m.part_rows) {  // the next head group of the item
          lr = tok = head = 0;
          ++part;
        }
      }
    }
  }
}

// The rows of a step with groups: a row's result is joined from the parts of its two items, that of its group's prefix and
// that of its own tokens, whole or cut, in their order (out = sum of 2^lse o / sum of 2^lse).  Rows of sequences without a
// prefix whose item is whole have their result already; those that do not fit are not touched.  A block first finds the items
// of its rows, while the two kernels before still run, and reads where these items' parts are; then kD / 8 lanes take a head,
// eight channels each, row after row, so that a row's parts are one read (of four at a time).
constexpr int kMergeThreads = 256, kMergeBlocks = 3;  // per SM
constexpr int kMergeRows = 16, kMergeRefs = 512;      // of a block, at most; row's units whose items fit shared memory

template <int kD>
__global__ void __launch_bounds__(kMergeThreads, kMergeBlocks)
extend_merge_kernel(const ExtendParams p, const ExtendList few, const int rows_each) {
  constexpr int kLanes = kD / 8, kHeads = kMergeThreads / kLanes;
  struct Row {
    int has;       // 0: nothing to do here, 1: own tokens alone, 2: a prefix too
    int first[2];  // first row of the item of either kind
    int rows[2];   // of a head group, of an item of a few rows; 0: of long chunks
  };
  __shared__ Row row_s[2][kMergeRows];  // of a step with long chunks and of one whose rows are all few
  __shared__ ItemRef ref_s[kMergeRefs][2];
  const int t0 = blockIdx.x * rows_each, count = min(rows_each, p.total_q - t0);
  {
    for (int r = 0; r < count;) {  // a sequence at a time, all its rows here at once
      int lo, n, past, g_lo = 0, g_hi = 0;
      const int t = t0 + r;
      const int b = ragged_sequence_of<kMergeThreads>(p.cu_q, p.seqlens, p.batch, p.total_q, p.max_seqlen, t, false,
                                                      p.dev_status, lo, n, past, [] {});
      const int prefix = b < 0 ? -1 : group_prefix(p, b, lo, n, past, g_lo, g_hi), here = b < 0 ? 1 : min(count - r, lo + n - t);
      for (int x = threadIdx.x; x < 2 * here; x += kMergeThreads) {
        const int y = r + (x >> 1), k = x & 1, first = k == 0 ? g_lo : lo, rows = k == 0 ? g_hi - g_lo : n, in = t0 + y - first;
        const bool wide = rows > p.thin_max;
        row_s[0][y].has = row_s[1][y].has = prefix < 0 ? 0 : prefix == 0 ? 1 : 2;
        row_s[0][y].first[k] = row_s[1][y].first[k] = first;
        row_s[0][y].rows[k] = row_s[1][y].rows[k] = rows * p.G;
        if (wide) {  // see SeqOf
          const int blocks = few_blocks(p, rows), each = (rows + blocks - 1) / blocks;
          row_s[0][y].first[k] += in / (2 * p.T) * (2 * p.T);
          row_s[0][y].rows[k] = 0;
          row_s[1][y].first[k] += in / each * each;
          row_s[1][y].rows[k] = min(each, rows - in / each * each) * p.G;
        }
      }
      r += here;
    }
  }
  __syncthreads();
  ptx::grid_dependency_wait();
  const ItemRef step = p.refs[2LL * p.total_q * p.n_units];
  if (step.first) return;  // left out
  const Row* rows_s = row_s[step.parts != 0];
  auto ref_of = [&](int r, int unit, int k) -> ItemRef {
    const Row& w = rows_s[r];
    if (w.has < (k == 0 ? 2 : 1)) return {0, 0};
    ItemRef x = p.refs[((size_t)k * p.total_q + w.first[k]) * p.n_units + unit];
    const int most = w.rows[k] == 0 ? p.n_teams : p.blocks;
    if (w.rows[k] == 0) x.parts = -x.parts;
    // never read outside of the workspace: what a block that gave up did not leave is passed over
    if (x.first < 0 || x.first >= most || x.parts < 0 || x.parts > most - x.first) x.parts = 0;
    return x;
  };
  const bool cached = count * p.n_units <= kMergeRefs;
  if (cached) {
    for (int x = threadIdx.x; x < 2 * count * p.n_units; x += kMergeThreads)
      ref_s[x >> 1][x & 1] = ref_of((x >> 1) / p.n_units, (x >> 1) % p.n_units, x & 1);
    __syncthreads();
  }
  const int lane = threadIdx.x % kLanes;
  for (int h = blockIdx.y * kHeads + threadIdx.x / kLanes; h < p.n_q; h += gridDim.y * kHeads) {
    const int group = h / p.G, unit = group / p.parts, member = group - unit * p.parts, head = h - group * p.G;
    for (int r = 0; r < count; ++r) {
      const Row& w = rows_s[r];
      const ItemRef ref0 = cached ? ref_s[r * p.n_units + unit][0] : ref_of(r, unit, 0);
      const ItemRef ref1 = cached ? ref_s[r * p.n_units + unit][1] : ref_of(r, unit, 1);
      const int total = ref0.parts + ref1.parts;
      if (w.has == 0 || (w.has == 1 && total <= 1)) continue;  // nothing to join
      const size_t row = (size_t)(t0 + r) * p.n_q + h;
      float top = -INFINITY, sum = 0.f;
      float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 1
      for (int x0 = 0; x0 < total; x0 += 4) {
        float ls[4];
        float4 v[4][2];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          ls[x] = -INFINITY;
          if (x0 + x < total) {
            const int k = x0 + x >= ref0.parts, part = k ? x0 + x - ref0.parts : x0 + x;
            const ItemRef ref = k ? ref1 : ref0;
            const float* lse = p.buffer[k].lse;
            const float* o = p.buffer[k].o;
            size_t at = row;
            if (ref.parts > 1) {  // the first part lies in its block's second slot, the others in the first
              const bool wide = w.rows[k] == 0;
              const ExtendList& list = wide ? p.list : few;
              const int block = (ref.first + part) * list.team + (wide ? member : 0);
              at = (size_t)(2 * block + (part == 0)) * list.slot_rows + ((t0 + r - w.first[k]) * p.G + head + member * w.rows[k]);
              lse = list.part_lse;
              o = list.part_o;
            }
            ls[x] = lse[at];
            const float4* from = reinterpret_cast<const float4*>(o + at * kD) + 2 * lane;
            v[x][0] = from[0];
            v[x][1] = from[1];
          }
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (ls[x] == -INFINITY) continue;  // the part saw no token of this row (and may have left no values)
          const float up = fmaxf(top, ls[x]), was = ex2(top - up), f = ex2(ls[x] - up);
          top = up;
          sum = fmaf(sum, was, f);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            acc[e].x = fmaf(f, v[x][e].x, acc[e].x * was);
            acc[e].y = fmaf(f, v[x][e].y, acc[e].y * was);
            acc[e].z = fmaf(f, v[x][e].z, acc[e].z * was);
            acc[e].w = fmaf(f, v[x][e].w, acc[e].w * was);
          }
        }
      }
      const float inv = sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        acc[e].x *= inv;
        acc[e].y *= inv;
        acc[e].z *= inv;
        acc[e].w *= inv;
      }
      if (p.out_is_f32) {
        float4* dst = reinterpret_cast<float4*>(reinterpret_cast<float*>(p.out) + row * kD) + 2 * lane;
        dst[0] = acc[0];
        dst[1] = acc[1];
      } else {
        reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) + row * kD)[lane] =
            make_uint4(pack2(acc[0].x, acc[0].y), pack2(acc[0].z, acc[0].w), pack2(acc[1].x, acc[1].y), pack2(acc[1].z, acc[1].w));
      }
      if (p.lse && lane == 0) p.lse[row] = sum != 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
    }
  }
}

// Lengths for the kernels that know no groups: -1, which they skip and report, where a sequence does not fit its group.
__global__ void extend_lengths_kernel(const ExtendParams p, int* seqlens) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= p.batch) return;
  int lo, n, past;
  int g_lo, g_hi;
  const bool fits = load_rows(p, b, lo, n, past) && (n == 0 || group_prefix(p, b, lo, n, past, g_lo, g_hi) >= 0);
  seqlens[b] = fits ? past : -1;
}

// Tensor map over one cache pool: dims (64 channels, token slot, channel half, head, block); a box brings box_tok tokens
// of one 64-channel half.
bool make_cache_map(CUtensorMap* map, const void* base, int d, long long tok_extent, int heads, long long blocks,
                    long long st_tok, long long st_head, long long st_blk, int box_tok) {
  const cuuint64_t dims[5] = {64, (cuuint64_t)tok_extent, (cuuint64_t)(d / 64), (cuuint64_t)heads, (cuuint64_t)blocks};
  const cuuint64_t strides[4] = {(cuuint64_t)st_tok * 2, 128, (cuuint64_t)st_head * 2, (cuuint64_t)st_blk * 2};
  const cuuint32_t box[5] = {64, (cuuint32_t)box_tok, 1, 1, 1};
  return make_tmap_bf16_sw128(map, base, 5, dims, strides, box);
}

// The same with boxes of whole rows: [channel half][box_tok tokens][64 channels].
bool make_pool_map(CUtensorMap* map, const void* base, int d, long long tok_extent, int heads, long long blocks,
                   long long st_tok, long long st_head, long long st_blk, int box_tok) {
  const cuuint64_t dims[5] = {64, (cuuint64_t)tok_extent, (cuuint64_t)(d / 64), (cuuint64_t)heads, (cuuint64_t)blocks};
  const cuuint64_t strides[4] = {(cuuint64_t)st_tok * 2, 128, (cuuint64_t)st_head * 2, (cuuint64_t)st_blk * 2};
  const cuuint32_t box[5] = {64, (cuuint32_t)box_tok, (cuuint32_t)(d / 64), 1, 1};
  return make_tmap_bf16_sw128(map, base, 5, dims, strides, box);
}

// The same for a pool whose heads lie behind one another in a block (stride_head = tokens * stride_tok) and whose rows
// have 128 channels: dims (64 channels, 8 tokens, channel half, group of 8 tokens of any head, block), so that one box
// brings whole rows, half as many boxes per tile (16-token pages were bound by the rate of boxes: 242 -> 190 us for 16
// sequences of 4k-32k tokens, 5 new rows each, 32/4/8 heads).
bool make_row_map(CUtensorMap* map, const void* base, int d, long long tok_extent, int heads, long long blocks,
                  long long st_tok, long long st_head, long long st_blk, int box_tok) {
  if (d != 128 || tok_extent % 8 != 0 || (heads > 1 && st_head != tok_extent * st_tok)) return false;
  const long long groups = tok_extent / 8 * heads;
  if (groups > 0x7fffffffLL) return false;
  const cuuint64_t dims[5] = {64, 8, 2, (cuuint64_t)groups, (cuuint64_t)blocks};
  const cuuint64_t strides[4] = {(cuuint64_t)st_tok * 2, 128, (cuuint64_t)st_tok * 16, (cuuint64_t)st_blk * 2};
  const cuuint32_t box[5] = {64, 8, 2, (cuuint32_t)(box_tok / 8), 1};
  return make_tmap_bf16_sw128(map, base, 5, dims, strides, box);
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  int G, T, groups, parts, region, thin_max;
  int blocks;              // of the thin kernel
  int n_teams;             // of the other one, parts blocks each
  int slot_rows, thin_rows;
};

int sm_count() {
  static std::atomic<int> cached{0};
  int n = cached.load();
  if (n == 0) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        n <= 0)
      n = 148;  // without a device (workspace sizes are asked on the host)
    else
      cached = n;
  }
  return n < kMaxBlocks ? n : kMaxBlocks;
}

// Head groups, rows per tile and teams; the same for the workspace's size and the launch.
Plan make_plan(const diffqkv_shape& s, int total_q, bool ranged) {
  Plan pl;
  const int columns = ranged ? kFewCols : kThinCols;
  const int per_k = s.n_q / s.n_k, per_v = s.n_q / s.n_v;
  int G = std::gcd(per_k, per_v);
  const bool nested = G == per_k || G == per_v;  // one kind of head groups lies within the other
  if (G > kRows) {  // the largest divisor that fits a tile
    int d = kRows;
    while (G % d != 0) --d;
    G = d;
  }
  pl.G = G;
  pl.T = kRows / G;
  pl.groups = s.n_q / G;
  // groups of one K head (V head) that differ in the other head only sit next to each other: a unit of at most four
  const int share = nested ? (per_k > per_v ? per_k : per_v) / G : 1;
  int parts = share < 4 ? share : 4;
  while (share % parts != 0 || pl.groups % parts != 0) --parts;
  pl.parts = parts;
  pl.region = parts == 1 ? columns : (parts == 2 ? columns / 2 : columns / 4);
  pl.thin_max = pl.region / G;
  pl.blocks = sm_count();
  pl.n_teams = pl.blocks / parts;
  const long long rows = 2LL * pl.T * G, asked = (long long)total_q * G, thin = (long long)pl.thin_max * G;
  pl.slot_rows = (int)(asked < rows ? asked : rows);
  pl.thin_rows = (int)(asked < thin ? asked : thin) * parts;
  return pl;
}

// Parts of the workspace; with a base their addresses.
size_t place(const Plan& pl, int d_v, char* base, ExtendList* wide, ExtendList* thin) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += up256(bytes);
    return base ? base + was : nullptr;
  };
  const int rows[2] = {pl.slot_rows, pl.thin_rows}, blocks[2] = {pl.n_teams * pl.parts, pl.blocks};
  ExtendList* lists[2] = {wide, thin};
  for (int i = 0; i < 2; ++i) {
    ExtendList l = {};
    l.meta = reinterpret_cast<ExtendMeta*>(take(sizeof(ExtendMeta) * kMaxBlocks));
    l.part_lse = reinterpret_cast<float*>(take(2 * sizeof(float) * (size_t)blocks[i] * rows[i]));
    l.part_o = reinterpret_cast<float*>(take(2 * sizeof(float) * (size_t)blocks[i] * rows[i] * d_v));
    l.slot_rows = rows[i];
    l.team = i == 0 ? pl.parts : 1;
    if (lists[i]) *lists[i] = l;
  }
  return at;
}

// Behind them, for a step with groups, the rows' two parts and where those are that were cut.
size_t place_buffers(const diffqkv_shape& s, const Plan& pl, int total_q, char* base, ExtendParams* p) {
  const size_t rows = (size_t)total_q * s.n_q;
  const size_t lse = up256(rows * sizeof(float)), o = up256(rows * s.d_v * sizeof(float));
  for (int i = 0; i < 2 && p; ++i) {
    p->buffer[i].lse = reinterpret_cast<float*>(base + i * (lse + o));
    p->buffer[i].o = reinterpret_cast<float*>(base + i * (lse + o) + lse);
  }
  if (p) p->refs = reinterpret_cast<ItemRef*>(base + 2 * (lse + o));
  return 2 * (lse + o) + up256(sizeof(ItemRef) * (2 * (size_t)total_q * (pl.groups / pl.parts) + 1));
}

bool dims_supported(const diffqkv_shape& s) {
  if (s.dtype != DIFFQKV_BF16 || !(s.scale > 0.f)) return false;
  return (s.d_qk == 128 && s.d_v == 128) || (s.d_qk == 64 && s.d_v == 64) || (s.d_qk == 64 && s.d_v == 128);
}

}  // namespace

size_t extend_workspace_bytes(const diffqkv_shape& s, int total_q, bool ranged) {
  const size_t simt = extend_simt_workspace_bytes(s, total_q);  // a cache may turn out to have no tensor map
  const size_t need = dims_supported(s) ? place(make_plan(s, total_q, ranged), s.d_v, nullptr, nullptr, nullptr) : 256;
  return need > simt ? need : simt;
}

size_t extend_groups_workspace_bytes(const diffqkv_shape& s, int total_q) {
  const size_t lengths = up256(sizeof(int) * (size_t)s.batch);  // see launch_extend_lengths
  const size_t need = dims_supported(s) ? place_buffers(s, make_plan(s, total_q, true), total_q, nullptr, nullptr) : 0;
  return need > lengths ? need : lengths;
}

cudaError_t launch_extend_lengths(const int* cu_q, int total_q, const diffqkv_cache& c, int batch, const ExtendRange& range,
                                  int* seqlens, cudaStream_t stream) {
  ExtendParams p = {};
  p.cu_q = cu_q; p.seqlens = c.seqlens; p.max_seqlen = c.max_seqlen;
  p.batch = batch; p.total_q = total_q;
  p.groups = range.groups; p.cu_groups = range.cu_groups; p.prefix_lens = range.prefix_lens; p.share = 2;
  extend_lengths_kernel<<<(unsigned)((batch + 127) / 128), 128, 0, stream>>>(p, seqlens);
  count_launch();
  return cudaGetLastError();
}

// cudaErrorNotSupported, with nothing launched, where the plain kernel has to take the call.
cudaError_t launch_extend(const void* q, const int* cu_q, int total_q, const diffqkv_cache& c, const diffqkv_shape& s,
                          const ExtendRange* range, void* workspace, void* out, float* lse, int* dev_status,
                          cudaStream_t stream) {
  if (!dims_supported(s) || c.max_seqlen < 1 || c.max_seqlen > 0x7ffffe00 || c.num_blocks < 1) return cudaErrorNotSupported;
  int box_tok = kKT;
  if (c.page_table) {
    if (c.page_size >= kKT) {
      if (c.page_size % kKT != 0) return cudaErrorNotSupported;
    } else {
      if (c.page_size < 8 || kKT % c.page_size != 0) return cudaErrorNotSupported;
      box_tok = c.page_size;
    }
  }
  Plan pl = make_plan(s, total_q, range != nullptr);
  // A window that hides nothing of the longest sequence: long chunks are the plain kernels' (1.5k-2k rows of 64-channel heads
  // 473, not 529 us; of 128 channels 540, not 510; two of 240 rows 39, not 42), few rows stay here (16 single rows behind 32k
  // tokens 247, not 269 us; 64 behind 1k-4k 95, not 120; four of 60 rows 19, not 31).
  const bool hides = range && (long long)range->window + range->sinks < c.max_seqlen;
  if (range && range->groups == 0 && !hides && total_q > (long long)s.batch * (kMidBlocks / 2) * pl.thin_max) {
    range = nullptr;
    pl = make_plan(s, total_q, false);
  }
  if (range) {  // both lists in 32 bits; see ranged_start
    const long long entries = (long long)range->groups + s.batch, units = pl.groups / pl.parts;
    const long long items = total_q / (2 * pl.T) * (range->groups > 0 ? 2LL : 1LL) + entries;
    if (items * units * (kRangedItemCost + kWideCost * (c.max_seqlen / kKT + 2LL)) > 0x7fffffffLL ||
        entries * units * (kFewItemCost + kFewMostCost * (c.max_seqlen / kFewT + 2LL)) > 0x7fffffffLL)
      return cudaErrorNotSupported;
  }
  CUtensorMap mq, mq_thin, mk, mv;
  {
    const cuuint64_t dims[4] = {64, (cuuint64_t)s.n_q, (cuuint64_t)total_q, (cuuint64_t)(s.d_qk / 64)};
    const cuuint64_t strides[3] = {(cuuint64_t)s.d_qk * 2, (cuuint64_t)s.n_q * s.d_qk * 2, 128};
    const cuuint32_t box[4] = {64, (cuuint32_t)pl.G, (cuuint32_t)pl.T, 1};
    const cuuint32_t thin[4] = {64, (cuuint32_t)pl.G, (cuuint32_t)pl.thin_max, 1};
    if (!make_tmap_bf16_sw128(&mq, q, 4, dims, strides, box)) return cudaErrorNotSupported;
    if (!range && pl.thin_max > 0 && !make_tmap_bf16_sw128(&mq_thin, q, 4, dims, strides, thin)) return cudaErrorNotSupported;
  }
  const long long tok_extent = c.page_table ? c.page_size : c.max_seqlen;
  auto cache_maps = [&]() -> bool {
    return make_cache_map(&mk, c.k_cache, s.d_qk, tok_extent, s.n_k, c.num_blocks, c.k_stride_tok, c.k_stride_head,
                          c.k_stride_blk, box_tok) &&
           make_cache_map(&mv, c.v_cache, s.d_v, tok_extent, s.n_v, c.num_blocks, c.v_stride_tok, c.v_stride_head,
                          c.v_stride_blk, box_tok);
  };
  if (!range && !cache_maps()) return cudaErrorNotSupported;
  CUtensorMap mk_few, mv_few;
  if (range && (!make_pool_map(&mk_few, c.k_cache, s.d_qk, tok_extent, s.n_k, c.num_blocks, c.k_stride_tok, c.k_stride_head,
                               c.k_stride_blk, box_tok < kFewT ? box_tok : kFewT) ||
                !make_pool_map(&mv_few, c.v_cache, s.d_v, tok_extent, s.n_v, c.num_blocks, c.v_stride_tok, c.v_stride_head,
                               c.v_stride_blk, box_tok < kFewT ? box_tok : kFewT)))
    return cudaErrorNotSupported;

  ExtendParams p = {};
  p.cu_q = cu_q; p.seqlens = c.seqlens; p.page_table = c.page_table;
  p.page_size = c.page_size; p.max_pages_per_seq = c.max_pages_per_seq; p.num_blocks = c.num_blocks; p.max_seqlen = c.max_seqlen;
  p.batch = s.batch; p.total_q = total_q; p.n_q = s.n_q;
  p.G = pl.G; p.T = pl.T; p.t_log2 = -1;
  for (int x = 0; x <= 7; ++x)
    if (pl.T == 1 << x) p.t_log2 = x;
  p.parts = pl.parts; p.n_units = pl.groups / pl.parts;
  p.thin_max = pl.thin_max; p.region = pl.region;
  p.blocks = pl.blocks; p.n_teams = pl.n_teams; p.team = pl.parts;
  p.heads_per_k = s.n_q / s.n_k; p.heads_per_v = s.n_q / s.n_v;
  p.k_parts = p.heads_per_k < p.heads_per_v ? pl.parts : 1;
  p.v_parts = p.heads_per_v < p.heads_per_k ? pl.parts : 1;
  p.thin_weight = 0.3f + 0.48f * (p.k_parts + p.v_parts);
  {  // 160 KB of tiles: K of two token tiles where there is room, the rest V; an even number where V tiles go in pairs
    const int slots = kRingBytes / (kKT * 2 * (s.d_qk > s.d_v ? s.d_qk : s.d_v));
    p.k_ring = 2 * p.k_parts < slots - p.v_parts ? 2 * p.k_parts : slots - p.v_parts;
    p.v_ring = slots - p.k_ring;
    if (s.d_v == 64 && p.v_parts % 2 == 0) p.v_ring &= ~1;
  }
  p.box_tok = box_tok;
  p.scale_log2 = s.scale * kLog2e;
  p.out = out; p.out_is_f32 = s.out_dtype == DIFFQKV_F32; p.lse = lse; p.dev_status = dev_status;
  ExtendList wide, thin;
  place(pl, s.d_v, static_cast<char*>(workspace), &wide, &thin);
  if (range) {
    // A tile of a few rows takes as long as its bytes, 1.85 thousand cycles for 48 KB, or as its products: about 2.2 thousand
    // cycles for four groups of 16 rows and 128 channels of either kind, that is four or five units, half of that for two
    // groups and twice for eight.
    const long long bytes = kFewT * 2LL * (p.k_parts * s.d_qk + p.v_parts * s.d_v);
    const int memory = (int)((4 * bytes + 24576) / 49152), products[3] = {2, 5, 10}, d = s.d_qk + s.d_v;
    for (int i = 0; i < 3; ++i)
      p.few_cost[i] = std::min(std::max(std::max(memory, (products[i] * d + 128) / 256), 1), kFewMostCost);
    p.thin_weight *= 0.42f / p.few_cost[0];  // tiles of half the tokens, in these units; the best of five for two mixtures
    p.mid_most = std::min(kMidMost * pl.blocks, kMidLong - 1);
    p.window = hides ? range->window : kNoWindow;  // window and sinks together stay within 32 bits
    p.sinks = hides ? range->sinks : 0;
    p.sink_tiles = (p.sinks + kKT - 1) / kKT;
    p.sink_few = (p.sinks + kFewT - 1) / kFewT;
    p.groups = range->groups; p.entries = range->groups + s.batch;
    p.cu_groups = range->cu_groups; p.prefix_lens = range->prefix_lens; p.share = range->share;
    if (p.groups > 0) place_buffers(s, pl, total_q, static_cast<char*>(workspace) + extend_workspace_bytes(s, total_q, true), &p);
  }
  const int thin_blocks = pl.thin_max > 0 ? pl.blocks : 0, blocks = pl.n_teams * pl.parts;

  // Which sequences are thin is known on the device alone, so both kernels are launched; the second may start as soon as
  // the first has, and takes the SMs that the first leaves (an SM has room for one block of either).  First comes the one
  // that has the more work if the rows are spread evenly: behind the other it starts on SMs in another order, away from
  // its team (prompts 447 instead of 434 us), and a step of thin sequences would wait for two launches (198, not 190 us).
  using ExtendFn = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const ExtendParams);
  const int dims = s.d_v == 64 ? 0 : s.d_qk == 128 ? 1 : 2;
  constexpr ExtendFn fns[2][3] = {
      {extend_attn_kernel<64, 64, false>, extend_attn_kernel<128, 128, false>, extend_attn_kernel<64, 128, false>},
      {extend_attn_kernel<64, 64, true>, extend_attn_kernel<128, 128, true>, extend_attn_kernel<64, 128, true>}};
  const ExtendFn fn = fns[range != nullptr][dims];
  cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kExtendSmem);
  if (err != cudaSuccess) return err;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  // Prefixes shared by many rows are long chunks: ranged steps with groups begin with these, whose start would otherwise
  // fall into the other kernel's stream of tiles (64 single rows behind 16k tokens: 111 -> 100 us).
  p.alone = range && total_q <= pl.thin_max;
  const bool wide_first = !p.alone && (thin_blocks == 0 || total_q > (long long)s.batch * pl.thin_max || (range && range->groups > 0));
  CUtensorMap mk_rows, mv_rows;  // of whole rows, for the kernels that take them
  p.head_groups = (int)(tok_extent / 8);
  p.k_rows = make_row_map(&mk_rows, c.k_cache, s.d_qk, tok_extent, s.n_k, c.num_blocks, c.k_stride_tok, c.k_stride_head,
                          c.k_stride_blk, box_tok);
  p.v_rows = make_row_map(&mv_rows, c.v_cache, s.d_v, tok_extent, s.n_v, c.num_blocks, c.v_stride_tok, c.v_stride_head,
                          c.v_stride_blk, box_tok);
  if (range && (!p.k_rows || !p.v_rows) && !cache_maps()) return cudaErrorNotSupported;
  auto launch_wide = [&]() -> cudaError_t {
    p.list = wide;
    p.first = wide_first;
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kExtendThreads);
    cfg.dynamicSmemBytes = kExtendSmem;
    cfg.numAttrs = wide_first && !range ? 0 : 1;
    const cudaError_t e = range ? cudaLaunchKernelEx(&cfg, fn, mq, p.k_rows ? mk_rows : mk, p.v_rows ? mv_rows : mv, p)
                                : cudaLaunchKernelEx(&cfg, fn, mq, mk, mv, p);
    if (e == cudaSuccess) count_launch();
    return e;
  };
  auto launch_thin = [&]() -> cudaError_t {
    if (thin_blocks == 0) return cudaSuccess;
    p.list = thin;
    p.first = !wide_first;
    if (range) return launch_extend_few(mk_few, mv_few, q, p, s.d_qk, s.d_v, thin_blocks, stream);
    return launch_extend_thin(mq_thin, p.k_rows ? mk_rows : mk, p.v_rows ? mv_rows : mv, p, s.d_qk, s.d_v, thin_blocks,
                              wide_first, stream);
  };
  if (p.alone) {
    if ((err = launch_thin()) != cudaSuccess) return err;
  } else {
    if ((err = wide_first ? launch_wide() : launch_thin()) != cudaSuccess) return err;
    if ((err = wide_first ? launch_thin() : launch_wide()) != cudaSuccess) return err;
  }
  p.list = wide;
  cfg.dynamicSmemBytes = 0;
  cfg.numAttrs = 1;
  if (p.groups > 0) {
    const int heads = kMergeThreads / (s.d_v / 8), across = (s.n_q + heads - 1) / heads, resident = kMergeBlocks * sm_count();
    int rows_each = (int)(((long long)total_q * across + resident - 1) / resident);
    if (rows_each > kMergeRows) rows_each = kMergeRows;
    cfg.gridDim = dim3((unsigned)((total_q + rows_each - 1) / rows_each), (unsigned)across);
    cfg.blockDim = dim3(kMergeThreads);
    err = cudaLaunchKernelEx(&cfg, s.d_v == 64 ? extend_merge_kernel<64> : extend_merge_kernel<128>, p, thin, rows_each);
  } else {
    const long long groups = kCombineThreads / (s.d_v / 8), rows = (long long)total_q * s.n_q, fill = sm_count() * kCombineBlocks;
    cfg.gridDim = dim3((unsigned)((rows + groups - 1) / groups < fill ? (rows + groups - 1) / groups : fill));
    cfg.blockDim = dim3(kCombineThreads);
    err = cudaLaunchKernelEx(&cfg, s.d_v == 64 ? extend_combine_kernel<64> : extend_combine_kernel<128>, p, thin, thin_blocks,
                             p.alone ? 0 : blocks);
  }
  if (err != cudaSuccess) return err;
  count_launch();
  return cudaGetLastError();
}

}  // namespace diffqkv
