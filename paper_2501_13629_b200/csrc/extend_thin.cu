// Chunk attention for sequences with a few new rows (decode, verification of guessed tokens): the thin half of
// diffqkv_extend; extend.cu has the mathematics and takes the longer chunks.
//
// A row tile of 128 matrix rows is nearly empty here, and the softmax of a nearly empty tile still takes 128 scores per
// row and thread.  So the products are transposed: the 128 cached tokens of a tile are the matrix rows,
//     S^T[token][column] = K q^T          (128 x N x d_qk)      column = (head group, row of the chunk, head of the group)
//     O^T[channel][column] += V^T P^T     (d_v x N x 128)
// with N <= 64 columns for all the query heads that share a K head (or a V head), so that K and V pass through an SM
// once for all of them, and the work of the softmax is proportional to the columns in use: one thread per token, N
// exponentials each, row sums kept per thread until the end of the segment.  P^T goes to the tensor core through shared
// memory (its B operand), 128 bytes per token, channels of V straight from their token-major tile (M-major A operand).
//
// The reference of a column (what its scores are taken from before the exponential) has to be one for all four warps of
// a softmax group, whose tokens meet in one accumulator.  It starts as the score of the segment's first token, which
// needs no search, and is raised to a tile's maximum when some score exceeds it by 2^24; the warps agree on that
// through one hardware barrier per tile.  That first score may be any number, or -inf, which counts as the lowest
// number: a raised column is formed from its scores again, not from distances to a reference far below.  Weights of up
// to 2^24 are harmless: bf16 and fp32 have the range, the relative precision of either does not depend on the magnitude,
// and the quotient takes the factor out again.
//
// Work: one flat list of (sequence, unit of heads, 128-token tile), divided evenly over one persistent block per SM (or
// over those that a step's long chunks leave), whose two softmax groups take alternate tiles and are joined at the end of a
// segment; cut items leave partial rows as in extend.cu.  A unit has up to four head groups that share their K or V head:
// one head group at a time, 16 sequences of 4k-32k tokens with 2-5 rows, 32/4/8 heads of 128, take 284 us instead of 190
// (187 since the scores' distances are formed in one step).
//
// Bound by memory where caches are long: those sequences (983 MB) take 182 us here, 5.4 TB/s (0.84 of a copy), plus the
// joining kernel; with row tiles as in extend.cu it was 300 us.  Short steps are bound by the chain of a block's start
// (8 thousand cycles to the first request: lengths, place in the list, page), its first tile (the code of every role comes
// from the second-level cache once: a warp's first tile takes 4-9 thousand cycles, later ones 2.2) and the joining kernel:
// 8 sequences of up to 2k tokens, 1-3 rows, 32/4/16 heads of 64, 25 us, of which 13 MB of cache are 2.
// Warp 0 TMA producer, one thread of warp 1 issues the products, warps 2-9 and 10-17 the softmax groups.  Every wait is
// bounded.
#include <type_traits>

#include "attn_math.cuh"
#include "extend.cuh"
#include "ptx.cuh"
#include "tcgen05.cuh"

namespace diffqkv {
namespace {

constexpr int kSoftmaxWarp0 = 2, kGroupWarps = 8;
constexpr int kHalfCols = kThinCols / 2;
constexpr float kThinThreshold = 24.f;  // log2 domain
constexpr float kLowest = -3.402823466e38f;
constexpr int kQRegion = 4 * 16384;  // two Q buffers and two P^T buffers of 16 KB

struct ThinSegment {
  int row_lo, n, past, head0;  // the sequence: first row, rows, tokens cached before; first head of the unit
  int ta, tb;                  // tiles
  int v0;                      // V tiles requested before the segment (the ring's position)
  int flags;
};
constexpr int kSegRing = 2;
constexpr int kSegEnd = 1, kSegWhole = 2, kSegFirst = 4;

struct Scratch {
  float m[2][kThinCols];        // reference maximum of every column, per softmax group; weights at a segment's end
  float part[2][4][kThinCols];  // per warp: maxima, or sums at a segment's end
  uint64_t bars[42];
  ThinSegment seg[kSegRing];
  long long seek_lo;
  int seek_b, seek_row, seek_n, seek_past;  // the sequence that this block begins with
  uint32_t tmem;
  int abort;
};
constexpr int kThinSmem = kQRegion + kRingBytes + (int)sizeof(Scratch);
static_assert(kThinSmem <= 232448, "shared memory of a block");

// The four warps of a (softmax group, half of the columns): does the condition hold anywhere; and a plain barrier.
__device__ __forceinline__ bool group_any(int id, bool x) {
  uint32_t y;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(y)
      : "r"((uint32_t)x), "r"(id)
      : "memory");
  return y != 0;
}
__device__ __forceinline__ void group_sync(int id) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(id) : "memory"); }

template <int kDQK, int kD>
__global__ void __launch_bounds__(kExtendThinThreads, 1)
extend_thin_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                   const __grid_constant__ CUtensorMap tmap_v, const ExtendParams p) {
  constexpr int kHalvesK = kDQK / 64, kHalves = kD / 64;
  constexpr int kKBytes = kKT * kDQK * 2, kVBytes = kKT * kD * 2;
  constexpr int kSlotBytes = kKBytes > kVBytes ? kKBytes : kVBytes;
  constexpr int kSlots = kRingBytes / kSlotBytes;  // 5 tiles of 32 KB or 10 of 16 KB: a ring of K, then one of V
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* q_s = smem;                     // [buffer][half][64 columns][128 B]
  unsigned char* p_s = smem + 2 * 16384;         // [group][128 tokens][128 B]
  unsigned char* ring_s = smem + kQRegion;
  Scratch& sc = *reinterpret_cast<Scratch*>(smem + kQRegion + kRingBytes);
  const uint32_t bar0 = ptx::smem_u32(sc.bars);
  const uint32_t full0 = bar0, empty0 = full0 + 8 * kSlots;
  const uint32_t q_full0 = empty0 + 8 * kSlots, q_empty0 = q_full0 + 16;
  const uint32_t s_full0 = q_empty0 + 16, p_full0 = s_full0 + 16, o_done0 = p_full0 + 16, o_free0 = o_done0 + 16;
  const uint32_t x_full = o_free0 + 16, x_empty = x_full + 8, drain = x_empty + 8;
  const uint32_t seg_full0 = drain + 8, seg_empty0 = seg_full0 + 8 * kSegRing;
  static_assert(2 * kSlots + 4 + 8 + 3 + 2 * kSegRing <= 42, "barriers");
  volatile int* abort_flag = &sc.abort;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if ((ptx::smem_u32(smem) & 1023u) != 0) {  // swizzled tiles start on multiples of 1024 bytes
    if (tid == 0) {
      report(p.dev_status, DIFFQKV_ERR_ALIGNMENT);
      p.list.meta[blockIdx.x].rows = 0;
    }
    ptx::grid_dependency_wait();
    return;
  }
  if (p.first) ptx::grid_launch_dependents();
  const int per_thread = (p.batch + kExtendThinThreads - 1) / kExtendThinThreads;
  const int b_lo = min(tid * per_thread, p.batch), b_hi = min(b_lo + per_thread, p.batch);
  Seq my = {};  // the thread's first sequence: there is seldom another
  if (b_lo < b_hi) my.load(p, b_lo);
  bool any = my.thin_tiles > 0;
  for (int b = b_lo + 1; b < b_hi; ++b) {
    Seq s;
    s.load(p, b);
    any |= s.thin_tiles > 0;
  }
  const int busy_threads = __syncthreads_count(any);
  if (busy_threads == 0) {  // a step without thin sequences (prompts): nothing to do here
    if (tid == 0) p.list.meta[blockIdx.x].rows = 0;
    ptx::grid_dependency_wait();
    return;
  }
  if (tid == 0) {
    sc.abort = 0;
    sc.seek_b = p.batch;
    sc.seek_lo = 0;
    for (int s = 0; s < kSlots; ++s) {
      ptx::mbar_init(full0 + 8 * s, 1);
      ptx::mbar_init(empty0 + 8 * s, 1);
    }
    for (int t = 0; t < 2; ++t) {
      ptx::mbar_init(q_full0 + 8 * t, 1);
      ptx::mbar_init(q_empty0 + 8 * t, 1);
      ptx::mbar_init(s_full0 + 8 * t, 1);
      ptx::mbar_init(p_full0 + 8 * t, kGroupWarps);
      ptx::mbar_init(o_done0 + 8 * t, 1);
      ptx::mbar_init(o_free0 + 8 * t, kGroupWarps);
    }
    ptx::mbar_init(x_full, kGroupWarps);
    ptx::mbar_init(x_empty, kGroupWarps);
    ptx::mbar_init(drain, 1);
    for (int s = 0; s < kSegRing; ++s) {
      ptx::mbar_init(seg_full0 + 8 * s, 1);
      ptx::mbar_init(seg_empty0 + 8 * s, 1 + 2 * kGroupWarps);
    }
    ptx::fence_barrier_init();
    ptx::prefetch_tmap(&tmap_q);
    ptx::prefetch_tmap(&tmap_k);
    ptx::prefetch_tmap(&tmap_v);
  }
  if (warp == 1) {
    tc::tmem_alloc(ptx::smem_u32(&sc.tmem), kTmemCols);
    tc::tmem_relinquish();
  }
  // ---- this block's range of the flat list of tiles
  long long* scan = reinterpret_cast<long long*>(&sc.part[0][0][0]);  // per warp: tiles, the other list's, chunks
  long long mine = 0, others = 0, total;  // others: the list of long chunks
  bool any_long = false;
  Seq s = my;
  for (int b = b_lo; b < b_hi;) {
    if (s.thin_tiles > 0) mine += (long long)p.n_units * (s.thin_tiles + kThinItemCost);
    if (s.n > 0) {
      others += p.n_units * s.cost(p);
      any_long = true;
    }
    if (++b < b_hi) s.load(p, b);
  }
  tc::fence_before_sync();
  any_long = __syncthreads_or(any_long);
  long long before = block_scan<kExtendThinThreads / 32>(mine, scan, total);
  tc::fence_after_sync();
  const uint32_t tmem = sc.tmem;
  if (any_long) block_scan<kExtendThinThreads / 32>(others, scan + 32, others);
  const int grid = any_long ? thin_blocks_left(p, wide_teams(p, others, total)) : p.blocks;  // the other kernel leaves
  if ((int)blockIdx.x >= grid) {
    if (tid == 0) p.list.meta[blockIdx.x].rows = 0;
    if (warp == 1) tc::tmem_dealloc(tmem, kTmemCols);
    ptx::grid_dependency_wait();
    return;
  }
  // Equal shares of the list, cut wherever they end; or, where that costs no block more than four tiles, equal chunks
  // that begin with their item: sum ceil(nt / chunk) <= total / chunk + items <= blocks, so every block has one
  // segment at most.  (A segment costs about as much as five tiles next to its tiles, and short lists would give most
  // blocks two: 8 sequences of up to 2k tokens, 32/4/16 heads of 64, 36 -> 26 us.)
  int chunk = 0;
  const int items = per_thread == 1 ? min(busy_threads * p.n_units, grid) : grid;
  if (items < grid && total < (1ll << 22)) {
    const uint32_t tiles = (uint32_t)total - items * kThinItemCost;
    chunk = (int)((tiles + grid - items - 1) / (grid - items));
    if (chunk > (int)(tiles / grid) + 4) chunk = 0;
  }
  int blocks = 0;  // that take part
  long long w0 = total, w1 = total;
  if (chunk > 0) {
    long long chunks;
    mine = (long long)p.n_units * ((my.thin_tiles + chunk - 1) / chunk);
    before = block_scan<kExtendThinThreads / 32>(mine, scan + 64, chunks);
    w0 = blockIdx.x;
    w1 = w0 < chunks ? w0 + 1 : w0;
  } else {
    blocks = shares(total, grid, kThinItemCost + 1);
    if ((int)blockIdx.x < blocks) {
      w0 = share_start(total, blockIdx.x, blocks);
      w1 = share_start(total, blockIdx.x + 1, blocks);
    }
  }
  if (w0 < w1 && before <= w0 && w0 < before + mine) {
    s = my;
    for (int b = b_lo;;) {
      const int nt = s.thin_tiles;
      const long long c = nt == 0 ? 0 : (long long)p.n_units * (chunk > 0 ? (nt + chunk - 1) / chunk : nt + kThinItemCost);
      if (w0 < before + c) {
        sc.seek_b = b;
        sc.seek_row = s.lo;
        sc.seek_n = s.rows;
        sc.seek_past = s.past;
        sc.seek_lo = before;
        break;
      }
      before += c;
      if (++b >= b_hi) break;
      s.load(p, b);
    }
  }
  __syncthreads();

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    // Lanes: token part of a tile, then channel half (where a box does not bring whole rows), then head.  As many heads as
    // fit are requested together: a request by the whole warp costs some 900 cycles, however many boxes it has.
    const int boxes_part = kKT / p.box_tok;
    const int my_part = lane % boxes_part;
    const int k_halves = p.k_rows ? 1 : kHalvesK, v_halves = p.v_rows ? 1 : kHalves;
    const int my_rest = lane / boxes_part;
    const int k_half = my_rest % k_halves, k_head = my_rest / k_halves, k_heads = 32 / (boxes_part * k_halves);
    const int v_half = my_rest % v_halves, v_head = my_rest / v_halves, v_heads = 32 / (boxes_part * v_halves);
    const uint32_t k_off = p.k_rows ? my_part * (p.box_tok * 256) : k_half * (kKT * 128) + my_part * (p.box_tok * 128);
    const uint32_t v_off = p.v_rows ? my_part * (p.box_tok * 256) : v_half * (kKT * 128) + my_part * (p.box_tok * 128);
    const uint32_t ring = ptx::smem_u32(ring_s), q_u32 = ptx::smem_u32(q_s);
    int ks = 0, vs = 0, k_count = 0, v_count = 0, segs = 0;  // ring places and tiles requested so far
    uint32_t kph = 0, vph = 0;
    bool ok = true;
    ExtendMeta m = {};
    auto load = [&](int b, int& lo, int& n, int& past) -> int {  // tiles of one unit of sequence b
      load_rows(p, b, lo, n, past);
      return n > 0 && n <= p.thin_max ? (past + n + kKT - 1) / kKT : 0;
    };
    auto hand_out = [&](const ThinSegment& d) -> bool {
      const int s = segs % kSegRing;
      if (!wait_warp(seg_empty0 + 8 * s, ((segs / kSegRing) & 1) ^ 1, abort_flag)) return false;
      if (lane == 0) {
        sc.seg[s] = d;
        ptx::mbar_arrive(seg_full0 + 8 * s);
      }
      __syncwarp();
      return true;
    };
    int chunk_lo = 0;
    int b = sc.seek_b, lo = sc.seek_row, n = sc.seek_n, past = sc.seek_past, nt = 0, u = 0;
    long long item_lo = sc.seek_lo;
    if (w0 < w1) {
      nt = (past + n + kKT - 1) / kKT;
      const long long in = w0 - item_lo;
      if (chunk > 0) {  // chunk `in` of the sequence: a range of one item, counted from the item's start
        const int per = (nt + chunk - 1) / chunk;
        u = (int)in / per;
        chunk_lo = ((int)in - u * per) * chunk;
      } else {
        const int size = nt + kThinItemCost;
        u = (int)quotient(in, size);
        item_lo += (long long)u * size;
      }
    } else {
      b = p.batch;
    }
    auto next_item = [&] {
      item_lo += nt + kThinItemCost;
      if (++u < p.n_units) return;
      u = 0;
      do {
        if (++b >= p.batch) return;
        nt = load(b, lo, n, past);
      } while (nt == 0);
    };
    while (ok && b < p.batch && item_lo < w1) {
      int ta, tb;
      if (chunk > 0) {
        ta = chunk_lo;
        tb = min(nt, chunk_lo + chunk);
      } else {
        ta = item_tile(w0 - item_lo, 1, nt, kThinItemCost);
        tb = item_tile(w1 - item_lo, 1, nt, kThinItemCost);
      }
      const int kv_len = past + n;
      const int head0 = u * p.parts * p.G;
      const int hk0 = head0 / p.heads_per_k, hv0 = head0 / p.heads_per_v;  // Eq. (idx)
      if (ta >= tb) {  // the share ends within the item's own cost
        next_item();
        continue;
      }
      if (ta == 0 && tb < nt) {
        m.rows = p.parts * n * p.G; m.part_rows = n * p.G; m.row_lo = lo; m.head0 = head0;
        m.parts = chunk > 0 ? (nt + chunk - 1) / chunk
                            : share_of(item_lo + last_tile(1, nt, kThinItemCost), total, blocks) - (int)blockIdx.x + 1;
      }
      if (!hand_out({lo, n, past, head0, ta, tb, v_count, (ta == 0 ? kSegFirst : 0) | (ta == 0 && tb == nt ? kSegWhole : 0)})) {
        ok = false;
        break;
      }
      auto fetch = [&](int tile) -> int {  // page of this lane's box (fetched two tiles ahead)
        if (!p.page_table) return b;
        const int tok = tile * kKT + my_part * p.box_tok;
        if (tile >= tb || tok >= kv_len) return 0;
        return p.page_table[(long long)b * p.max_pages_per_seq + tok / p.page_size];
      };
      // The tiles of the K heads (is_k) or of the V heads of token tile `tile`, whose page is `page`.
      auto request = [&](auto is_k, int tile, int page) __attribute__((always_inline)) {
        constexpr bool kIsK = decltype(is_k)::value;
        const int tok = tile * kKT;
        const int parts_valid = min(boxes_part, (kv_len - tok + p.box_tok - 1) / p.box_tok);
        if (my_part < parts_valid && (page < 0 || page >= p.num_blocks)) {  // never read outside the pool: flag it, block 0 instead
          report(p.dev_status, DIFFQKV_ERR_INDEX);
          page = 0;
        }
        const int first = tok + my_part * p.box_tok;
        const int slot_tok = p.page_table ? first % p.page_size : first;
        const int count = kIsK ? p.k_parts : p.v_parts, together = kIsK ? k_heads : v_heads;
        const int ring_size = kIsK ? p.k_ring : p.v_ring, mine = kIsK ? k_head : v_head;
        const uint32_t bytes = (uint32_t)(parts_valid * p.box_tok * (kIsK ? kHalvesK : kHalves)) * 128u;
        int& pos = kIsK ? ks : vs;
        uint32_t& ph = kIsK ? kph : vph;
        for (int x0 = 0; x0 < count; x0 += together) {
          const int now = min(together, count - x0);  // heads of this request
          int place = pos + mine;
          uint32_t parity = ph;
          if (place >= ring_size) { place -= ring_size; parity ^= 1; }
          const int slot = (kIsK ? 0 : p.k_ring) + place;
          const bool here = mine < now;
          // every head as soon as its own place is free (the bytes are announced by one lane, in any order with the copies:
          // the barrier cannot complete before)
          const bool fine = !here || ptx::mbar_wait(empty0 + 8 * slot, parity ^ 1, abort_flag);
          if (here && fine) {
            const uint32_t bar = full0 + 8 * slot, dst = ring + slot * kSlotBytes + (kIsK ? k_off : v_off);
            if (lane == mine * boxes_part * (kIsK ? k_halves : v_halves)) ptx::mbar_arrive_expect_tx(bar, bytes);
            if (my_part < parts_valid) {
              const int head = (kIsK ? hk0 : hv0) + x0 + mine;
              const CUtensorMap* map = kIsK ? &tmap_k : &tmap_v;
              if (kIsK ? p.k_rows : p.v_rows) ptx::tma_load_5d(dst, map, bar, 0, 0, 0, head * p.head_groups + slot_tok / 8, page);
              else ptx::tma_load_5d(dst, map, bar, 0, slot_tok, kIsK ? k_half : v_half, head, page);
            }
          }
          if (!__all_sync(0xffffffffu, fine)) { ok = false; return; }
          pos += now;
          if (pos >= ring_size) { pos -= ring_size; ph ^= 1; }
          (kIsK ? k_count : v_count) += now;
        }
      };
      // K runs a tile ahead of V: a V tile waits for the softmax of its scores anyway, and what waits holds a place
      int page0 = fetch(ta), page1 = fetch(ta + 1);
      request(std::true_type{}, ta, page0);
      if (!ok) break;
      // the segment's Q: rows of every head group behind one another, thin_max tokens each
      const int qb = segs & 1;
      if (!wait_warp(q_empty0 + 8 * qb, ((segs >> 1) & 1) ^ 1, abort_flag)) { ok = false; break; }
      if (lane == 0) {
        ptx::mbar_arrive_expect_tx(q_full0 + 8 * qb, (uint32_t)(p.parts * kHalvesK * p.G * p.thin_max) * 128u);
        for (int g = 0; g < p.parts; ++g)
#pragma unroll
          for (int h = 0; h < kHalvesK; ++h)
            ptx::tma_load_4d(q_u32 + qb * 16384 + h * (kThinCols * 128) + g * p.region * 128, &tmap_q, q_full0 + 8 * qb, 0,
                             head0 + g * p.G, lo, h);
      }
      __syncwarp();
      for (int tile = ta; tile < tb && ok; ++tile) {
        const int page2 = fetch(tile + 2);
        if (tile + 1 < tb) request(std::true_type{}, tile + 1, page1);
        if (ok) request(std::false_type{}, tile, page0);
        page0 = page1;
        page1 = page2;
      }
      if (!ok) break;
      ++segs;
      if (chunk > 0) break;
      next_item();
    }
    if (ok) ok = hand_out({0, 0, 0, 0, 0, 0, 0, kSegEnd});
    if (lane == 0) p.list.meta[blockIdx.x] = m;
    if (!ok) {
      report(p.dev_status, DIFFQKV_ERR_TIMEOUT);
      // give copies in flight a bounded chance to land before the block's shared memory is released
      for (int s = 0; s < min(k_count, p.k_ring); ++s)
        ptx::mbar_wait(full0 + 8 * s, (uint32_t)((k_count - s + p.k_ring - 1) / p.k_ring - 1) & 1u, nullptr);
      for (int s = 0; s < min(v_count, p.v_ring); ++s)
        ptx::mbar_wait(full0 + 8 * (p.k_ring + s), (uint32_t)((v_count - s + p.v_ring - 1) / p.v_ring - 1) & 1u, nullptr);
      for (int s = max(0, segs - 1); s <= segs; ++s) ptx::mbar_wait(q_full0 + 8 * (s & 1), (uint32_t)(s >> 1) & 1u, nullptr);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (one thread)
    constexpr uint32_t hi = tc::smem_desc_hi_sw128(1024);
    if (ptx::elect_one()) {
      const uint32_t q_lo = tc::smem_desc_lo(ptx::smem_u32(q_s), 16), r_lo = tc::smem_desc_lo(ptx::smem_u32(ring_s), 16);
      // V^T: the two 64-channel chunks of M are half a tile apart.  With 64 channels they are the tiles of two V heads,
      // neighbours in the ring of V (whose length is even then, so that a pair never wraps), or the same
      // tile twice: lanes 0 .. 63 of the accumulator belong to even heads, 64 .. 127 to odd ones or to nobody.  A
      // product of 128 x N x 16 takes about 100 cycles whatever N is (its A operand comes from shared memory).
      const int v_step = kHalves == 1 && p.v_parts % 2 == 0 ? 2 : 1;
      // A tile is [half][128 tokens][128 B], or, where boxes bring whole rows, [16 groups of 8 tokens][half][8][128 B].
      const uint32_t v_lo = tc::smem_desc_lo(ptx::smem_u32(ring_s), p.v_rows ? 1024 : kHalves == 2 || v_step == 2 ? kKT * 128 : 0);
      const uint32_t k_hi = tc::smem_desc_hi_sw128(p.k_rows ? 2048 : 1024), v_hi = tc::smem_desc_hi_sw128(p.v_rows ? 2048 : 1024);
      const uint32_t k_half = (p.k_rows ? 1024 : kKT * 128) >> 4;  // from the first 64 channels of K to the others
      const uint32_t v_16 = (p.v_rows ? 4096 : 2048) >> 4;         // 16 tokens of V
      const uint32_t p_lo = tc::smem_desc_lo(ptx::smem_u32(p_s), 16);
      bool ok = true;
      int ks = 0, vs = 0, segs = 0;  // ring slots of the next K tile to score and the next V tile to use
      uint32_t kph = 0, vph = 0, tp0 = 0, tp1 = 0, of0 = 1, of1 = 1;
      auto step = [](int& s, uint32_t& ph, int by, int ring) { s += by; if (s >= ring) { s -= ring; ph ^= 1; } };
      for (;; ++segs) {
        const int sl = segs % kSegRing;
        if (!ptx::mbar_wait(seg_full0 + 8 * sl, (segs / kSegRing) & 1, abort_flag)) { ok = false; break; }
        const int flags = sc.seg[sl].flags, tiles = sc.seg[sl].tb - sc.seg[sl].ta, n = sc.seg[sl].n;
        ptx::mbar_arrive(seg_empty0 + 8 * sl);
        if (flags & kSegEnd) break;
        const int qb = segs & 1;
        const uint32_t cols = (uint32_t)((n * p.G + 15) & ~15);        // of a head group
        const uint32_t all = (uint32_t)((p.parts - 1) * p.region) + cols;
        // S^T: K and Q both K-major; O^T: V is M-major, P^T N-major
        const uint32_t id_s = tc::idesc_bf16_f32(kKT, 0, 0, 0) | ((p.k_parts > 1 ? cols : all) >> 3 << 17);
        const uint32_t id_o = tc::idesc_bf16_f32(128, 0, 1, 1) |
                              ((p.v_parts == 1 ? all : v_step == 2 ? p.region + cols : cols) >> 3 << 17);
        if (!ptx::mbar_wait(q_full0 + 8 * qb, (segs >> 1) & 1, abort_flag)) { ok = false; break; }
        auto scores = [&](int i) {  // S^T of tile i, for group i & 1
          const uint32_t d = tmem + (i & 1) * 128;  // free: the group's last weights have been announced
          for (int x = 0; x < p.k_parts; ++x) {
            if (!ptx::mbar_wait(full0 + 8 * ks, kph, abort_flag)) { ok = false; return; }
            tc::fence_after_sync();
            const uint32_t ka = r_lo + ks * (kSlotBytes >> 4);
            const uint32_t qa = q_lo + ((qb * 16384 + x * p.region * 128) >> 4);
            tc::mma_ss_halves<false>(d + x * p.region, ka, k_hi, qa, hi, id_s);
#pragma unroll
            for (int k = 1; k < kDQK / 16; ++k)
              tc::mma_ss_halves<true>(d + x * p.region, ka + (k / 4) * k_half + (((k % 4) * 32) >> 4), k_hi,
                                      qa + (((k / 4) * (kThinCols * 128) + (k % 4) * 32) >> 4), hi, id_s);
            tc::commit(empty0 + 8 * ks);
            step(ks, kph, 1, p.k_ring);
          }
          tc::commit(s_full0 + 8 * (i & 1));
          if (i + 1 == tiles) tc::commit(q_empty0 + 8 * qb);
        };
        scores(0);
        for (int i = 0; i < tiles && ok; ++i) {
          // Whichever is there first: K of tile i + 1, for its scores, or the weights of tile i, for the product with its V
          // (which gives the places back).
          const int t = i & 1;
          bool ahead = i + 1 < tiles;
          if (ahead) {
            const int which = ptx::mbar_wait_either(full0 + 8 * ks, kph, p_full0 + 8 * t, t == 0 ? tp0 : tp1, abort_flag);
            if (which == 1) {
              scores(i + 1);
              ahead = false;
            }
            ok = ok && which != 0;
            if (!ok) break;
          }
          if (i < 2) {  // the accumulator of the segment before has been read out
            if (!ptx::mbar_wait(o_free0 + 8 * t, t == 0 ? of0 : of1, abort_flag)) { ok = false; break; }
            if (t == 0) of0 ^= 1; else of1 ^= 1;
          }
          if (!ptx::mbar_wait(p_full0 + 8 * t, t == 0 ? tp0 : tp1, abort_flag)) { ok = false; break; }
          if (t == 0) tp0 ^= 1; else tp1 ^= 1;
          const uint32_t d = tmem + 256 + t * kThinCols;
          for (int x = 0; x < p.v_parts; x += v_step) {
            for (int y = 0; y < v_step && ok; ++y) ok = ptx::mbar_wait(full0 + 8 * (p.k_ring + vs + y), vph, abort_flag);
            if (!ok) break;
            tc::fence_after_sync();
            const uint32_t va = v_lo + (p.k_ring + vs) * (kSlotBytes >> 4);
            const uint32_t pa = p_lo + ((t * 16384 + x * p.region * 2) >> 4);
#pragma unroll
            for (int k = 0; k < kKT / 16; ++k) {  // 16 tokens at a time: 2048 bytes of P^T
              if (k == 0 && i < 2) tc::mma_ss_halves<false>(d + x * p.region, va, v_hi, pa, hi, id_o);
              else tc::mma_ss_halves<true>(d + x * p.region, va + k * v_16, v_hi, pa + ((k * 2048) >> 4), hi, id_o);
            }
            for (int y = 0; y < v_step; ++y) tc::commit(empty0 + 8 * (p.k_ring + vs + y));
            step(vs, vph, v_step, p.v_ring);
          }
          if (!ok) break;
          tc::commit(o_done0 + 8 * t);
          if (ahead) scores(i + 1);
        }
        if (!ok) break;
      }
      if (!ok) report(p.dev_status, DIFFQKV_ERR_TIMEOUT);
      tc::commit(drain);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ softmax groups
    // Eight warps each: four for the token quarters of a tile, twice, for the lower and the upper 32 columns.  The four
    // warps of a (group, half) decide together, so they meet at a hardware barrier; they leave together as well (a warp
    // whose wait ran out says so at the next barrier), so none is left waiting there.
    const int t = (warp - kSoftmaxWarp0) >> 3;
    const int half = ((warp - kSoftmaxWarp0) >> 2) & 1;
    const int quarter = warp & 3;          // tensor-memory lanes this warp may touch
    const int wq = (warp - kSoftmaxWarp0) & 3;
    const int r = quarter * 32 + lane;     // token of a tile; channel of the accumulator
    const int c0 = half * kHalfCols;       // first column of this warp
    const int bar_id = 1 + t * 2 + half;
    const uint32_t s_taddr = tmem + ((uint32_t)(quarter * 32) << 16) + t * 128 + c0;
    const uint32_t o_taddr = tmem + ((uint32_t)(quarter * 32) << 16) + 256 + c0;
    unsigned char* p_row = p_s + t * 16384 + r * 128;
    float* m = sc.m[t] + c0;
    uint32_t par = 0, xpar = 0;
    int other = 0;  // tiles of the other group in earlier segments
    bool ok = true;
    for (uint32_t segs = 0;; ++segs) {
      const ThinSegment& w = sc.seg[segs % kSegRing];
      ok = wait_warp(seg_full0 + 8 * (segs % kSegRing), (segs / kSegRing) & 1, abort_flag);
      // Group 1 hands its sums and maxima over at a segment's end: it may write there again once they have been read.
      if (ok && t == 1 && !(w.flags & kSegEnd) && w.tb - w.ta > 1) ok = wait_warp(x_empty, xpar ^ 1, abort_flag);
      if (group_any(bar_id, !ok)) { ok = false; break; }
      if (w.flags & kSegEnd) break;
      const int tiles = w.tb - w.ta;
      const int used = w.n * p.G;  // columns of a head group in use
      uint32_t mask = 0;           // groups of eight columns of this half that hold some
#pragma unroll
      for (int q = 0; q < kHalfCols / 8; ++q)
        if ((c0 + q * 8) / p.region < p.parts && ((c0 + q * 8) & (p.region - 1)) < used) mask |= 1u << q;
      float l[kHalfCols];
#pragma unroll
      for (int c = 0; c < kHalfCols; ++c) l[c] = 0.f;
      bool later = false;  // not the segment's first tile of this group
#pragma unroll 1
      for (int i = t; i < tiles; i += 2, par ^= 1, later = true) {
        ok = wait_warp(s_full0 + 8 * t, par, abort_flag) && ok;
        tc::fence_after_sync();
        float x[kHalfCols];
        const int k0 = (w.ta + i) * kKT;
        auto load_scores = [&] {  // they stay in tensor memory until this tile's weights are announced
#pragma unroll
          for (int q = 0; q < kHalfCols / 8; ++q)
            if (mask >> q & 1) tc::ld_32x32b_x8(s_taddr + q * 8, *reinterpret_cast<uint32_t(*)[8]>(&x[q * 8]));
          tc::wait_ld();
          if (k0 + kKT > w.past + 1) {  // the tile reaches past some row's position
            const int hidden = (k0 + r - w.past) * p.G;  // columns of a group below this belong to rows before the token
#pragma unroll
            for (int q = 0; q < kHalfCols / 8; ++q)
              if (mask >> q & 1) {
                const int first = hidden - ((c0 + q * 8) & (p.region - 1));
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (e < first) x[q * 8 + e] = -INFINITY;
              }
          }
        };
        load_scores();
        // ---- scores on the scale of base 2, from the reference: the score of the segment's first token of this group to
        // begin with (a row that does not see it sees none of the tile)
        if (!later) {
          if (quarter == 0 && lane == 0) {
            // -inf counts as the lowest number, which any other raises
            auto start = [&](float y) { y *= p.scale_log2; return y == -INFINITY ? kLowest : y; };
#pragma unroll
            for (int q = 0; q < kHalfCols / 8; ++q)
              if (mask >> q & 1) {
#pragma unroll
                for (int c = q * 8; c < q * 8 + 8; c += 4)
                  *reinterpret_cast<float4*>(m + c) = make_float4(start(x[c]), start(x[c + 1]), start(x[c + 2]), start(x[c + 3]));
              }
          }
          group_sync(bar_id);
        }
        bool over = !ok;
#pragma unroll
        for (int q = 0; q < kHalfCols / 8; ++q)
          if (mask >> q & 1) {
            const int end = used - ((c0 + q * 8) & (p.region - 1));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int c = q * 8 + e;
              x[c] = fmaf(x[c], p.scale_log2, -m[c]);
              over |= x[c] > kThinThreshold && e < end;
            }
          }
        if (group_any(bar_id, over)) {
          // ---- largest score of every column in this tile; the reference goes up where it is passed
          load_scores();
          float y[kHalfCols / 2];  // over the lanes, half of the columns in every step; lane c ends with column c
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float give = lane & 16 ? x[c] : x[c + 16], keep = lane & 16 ? x[c + 16] : x[c];
            y[c] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, 16));
          }
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) {
#pragma unroll
            for (int c = 0; c < o; ++c) {
              const float give = lane & o ? y[c] : y[c + o], keep = lane & o ? y[c + o] : y[c];
              y[c] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, o));
            }
          }
          const float top = y[0];
          sc.part[t][wq][c0 + lane] = top;
          if (later) ok = wait_warp(o_done0 + 8 * t, par ^ 1, abort_flag) && ok;
          if (group_any(bar_id, !ok)) { ok = false; break; }
          if (wq == 0) {  // a lane per column
            const float largest = p.scale_log2 * fmaxf(fmaxf(top, sc.part[t][1][c0 + lane]),
                                                       fmaxf(sc.part[t][2][c0 + lane], sc.part[t][3][c0 + lane]));
            const float was = m[lane], now = largest - was > kThinThreshold ? largest : was;
            sc.part[t][0][c0 + lane] = now != was ? ex2(was - now) : 1.f;
            m[lane] = now;
          }
          group_sync(bar_id);
          const float* alphas = &sc.part[t][0][c0];
          tc::fence_after_sync();
#pragma unroll
          for (int q = 0; q < kHalfCols / 8; ++q) {
            if (!(mask >> q & 1)) continue;
            uint32_t o[8];
            if (later) {
              tc::ld_32x32b_x8(o_taddr + t * kThinCols + q * 8, o);
              tc::wait_ld();
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x[q * 8 + e] = fmaf(x[q * 8 + e], p.scale_log2, -m[q * 8 + e]);
              if (later) {
                const float alpha = alphas[q * 8 + e];
                l[q * 8 + e] *= alpha;
                o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
              }
            }
            if (later) tc::st_32x32b_x8(o_taddr + t * kThinCols + q * 8, o);
          }
          if (later) tc::wait_st();
        } else if (later) {  // the last product of this group has read its P^T
          ok = wait_warp(o_done0 + 8 * t, par ^ 1, abort_flag) && ok;
        }
        // ---- P^T = 2^x as packed bf16, one row of 128 bytes per token, 16-byte chunks exclusive-ored with the row
#pragma unroll
        for (int q = 0; q < kHalfCols / 8; ++q)
          if (mask >> q & 1) {
            uint32_t y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p0 = ex2(x[q * 8 + 2 * e]), p1 = ex2(x[q * 8 + 2 * e + 1]);
              l[q * 8 + 2 * e] += p0;
              l[q * 8 + 2 * e + 1] += p1;
              y[e] = pack2(p0, p1);
            }
            *reinterpret_cast<uint4*>(p_row + (((half * 4 + q) ^ (r & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
          }
        if (k0 + kKT > w.past + w.n) {
          // V rows past the sequence end hold whatever followed in memory: zero them (0 * NaN would poison the product).
          // Where the ring has room for one tile's V the tile before, the other group's, may still wait for its own, in the
          // place that this one's will have: until its product is done a wait for this V could take the phase before for
          // its own.  (In a longer ring that place was the tile's before, whose product this group has waited for, or an
          // earlier segment's, whose products had all been issued.)
          if (i > 0 && p.v_ring < 2 * p.v_parts) ok = wait_warp(o_done0 + 8 * (1 - t), (other + ((i - 1) >> 1)) & 1, abort_flag) && ok;
          if (half == 0 && r >= w.past + w.n - k0) {
            for (int y = 0; y < p.v_parts; ++y) {
              const int at = w.v0 + i * p.v_parts + y, slot = p.k_ring + at % p.v_ring;
              ok = ok && ptx::mbar_wait(full0 + 8 * slot, (at / p.v_ring) & 1, abort_flag);
#pragma unroll
              for (int h = 0; h < kHalves; ++h) {
                uint4* dst = reinterpret_cast<uint4*>(ring_s + slot * kSlotBytes +
                                                      (p.v_rows ? (r / 8) * 2048 + h * 1024 + (r % 8) * 128 : h * (kKT * 128) + r * 128));
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[e] = make_uint4(0, 0, 0, 0);
              }
            }
          }
        }
        ptx::fence_proxy_async();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(p_full0 + 8 * t);
      }
      // ---- the segment's result: sums over the lanes (every lane ends up with one column), then over the warps
      if (t < tiles) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
          for (int c = 0; c < o; ++c) {
            const bool up = lane & o;
            const float give = up ? l[c] : l[c + o], keep = up ? l[c + o] : l[c];
            l[c] = keep + __shfl_xor_sync(0xffffffffu, give, o);
          }
        }
        ok = wait_warp(o_done0 + 8 * t, par ^ 1, abort_flag) && ok;
        if (group_any(bar_id, !ok)) { ok = false; break; }  // also: the last raise has read its maxima
        tc::fence_after_sync();
        sc.part[t][wq][c0 + lane] = l[0];
      }
      other += t == 0 ? tiles >> 1 : (tiles + 1) >> 1;
      const bool join = tiles > 1;
      if (t == 1) {
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          if (join) ptx::mbar_arrive(x_full);
          ptx::mbar_arrive(seg_empty0 + 8 * (segs % kSegRing));
        }
        if (join) xpar ^= 1;
        continue;
      }
      if (join) {
        ok = wait_warp(x_full, xpar, abort_flag);
        xpar ^= 1;
        tc::fence_after_sync();
      }
      if (group_any(bar_id, !ok)) { ok = false; break; }
      const bool whole = w.flags & kSegWhole;
      const long long prow0 = (2LL * blockIdx.x + ((w.flags & kSegFirst) ? 1 : 0)) * p.list.slot_rows;
      if (wq == 0) {  // a lane per column: the two groups' weights in the result, the log-sum-exp
        const int c = c0 + lane, g = c / p.region, lc = c & (p.region - 1);
        const float l0 = sc.part[0][0][c] + sc.part[0][1][c] + sc.part[0][2][c] + sc.part[0][3][c];
        const float l1 = join ? sc.part[1][0][c] + sc.part[1][1][c] + sc.part[1][2][c] + sc.part[1][3][c] : 0.f;
        const float m0 = l0 != 0.f ? sc.m[0][c] : -INFINITY, m1 = l1 != 0.f ? sc.m[1][c] : -INFINITY;
        const float top = fmaxf(m0, m1);
        const float e0 = l0 != 0.f ? exp2f(m0 - top) : 0.f, e1 = l1 != 0.f ? exp2f(m1 - top) : 0.f;
        const float sum = l0 * e0 + l1 * e1, inv = sum != 0.f ? 1.f / sum : 0.f;
        sc.m[0][c] = e0 * inv;
        if (join) sc.m[1][c] = e1 * inv;
        if (g < p.parts && lc < used) {
          const float lse2 = sum != 0.f ? top + log2f(sum) : -INFINITY;
          const int token = lc / p.G;
          if (!whole) p.list.part_lse[prow0 + g * used + lc] = lse2;
          else if (p.lse) p.lse[(long long)(w.row_lo + token) * p.n_q + w.head0 + g * p.G + lc - token * p.G] = lse2 * kLn2;
        }
      }
      group_sync(bar_id);
#pragma unroll 1
      for (int q = 0; q < kHalfCols / 8; ++q) {
        if (!(mask >> q & 1)) continue;
        uint32_t o0[8], o1[8];
        tc::ld_32x32b_x8(o_taddr + q * 8, o0);
        if (join) tc::ld_32x32b_x8(o_taddr + kThinCols + q * 8, o1);
        tc::wait_ld();
        const int c = c0 + q * 8, g = c / p.region, lc = c & (p.region - 1);
        // the lanes that hold this head group's channels
        const bool mine = kHalves == 2 || (r < 64) == (p.v_parts % 2 != 0 || g % 2 == 0);
        const int ch = r & (kD - 1);
        int token = lc / p.G, h = lc - token * p.G;
        long long at = whole ? ((long long)(w.row_lo + token) * p.n_q + w.head0 + g * p.G + h) * kD + ch
                             : (prow0 + g * used + lc) * kD + ch;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float y = __uint_as_float(o0[e]) * sc.m[0][c + e];
          if (join) y = fmaf(__uint_as_float(o1[e]), sc.m[1][c + e], y);
          if (lc + e < used && mine) {
            if (!whole) p.list.part_o[at] = y;
            else if (p.out_is_f32) reinterpret_cast<float*>(p.out)[at] = y;
            else reinterpret_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(y);
          }
          at += kD;
          if (whole && ++h == p.G) {  // the next token's first head
            h = 0;
            at += (long long)(p.n_q - p.G) * kD;
          }
        }
      }
      group_sync(bar_id);  // the weights have been read
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        ptx::mbar_arrive(o_free0);
        if (join) {
          ptx::mbar_arrive(o_free0 + 8);
          ptx::mbar_arrive(x_empty);
        }
        ptx::mbar_arrive(seg_empty0 + 8 * (segs % kSegRing));
      }
    }
    if (!ok) report(p.dev_status, DIFFQKV_ERR_TIMEOUT);
  }

  // ---- teardown: all products this block issued must be done before its tensor memory is released
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    ptx::mbar_wait(drain, 0, nullptr);
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, kTmemCols);
  }
  ptx::grid_dependency_wait();  // see the kernel for longer chunks
}

}  // namespace

cudaError_t launch_extend_thin(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const ExtendParams& p,
                               int d_qk, int d_v, int blocks, bool second, cudaStream_t stream) {
  using Fn = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const ExtendParams);
  const Fn fn = d_v == 64 ? extend_thin_kernel<64, 64> : (d_qk == 128 ? extend_thin_kernel<128, 128> : extend_thin_kernel<64, 128>);
  const cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kThinSmem);
  if (err != cudaSuccess) return err;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kExtendThinThreads);
  cfg.dynamicSmemBytes = kThinSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = second ? 1 : 0;
  const cudaError_t launched = cudaLaunchKernelEx(&cfg, fn, mq, mk, mv, p);
  if (launched == cudaSuccess) count_launch();
  return launched;
}

}  // namespace diffqkv
