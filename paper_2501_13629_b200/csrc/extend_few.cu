// Sequences with a few new rows, and prefixes shared by a few rows, of the ranged steps (diffqkv_extend_window,
// diffqkv_extend_shared): the other half of extend.cu, which has the mathematics and takes the longer chunks.
//
// Such steps are short: a window of 4k tokens, the tokens behind a shared prefix.  extend_thin.cu's way, which plain steps
// take, costs 18 us of starts, first tiles and ends however little there is to do, because every role's straight code is
// fetched once (about 10 cycles an instruction); 16 sequences with a window of 1k tokens took it 24 us, of which the cache is
// 4.  So here all warps but one run the same short loop, on warp-level products, and the same step takes 16 us.
//
// Work: one flat list of (entry, block of rows, unit of heads, 64-token tile), where the tiles that no row sees are left out,
// divided over one persistent block an SM, or over those that the step's long chunks leave; cut items leave partial rows as
// in extend.cu.  An entry is one block of rows, or several that read the same tokens (see kMidMost).  A unit's K and V heads
// (one of either kind, up to four of the other) pass an SM once for all of its query heads.
//
// Per block: warp 8 requests whole tiles by TMA into a ring of stages.  The other eight share a tile's 128 columns at most,
// (16 rows of one head group) x (tokens): one, two, four or up to eight such row groups have 8, 4, 2 or one warp each, which
// take 32 tokens of a tile, or both halves of it (with 4 or 8 warps to a row group those of every second or fourth tile), and
// are joined through shared memory at the end of a segment.  A warp holds its rows' queries and their accumulator in
// registers,
//     S[16 rows x 32 tokens] = Q K^T,   O[16 x d_v] += P V        (P from registers, K and V by ldmatrix)
// with the running reference of a row raised only when passed by 2^8, as in extend.cu; statistics and sums are fp32, the
// weights are rounded to bf16 for the second product.  V rows that no row of the sequence sees are cleared first: their
// boxes may not have been read.
//
// Bound, for up to two row groups, by memory (a 48 KB tile in 1.85 thousand cycles), for more by the warps' chain of products
// and softmax (2.2 thousand for four, twice that for eight): 32 sequences of 2-5 rows of 32/4/8 heads behind windows of 4k
// tokens (405 MB) take 83 us, 4.9 TB/s, the warp-level tensor pipe active 28 % (87 us with the join).  Started, a
// block has its first tile after 9 thousand cycles; the step of 16 rows has little else.
#include "attn_math.cuh"
#include "extend.cuh"
#include "ptx.cuh"

namespace diffqkv {
namespace {

constexpr int kWarps = 8, kThreads = (kWarps + 1) * 32;
constexpr int kMaxStages = 8;
constexpr float kFewThreshold = 8.f;  // log2 domain
constexpr int kMaxSmem = 232448;

struct FewSegment {  // as the producer hands it to the other warps, through a ring in shared memory
  int lo, n, past, end, start;  // see SeqOf
  int low, skip;                // first token behind the sinks that the first row sees; tiles skipped in front of it
  int unit, ta, tb, dst, flags;
};
constexpr int kSegRing = 4;
constexpr int kSegEnd = 1, kSegWhole = 2, kSegFirst = 4;
template <int kD>
struct Scratch {
  float4 o[4][kD / 8][32];  // accumulators handed from warp to warp, a register of all lanes behind one another
  float2 ml[4][16];         // their rows' reference and sum
  RangedScan<kWarps + 1> scan;
  uint32_t chunks[kWarps + 1];
  uint64_t full[kMaxStages], empty[kMaxStages], seg_full[kSegRing], seg_empty[kSegRing];
  FewSegment seg[kSegRing];
  int abort;
};

template <int kDQK, int kD>
__global__ void __launch_bounds__(kThreads, 1)
extend_few_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                  const __nv_bfloat16* __restrict__ q, const ExtendParams p) {
  constexpr int HK = kDQK / 64, HV = kD / 64;
  constexpr int kKBytes = kFewT * kDQK * 2, kVBytes = kFewT * kD * 2;
  constexpr int kItem = kFewItemCost;
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t stage_bytes = p.k_parts * kKBytes + p.v_parts * kVBytes;
  Scratch<kD>& sc = *reinterpret_cast<Scratch<kD>*>(smem + p.few_stages * stage_bytes);
  const uint32_t ring = ptx::smem_u32(smem), full0 = ptx::smem_u32(sc.full), empty0 = ptx::smem_u32(sc.empty);
  const uint32_t seg_full0 = ptx::smem_u32(sc.seg_full), seg_empty0 = ptx::smem_u32(sc.seg_empty);
  volatile int* abort_flag = &sc.abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if ((ring & 1023u) != 0) {  // swizzled tiles start on multiples of 1024 bytes
    if (tid == 0) {
      report(p.dev_status, DIFFQKV_ERR_ALIGNMENT);
      p.list.meta[blockIdx.x].rows = 0;
    }
    ptx::grid_dependency_wait();
    return;
  }
  if (p.first) {  // see extend.cu
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
  }
  if (tid < kMaxStages + kSegRing) {  // full and empty, of the stages and behind them of the segments
    const bool seg = tid >= kMaxStages;
    ptx::mbar_init(seg ? seg_full0 + 8 * (tid - kMaxStages) : full0 + 8 * tid, 1);
    ptx::mbar_init(seg ? seg_empty0 + 8 * (tid - kMaxStages) : empty0 + 8 * tid, kWarps);
    ptx::fence_barrier_init();
  }
  if (tid == 0) {
    sc.abort = 0;
    ptx::prefetch_tmap(&tmap_k);
    ptx::prefetch_tmap(&tmap_v);
  }
  // ---- this block's share of the list
  using Seq = SeqOf<true>;
  Seq my;
  const RangedStart at = ranged_start(p, sc.scan, my, p.alone && blockIdx.x == 0);
  const uint32_t total = at.few;
  // Equal shares of the list, cut wherever they end; or, where that costs no block more than six tiles, equal chunks that
  // begin with their item (see extend_thin.cu), so that every block has one segment at most.  A chunk is that many of the
  // cheapest tiles, rounded up of others (42 rows in two groups, whose tiles cost more than twice their own tokens': 29 us,
  // 36 with as many of either).
  const int grid = at.wide == 0 ? p.blocks : thin_blocks_left(p, ranged_wide_teams(p, at.wide, total));  // what the other kernel leaves
  int chunk = 0, blocks = 0;  // blocks: that take part
  uint32_t w0 = 0, w1 = 0, before = at.before_few;
  auto chunk_of = [&](const Seq& s) -> int {
    const int cost = s.few_cost(p);
    return cost == p.few_cost[0] ? chunk : (chunk * p.few_cost[0] + cost - 1) / cost;
  };
  auto chunks_of = [&](const Seq& s) -> int {
    const int each = chunk_of(s);
    return s.blocks * ((s.thin_tiles + each - 1) / each);
  };
  if (total > 0 && (int)blockIdx.x < grid) {
    const int items = at.single ? min(at.busy * p.n_units, grid) : grid;
    if (items < grid) {
      const uint32_t tiles = (total - items * kItem + p.few_cost[0] - 1) / (uint32_t)p.few_cost[0];  // or more
      chunk = (int)((tiles + grid - items - 1) / (uint32_t)(grid - items));
      if (chunk > (int)(tiles / (uint32_t)grid) + 6) chunk = 0;
    }
    if (chunk > 0) {  // the list of chunks instead
      uint32_t x = my.thin_tiles > 0 ? p.n_units * chunks_of(my) : 0;
      const uint32_t mine = x;
#pragma unroll 1
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (lane == 31) sc.chunks[warp] = x;
      __syncthreads();
      uint32_t all = 0;
      before = x - mine;
#pragma unroll 1
      for (int w = 0; w <= kWarps; ++w) {
        if (w < warp) before += sc.chunks[w];
        all += sc.chunks[w];
      }
      w0 = blockIdx.x;
      w1 = w0 < all ? w0 + 1 : w0;
    } else {
      blocks = ranged_shares(total, grid, kItem + kFewMostCost);
      if ((int)blockIdx.x < blocks) {
        w0 = ranged_share_start(total, blockIdx.x, blocks);
        w1 = ranged_share_start(total, blockIdx.x + 1, blocks);
      }
    }
  }
  if (w0 >= w1) {  // nothing to do: a step of long chunks, or fewer tiles than blocks
    if (tid == 0) p.list.meta[blockIdx.x].rows = 0;
    ptx::grid_dependency_wait();
    return;
  }
  ranged_seek(p, sc.scan, at, my, w0, before, [&](const Seq& s) -> uint32_t {
    return p.n_units * (uint32_t)(chunk > 0 ? (s.thin_tiles > 0 ? chunks_of(s) : 0) : s.few_unit(p));
  });
  __syncthreads();

  const int bt_shift = 31 - __clz(p.box_tok);
  int stage = 0;
  uint32_t phase = 0;
  auto step = [&]() {
    if (++stage == p.few_stages) {
      stage = 0;
      phase ^= 1;
    }
  };

  if (warp == kWarps) {
    // ------------------------------------------------------------------ TMA producer
    // Lane: token part of a tile, then head; a box brings all channels of a part.
    const int parts = kFewT >> bt_shift, my_part = lane & (parts - 1), my_head = lane / parts, together = 32 / parts;
    const int heads = p.k_parts + p.v_parts;
    const uint32_t part_bytes = p.box_tok * 128u;
    int count = 0, segs = 0;
    bool ok = true;
    ExtendMeta m = {};
    int e = sc.scan.e, u, chunk_lo = 0;  // u: unit, and block of rows n_units further on
    Seq x = sc.scan.seq;
    int nt = x.thin_tiles, cost = x.few_cost(p);
    uint32_t item_lo = sc.scan.lo;
    if (chunk > 0) chunk = chunk_of(x);  // of the block's one item
    {
      const uint32_t in = w0 - item_lo, per = chunk > 0 ? (nt + chunk - 1) / chunk : cost * nt + kItem;
      u = (int)(in / per);
      if (chunk > 0) chunk_lo = (int)(in - u * per) * chunk;
      else item_lo += u * per;
    }
    auto next_item = [&]() {
      item_lo += cost * nt + kItem;
      if (item_lo >= w1 || ++u < p.n_units * x.blocks) return;
      u = 0;
      do {
        if (++e >= p.entries) return;
        x.load(p, e);
        x.choose(at.all_few);
        nt = x.thin_tiles;
        cost = x.few_cost(p);
      } while (nt == 0);
    };
    auto hand_out = [&](const FewSegment& d, volatile int* abort) -> bool {
      const int at = segs % kSegRing;
      if (!wait_warp(seg_empty0 + 8 * at, ((segs / kSegRing) & 1) ^ 1, abort)) return false;
      if (lane == 0) {
        sc.seg[at] = d;
        ptx::mbar_arrive(seg_full0 + 8 * at);  // releases the stores above
      }
      __syncwarp();
      ++segs;
      return true;
    };
    while (ok && e < p.entries && item_lo < w1) {
      int ta, tb;
      if (chunk > 0) {
        ta = chunk_lo;
        tb = min(nt, chunk_lo + chunk);
      } else {
        ta = w0 > item_lo ? item_tile(w0 - item_lo, cost, nt, kItem) : 0;
        tb = item_tile(w1 - item_lo, cost, nt, kItem);
        if (ta >= tb) {  // the share begins, or ends, within the item's own cost
          next_item();
          continue;
        }
      }
      const int low = max(x.low(p, 0), 0), skip = x.skip_few(p);
      const int block = u / p.n_units, unit = u - block * p.n_units, tok0 = block * x.block_rows;
      const int lo = x.lo + tok0, rows = min(x.block_rows, x.rows - tok0);
      const int head0 = unit * p.parts * p.G, hk0 = head0 / p.heads_per_k, hv0 = head0 / p.heads_per_v;  // Eq. (idx)
      if (!hand_out({lo, rows, x.past + tok0, x.end, x.start, low, skip, unit, ta, tb, x.dst,
                     (ta == 0 ? kSegFirst : 0) | (ta == 0 && tb == nt ? kSegWhole : 0)}, abort_flag)) {
        ok = false;
        break;
      }
      if (ta == 0 && tb < nt) {
        m.rows = p.parts * rows * p.G; m.part_rows = rows * p.G; m.row_lo = lo; m.head0 = head0;
        m.parts = chunk > 0 ? (nt + chunk - 1) / chunk
                            : share_of((long long)item_lo + last_tile(cost, nt, kItem), total, blocks) - (int)blockIdx.x + 1;
      }
      if (ta == 0 && p.groups > 0 && lane == 0)
        p.refs[((x.dst == kDstPrefix ? 0LL : p.total_q) + lo) * p.n_units + unit] = {(int)blockIdx.x, tb < nt ? m.parts : 1};
      auto token_of = [&](int tile) -> int { return ((tile >= p.sink_few ? tile + skip : tile) << 6) + my_part * p.box_tok; };
      auto wanted = [&](int tok) -> bool { return tok < x.end && (tok < p.sinks || tok + p.box_tok > low); };
      auto fetch = [&](int tile) -> int {  // page of this lane's box
        if (!p.page_table) return x.tab;
        const int tok = token_of(tile);
        if (tile >= tb || !wanted(tok)) return 0;
        return p.page_table[(long long)x.tab * p.max_pages_per_seq + tok / p.page_size];
      };
      int page = fetch(ta);
      for (int tile = ta; tile < tb; ++tile) {
        const int page_next = fetch(tile + 1);
        const int tok = token_of(tile);
        const bool reads = wanted(tok);
        if (reads && (page < 0 || page >= p.num_blocks)) {  // never read outside the pool: flag it, block 0 instead
          report(p.dev_status, DIFFQKV_ERR_INDEX);
          page = 0;
        }
        const int slot = p.page_table ? tok % p.page_size : tok;
        const int valid = __popc(__ballot_sync(0xffffffffu, reads && my_head == 0));
        if (!wait_warp(empty0 + 8 * stage, phase ^ 1, abort_flag)) { ok = false; break; }
        const uint32_t bar = full0 + 8 * stage;
        if (lane == 0) ptx::mbar_arrive_expect_tx(bar, valid * part_bytes * (p.k_parts * HK + p.v_parts * HV));
        __syncwarp();
        if (reads) {
          const uint32_t dst = ring + stage * stage_bytes;
          for (int h = my_head; h < heads; h += together) {
            const int v = h - p.k_parts;
            if (v < 0) ptx::tma_load_5d(dst + h * kKBytes + my_part * (part_bytes * HK), &tmap_k, bar, 0, slot, 0, hk0 + h, page);
            else ptx::tma_load_5d(dst + p.k_parts * kKBytes + v * kVBytes + my_part * (part_bytes * HV), &tmap_v, bar, 0, slot, 0, hv0 + v, page);
          }
        }
        page = page_next;
        ++count;
        step();
      }
      if (!ok || chunk > 0) break;
      next_item();
    }
    if (!p.first) ptx::grid_launch_dependents();  // see extend.cu
    FewSegment end = {};
    end.flags = kSegEnd;
    if (!hand_out(end, nullptr)) ok = false;  // in any case: the other warps leave together
    if (lane == 0) p.list.meta[blockIdx.x] = m;
    if (!ok) {
      report(p.dev_status, DIFFQKV_ERR_TIMEOUT);
      // give copies in flight a bounded chance to land before the block's shared memory is released
      for (int s = 0; s < min(count, p.few_stages); ++s)
        ptx::mbar_wait(full0 + 8 * s, (uint32_t)((count - s + p.few_stages - 1) / p.few_stages - 1) & 1u, nullptr);
    }
  } else {
    // ------------------------------------------------------------------ products and softmax
    const int g8 = lane >> 2, t4 = lane & 3;  // row and column pair of the fragments
    // Row r, 64-channel half h of a head tile lies at ((r / box_tok) H + h) box_tok + r % box_tok times 128 bytes, its 16-byte
    // pieces exclusive-ored with r mod 8.  Of the rows that a lane addresses (ldmatrix) r mod 8 is lane mod 8 always, so
    // that a step's addresses are a base and constants: rows 16 and 32 further down, the other half, and the pieces.
    const int box = p.box_tok;
    auto row_at = [&](int r, int H) -> uint32_t { return (uint32_t)(((r >> bt_shift) * H << bt_shift) + (r & (box - 1))) << 7; };
    const uint32_t half_at = (uint32_t)box << 7;
    const uint32_t k_lane = row_at((lane & 7) + 8 * (lane >> 4), HK) + ((((lane >> 3) & 1) ^ (lane & 7)) << 4);
    const uint32_t v_lane = row_at(lane & 15, HV) + (((lane >> 4) ^ (lane & 7)) << 4);
    const uint32_t k_16 = row_at(16, HK), k_32 = row_at(32, HK), v_16 = row_at(16, HV), v_32 = row_at(32, HV);
    bool dead = false;  // a wait for tiles ran out: go on without waiting, so that all warps meet at the barriers below
    for (uint32_t segs = 0;; ++segs) {
      const FewSegment& w = sc.seg[segs % kSegRing];  // released at the end of the segment
      // the producer hands an end out even where it gives up, long before this limit, so that all warps take the same way
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(seg_full0 + 8 * (segs % kSegRing), (segs / kSegRing) & 1, nullptr,
                                                  8 * ptx::kWaitLimitNs))) {
        dead = true;
        break;
      }
      if (w.flags & kSegEnd) break;
      const int used = w.n * p.G;                                            // rows of a head group
      const int blocks16 = (used + 15) >> 4, all16 = p.parts * blocks16;     // at most 8
      const int mshift = all16 > 1 ? 32 - __clz(all16 - 1) : 0, slices = kWarps >> mshift;
      const int mt = warp & ((1 << mshift) - 1), slice = warp >> mshift;
      const int group = mt / blocks16, r0 = (mt - group * blocks16) << 4;
      const bool active = mt < all16;
      // ---- the warp's rows r0 + g8 and r0 + g8 + 8 of the head group: queries, the tokens that they see
      auto out_row = [&](int r) -> long long {
        const int tok = r / p.G;
        return (long long)(w.lo + tok) * p.n_q + (w.unit * p.parts + group) * p.G + (r - tok * p.G);
      };
      uint32_t qf[kDQK / 16][4];
      int last[2], first[2];  // up to last, from first on (and the sinks)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int r = r0 + g8 + 8 * y, tok = r / p.G;
        const bool here = active && r < used;
        last[y] = min(w.past + tok, w.end - 1);
        first[y] = max(w.start, w.past + tok + 1 - p.window);
        const uint32_t* src = reinterpret_cast<const uint32_t*>(q + (here ? out_row(r) : 0) * kDQK) + t4;
#pragma unroll
        for (int ks = 0; ks < kDQK / 16; ++ks) {
          qf[ks][y] = here ? src[ks * 8] : 0u;
          qf[ks][y + 2] = here ? src[ks * 8 + 4] : 0u;
        }
      }
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
      float acc[kD / 8][4];
#pragma unroll
      for (int c = 0; c < kD / 8; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[c][e] = 0.f;
      const uint32_t k_off = (p.k_parts > 1 ? group : 0) * kKBytes;
      const uint32_t v_off = p.k_parts * kKBytes + (p.v_parts > 1 ? group : 0) * kVBytes;
      const int low = w.low, end = w.end, tb = w.tb;
      // The slices of a row group: one takes both halves of a tile, two one each, four or eight those of every second or
      // fourth tile.
      const int half0 = (slice & 1) * 32, halves = slices == 1 ? 64 : half0 + 32;
      const int turn = slice >> 1, turns = slices > 1 ? (slices >> 1) - 1 : 0;
#pragma unroll 1
      for (int i = w.ta; i < tb; ++i) {
        if (!dead && !wait_warp(full0 + 8 * stage, phase, abort_flag)) dead = true;
        const int k0 = (i >= p.sink_few ? i + w.skip : i) << 6;
        const uint32_t base = ring + stage * stage_bytes;
        const bool mine = active && !dead && ((i - w.ta) & turns) == turn;
#pragma unroll 1
        for (int r = half0; r < halves; r += 32) {
          const int t0 = k0 + r;  // first of 32 tokens
          if (!mine || t0 >= end || (t0 + 32 <= low && t0 >= p.sinks)) continue;  // the same for the whole warp
          const bool edge = t0 + 32 > end || (t0 < low && t0 + 32 > p.sinks);     // some are seen by no row
          // ---- scores
          float s[4][4];
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e >> 2][e & 3] = 0.f;
          const uint32_t k_at = base + k_off + k_lane + (r ? k_32 : 0u);
#pragma unroll
          for (int ks = 0; ks < kDQK / 16; ++ks) {
            const uint32_t at = k_at + (ks / 4) * half_at;
            uint32_t b[4], d[4];
            ptx::ldmatrix_x4(at ^ ((ks % 4) << 5), b);
            ptx::ldmatrix_x4((at + k_16) ^ ((ks % 4) << 5), d);
            ptx::mma_bf16_16816(s[0], qf[ks], b[0], b[1]);
            ptx::mma_bf16_16816(s[1], qf[ks], b[2], b[3]);
            ptx::mma_bf16_16816(s[2], qf[ks], d[0], d[1]);
            ptx::mma_bf16_16816(s[3], qf[ks], d[2], d[3]);
          }
          if (t0 + 31 > min(last[0], last[1]) || (t0 < max(first[0], first[1]) && t0 + 32 > p.sinks)) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int tok = t0 + (e >> 2) * 8 + 2 * t4 + (e & 1), y = (e >> 1) & 1;
              if (tok > last[y] || (tok < first[y] && tok >= p.sinks)) s[e >> 2][e & 3] = -INFINITY;
            }
          }
          // ---- softmax over the 32 tokens: four lanes a row
          float alpha[2];
          bool raise = false;
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float mx = fmaxf(s[0][2 * y], s[0][2 * y + 1]);
#pragma unroll
            for (int h = 1; h < 4; ++h) mx = max3(mx, s[h][2 * y], s[h][2 * y + 1]);
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)) * p.scale_log2;
            const bool up = mx > m[y] + kFewThreshold;
            alpha[y] = up ? ex2(m[y] - mx) : 1.f;
            if (up) m[y] = mx;
            raise |= up;
          }
          if (__any_sync(0xffffffffu, raise)) {
            l[0] *= alpha[0];
            l[1] *= alpha[1];
#pragma unroll
            for (int c = 0; c < kD / 8; ++c) {
              acc[c][0] *= alpha[0]; acc[c][1] *= alpha[0];
              acc[c][2] *= alpha[1]; acc[c][3] *= alpha[1];
            }
          }
          uint32_t pf[2][4];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float neg = m[y] == -INFINITY ? 0.f : -m[y];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const float a = ex2(fmaf(s[h][2 * y], p.scale_log2, neg)), b = ex2(fmaf(s[h][2 * y + 1], p.scale_log2, neg));
              l[y] += a + b;
              pf[h >> 1][2 * (h & 1) + y] = pack2(a, b);
            }
          }
          // ---- V rows that no row sees hold anything: 0 * NaN would poison the product
          if (edge) {
            const int tok = t0 + lane;
            if (tok >= end || (tok < low && tok >= p.sinks)) {
              unsigned char* dst = smem + stage * stage_bytes + v_off + row_at(r + lane, HV);
#pragma unroll 1
              for (int c = 0; c < HV * 8; ++c)
                *reinterpret_cast<uint4*>(dst + (c >> 3) * half_at + (((c ^ lane) & 7) << 4)) = make_uint4(0, 0, 0, 0);
            }
            ptx::fence_proxy_async();  // before the next TMA write
            __syncwarp();
          }
          // ---- O += P V, 16 tokens at a time
          const uint32_t v_at = base + v_off + v_lane + (r ? v_32 : 0u);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int c = 0; c < kD / 16; ++c) {
              uint32_t b[4];
              ptx::ldmatrix_x4_trans((v_at + h * v_16 + (c / 4) * half_at) ^ ((c % 4) << 5), b);
              ptx::mma_bf16_16816(acc[2 * c], pf[h], b[0], b[1]);
              ptx::mma_bf16_16816(acc[2 * c + 1], pf[h], b[2], b[3]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(empty0 + 8 * stage);
        step();
      }
      // ---- the segment's result: sums over the four lanes of a row, then the slices pairwise, the upper half to the lower
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        l[y] += __shfl_xor_sync(0xffffffffu, l[y], 1);
        l[y] += __shfl_xor_sync(0xffffffffu, l[y], 2);
      }
#pragma unroll 1
      for (int h = slices >> 1; h > 0; h >>= 1) {
        const int at = ((slice & (h - 1)) << mshift) | mt;
        if (slice >= h && slice < 2 * h) {
#pragma unroll
          for (int c = 0; c < kD / 8; ++c) sc.o[at][c][lane] = make_float4(acc[c][0], acc[c][1], acc[c][2], acc[c][3]);
          if (t4 == 0) {
            sc.ml[at][g8] = make_float2(m[0], l[0]);
            sc.ml[at][g8 + 8] = make_float2(m[1], l[1]);
          }
        }
        ptx::named_barrier_sync(1, kWarps * 32);
        if (slice < h) {
          float wa[2], wb[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float2 o = sc.ml[at][g8 + 8 * y];
            const float top = fmaxf(m[y], o.x), ref = top == -INFINITY ? 0.f : top;
            wa[y] = ex2(m[y] - ref);
            wb[y] = ex2(o.x - ref);
            l[y] = l[y] * wa[y] + o.y * wb[y];
            m[y] = top;
          }
#pragma unroll
          for (int c = 0; c < kD / 8; ++c) {
            const float4 o = sc.o[at][c][lane];
            acc[c][0] = fmaf(o.x, wb[0], acc[c][0] * wa[0]);
            acc[c][1] = fmaf(o.y, wb[0], acc[c][1] * wa[0]);
            acc[c][2] = fmaf(o.z, wb[1], acc[c][2] * wa[1]);
            acc[c][3] = fmaf(o.w, wb[1], acc[c][3] * wa[1]);
          }
        }
        ptx::named_barrier_sync(1, kWarps * 32);
      }
      if (slice == 0) {
        const bool whole = w.flags & kSegWhole, to_out = whole && w.dst == kDstOut;
        const bool as_f32 = !to_out || p.out_is_f32;
        float* dst32 = to_out ? reinterpret_cast<float*>(p.out) : whole ? p.buffer[w.dst - 1].o : p.list.part_o;
        const long long prow = (2LL * blockIdx.x + ((w.flags & kSegFirst) ? 1 : 0)) * p.list.slot_rows + group * used;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int lr = r0 + g8 + 8 * y;
          if (!active || lr >= used) continue;
          const float inv = l[y] != 0.f ? 1.f / l[y] : 0.f, lse2 = l[y] != 0.f ? m[y] + log2f(l[y]) : -INFINITY;
          const long long row = whole ? out_row(lr) : prow + lr;
          if (t4 == 0) {
            if (!whole) p.list.part_lse[row] = lse2;
            else if (!to_out) p.buffer[w.dst - 1].lse[row] = lse2;
            else if (p.lse) p.lse[row] = lse2 * kLn2;
          }
#pragma unroll
          for (int c = 0; c < kD / 8; ++c) {
            const float a = acc[c][2 * y] * inv, b = acc[c][2 * y + 1] * inv;
            if (as_f32) *reinterpret_cast<float2*>(dst32 + row * kD + c * 8 + 2 * t4) = make_float2(a, b);
            else *reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(p.out) + row * kD + c * 8 + 2 * t4) = pack2(a, b);
          }
        }
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(seg_empty0 + 8 * (segs % kSegRing));
    }
    if (dead) report(p.dev_status, DIFFQKV_ERR_TIMEOUT);
  }
  ptx::grid_dependency_wait();  // see extend.cu: the second of the two kernels ends behind the first
}

}  // namespace

cudaError_t launch_extend_few(const CUtensorMap& mk, const CUtensorMap& mv, const void* q, ExtendParams p, int d_qk, int d_v,
                              int blocks, cudaStream_t stream) {
  using Fn = void (*)(const CUtensorMap, const CUtensorMap, const __nv_bfloat16*, const ExtendParams);
  const Fn fn = d_v == 64 ? extend_few_kernel<64, 64> : d_qk == 128 ? extend_few_kernel<128, 128> : extend_few_kernel<64, 128>;
  if (p.box_tok > kFewT) p.box_tok = kFewT;
  const int stage = kFewT * 2 * (p.k_parts * d_qk + p.v_parts * d_v);
  const int scratch = d_v == 64 ? (int)sizeof(Scratch<64>) : (int)sizeof(Scratch<128>);
  p.few_stages = (kMaxSmem - scratch) / stage;
  if (p.few_stages > kMaxStages) p.few_stages = kMaxStages;
  const int smem = p.few_stages * stage + scratch;
  const cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (err != cudaSuccess) return err;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t launched = cudaLaunchKernelEx(&cfg, fn, mk, mv, static_cast<const __nv_bfloat16*>(q), p);
  if (launched == cudaSuccess) count_launch();
  return launched;
}

}  // namespace diffqkv
