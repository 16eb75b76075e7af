// Attention of a tree of drafted tokens over the compressed cache (stief_tree_attention).  Node i of sequence b attends the
// context, positions 0 .. ctx_b - 1, and the drafted nodes in its mask row, whose rows are cached behind the context:
//   out_i = softmax(q_i' K_down[S_i]^T / sqrt(128)) V_down[S_i] U_v^T,   q_i' = q_i U_k.
// A tree has few query rows (nodes x heads of the group) and a long cache, so the cache is what has to be streamed: every
// row of it once per (sequence, KV head).  Three launches, each started while the one before it still runs:
//   project_kernel   q' = q U_k in fp32, kept as two bf16 terms (value and remainder, 16 significant bits: with the value alone
//                    the scores' error was as large as all others together), rows packed per (sequence, KV head)
//   tree_kernel      one persistent CTA per SM.  A unit is (sequence, KV head, up to 256 query rows,
//                    128 at key ranks above 64, whose Q' fills the shared memory); the units' blocks of 128
//                    positions lie end to end on one axis (each unit preceded by kPad blocks' worth of start-up cost) and
//                    every CTA takes an equal range of it, so that ragged lengths and few units fill the GPU alike.  What a
//                    CTA finds in one unit, a segment, leaves a partial result: unnormalised mix, reference, sum.
//   combine_kernel   joins the segments of 16 rows (log-sum-exp), normalises, back-projects and writes them.
//
// tree_kernel, 384 threads: two row tiles of 128 rows.  With at most 128 rows both tiles hold the SAME rows and take
// alternate blocks (two independent softmax streams, joined like segments): one stream is bound by the latency of its chain
// scores -> softmax -> P V.  With more, each tile has its own rows and both use every block.
// TMEM gives a warp 32 lanes, so 32 rows would keep one warp of four at work; with at most 64 or 32 rows a tile therefore holds
// them twice or four times, each copy takes its half or quarter of a block's columns (P is zero elsewhere, the wasted products
// cost nothing here) and is joined with the others when the segment ends.
//   warps 0-3, 4-7  softmax of tile 0 / 1, thread = row = TMEM lane, 128 scores in registers; warps without rows skip
//   warps 8, 11     cache pages by TMA into a ring of blocks, two pages of keys and two of values of one KV head; Q' tiles
//   warps 9, 10     MMA issue, a warp per tile:  S = Q' K^T (N = 128; Q' as value and remainder), O += P V (N = r_v)
// TMEM (512 columns): per tile 128 for S and 128 for O; with r_v <= 64 half of O's are free and hold P, and the next scores are
// made while the softmax still works; with more P lies over S.  Everything else follows the prompt kernel (stief_prompt.cu).
//
// What bounds it.  Up to 64 rows the memory: 4 sequences of 32768 tokens at ranks 64/64 are 269 MB, 42 us at the measured copy
// rate; 8 / 16 nodes of 4 heads take 71 / 75 us, of which the stream takes 45, the first scores come 7 us after the start
// (projection, launch, and the first pages behind those of all other SMs), CTAs end over 8 us, and joining takes 6.  From 65
// rows on the softmax, of which two warps share a scheduler: loading 32 rows of 128 scores, their maximum, exponentials and P
// take 3250 cycles when the two are half a step apart (1024 each of the special-function units') and 4040 side by side; 32
// nodes take 87 us and 64 nodes, 256 rows, 127 us.  At ranks 128/128, 537 MB and a ring of two blocks, 16 / 64 nodes take 138 / 260 us.
// These are bursts of five calls replayed from a graph, at 1965 MHz; without pauses the power limit brings the clock down, and
// 8 / 16 / 32 / 64 nodes called one by one take 74 / 76 / 86 / 132 us at 1890 / 1852 / 1875 / 1777 MHz.
//
// The steps to this form were timed in such bursts, before far scores (stief_softmax.cuh, 1 to 2 %), on a card where 32 / 64 nodes
// took 80 / 117 us: with a ring of three or four blocks instead of five 32 nodes took 94 and 86.  An issuing warp runs beside two
// softmax warps and needs 100 to 180 cycles for a wait that is over already: with a barrier per page and P in two halves it was
// the slowest part (64 nodes 136 us).  Tried and slower: a share of the exponentials as a
// polynomial (64 nodes 136 and 149 against 118 us for an eighth and a quarter), turns of the softmax warps themselves (145 to
// 151 against 134 to 141), pages brought to L2 one to four blocks ahead of the ring (32 nodes 86 to 88 against 80: a fetching
// warp's time), waits tested ahead of the work before them (64 nodes 117 to 120 against 117).
#pragma once

#include <cfloat>

#include "stief_softmax.cuh"
#include "stief_tree.h"
#include "stief_umma.cuh"

namespace stief {
namespace tree {

using namespace tc;

constexpr int kThreads = 384;
constexpr int kRows = 128;                      // rows of a tile
constexpr int kBlock = 128;                     // positions of a block: two pages
constexpr int kSmemLimit = 232448;
constexpr int kHeadBytes = 5120;                // prefix sums (4352), barriers (512)
constexpr int kJoinBytes = 14336;               // joining the copies of rows, per tile 1024 of references and sums, 6144 of values
__host__ __device__ constexpr int join_bytes(int RV) { return RV <= 64 ? kJoinBytes : 0; }
constexpr int kMaxStages = 12;
constexpr int kTmemCols = 512;
constexpr float kRescaleLog2 = 8.0f;
// The looks at a barrier that nothing depends on: how many at most, and from how many blocks of a segment on the tiles are
// paced.  Only tiles of their own rows are: with alternate blocks the ring's order already keeps them apart (paced, on the same
// card, 32 nodes 78 against 80 us, but 26 ragged 98 against 97 and 8 nodes 70 against 69).
constexpr int kPacePolls = 64, kPacedBlocks = 8, kLooks = 1 << 12;

// Sequence b as every kernel sees it
struct Seq {
  int ctx, n, blocks, units;                    // context, nodes, blocks of positions, units per KV head (0: nothing to do)
};
__device__ __forceinline__ Seq sequence(const Args& a, int b) {
  Seq s;
  s.ctx = a.Bt.seq_lens[b];
  s.n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.n_q) : a.n_q;
  const bool fits = s.ctx >= 0 && s.ctx <= (1 << 30) && ((long long)s.ctx + s.n + kPage - 1) / kPage <= a.Bt.max_pages;      // positions are counted in int
  if (!fits && s.n > 0) report(a.status, STIEF_ERR_BOUNDS);
  if (!fits) s.n = 0;
  s.blocks = s.n > 0 ? (s.ctx + s.n + kBlock - 1) / kBlock : 0;
  s.units = (s.n * a.L.G + a.unit_rows - 1) / a.unit_rows;
  return s;
}
__device__ __forceinline__ int sequence_cost(const Args& a, const Seq& s) { return a.L.Hkv * s.units * (s.blocks + kPad); }
// First position of the axis that CTA i of n takes
__device__ __forceinline__ int range_start(int i, int n, int total) { return (int)((long long)i * total / n); }
__device__ __forceinline__ int cta_count(const Args& a, int total) { return min(a.n_cta, total); }

// Copies of the rows in a tile.  With r_v > 64 a page takes the memory so long that one copy keeps up; and a segment of
// one block per tile gains less from them (0.6 us) than joining them costs (2.8 us; at five blocks it is the other way round).
constexpr int kFewBlocks = 2;
__device__ __forceinline__ int replicas_of(int rows, int r_v, int blocks) { return r_v > 64 || blocks <= kFewBlocks ? 1 : rows <= 32 ? 4 : rows <= 64 ? 2 : 1; }

struct Segment {
  int b, h, unit, slot;                         // unit: row block within the (sequence, KV head)
  int ctx, n, rows;                             // rows of the unit
  int j0, cnt;                                  // blocks [j0, j0 + cnt)
  int replicas;                                 // copies of the rows in a tile (see tree_kernel): 1, 2 or 4
  bool dual, valid;
};

struct Walk {
  int pos, hi, b, cta;
  __device__ __forceinline__ void start(const Args& a, const int* pref) {
    const int total = pref[a.Bt.B], n = cta_count(a, total);
    cta = blockIdx.x;
    pos = hi = b = 0;
    if (cta < n) {
      pos = range_start(cta, n, total);
      hi = range_start(cta + 1, n, total);
    }
  }
  __device__ __forceinline__ Segment next(const Args& a, const int* pref) {
    Segment g;
    g.valid = false;
    g.cnt = 0;
    while (pos < hi) {
      while (pref[b + 1] <= pos) ++b;
      const Seq s = sequence(a, b);
      const int len = s.blocks + kPad, r = pos - pref[b], u = r / len, first = pref[b] + u * len;
      const int end = min(hi, first + len);
      g.j0 = max(pos - first - kPad, 0);
      g.cnt = end - first - kPad - g.j0;
      pos = end;
      if (g.cnt <= 0) continue;
      g.b = b;
      g.h = u / s.units;
      g.unit = u - g.h * s.units;
      g.slot = cta + (b * a.L.Hkv + g.h) * a.max_units + g.unit;
      g.ctx = s.ctx;
      g.n = s.n;
      g.rows = min(s.n * a.L.G - g.unit * a.unit_rows, a.unit_rows);
      g.dual = g.rows <= kRows;
      g.replicas = replicas_of(g.rows, a.L.r_v, g.cnt);
      g.valid = true;
      break;
    }
    return g;
  }
};

// Blocks of a segment that tile t works on
__device__ __forceinline__ int tile_blocks(const Segment& g, int t) { return g.dual ? (g.cnt + 1 - t) >> 1 : g.cnt; }

// 32 positions from node index s on (negative: context): which of them a row with mask words `m` sees
__device__ __forceinline__ uint32_t seen32(const uint32_t* m, int s, int n) {
  if (s <= -32) return ~0u;
  if (s >= n) return 0u;
  uint32_t w;
  if (s < 0) {
    w = m[0] << -s;
  } else {
    const int i = s >> 5;
    w = __funnelshift_r(m[i], (i + 1) * 32 < n ? m[i + 1] : 0u, s & 31);
  }
  if (n - s < 32) w &= (1u << (n - s)) - 1u;
  return s < 0 ? w | ((1u << -s) - 1u) : w;
}

template <int RK, int RV>
__global__ void __launch_bounds__(kThreads, 1)
tree_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmQ32, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const Args a) {
  constexpr Blocks bk{(RK % 64 == 0) ? 64 : (RK % 32 == 0) ? 32 : 16, 0, 0, 0}, bv{(RV % 64 == 0) ? 64 : (RV % 32 == 0) ? 32 : 16, 0, 0, 0};
  constexpr int kSpanK = 2 * bk.bw, kSpanV = 2 * bv.bw, kNbK = RK / bk.bw, kNbV = RV / bv.bw;       // see Blocks in stief_tc.cuh
  constexpr int kLayK = kSpanK == 128 ? 2 : kSpanK == 64 ? 4 : 6, kLayV = kSpanV == 128 ? 2 : kSpanV == 64 ? 4 : 6;
  constexpr bool kOwnP = RV <= 64;              // P has TMEM columns of its own: 192 .. 255 of the tile's
  constexpr int kColP = kOwnP ? 192 : 0;
  constexpr int kBlockK = kBlock * RK * 2, kBlockV = kBlock * RV * 2, kQBytes = kRows * RK * 2;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int* pref = reinterpret_cast<int*>(smem);
  uint8_t* ctrl_ptr = smem + 4352;
  const uint32_t ctrl = smem_u32(ctrl_ptr);
  const uint32_t q_smem = smem_u32(smem) + kHeadBytes + join_bytes(RV), ring = q_smem + a.q_regions * kQBytes;
  const int nst = a.nst;
  const uint32_t ring_v = ring + nst * kBlockK; // the blocks' keys, then their values, each one operand of 128 rows
  uint8_t* ring_v_ptr = smem + kHeadBytes + join_bytes(RV) + a.q_regions * kQBytes + nst * kBlockK;
  auto full_bar = [&](int s) { return ctrl + s * 8; };
  auto empty_bar = [&](int s) { return ctrl + (12 + s) * 8; };
  const uint32_t q_full = ctrl + 24 * 8, q_empty = ctrl + 26 * 8;
  auto s_full = [&](int t) { return ctrl + (28 + t) * 8; };
  auto p_full = [&](int t, int half) { return ctrl + (30 + 2 * t + half) * 8; };
  auto o_full = [&](int t) { return ctrl + (34 + t) * 8; };
  auto s_free = [&](int t) { return ctrl + (36 + t) * 8; };
  auto p_free = [&](int t) { return ctrl + (38 + t) * 8; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl_ptr + 40 * 8);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl_ptr + 40 * 8 + 4);
  int32_t* status = a.status;
  launch_dependents();
  if (q_smem & 1023u) {                         // the swizzled tiles need it; dynamic shared memory starts there
    report(status, STIEF_ERR_CUDA);
    return;
  }

  for (int b = tid; b < a.Bt.B; b += kThreads) pref[b + 1] = sequence_cost(a, sequence(a, b));
  if (tid == 0) {
    pref[0] = 0;
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(full_bar(s), 2);                // a block's keys and its values
      mbar_init(empty_bar(s), 2);               // one arrival from each tile's issuer
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s_full(t), 1);
      mbar_init(p_full(t, 0), 4);
      mbar_init(p_full(t, 1), 4);
      mbar_init(o_full(t), 1);
      mbar_init(s_free(t), 4);
      mbar_init(p_free(t), 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 2);                      // one arrival from each tile's issuer
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 8) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
  __syncthreads();
  if (warp == 0) {                              // running sums of the costs
    int carry = 0;
    for (int b0 = 0; b0 < a.Bt.B; b0 += 32) {
      int x = b0 + lane < a.Bt.B ? pref[b0 + lane + 1] : 0;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      if (b0 + lane < a.Bt.B) pref[b0 + lane + 1] = carry + x;
      carry += __shfl_sync(0xffffffffu, x, 31);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  Walk walk;
  walk.start(a, pref);
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");      // 384 x 168 registers at launch = 256 x 200 + 128 x 104
    if (warp == 8 || warp == 11) {
      // ---------------------------------------------------------------------------------------- cache pages, Q' tiles
      // One warp fetches the K halves of the pages, the other the V halves (a warp needs some 500 cycles per page for both,
      // which is what a page of ranks 48/48 may take in all) and the queries.  The first of these come from the kernel before,
      // which is over about when this one starts; later ones wait for their place, and pages go ahead of them meanwhile.
      const bool keys = warp == 8;
      if (lane == 0) {
        tma_prefetch_desc(keys ? &tmK : &tmV);
        if (!keys) tma_prefetch_desc(&tmQ);
      }
      int st = 0, use = 0, kt = 0;                              // ring position, segments so far
      const int parts = a.L.U_k ? 2 : 1, q_rows = a.Bt.B * a.L.Hkv * (a.n_q * a.L.G);         // given queries have no remainder
      bool first_q = true;
      for (Segment g = walk.next(a, pref); g.valid; g = walk.next(a, pref)) {
        const int first = 2 * g.j0, pages = min(2 * g.cnt, (g.ctx + g.n + kPage - 1) / kPage - first);
        const int* bt = a.Bt.block_table + (size_t)g.b * a.Bt.max_pages + first;
        bool q_due = !keys;                                     // the segment's queries are still to be sent
        auto send_queries = [&](bool wait) {                    // lane 0
          if (first_q) {
            grid_dependency_wait();                             // project_kernel has written them, with ordinary stores
            asm volatile("fence.proxy.async;" ::: "memory");
            first_q = false;
          }
          if (kt > 0) {
            if (wait) mbar_wait(q_empty, (kt - 1) & 1, abort_flag, status);
            else if (!mbar_test_wait(q_empty, (kt - 1) & 1)) return;
          }
          ++kt;
          q_due = false;
          const int row0 = (g.b * a.L.Hkv + g.h) * (a.n_q * a.L.G) + g.unit * a.unit_rows, wrap = kRows / g.replicas, tiles = g.dual ? 1 : 2;
          mbar_arrive_expect_tx(q_full, tiles * parts * kQBytes);
          for (int t = 0; t < tiles; ++t)
            for (int x = 0; x < parts; ++x) {
              const int row = row0 + t * kRows + x * q_rows;
#pragma unroll
              for (int i = 0; i < kNbK; ++i) {
                const uint32_t dst = q_smem + (2 * t + x) * kQBytes + i * kRows * kSpanK;
                if (g.replicas == 1) tma_load_2d(dst, &tmQ, i * bk.bw, row, q_full);
                else
                  for (int r = 0; r < kRows; r += 32) tma_load_2d(dst + r * kSpanK, &tmQ32, i * bk.bw, row + r % wrap, q_full);
              }
            }
        };
        int ids = lane < pages ? bt[lane] : 0;
        if (lane == 0 && q_due && first_q) send_queries(true);
        for (int j0 = 0; j0 < pages; j0 += 32) {
          const int nxt = j0 + 32 + lane < pages ? bt[j0 + 32 + lane] : 0;     // a batch of page ids ahead
          const int cnt = min(32, pages - j0);
          for (int jj = 0; jj < cnt; jj += 2) {
            const int here = min(2, cnt - jj);
            int pg[2] = {__shfl_sync(0xffffffffu, ids, jj), __shfl_sync(0xffffffffu, ids, jj + 1)};
            if (lane == 0) {
              if (use > 0) {
                if (q_due) send_queries(!mbar_test_wait(empty_bar(st), (use - 1) & 1));        // no block to fetch: wait for the queries' place
                mbar_wait(empty_bar(st), (use - 1) & 1, abort_flag, status);
              }
              const uint32_t dst = keys ? ring + st * kBlockK : ring_v + st * kBlockV;
              mbar_arrive_expect_tx(full_bar(st), (keys ? kBlockK : kBlockV) / 2 * here);
#pragma unroll
              for (int p = 0; p < 2; ++p) {
                if (p >= here) continue;
                if (pg[p] < 0 || pg[p] >= a.L.num_pages) {
                  report(status, STIEF_ERR_BOUNDS);
                  pg[p] = 0;
                }
                const int row = (pg[p] * a.L.Hkv + g.h) * kPage;
                if (keys) {
#pragma unroll
                  for (int i = 0; i < kNbK; ++i) tma_load_2d(dst + (i * kBlock + p * kPage) * kSpanK, &tmK, i * bk.bw, row, full_bar(st));
                } else {
#pragma unroll
                  for (int i = 0; i < kNbV; ++i) tma_load_2d(dst + (i * kBlock + p * kPage) * kSpanV, &tmV, i * bv.bw, row, full_bar(st));
                }
              }
              if (++st == nst) {
                st = 0;
                ++use;
              }
            }
          }
          ids = nxt;
        }
        if (lane == 0 && q_due) send_queries(true);
        __syncwarp();
      }
      if (!keys && first_q) grid_dependency_wait();             // a CTA without work, too, ends after the kernel before it
    } else {
      // ---------------------------------------------------------------------------------------- MMA issue, tile t
      const int t = uniform(warp) - 9;
      const uint32_t tmem_u = uniform(tmem_base) + t * 256, ring_u = uniform(ring), ring_v_u = uniform(ring_v), ctrl_u = uniform(ctrl);
      const uint32_t q_u = uniform(q_smem);
      const int parts = a.L.U_k ? 2 : 1;
      uint32_t qa = 0;                                                         // this tile's Q' operand, its remainder one region on
      constexpr uint32_t kHiK = (uint32_t)((((uint64_t)(8 * kSpanK >> 4) << 32) | (1ull << 46) | ((uint64_t)kLayK << 61)) >> 32);
      constexpr uint32_t kHiV = (uint32_t)((((uint64_t)(8 * kSpanV >> 4) << 32) | (1ull << 46) | ((uint64_t)kLayV << 61)) >> 32);
      const uint32_t id_qk = idesc_bf16_f32(kRows, kPage), id_qk2 = idesc_bf16_f32(kRows, kBlock), id_pv = idesc_bf16_f32_bmn(kRows, RV);
      auto bar = [&](int i) { return ctrl_u + i * 8; };                        // as numbered above
      int st = 0, use = 0, kt = 0, n = 0, others = 0;                          // ring position of the next block; blocks of the other tile
      // Both tiles see every block land, in order, the other tile's too, and both give it back: a barrier's parity tells a slot's
      // block from the one before and the one behind it only to who keeps step with them.  `skip` blocks of the other tile, then
      // this one's, whose slot is kept; without `wait` only as far as they have landed, and whether that was all.
      int skip = 0, cur = 0, nxt = 0;
      auto step = [&]() {
        if (++st == nst) {
          st = 0;
          ++use;
        }
      };
      auto observe = [&](bool wait, bool own) {
        for (; skip > 0; --skip) {
          if (wait) mbar_wait_warp(bar(st), use & 1, abort_flag, status);
          else if (!__all_sync(0xffffffffu, mbar_test_wait(bar(st), use & 1))) return false;
          if (lane == 0) mbar_arrive(bar(12 + st));
          __syncwarp();
          step();
        }
        if (!own) return true;
        if (wait) mbar_wait_warp(bar(st), use & 1, abort_flag, status);
        else if (!__all_sync(0xffffffffu, mbar_test_wait(bar(st), use & 1))) return false;
        nxt = st;
        step();
        return true;
      };
      // The tiles' scores are issued in turn, each when the other's last have been read: the softmax of one then loads and looks for
      // its maximum while the other's has the special-function units (64 nodes 133 -> 118 us).  Only pace, not order: the look
      // has an end, and a wrong answer (a parity is one bit) costs nothing but the shift.
      auto pace = [&](int phase) {
        for (int i = 0; i < kPacePolls && !__all_sync(0xffffffffu, mbar_test_wait(bar(37 - t), phase & 1)); ++i) {
        }
      };
      auto score = [&](int pages, int slot, bool last) {                       // S = Q' K^T, 64 columns per page
        const uint32_t ka = desc_lo(16, ring_u + slot * kBlockK), idesc = pages == 2 ? id_qk2 : id_qk;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int k = 0; k < RK / 16; ++k) {
            if (x >= parts) continue;
            constexpr int kPer = bk.bw / 16;                                   // K steps per swizzled block of columns
            const uint32_t off = (uint32_t)((k / kPer) * kRows * kSpanK + (k % kPer) * 32) >> 4;           // kRows == kBlock
            umma_ss(tmem_u, qa + x * (kQBytes >> 4) + off, kHiK, ka + off, kHiK, idesc, x > 0 || k > 0 ? 1u : 0u);
          }
        umma_commit_warp(bar(28 + t));
        if (last) umma_commit_warp(bar(26));
      };
      for (Segment g = walk.next(a, pref); uniform((int)g.valid); g = walk.next(a, pref)) {
        const int cnt = uniform(g.cnt), j0 = uniform(g.j0), len = uniform(g.ctx + g.n);
        const bool dual = uniform((int)g.dual) != 0;
        const int pages = min(2 * cnt, (len + kPage - 1) / kPage - 2 * j0);    // pages of the segment
        const int steps = dual ? (cnt + 1 - t) >> 1 : cnt, stride = dual ? 2 : 1, at = dual ? t : 0;
        if (steps == 0) {                                                      // a lone block: the other tile's
          skip = cnt;
          observe(true, false);
          mbar_wait_warp(bar(24), kt & 1, abort_flag, status);
          ++kt;
          others += cnt;
          if (lane == 0) mbar_arrive(bar(26));
          __syncwarp();
          continue;
        }
        qa = desc_lo(16, q_u + (dual ? 0 : 2 * t) * kQBytes);
        int here = min(2, pages - 2 * at);
        skip = at;
        observe(true, true);
        cur = nxt;
        mbar_wait_warp(bar(24), kt & 1, abort_flag, status);
        tc_fence_after();
        const bool paced = kOwnP && !dual && cnt >= kPacedBlocks;
        const int others_steps = dual ? (cnt + t) >> 1 : cnt;
        if (paced && t == 1) pace(others);
        score(here, cur, steps == 1);
        for (int s = 0; s < steps; ++s) {
          // Where the next block has landed already, all that its scores need is dealt with ahead of P, so that from P on only
          // products are issued; where it has not, P is not kept waiting for it (nor the slot that its product gives back:
          // with three blocks in the ring that alone doubled the time).
          bool early = false;
          int want = 0;
          if (s + 1 < steps) {
            want = min(2, pages - 2 * (at + (s + 1) * stride));
            skip = dual ? 1 : 0;                                               // the other tile's block lies between
            for (int i = 0; i < kLooks; ++i) {                                 // while P is not there yet, scores may be issued at any time
              early = observe(false, true);
              if (early || !kOwnP || __all_sync(0xffffffffu, mbar_test_wait(bar(31 + 2 * t), n & 1))) break;
            }
            if (early && kOwnP) {                                              // S is free once it has been read
              mbar_wait_warp(bar(36 + t), n & 1, abort_flag, status);
              if (paced && s + t < others_steps) pace(others + s + t);
              tc_fence_after();
              score(want, nxt, s + 2 == steps);
            }
          }
          const uint32_t va = desc_lo(kBlock * kSpanV, ring_v_u + cur * kBlockV);
#pragma unroll
          for (int k = 0; k < kBlock / 16; ++k) {                              // O += P V
            if (kOwnP ? k == 0 : k % 4 == 0) {
              mbar_wait_warp(bar(30 + 2 * t + (kOwnP || k > 0 ? 1 : 0)), n & 1, abort_flag, status);
              tc_fence_after();
            }
            if (k < 4 || here == 2) umma_ts(tmem_u + 128, tmem_u + kColP + 8 * k, va + (uint32_t)(k * 16 * kSpanV >> 4), kHiV, id_pv, s > 0 || k > 0 ? 1u : 0u);
          }
          if (kOwnP) umma_commit_warp(bar(38 + t));
          if (s + 1 == steps) {
            umma_commit_warp(bar(34 + t));
            umma_commit_warp(bar(12 + cur));
          } else if (!early) {
            umma_commit_warp(bar(12 + cur));
            observe(true, true);
            if (kOwnP) mbar_wait_warp(bar(36 + t), n & 1, abort_flag, status); // S has been read long ago
            tc_fence_after();
            score(want, nxt, s + 2 == steps);
          } else {
            if (!kOwnP) score(want, nxt, s + 2 == steps);
            umma_commit_warp(bar(12 + cur));
          }
          ++n;
          here = want;
          cur = nxt;
        }
        if (dual) {                                                            // blocks behind this tile's last
          skip = cnt - 1 - (at + (steps - 1) * 2);
          observe(true, false);
        }
        others += others_steps;
        ++kt;
      }
    }
  } else {
    // ------------------------------------------------------------------------------------------ softmax, partial results
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    const int t = warp >> 2, q4 = warp & 3, lane_row = 32 * q4 + lane;
    const uint32_t t_s = tmem_base + ((uint32_t)(32 * q4) << 16) + t * 256, t_o = t_s + 128, t_p = t_s + kColP;
    const float c = kLog2e * rsqrtf((float)kD);
    int n = 0, kt = 0, ring_block = 0;                          // blocks and segments of this tile so far; blocks of both
    auto arrive_warp = [&](uint32_t bar) {
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    for (Segment g = walk.next(a, pref); g.valid; g = walk.next(a, pref)) {
      const int len = g.ctx + g.n, block0 = ring_block;
      ring_block += g.cnt;
      const int steps = tile_blocks(g, t);
      if (steps == 0) continue;
      const int wrap = kRows / g.replicas, replica = lane_row / wrap, row = lane_row - replica * wrap;
      const int base_row = g.dual ? 0 : t * kRows, urow = base_row + row;
      const bool row_valid = urow < g.rows, warp_live = base_row + row - lane < g.rows;
      const int node = min(g.unit * a.unit_rows + urow, g.n * a.L.G - 1) / a.L.G;
      const uint32_t* mask = a.mask + ((size_t)g.b * a.n_q + node) * a.mask_words;
      float m_ref = 0.f, l = 0.f;
      // One block, of whose 128 columns this thread takes kCols: all of them, or with the rows there twice or four times
      // its copy's half or quarter, P being zero elsewhere.
      auto block = [&](auto cols_tag, int s_i, int p0) {
        constexpr int kCols = decltype(cols_tag)::value, kWords = kCols / 2;
        static_assert(kCols == 128 || kOwnP, "copies have P's own columns");
        const int col0 = kCols == 128 ? 0 : replica * kCols;
        uint32_t sv[kCols];
        float* s = reinterpret_cast<float*>(sv);
#pragma unroll
        for (int i = 0; i < kCols / 32; ++i) tmem_ld32(t_s + col0 + 32 * i, sv + 32 * i);
        tmem_ld_wait();
        if (kOwnP) {
          tc_fence_before();
          arrive_warp(s_free(t));
        }
        if (p0 + kBlock > g.ctx) {                              // the drafted nodes, and what lies behind them
#pragma unroll
          for (int w = 0; w < kCols / 32; ++w) {
            const uint32_t seen = seen32(mask, p0 + col0 + 32 * w - g.ctx, g.n);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!((seen >> i) & 1u)) s[32 * w + i] = -INFINITY;
          }
        }
        float mx;
        {
          float m[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
          for (int i = 4; i < kCols - 4; i += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = max3(m[e], s[i + 2 * e], s[i + 2 * e + 1]);
          mx = fmaxf(max3(max3(m[0], s[kCols - 4], s[kCols - 3]), m[1], m[2]), max3(m[3], s[kCols - 2], s[kCols - 1]));
        }
        if (kOwnP && n > 0) {                                   // the product of the block before is complete
          mbar_wait(p_free(t), (n - 1) & 1, abort_flag, status);
          tc_fence_after();
        }
        if (s_i == 0) {
          m_ref = fmaxf(mx, -FLT_MAX);                          // a row that sees nothing here keeps p = 0 and l = 0
          l = 0.f;
        } else if (const bool grown = (mx - m_ref) * c > kRescaleLog2; __any_sync(0xffffffffu, grown)) {
          const float f = grown ? reference_weight(m_ref, mx, c) : 1.0f;    // a row's bits do not depend on its neighbours
          if (grown) m_ref = mx;
          l *= f;
#pragma unroll 1
          for (int c0 = 0; c0 < RV; c0 += 16) {                 // (where P lies over S, S implies that product)
            uint32_t v[16];
            tmem_ld16(t_o + c0, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
            tmem_st16(t_o + c0, v);
          }
        }
        if (kCols < 128 && s_i == 0) {                          // the other copies' columns, in P's own: once
          const uint32_t zero[16] = {};
#pragma unroll 1
          for (int w = 0; w < 64; w += 16)
            if (w / kWords != replica) tmem_st16(t_p + w, zero);
        }
        const float c_row = exponent_scale(m_ref, c);
        const uint64_t c2 = pack2(c_row, c_row), neg2 = pack2(-m_ref * c_row, -m_ref * c_row);
        uint64_t sum[2] = {0ull, 0ull};                         // pairs of +0
#pragma unroll
        for (int q = 0; q < kCols / 32; ++q) {                  // probabilities as bf16 pairs
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float x0, x1;
            unpack2(fma2(pack2(s[32 * q + 2 * i], s[32 * q + 2 * i + 1]), c2, neg2), x0, x1);
            const float e0 = fast_exp2(x0), e1 = fast_exp2(x1);
            sum[i & 1] = add2(sum[i & 1], pack2(e0, e1));
            pk[i] = pack_bf16(e0, e1);
          }
          tmem_st16(t_p + col0 / 2 + 16 * q, pk);
          if (!kOwnP && q == 1) {                               // the first page's may be used already
            tmem_st_wait();
            tc_fence_before();
            arrive_warp(p_full(t, 0));
          }
        }
        tmem_st_wait();
        tc_fence_before();
        arrive_warp(p_full(t, 1));
        float a0, a1;
        unpack2(add2(sum[0], sum[1]), a0, a1);
        l += a0 + a1;
      };
      for (int s_i = 0; s_i < steps; ++s_i, ++n) {
        const int j = g.dual ? 2 * s_i + t : s_i, p0 = (g.j0 + j) * kBlock;
        mbar_wait(s_full(t), n & 1, abort_flag, status);
        tc_fence_after();
        if (p0 + kBlock > len) {
          // Rows behind the sequence's end: whatever bits they have (NaN included) must not reach the accumulator through
          // 0 * x.  Every tile that uses the block zeroes them, up to the end of its last page.
          const int dead = len - p0, rows = (dead > kPage ? kBlock : kPage) - dead, idx = block0 + j, stg = idx % nst;
          mbar_wait(full_bar(stg), (idx / nst) & 1, abort_flag, status);
          uint8_t* v = ring_v_ptr + stg * kBlockV + dead * kSpanV;
          constexpr int kCpr = kSpanV / 16, kPerRow = RV / 8;
          for (int e = lane_row; e < rows * kPerRow; e += kRows) {
            const int r = e / kPerRow, ch = e % kPerRow;
            *reinterpret_cast<uint4*>(v + (ch / kCpr) * kBlock * kSpanV + r * kSpanV + (ch % kCpr) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async_smem();
        }
        if (!warp_live) {                                       // none of the warp's rows exists
          if (kOwnP) {                                          // not before the others have published the block before
            arrive_warp(s_free(t));
            if (n > 0) mbar_wait(p_free(t), (n - 1) & 1, abort_flag, status);
          }
          if (!kOwnP) arrive_warp(p_full(t, 0));
          arrive_warp(p_full(t, 1));
        } else if (!kOwnP || g.replicas == 1) {                 // copies only where r_v <= 64 (replicas_of)
          block(std::integral_constant<int, 128>{}, s_i, p0);
        } else if constexpr (kOwnP) {
          if (g.replicas == 2) block(std::integral_constant<int, 64>{}, s_i, p0);
          else block(std::integral_constant<int, 32>{}, s_i, p0);
        }
      }
      // ---- the segment's partial result, [slot][RV / 4][128 lanes] float4: a warp writes 512 contiguous bytes
      mbar_wait(o_full(t), kt & 1, abort_flag, status);
      ++kt;
      tc_fence_after();
      const size_t slot = (size_t)g.slot * 2 + t;
      float4* po = reinterpret_cast<float4*>(a.part_o) + slot * (RV / 4) * kRows + row;
      float2* pml = reinterpret_cast<float2*>(a.part_ml) + slot * kRows + row;
      float weight = 1.0f, top = m_ref, total_l = l;
      if (RV <= 64 && g.replicas > 1) {                         // a row's copies are joined here, 16 channels at a time
        uint8_t* join = smem + kHeadBytes + t * (kJoinBytes / 2);
        float2* copy_ml = reinterpret_cast<float2*>(join);      // [copy][row]
        float4* copy_o = reinterpret_cast<float4*>(join + 1024);        // [copy - 1][four channels][row]
        auto meet = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(1 + t) : "memory"); };
        copy_ml[lane_row] = make_float2(top, l);
        meet();
        for (int i = 0; i < g.replicas; ++i) top = fmaxf(top, copy_ml[i * wrap + row].x);
        total_l = 0.f;
        for (int i = 0; i < g.replicas; ++i) {
          const float2 x = copy_ml[i * wrap + row];
          total_l = fmaf(x.y, reference_weight(x.x, top, c), total_l);
        }
        weight = reference_weight(m_ref, top, c);
#pragma unroll 1
        for (int c0 = 0; c0 < RV; c0 += 16) {
          uint32_t v[16];
          tmem_ld16(t_o + c0, v);
          tmem_ld_wait();
          float* o = reinterpret_cast<float*>(v);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] *= weight;
          if (replica > 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) copy_o[((replica - 1) * 4 + i) * wrap + row] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          }
          meet();
          if (replica == 0) {
            for (int k = 0; k + 1 < g.replicas; ++k)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float4 x = copy_o[(k * 4 + i) * wrap + row];
                o[4 * i] += x.x;
                o[4 * i + 1] += x.y;
                o[4 * i + 2] += x.z;
                o[4 * i + 3] += x.w;
              }
            if (row_valid) {
#pragma unroll
              for (int i = 0; i < 4; ++i) po[(size_t)(c0 / 4 + i) * kRows] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
          }
          meet();
        }
      } else if (warp_live) {
#pragma unroll 1
        for (int c0 = 0; c0 < RV; c0 += 16) {
          uint32_t v[16];
          tmem_ld16(t_o + c0, v);
          tmem_ld_wait();
          if (row_valid) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              po[(size_t)(c0 / 4 + i) * kRows] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
          }
        }
      }
      if (replica == 0 && row_valid) *pml = make_float2(top, total_l);
      tc_fence_before();                                        // ordered before this tile's next P by the arrival that publishes it
    }
  }

  if (*abort_flag) let_copies_land();           // a wait ran out: nobody has waited for the ring's last copies
  tc_fence_before();
  __syncthreads();
  if (warp == 8) tmem_dealloc(tmem_base, kTmemCols);
}

struct Launch {
  Args a;
  CUtensorMap tmQ, tmQ32, tmK, tmV;         // tmQ32: boxes of 32 rows, for rows that a tile holds several times
  int grid, smem;
};

}  // namespace tree

// One launcher per key rank (each its own translation unit)
cudaError_t launch_tree_rk32(const tree::Launch& l, cudaStream_t st);
cudaError_t launch_tree_rk48(const tree::Launch& l, cudaStream_t st);
cudaError_t launch_tree_rk64(const tree::Launch& l, cudaStream_t st);
cudaError_t launch_tree_rk96(const tree::Launch& l, cudaStream_t st);
cudaError_t launch_tree_rk128(const tree::Launch& l, cudaStream_t st);

}  // namespace stief
