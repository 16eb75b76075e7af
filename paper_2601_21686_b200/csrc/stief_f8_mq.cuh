// Attention of several causal query rows per head over the 8-bit floating-point cache (chunked prefill, speculative decode):
//     out_i = softmax(q_i' (c_k S_k)[0..p_i]^T / sqrt(128)) (c_v S_v)[0..p_i] U_v^T,   q_i' = q_i U_k,
// on the 5th-generation tensor cores, in the form of stief_mq.cuh: the same work units (sequence, KV head, 256 query rows in two
// tiles of 128), the same split of a long page range into parts.  What the codes change:
//   operands   kind::f16 products want both operands in one 16-bit type, so every page is expanded once per CTA, for both
//              tiles, from codes to f16 (exact, one conversion per two codes), by warps of their own: they read the page's codes
//              from a ring that 1-D bulk copies fill and write the K and V blocks, swizzled as tcgen05.mma reads them, into the
//              ring of operands.  Value rows past the end of the sequence are written as zeros there, so that what
//              unspecified codes stand for (NaN) cannot reach the accumulator through 0 * x.
//   queries    Q' is rounded to f16 once (11 bits), each row first scaled by the power of two that brings its largest element to
//              2^11 .. 2^12: f16's range is no limit, and a row's factor goes into its exponents.
//   scales     powers of two.  The key scale joins a page's exponent factor.  The value scale 2^e joins the exponent itself: the
//              weight of a position is w = 2^(x + e - ref), ref going by the largest x + e of the row, so weights of pages
//              whose scales lie far apart keep their precision; the row sum takes w 2^-e under a reference of its own (both
//              references: kTopWeight in stief_f8.cuh).
//   weights    f16 (11 bits, where bf16 would leave 8), at most 2^15: the reference is moved when a row's largest has grown by
//              more than 2^8, and w = 2^7 at the reference.
// A step is a block of two pages, 128 positions: waits, TMEM round trips and reductions are paid once per 128 scores of a row.
// 512 threads, registers split by role (setmaxnreg):
//   warp 0        fetches the codes of the pages, keys and values of a page apart
//   warps 1, 2    MMA issue, one per tile (control flow and descriptors in uniform registers, stief_umma.cuh).  Up to r_v = 64 the
//                 weights have TMEM columns of their own and the next block's scores are issued ahead of P V; above, P lies
//                 over the scores and the next scores follow P V
//   warps 4-11    softmax and epilogue, four per tile; thread = row = TMEM lane
//   warps 12-15   fill the ring of operands: expand the pages; raw queries, U_k and U_v come straight into it by TMA
// TMEM, per tile 256 columns: scores 0-127 (also Q' at the start of a unit and OUT at its end), P 128-191 and O 192-255, or O 128-255.
// Measured (32 query heads over 8): 2048 tokens over 16384 at ranks 64/64 553 to 563 us with scales that vary from page to page and 525
// with one (465 and 495 TFLOP/s), 96/128 592 and 558, 128/128 617 and 582 (893); 512 over 8192 94 (two parts), 256 over 4096 41 (four).
// A step of two pages for both tiles takes 2.1 to 2.4 us: the softmax of 2 x 128 x 128 scores, half of it on the special-function units,
// then the waits between the roles; the tensor pipe is busy for a fifth (64/64) to two fifths of it.  A unit costs another 8 to 10 us for its
// queries, its first page and its epilogue.  (Scores with a standard deviation of 72 in base 2 move the accumulators in most steps: 580,
// 694 and 886 us.)
// Every wait is bounded (see mbar_wait): on a timeout the status word says so, later waits return at once, every role walks
// to the end of its loops and TMEM is released.
#pragma once

#include "stief_f8.cuh"
#include "stief_mq.cuh"
#include "stief_umma.cuh"

namespace stief {
namespace f8mq {

using namespace tc;

constexpr int kThreads = 512;
constexpr int kRows = mq::kRows;
constexpr int kBlock = 2 * kPage;                // positions per step
constexpr int kCtrlBytes = 1408, kListOffset = 768;
constexpr int kListed = 96;                      // sequences whose units can be listed (see Work)
constexpr int kMinStages = 4, kMaxStages = 8, kMinCodeSlots = 4, kMaxCodeSlots = 16;
constexpr int kScaleSlots = 8;                   // blocks whose scales are kept: more than the operand ring holds
constexpr int kPacePolls = 64, kPacedBlocks = 8;           // looks at the other tile; blocks from which on turns pay (2048 over 16384, 128/128: 795 us without, 644 with)
constexpr float kFarReference = 1024.f;
constexpr float kHeadroomLog2 = 7.0f;            // weights are 2^7 at the reference; it is moved when one would exceed 2^kTopWeight

struct Args {
  mq::Args m;                    // layer, batch, rows, outputs, parts; m.nst and m.qp_bytes as there, the pools in m.L are unused
  f8::Pools P;
  const __nv_bfloat16* q;        // read directly where the key side has no basis
  long long q_stride_b, q_stride_t;
  int n_code;                    // slots of the ring of codes
};

// One stage of the operand ring: K or V of a block, half a raw query tile, or a basis; one slot of codes: one side of a page, and scales
__host__ __device__ constexpr int stage_bytes(int rk, int rv) { return 256 * (rk > rv ? (rk > 64 ? rk : 64) : (rv > 64 ? rv : 64)); }
__host__ __device__ constexpr int slot_bytes(int rk, int rv) { return kPage * (rk > rv ? rk : rv) + 128; }

// instruction descriptors of kind::f16 with f16 operands (format 0) and fp32 accumulators; B K-major, or MN-major (bit 16)
__device__ __forceinline__ uint32_t idesc_f16_f32(int M, int N) { return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }
__device__ __forceinline__ uint32_t idesc_f16_f32_bmn(int M, int N) { return idesc_f16_f32(M, N) | (1u << 16); }

// A unit as every role derives it: pages and blocks.  With two streams over the same rows (dual) the tiles take alternate blocks.
struct Unit : mq::Unit {
  int blocks;                    // of the unit, in the ring
  int nb[2];                     // of each tile
  int last[2];                   // first position behind the pages that the tile's rows may attend in this unit
};
__device__ __forceinline__ Unit block_unit(const mq::Args& a, int u, int TT) {
  Unit w;
  static_cast<mq::Unit&>(w) = mq::decode_unit(a, u, TT);
  w.blocks = (w.cnt + 1) >> 1;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    w.nb[t] = a.dual ? (w.blocks + 1 - t) >> 1 : (w.np[t] + 1) >> 1;
    w.last[t] = (w.p_lo + (a.dual ? w.cnt : w.np[t])) * kPage;
  }
  return w;
}

// The units that hold work, longest sequences first and the latest query tokens of each first, so that CTAs get equal numbers of
// them: in a ragged batch many of the units that n_q allows for are empty.  Kept in shared memory for up to kListed sequences;
// beyond, units are taken as they are numbered, empty ones among them (up to 512 query tokens in every 16th sequence of up to 2048, up to
// 30 in the others: 96 sequences 250 us, 97 323).
struct Work {
  const int* first;              // [B + 1], by place in the order: pairs of tiles before it
  const uint16_t* order;         // [B]: the sequence at a place
  int B, pairs;                  // pairs < 0: no list
  __device__ __forceinline__ int count(const mq::Args& a, int n_units) const { return pairs < 0 ? n_units : pairs * a.L.Hkv * a.n_split; }
  __device__ __forceinline__ int unit(const mq::Args& a, int v, int TT) const {      // the number that decode_unit knows it by
    if (pairs < 0) return v;
    const int r = v / a.n_split, p = r / a.L.Hkv;
    int lo = 0, hi = B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= p) lo = mid;
      else hi = mid;
    }
    const int n_t2 = (a.n_q + 2 * TT - 1) / (2 * TT), t2 = first[lo + 1] - 1 - p;
    return (((n_t2 - 1 - t2) * B + order[lo]) * a.L.Hkv + r % a.L.Hkv) * a.n_split + v % a.n_split;
  }
};
// Called by all threads; `scratch`: 2 kListed words.  Ends with a barrier.
__device__ __forceinline__ Work list_work(const mq::Args& a, int TT, int* first, uint16_t* order, int* scratch) {
  Work w{first, order, a.Bt.B, -1};
  const int B = a.Bt.B, tid = threadIdx.x;
  if (B > kListed) return w;
  int *lens = scratch, *tiles = scratch + kListed;
  int len = 0, nt = 0;
  if (tid < B) {
    const int ql = min(max(a.q_lens ? a.q_lens[tid] : a.n_q, 0), a.n_q);
    len = a.Bt.seq_lens[tid];
    if (ql > 0 && (len < ql || (len - 1) / kPage + 1 > a.Bt.max_pages)) {   // fewer cached tokens than query rows, or a table too short
      if (blockIdx.x == 0) report(a.status, STIEF_ERR_BOUNDS);
    } else {
      nt = (ql + 2 * TT - 1) / (2 * TT);
    }
    lens[tid] = len;
  }
  __syncthreads();
  if (tid < B) {
    int rank = 0;
    for (int i = 0; i < B; ++i) rank += lens[i] > len || (lens[i] == len && i < tid);
    order[rank] = (uint16_t)tid;
    tiles[rank] = nt;
  }
  __syncthreads();
  if (tid == 0) {
    int sum = 0;
    for (int i = 0; i < B; ++i) {
      first[i] = sum;
      sum += tiles[i];
    }
    first[B] = sum;
  }
  fence_proxy_async_smem();                      // the scratch becomes a target of asynchronous copies
  __syncthreads();
  w.pairs = first[B];
  return w;
}

static_assert((72 + 2) * 8 + kScaleSlots * 16 <= kListOffset && kListOffset + (kListed + 1) * 4 + kListed * 2 <= kCtrlBytes, "control words");

template <int RK, int RV>
__global__ void __launch_bounds__(kThreads, 1)
f8_mq_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmUk, const __grid_constant__ CUtensorMap tmUv,
             const Args args) {
  extern __shared__ uint8_t smem_raw[];
  const mq::Args& a = args.m;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const int nst = a.nst, n_code = args.n_code;
  constexpr int kStage = stage_bytes(RK, RV), kSlot = slot_bytes(RK, RV);
  constexpr bool kOwnP = RV <= 64;               // P has TMEM columns of its own
  constexpr int kP = kOwnP ? 128 : 0, kO = kOwnP ? 192 : 128;
  const uint32_t ring = base;
  const uint32_t qp = ring + nst * kStage;                      // Q' / O_down operands, one region per tile
  const uint32_t codes = qp + 2 * a.qp_bytes;
  const uint32_t ctrl = codes + n_code * kSlot;
  uint8_t *qp_ptr = base_ptr + (qp - base), *codes_ptr = base_ptr + (codes - base), *ctrl_ptr = base_ptr + (ctrl - base);
  enum Bar { kFull = 0, kEmpty = 8, kCodeFull = 16, kCodeEmpty = 32, kSFull = 48, kSFree = 50, kPFull = 52, kPvDone = 56, kQacc = 58, kQReady = 60,
             kOFull = 62, kOdReady = 64, kOutFull = 66, kUnitDone = 68, kTurn = 70, kBars = 72 };
  auto bar_at = [&](int i) { return ctrl + i * 8; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl_ptr + kBars * 8);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl_ptr + kBars * 8 + 4);
  float4* block_scales = reinterpret_cast<float4*>(ctrl_ptr + (kBars + 2) * 8);     // [kScaleSlots]: (key, value) of both pages

  const int G = a.L.G, Hkv = a.L.Hkv;
  const bool fold_k = a.L.U_k == nullptr, fold_v = a.L.U_v == nullptr;
  const int TT = kRows / G;                                     // query tokens per tile (rows from TT G on are not used)
  const Blocks bk = blocks_of(RK), bv = blocks_of(RV);
  const int n_units = ((a.n_q + 2 * TT - 1) / (2 * TT)) * a.Bt.B * Hkv * a.n_split;
  const bool backproj = !fold_v && a.n_split == 1;               // else the compressed (partial) result leaves the kernel
  int32_t* status = a.status;

  launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(bar_at(kFull + s), 4);            // one arrival from each filling warp
      mbar_init(bar_at(kEmpty + s), 2);           // one arrival from each tile's issuer
    }
    for (int s = 0; s < kMaxCodeSlots; ++s) {
      mbar_init(bar_at(kCodeFull + s), 1);
      mbar_init(bar_at(kCodeEmpty + s), 4);       // one arrival from each filling warp
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(bar_at(kSFull + t), 1);
      mbar_init(bar_at(kSFree + t), 4);           // one arrival per softmax warp of the tile
      mbar_init(bar_at(kPFull + 2 * t), 4);
      mbar_init(bar_at(kPFull + 2 * t + 1), 4);
      mbar_init(bar_at(kPvDone + t), 1);
      mbar_init(bar_at(kQacc + t), 1);
      mbar_init(bar_at(kQReady + t), 4);
      mbar_init(bar_at(kOFull + t), 1);
      mbar_init(bar_at(kOdReady + t), 4);
      mbar_init(bar_at(kOutFull + t), 1);
      mbar_init(bar_at(kUnitDone + t), 4);
      mbar_init(bar_at(kTurn + t), 1);
    }
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 1) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), mq::kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  grid_dependency_wait();                                       // the setup above ran beside the kernel before; everything below reads its results
  const Work work = list_work(a, TT, reinterpret_cast<int*>(ctrl_ptr + kListOffset), reinterpret_cast<uint16_t*>(ctrl_ptr + kListOffset + (kListed + 1) * 4),
                              reinterpret_cast<int*>(codes_ptr));
  const int n_work = work.count(a, n_units), grid = gridDim.x;
  // Units of CTA c: there and back, so that who had a longest unit of one round gets a shortest of the next
  auto taken = [&](int r) { return r * grid + (r & 1 ? grid - 1 - (int)blockIdx.x : (int)blockIdx.x); };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");       // 512 x 128 registers at launch = 256 x 176 + 128 x 80 + 128 x 80
    if (warp == 0) {
      // ---------------------------------------------------------------------------------------- codes of the pages
      int cs = 0, use = 0;                                      // slot of the next codes, times it has been used
      auto fetch = [&](const uint8_t* src, uint32_t bytes, const float* scales) {
        if (use > 0) mbar_wait(bar_at(kCodeEmpty + cs), (use - 1) & 1, abort_flag, status);
        const uint32_t dst = codes + cs * kSlot, bar = bar_at(kCodeFull + cs);
        mbar_arrive_expect_tx(bar, bytes + (scales ? f8::kScalesPerTile * 4 : 0));
        bulk_load_1d(dst, src, bytes, bar);
        if (scales) bulk_load_1d(dst + kSlot - 128, scales, f8::kScalesPerTile * 4, bar);
        if (++cs == n_code) {
          cs = 0;
          ++use;
        }
      };
      for (int r = 0; r * grid < n_work; ++r) {
        const int u = taken(r);
        if (u >= n_work) continue;
        const Unit w = block_unit(a, work.unit(a, u, TT), TT);
        if (!w.valid) continue;
        const int* bt = a.Bt.block_table + (size_t)w.b * a.Bt.max_pages;
        int ids = lane < w.cnt ? bt[w.p_lo + lane] : 0;
        for (int j0 = 0; j0 < w.cnt; j0 += 32) {
          const int nxt = j0 + 32 + lane < w.cnt ? bt[w.p_lo + j0 + 32 + lane] : 0;    // the next batch, a batch ahead
          const int cnt = min(32, w.cnt - j0);
          for (int jj = 0; jj < cnt; jj += 2) {
            int pg[2] = {__shfl_sync(0xffffffffu, ids, jj), __shfl_sync(0xffffffffu, ids, (jj + 1) & 31)};
            if (lane == 0) {
              const int both = jj + 1 < cnt ? 2 : 1;
              size_t tile[2];
              for (int i = 0; i < both; ++i) {
                if (pg[i] < 0 || pg[i] >= a.L.num_pages) {
                  report(status, STIEF_ERR_BOUNDS);
                  pg[i] = 0;
                }
                tile[i] = (size_t)pg[i] * Hkv + w.h;
              }
              for (int i = 0; i < both; ++i) fetch(args.P.k_codes + tile[i] * (kPage * RK), kPage * RK, args.P.scales + tile[i] * f8::kScalesPerTile);
              for (int i = 0; i < both; ++i) fetch(args.P.v_codes + tile[i] * (kPage * RV), kPage * RV, nullptr);
            }
          }
          ids = nxt;
        }
      }
    } else if (warp < 3) {
      // ---------------------------------------------------------------------------------------- MMA issue, tile mt
      // Both issuers walk ALL ring items in order; an item one has no use for is released with a plain arrive once it has
      // landed, so each stage always collects two arrivals.
      const int mt = uniform(warp) - 1;
      const uint32_t t_s = uniform(tmem_base) + mt * 256, t_p = t_s + kP, t_o = t_s + kO;
      const uint32_t ring_u = uniform(ring), ctrl_u = uniform(ctrl), qp_u = uniform(qp) + mt * uniform(a.qp_bytes);
      auto bar = [&](int i) { return ctrl_u + i * 8; };
      const uint32_t id_qk = idesc_f16_f32(kRows, kBlock), id_pv = idesc_f16_f32_bmn(kRows, RV);
      const uint32_t id_pj = idesc_bf16_f32_bmn(kRows, RK), id_bp = idesc_bf16_f32(kRows, kD);
      const uint32_t hi_k = desc_hi(desc_template(bk.layout, 16, 8 * bk.span)), hi_v = desc_hi(desc_template(bv.layout, 16, 8 * bv.span));
      const uint32_t hi_q = desc_hi(desc_template(2, 16, 1024));
      constexpr int nk = RK / 16, nv = RV / 16;
      // descriptor offset (in 16-byte units) of K step k of a K-major operand of 128 rows: inside a block 2 units per step, then the
      // next block
      const int lgk = bk.bw == 64 ? 2 : bk.bw == 32 ? 1 : 0, lgv = bv.bw == 64 ? 2 : bv.bw == 32 ? 1 : 0;
      auto koff = [](int k, int lg, uint32_t blk) { return (uint32_t)(k >> lg) * blk + (uint32_t)(k & ((1 << lg) - 1)) * 2u; };
      const uint32_t kblk = (uint32_t)(kRows * bk.span) >> 4, vblk = (uint32_t)(kRows * bv.span) >> 4;
      const uint32_t pv_b = (uint32_t)(16 * bv.span) >> 4;                       // V block: 16 rows per K step
      const uint32_t dq = desc_lo(16, qp_u);                                     // this tile's Q' operand, and its O_down operand
      const int nst_u = uniform(nst);
      const bool dual = uniform(a.dual) != 0, fold_k_u = uniform((int)fold_k) != 0, backproj_u = uniform((int)backproj) != 0;
      int st = 0, use = 0, kt = 0, n = 0, others = 0;                            // n: blocks of this tile so far; of the other tile
      auto consume = [&](uint32_t& addr, int& stage) {                           // next item of the ring, once it has landed
        mbar_wait_warp(bar(kFull + st), use & 1, abort_flag, status);
        addr = ring_u + st * kStage;
        stage = st;
        if (++st == nst_u) {
          st = 0;
          ++use;
        }
      };
      auto drop = [&](int items) {                                               // items this tile has no use for
        for (int i = 0; i < items; ++i) {
          uint32_t addr;
          int stage;
          consume(addr, stage);
          if (lane == 0) mbar_arrive(bar(kEmpty + stage));
          __syncwarp();
        }
      };
      for (int r = 0; r * grid < n_work; ++r) {
        const int u = taken(r);
        if (u >= n_work) continue;
        const Unit w = block_unit(a, work.unit(a, u, TT), TT);
        if (uniform((int)w.valid) == 0) continue;
        const int nb0 = uniform(w.nb[0]), nb1 = uniform(w.nb[1]), blocks = uniform(w.blocks);
        const int nb = mt ? nb1 : nb0;
        const bool active = nb > 0;
        if (!fold_k_u) {                                                         // each tile has U_k and its two halves of raw queries in the ring
          if (mt == 1 && nb0 > 0) drop(3);
          if (active) {
            uint32_t ua, qa;
            int us, qs;
            consume(ua, us);
            if (kt > 0) mbar_wait_warp(bar(kUnitDone + mt), (kt - 1) & 1, abort_flag, status);   // the tile's TMEM columns are free
            const uint32_t db = desc_lo(kD * bk.span, ua);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              consume(qa, qs);
              tc_fence_after();
              const uint32_t da = desc_lo(16, qa);
#pragma unroll
              for (int k = 0; k < 4; ++k)
                umma_ss(t_s, da + 2u * k, hi_q, db + (uint32_t)((4 * half + k) * bk.span), hi_k, id_pj, half + k > 0 ? 1u : 0u);
              umma_commit_warp(bar(kEmpty + qs));
            }
            umma_commit_warp(bar(kQacc + mt));
            umma_commit_warp(bar(kEmpty + us));
          }
          if (mt == 0 && nb1 > 0) drop(3);
        }
        if (active) {
          mbar_wait_warp(bar(kQReady + mt), kt & 1, abort_flag, status);
          tc_fence_after();
        }
        int jb = 0;                                                              // next block in the ring
        auto to_own = [&]() {                                                    // past the blocks of the other tile; is there one of this tile's?
          while (jb < blocks && !(dual ? (jb & 1) == mt : jb < nb)) {
            drop(2);
            ++jb;
          }
          return jb < blocks;
        };
        auto score = [&]() {                                                     // S = Q' K^T of block jb
          uint32_t ka;
          int ks;
          consume(ka, ks);
          tc_fence_after();
          const uint32_t db = desc_lo(16, ka);
#pragma unroll
          for (int k = 0; k < nk; ++k) umma_ss(t_s, dq + koff(k, lgk, kblk), hi_k, db + koff(k, lgk, kblk), hi_k, id_qk, k > 0 ? 1u : 0u);
          umma_commit_warp(bar(kSFull + mt));
          umma_commit_warp(bar(kEmpty + ks));
        };
        // Tiles of their own rows take turns: left alone they fall into step, want the special-function units at the same time and
        // leave them idle at the same time.  With P in columns of its own a tile's scores are issued when the other's last have been
        // read; with P over the scores, P V and the next scores of the two tiles alternate.  Only pace, not order: the look has an
        // end, and a wrong answer (a parity is one bit) costs nothing but the shift.
        const int theirs = mt ? nb0 : nb1;
        const bool paced = !dual && nb0 >= kPacedBlocks && nb1 >= kPacedBlocks;
        auto pace = [&](int block) {
          if (!paced || block < 0 || block >= theirs) return;
          for (int i = 0; i < kPacePolls && !__all_sync(0xffffffffu, mbar_test_wait(bar((kOwnP ? kSFree : kTurn) + 1 - mt), (others + block) & 1)); ++i) {
          }
        };
        bool have = to_own(), first = true;
        int own = 0;                                                             // blocks of this tile in the unit so far
        if (have) {
          if (kOwnP && mt == 1) pace(0);
          score();
        }
        while (have) {
          uint32_t va;
          int vs;
          consume(va, vs);
          ++jb;
          bool more = false;
          if constexpr (kOwnP) {
            more = to_own();
            if (more) {
              mbar_wait_warp(bar(kSFree + mt), n & 1, abort_flag, status);       // the scores of block n are in registers
              pace(own + mt);
              tc_fence_after();
              score();
            }
          }
          if constexpr (!kOwnP) pace(own - 1 + mt);
          const uint32_t db = desc_lo(kBlock * bv.span, va);
#pragma unroll
          for (int k = 0; k < kBlock / 16; ++k) {
            if (k == 0 || k == 4) {
              mbar_wait_warp(bar(kPFull + 2 * mt + (k >> 2)), n & 1, abort_flag, status);
              tc_fence_after();
            }
            umma_ts(t_o, t_p + 8 * k, db + (uint32_t)k * pv_b, hi_v, id_pv, (!first || k > 0) ? 1u : 0u);
          }
          umma_commit_warp(bar(kPvDone + mt));
          umma_commit_warp(bar(kEmpty + vs));
          first = false;
          ++n;
          ++own;
          if constexpr (!kOwnP) {
            more = to_own();
            if (more) score();
            if (lane == 0) mbar_arrive(bar(kTurn + mt));
            __syncwarp();
          }
          have = more;
        }
        if (active) umma_commit_warp(bar(kOFull + mt));
        if (backproj_u) {
          // OUT = O_down U_v^T with O_down handed over as two bf16 terms (value, then residual): two accumulating passes into the
          // tile's score columns, which are idle by now
          if (active) {
            uint32_t ua;
            int us;
            consume(ua, us);
            const uint32_t db = desc_lo(16, ua);
            for (int pass = 0; pass < 2; ++pass) {
              mbar_wait_warp(bar(kOdReady + mt), pass, abort_flag, status);
              tc_fence_after();
#pragma unroll
              for (int k = 0; k < nv; ++k) umma_ss(t_s, dq + koff(k, lgv, vblk), hi_v, db + koff(k, lgv, vblk), hi_v, id_bp, (pass > 0 || k > 0) ? 1u : 0u);
              umma_commit_warp(bar(kOutFull + mt));
            }
            umma_commit_warp(bar(kEmpty + us));
          } else {
            drop(1);
          }
        }
        kt += active;
        others += theirs;
      }
    }
  } else if (warp >= 12) {
    // ------------------------------------------------------------------------------------------ the ring of operands
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    const int et = tid - 12 * 32;                               // 0 .. 127
    int st = 0, use = 0, cs = 0, cuse = 0, blk = 0;
    // All items are filled from here, in order (whoever waits for a stage has seen every earlier phase of its barrier): raw queries
    // and bases are TMA loads that one thread issues.
    auto acquire = [&]() {
      if (use > 0) mbar_wait(bar_at(kEmpty + st), (use - 1) & 1, abort_flag, status);
    };
    auto advance = [&]() {
      if (++st == nst) {
        st = 0;
        ++use;
      }
    };
    auto load = [&](uint32_t bytes, auto issue) {
      acquire();
      __syncwarp();
      if (lane == 0) {
        if (warp == 12) {
          mbar_arrive_expect_tx(bar_at(kFull + st), bytes);
          issue(ring + st * kStage, bar_at(kFull + st));
        } else {
          mbar_arrive(bar_at(kFull + st));
        }
      }
      advance();
    };
    auto named_barrier = [&]() { asm volatile("bar.sync 1, 128;" ::: "memory"); };      // of the four warps
    auto publish = [&]() {                                      // the stage is written
      fence_proxy_async_smem();                                 // generic writes -> visible to the tensor core's reads
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_at(kFull + st));
      advance();
    };
    // One side of a block: codes of the next one or two slots -> the current stage.  A thread has the same pieces of 16 codes of every
    // page, 64 R / 16 of them over 128 threads: `off` is where a piece's first 8 values go in the block, the other 8 go to the
    // neighbouring 16 bytes, the second page 64 rows on.  Rows from `live` on are written as zeros (also those of a second page
    // that is not there: its weights are zeros).
    auto expand = [&](auto rank_tag, const auto& off, uint32_t page_bytes, int pages, int live, float2* scales) {
      constexpr int R = decltype(rank_tag)::value, NP = (R * 4 + 127) / 128;
      acquire();
      uint8_t* dst = base_ptr + st * kStage;
#pragma unroll 1
      for (int pg = 0; pg < pages; ++pg) {
        const uint8_t* src = codes_ptr + cs * kSlot;
        mbar_wait(bar_at(kCodeFull + cs), cuse & 1, abort_flag, status);
        uint4 w[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i)
          if (R % 32 == 0 || et + 128 * i < R * 4) w[i] = reinterpret_cast<const uint4*>(src)[et + 128 * i];
        if (scales) scales[pg] = *reinterpret_cast<const float2*>(src + kSlot - 128);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          if (R % 32 == 0 || et + 128 * i < R * 4) {
            uint4 lo, hi;
            f8::expand4(w[i].x, lo.x, lo.y);
            f8::expand4(w[i].y, lo.z, lo.w);
            f8::expand4(w[i].z, hi.x, hi.y);
            f8::expand4(w[i].w, hi.z, hi.w);
            *reinterpret_cast<uint4*>(dst + off[i]) = lo;
            *reinterpret_cast<uint4*>(dst + (off[i] ^ 16u)) = hi;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_at(kCodeEmpty + cs));
        if (++cs == n_code) {
          cs = 0;
          ++cuse;
        }
        dst += page_bytes;
      }
      if (live < kBlock) {
        const Blocks bl = blocks_of(R);
        dst = base_ptr + st * kStage;
        named_barrier();                                        // other threads' values are in place before they are overwritten
#pragma unroll 1
        for (int e = et; e < (kBlock - live) * (R / 8); e += 128)
          *reinterpret_cast<uint4*>(dst + block_offset(bl, kBlock, live + e / (R / 8), e % (R / 8) * 8)) = make_uint4(0u, 0u, 0u, 0u);
      }
    };
    uint32_t k_off[(RK * 4 + 127) / 128], v_off[(RV * 4 + 127) / 128];
#pragma unroll
    for (int i = 0; i < (RK * 4 + 127) / 128; ++i) k_off[i] = block_offset(bk, kBlock, (et + 128 * i) / (RK / 16), (et + 128 * i) % (RK / 16) * 16);
#pragma unroll
    for (int i = 0; i < (RV * 4 + 127) / 128; ++i) v_off[i] = block_offset(bv, kBlock, (et + 128 * i) / (RV / 16), (et + 128 * i) % (RV / 16) * 16);
    if (et == 0) {
      if (!fold_k) {
        tma_prefetch_desc(&tmQ);
        tma_prefetch_desc(&tmUk);
      }
      if (backproj) tma_prefetch_desc(&tmUv);
    }
    for (int r = 0; r * grid < n_work; ++r) {
      const int u = taken(r);
      if (u >= n_work) continue;
      const Unit w = block_unit(a, work.unit(a, u, TT), TT);
      if (!w.valid) continue;
      if (!fold_k) {
        for (int t = 0; t < 2; ++t) {
          if (w.nb[t] == 0) continue;
          load(kD * RK * 2, [&](uint32_t dst, uint32_t bar) {
            for (int i = 0; i < bk.nb; ++i) tma_load_3d(dst + i * kD * bk.span, &tmUk, i * bk.bw, 0, a.L.uk_stride ? w.h : 0, bar);
          });
          for (int half = 0; half < 2; ++half)
            load((uint32_t)(TT * G) * kD, [&](uint32_t dst, uint32_t bar) { tma_load_4d(dst, &tmQ, 64 * half, w.h * G, w.tok0[t], w.b, bar); });
        }
      }
      for (int jb = 0; jb < w.blocks; ++jb, ++blk) {
        const bool both = 2 * jb + 1 < w.cnt;
        const int live = w.seq_len - (w.p_lo + 2 * jb) * kPage;             // rows of the block that belong to the sequence
        const int pages = both ? 2 : 1;
        float2 sc[2] = {make_float2(1.f, 1.f), make_float2(1.f, 1.f)};
        expand(std::integral_constant<int, RK>{}, k_off, kPage * bk.span, pages, kBlock, sc);      // keys: positions that nobody attends are masked
        if (et == 0) block_scales[blk % kScaleSlots] = make_float4(sc[0].x, sc[0].y, sc[1].x, sc[1].y);
        publish();
        expand(std::integral_constant<int, RV>{}, v_off, kPage * bv.span, pages, min(live, pages * kPage), nullptr);
        publish();
      }
      if (backproj)
        load(kD * RV * 2, [&](uint32_t dst, uint32_t bar) {
          for (int i = 0; i < bv.nb; ++i) tma_load_3d(dst + i * kD * bv.span, &tmUv, i * bv.bw, 0, a.L.uv_stride ? w.h : 0, bar);
        });
    }
  } else {
    // ------------------------------------------------------------------------------------------ softmax / epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    const int t = (warp - 4) >> 2;                              // the tile this warp works for
    const int q4 = warp & 3;                                    // TMEM lane quarter this warp may access
    const int row = 32 * q4 + lane;                             // row of the tile = TMEM lane
    const uint32_t t_s = tmem_base + ((uint32_t)(32 * q4) << 16) + t * 256, t_p = t_s + kP, t_o = t_s + kO;
    uint8_t* my_qp = qp_ptr + t * a.qp_bytes;
    const float c = kLog2e * rsqrtf((float)kD);                 // scores are scaled by 1/sqrt(d_h); exponent in base 2
    const int d_out = fold_v ? RV : kD;
    int kt = 0, n = 0, blk = 0;                                 // units and blocks of this tile so far; blocks of the ring before the unit
    auto arrive_warp = [&](uint32_t bar) {                      // after every lane's shared/TMEM accesses are ordered
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    for (int r = 0; r * grid < n_work; ++r) {
      const int u = taken(r);
      if (u >= n_work) continue;
      const Unit w = block_unit(a, work.unit(a, u, TT), TT);
      if (!w.valid) continue;
      const int blk0 = blk;
      blk += w.blocks;
      if (w.nb[t] == 0) continue;
      const int nb = w.nb[t];
      const int tok = w.tok0[t] + row / G, g = row - (row / G) * G;
      const bool row_valid = tok < w.q_len && row < TT * G;
      // first position that the row does not attend; rows past the end behave like the last valid token
      const int end = min(w.q_start + min(tok, w.q_len - 1) + 1, w.last[t]);

      // ---- Q' as f16 into the A operand of the score products, each row scaled by a power of two of its own
      float c_row;
      {
        float top = 0.f;
        const uint4* qrow = reinterpret_cast<const uint4*>(args.q + (size_t)w.b * args.q_stride_b + (size_t)tok * args.q_stride_t + (size_t)(w.h * G + g) * RK);
        auto piece = [&](int c0, float (&x)[16]) {              // elements c0 .. c0 + 15 of the row
          if (fold_k) {
            uint4 v0 = make_uint4(0u, 0u, 0u, 0u), v1 = v0;
            if (row_valid) {
              v0 = qrow[c0 / 8];
              v1 = qrow[c0 / 8 + 1];
            }
            const uint32_t v[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              x[2 * i] = bf16_lo(v[i]);
              x[2 * i + 1] = bf16_hi(v[i]);
            }
          } else {
            tmem_ld16(t_s + c0, *reinterpret_cast<uint32_t(*)[16]>(&x));
            tmem_ld_wait();
          }
        };
        if (!fold_k) {
          mbar_wait(bar_at(kQacc + t), kt & 1, abort_flag, status);
          tc_fence_after();
        }
        for (int c0 = 0; c0 < RK; c0 += 16) {
          float x[16];
          piece(c0, x);
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
        }
        const int e = top > 0.f ? min(max((int)(__float_as_uint(top) >> 23) - 127, -112), 126) - 11 : 0;
        const float norm = f8::pow2(-e);
        c_row = row_valid ? f8::pow2(e) * c : 0.f;              // rows of no token (what stands there may be anything) do not ask for the form for far scores
        for (int c0 = 0; c0 < RK; c0 += 16) {
          float x[16];
          piece(c0, x);
          uint32_t pk[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) pk[i] = f8::pack_f16(x[2 * i] * norm, x[2 * i + 1] * norm);
          *reinterpret_cast<uint4*>(my_qp + block_offset(bk, kRows, row, c0)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
          *reinterpret_cast<uint4*>(my_qp + block_offset(bk, kRows, row, c0 + 8)) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
        }
        fence_proxy_async_smem();
        tc_fence_before();
        arrive_warp(bar_at(kQReady + t));
      }

      float m = -INFINITY, em = 0.f, l = 0.f, n_ref = f8::kNoSum;      // both parts of the reference; row sum and its reference
      for (int jo = 0; jo < nb; ++jo, ++n) {
        const int j = a.dual ? 2 * jo + t : jo;                 // the block within the unit's range
        mbar_wait(bar_at(kSFull + t), n & 1, abort_flag, status);
        tc_fence_after();
        uint32_t sv[kBlock];
        float* s = reinterpret_cast<float*>(sv);
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld32(t_s + 32 * i, sv + 32 * i);
        // written before the arrival that these scores' product waited for; overwritten eight blocks on
        const float4 sc = block_scales[(blk0 + j) % kScaleSlots];
        tmem_ld_wait();
        if constexpr (kOwnP) {
          tc_fence_before();
          arrive_warp(bar_at(kSFree + t));
        }
        const int p0 = (w.p_lo + 2 * j) * kPage;
        const bool edge = p0 + kBlock > end;
        if (edge) {                                             // positions after the row's own, and pages that are not in the unit
#pragma unroll
          for (int i = 0; i < kBlock; ++i)
            if (p0 + i >= end) s[i] = -INFINITY;
        }
        // exponents x = s f + e of the two pages; f is above zero, so that masked scores stay -inf
        const float f0 = fmaxf(f8::score_factor(c_row, sc.x), 1e-37f), f1 = fmaxf(f8::score_factor(c_row, sc.z), 1e-37f);
        const float e0 = f8::scale_exponent(sc.y), e1 = f8::scale_exponent(sc.w);
        float x_page[2];                                        // largest score of each page
        {
          float m[4] = {s[0], s[1], s[64], s[65]};
#pragma unroll
          for (int i = 2; i < 62; i += 4)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              m[2 * h] = max3(m[2 * h], s[64 * h + i], s[64 * h + i + 1]);
              m[2 * h + 1] = max3(m[2 * h + 1], s[64 * h + i + 2], s[64 * h + i + 3]);
            }
          x_page[0] = __fmul_rn(fmaxf(max3(m[0], s[62], s[63]), m[1]), f0);
          x_page[1] = __fmul_rn(fmaxf(max3(m[2], s[126], s[127]), m[3]), f1);
        }
        // P and the accumulator are idle once the block before is mixed (with P over the scores, these scores came after that)
        auto mixed = [&]() {
          if constexpr (kOwnP) {
            if (n > 0) {
              mbar_wait(bar_at(kPvDone + t), (n - 1) & 1, abort_flag, status);
              tc_fence_after();
            }
          }
        };
        float r = 1.f;                                          // what a moved reference leaves of the accumulator
        bool moved = false;                                     // for a row of the warp
        bool vanish[2];
        {
          // log2 of each page's largest weight (infinity: the row has attended nothing before)
          float beyond[2] = {x_page[0] - m, x_page[1] - m}, above[2] = {beyond[0] + (e0 - em), beyond[1] + (e1 - em)};
          const float most = fmaxf(above[0], above[1]);
          const bool grown = jo == 0 || most > f8::kTopWeight;
          if (jo > 0) moved = __any_sync(0xffffffffu, grown);
          if (grown) {
            const bool second = (x_page[1] - x_page[0]) + (e1 - e0) > 0.f;
            r = fast_exp2(kHeadroomLog2 - most);
            m = second ? x_page[1] : x_page[0];                 // -inf when a part of a split range begins behind the row's position
            em = (second ? e1 : e0) - kHeadroomLog2;
            beyond[0] = x_page[0] - m;
            beyond[1] = x_page[1] - m;
            above[0] = beyond[0] + (e0 - em);
            above[1] = beyond[1] + (e1 - em);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) vanish[h] = f8::may_vanish(beyond[h], above[h]);
        }
        const float ref = m > -INFINITY ? m : 0.f;
        {
          const float x_top = fmaxf(x_page[0], x_page[1]), n_old = n_ref;
          n_ref = x_top > n_ref + f8::kSumGrown ? x_top : n_ref;
          l *= fast_exp2(n_old - n_ref);
        }
        // Exponents as one fma with (e - E) - M where that is good to 2^-14; with scores far from zero (references beyond 2^10) the
        // rounded x is what counts, less M, then the scales.  That form also serves pages whose weights vanish: exponentials by the page's
        // own largest score, for the sum alone.  A warp takes it if a row of it needs it; the other rows then add zeros to the first form, so
        // that a row's bits do not depend on its neighbours.  A page at a time: its weights are mixed while the next one's are made.
        auto weights = [&](auto far_tag) {
          constexpr bool kFar = decltype(far_tag)::value;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float f = h ? f1 : f0, shift = (h ? e1 : e0) - em, mix = vanish[h] ? 0.f : 1.f;
            float first = shift - ref, less = 0.f, rest = 0.f;
            if constexpr (kFar) {
              if (vanish[h] || fabsf(ref) > kFarReference) {
                first = 0.f;
                less = vanish[h] ? -x_page[h] : -ref;
                rest = vanish[h] ? 0.f : shift;
              }
            }
            const uint64_t f2 = pack2(f, f), first2 = pack2(first, first), less2 = pack2(less, less), rest2 = pack2(rest, rest);
            uint64_t sum2 = pack2(0.f, 0.f);
            uint32_t pk[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              uint64_t x2 = fma2(pack2(s[64 * h + 2 * i], s[64 * h + 2 * i + 1]), f2, first2);
              if constexpr (kFar) x2 = add2(add2(x2, less2), rest2);
              float x0, x1;
              unpack2(x2, x0, x1);
              x0 = fast_exp2(x0);
              x1 = fast_exp2(x1);
              sum2 = add2(sum2, pack2(x0, x1));
              pk[i] = kFar ? f8::pack_f16(x0 * mix, x1 * mix) : f8::pack_f16(x0, x1);
            }
            if (h == 0) mixed();
            tmem_st16(t_p + 32 * h, *reinterpret_cast<uint32_t(*)[16]>(&pk[0]));
            tmem_st16(t_p + 32 * h + 16, *reinterpret_cast<uint32_t(*)[16]>(&pk[16]));
            if (h == 0 && moved) {                              // as late as the weights allow: P V of the block before has to be through
#pragma unroll 1
              for (int c0 = 0; c0 < RV; c0 += 16) {
                uint32_t v[16];
                tmem_ld16(t_o + c0, v);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * r);
                tmem_st16(t_o + c0, v);
              }
            }
            float a0, a1;
            unpack2(sum2, a0, a1);
            // what the sum counts for (with an end, so that a page of which the row attends nothing, sum 0, meets no infinity)
            l = fmaf(a0 + a1, fast_exp2(kFar && vanish[h] ? x_page[h] - n_ref : fminf((m - n_ref) - shift, 126.f)), l);
            tmem_st_wait();
            tc_fence_before();
            arrive_warp(bar_at(kPFull + 2 * t + h));
          }
        };
        if (__any_sync(0xffffffffu, (fabsf(ref) > kFarReference || vanish[0] || vanish[1]))) weights(std::true_type{});
        else weights(std::false_type{});
      }

      // ---- epilogue of the unit
      mbar_wait(bar_at(kOFull + t), kt & 1, abort_flag, status);
      tc_fence_after();
      const float half = fast_exp2(0.5f * ((m - n_ref) + em));      // in two steps: beyond fp32's exponents where scales lie far apart
      const float inv = half / l;
      __nv_bfloat16* orow = a.out + (size_t)w.b * a.out_stride_b + (size_t)tok * a.out_stride_t + (size_t)(w.h * G + g) * d_out;
      if (a.n_split > 1) {
        // partial result of this part of the page range: its mix, and its row sum with the reference (base-2 units)
        const size_t prow = (((size_t)w.b * a.n_q + tok) * a.L.Hq + w.h * G + g) * a.n_parts + (a.dual ? 2 * w.split + t : w.split);
        for (int c0 = 0; c0 < RV; c0 += 16) {
          uint32_t v[16];
          tmem_ld16(t_o + c0, v);
          tmem_ld_wait();
          if (row_valid) {
            float4* dst = reinterpret_cast<float4*>(a.part_o + prow * RV + c0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              dst[i] = make_float4(__uint_as_float(v[4 * i]) * half * inv, __uint_as_float(v[4 * i + 1]) * half * inv,
                                   __uint_as_float(v[4 * i + 2]) * half * inv, __uint_as_float(v[4 * i + 3]) * half * inv);
          }
        }
        if (row_valid) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(n_ref, l);
      } else if (fold_v) {
        for (int c0 = 0; c0 < RV; c0 += 16) {
          uint32_t v[16], pk[8];
          tmem_ld16(t_o + c0, v);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * half);
          pack16(v, inv, pk);
          if (row_valid) {
            *reinterpret_cast<uint4*>(orow + c0) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            *reinterpret_cast<uint4*>(orow + c0 + 8) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
          }
        }
      } else {
        // O_down = O / l goes to the back-projection as bf16(x) and then bf16(x - bf16(x)): two accumulating passes keep about 16
        // significant bits, so the result is rounded once, at the output
        for (int pass = 0; pass < 2; ++pass) {
          for (int c0 = 0; c0 < RV; c0 += 16) {
            uint32_t v[16], pk[8];
            tmem_ld16(t_o + c0, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float x0 = __uint_as_float(v[2 * i]) * half * inv, x1 = __uint_as_float(v[2 * i + 1]) * half * inv;
              uint32_t hi, lo;
              split_bf16(x0, x1, hi, lo);
              pk[i] = pass ? lo : hi;
            }
            *reinterpret_cast<uint4*>(my_qp + block_offset(bv, kRows, row, c0)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            *reinterpret_cast<uint4*>(my_qp + block_offset(bv, kRows, row, c0 + 8)) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
          }
          fence_proxy_async_smem();
          tc_fence_before();
          arrive_warp(bar_at(kOdReady + t));
          mbar_wait(bar_at(kOutFull + t), pass, abort_flag, status);     // the pass has read the operand (after the second: OUT is complete)
          tc_fence_after();
        }
        for (int c0 = 0; c0 < kD; c0 += 16) {
          uint32_t v[16], pk[8];
          tmem_ld16(t_s + c0, v);
          tmem_ld_wait();
          pack16(v, 1.0f, pk);
          if (row_valid) {
            *reinterpret_cast<uint4*>(orow + c0) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            *reinterpret_cast<uint4*>(orow + c0 + 8) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
          }
        }
      }
      if (row_valid && a.out_lse && a.n_split == 1)
        a.out_lse[((size_t)w.b * a.n_q + tok) * a.L.Hq + w.h * G + g] = kLn2 * (n_ref + log2f(l));
      tc_fence_before();
      arrive_warp(bar_at(kUnitDone + t));                       // the tile's TMEM columns and operand region are free
      ++kt;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem_base, mq::kTmemCols);
}

// Measured: 0.25 (r_v 32, 64) to 0.5 us (128) for a thousand rows of two parts, on top of 10 us for a launch that waits for
// another; a block of 256 threads that fetches the next tile's references early took as long.
// Merges the parts of a split page range (by their sums and references), back-projects and writes the rows.  The rows of a
// (sequence, KV head), token by token and its G heads in turn, are taken in tiles of `tile_rows` <= 16; a block keeps U_v as operands
// of mma.sync in registers and goes through every gridDim.x-th tile.  Rows go to the product as bf16(x) and bf16(x - bf16(x)), as
// without parts.  A part that had no block for the row's tile was never written and is left out by redoing the range arithmetic of
// decode_unit.
constexpr int kCombineThreads = 128, kCombineRows = 16, kMaxParts = 64;
template <int RV>
__global__ void __launch_bounds__(kCombineThreads)
f8_mq_combine_kernel(const mq::Args a, int tile_rows) {
  constexpr int kPitch = RV + 8, NK = RV / 16;                    // rows 16 (odd) bytes apart: conflict-free ldmatrix
  __shared__ __align__(16) __nv_bfloat16 terms[2][kCombineRows][kPitch];
  __shared__ float weight[kCombineRows][kMaxParts + 1];
  launch_dependents();
  grid_dependency_wait();
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = a.L.G, TT = kRows / G, NP = a.n_parts;
  int ql = a.q_lens ? a.q_lens[b] : a.n_q;
  ql = min(max(ql, 0), a.n_q);
  const int sl = a.Bt.seq_lens[b], q_start = sl - ql;
  if (q_start < 0 || (sl - 1) / kPage + 1 > a.Bt.max_pages) return;
  const int rows = ql * G;
  if ((int)blockIdx.x * tile_rows >= rows) return;
  const bool fold_v = a.L.U_v == nullptr;
  // Output channels of the warp: 32 warp + 8 (column / 2) + 2 j + column % 2 for column 0 .. 7 of its j-th product, so that a thread's
  // share of a row is 8 neighbours.
  uint32_t u[NK][4][2];
  if (!fold_v) {
    const __nv_bfloat16* Uv = a.L.U_v + (size_t)h * a.L.uv_stride;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = lane >> 2;
      const __nv_bfloat16* src = Uv + (32 * warp + 8 * (col >> 1) + 2 * j + (col & 1)) * RV + 2 * (lane & 3);
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        u[k][j][0] = __ldg(reinterpret_cast<const uint32_t*>(src + 16 * k));
        u[k][j][1] = __ldg(reinterpret_cast<const uint32_t*>(src + 16 * k + 8));
      }
    }
  }
  for (int r0 = blockIdx.x * tile_rows; r0 < rows; r0 += gridDim.x * tile_rows) {
    const int nr = min(tile_rows, rows - r0);
    {                                                           // weights of the rows' parts over the row sum: eight threads a row
      const int r = tid >> 3, p8 = tid & 7;
      const bool live = r < nr;
      const int tok = (r0 + min(r, nr - 1)) / G, g = r0 + min(r, nr - 1) - tok * G;
      // pages of the row's tile and of the unit (both tiles), as decode_unit derives them
      const int t2 = tok / (2 * TT), first = t2 * 2 * TT;
      int full[2] = {0, 0};
      for (int t = 0; t < 2; ++t)
        if (first + t * TT < ql) full[t] = (q_start + min(first + (t + 1) * TT, ql) - 1) / kPage + 1;
      const uint32_t all = max(full[0], full[1]);               // times 32 parts below 2^31
      const int mine = full[(tok - first) / TT];
      auto exists = [&](int i) {
        const uint32_t sp = a.dual ? i >> 1 : i;
        const int lo = (int)(sp * all / (uint32_t)a.n_split), hi = min((int)((sp + 1) * all / (uint32_t)a.n_split), mine);
        return a.dual ? (i & 1) < (hi - lo + 1) >> 1 : hi > lo;
      };
      const size_t row = ((size_t)b * a.n_q + tok) * a.L.Hq + h * G + g;
      float m[kMaxParts / 8], l[kMaxParts / 8], M = -INFINITY, den = 0.f;
#pragma unroll
      for (int i = 0; i < kMaxParts / 8; ++i) {
        const int p = p8 + 8 * i;
        m[i] = -INFINITY;
        l[i] = 0.f;
        if (live && p < NP && exists(p)) {
          const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (row * NP + p) * 2);
          m[i] = ml.x;
          l[i] = ml.y;
        }
        M = fmaxf(M, m[i]);
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
#pragma unroll
      for (int i = 0; i < kMaxParts / 8; ++i) {
        const bool some = l[i] > 0.f || l[i] != l[i];           // a part that the row attends nothing of has l = 0
        m[i] = some ? l[i] * fast_exp2(m[i] - M) : 0.f;
        den += m[i];
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
      const float inv = 1.f / den;
#pragma unroll
      for (int i = 0; i < kMaxParts / 8; ++i)
        if (live && p8 + 8 * i < NP) weight[r][p8 + 8 * i] = m[i] == 0.f ? 0.f : m[i] * inv;
      if (live && p8 == 0 && a.out_lse) a.out_lse[row] = kLn2 * (M + log2f(den));
    }
    __syncthreads();
    const size_t row0 = ((size_t)b * a.n_q * a.L.Hq + h * G);
    auto part_row = [&](int r) {                                // the row among all: rows of a token are Hq apart
      const int tok = (r0 + r) / G;
      return row0 + (size_t)tok * a.L.Hq + (r0 + r - tok * G);
    };
    constexpr int NE = (kCombineRows * RV / 4 + kCombineThreads - 1) / kCombineThreads;
    const float4* src[NE];
    float4 x[NE];
    int er[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int e = tid + kCombineThreads * i;
      er[i] = e / (RV / 4) < nr ? e / (RV / 4) : -1;
      src[i] = reinterpret_cast<const float4*>(a.part_o + part_row(max(er[i], 0)) * NP * RV) + e % (RV / 4);
      x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll 2
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        const float wgt = er[i] >= 0 ? weight[er[i]][p] : 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (wgt != 0.f) v = __ldcs(src[i] + (size_t)p * (RV / 4));
        x[i].x = fmaf(v.x, wgt, x[i].x);
        x[i].y = fmaf(v.y, wgt, x[i].y);
        x[i].z = fmaf(v.z, wgt, x[i].z);
        x[i].w = fmaf(v.w, wgt, x[i].w);
      }
    auto out_row = [&](int r, int d_out) {
      const int tok = (r0 + r) / G;
      return a.out + (size_t)b * a.out_stride_b + (size_t)tok * a.out_stride_t + (size_t)(h * G + r0 + r - tok * G) * d_out;
    };
    if (fold_v) {
#pragma unroll
      for (int i = 0; i < NE; ++i)
        if (er[i] >= 0)
          *reinterpret_cast<uint2*>(out_row(er[i], RV) + (tid + kCombineThreads * i) % (RV / 4) * 4) = make_uint2(pack_bf16(x[i].x, x[i].y), pack_bf16(x[i].z, x[i].w));
    } else {
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        const int e = tid + kCombineThreads * i;
        if (e < kCombineRows * RV / 4) {                        // rows that the tile does not have are zeros
          uint32_t hi[2], lo[2];
          split_bf16(x[i].x, x[i].y, hi[0], lo[0]);
          split_bf16(x[i].z, x[i].w, hi[1], lo[1]);
          *reinterpret_cast<uint2*>(&terms[0][e / (RV / 4)][e % (RV / 4) * 4]) = make_uint2(hi[0], hi[1]);
          *reinterpret_cast<uint2*>(&terms[1][e / (RV / 4)][e % (RV / 4) * 4]) = make_uint2(lo[0], lo[1]);
        }
      }
      __syncthreads();
      float acc[4][4] = {};
      const uint32_t at = smem_u32(&terms[0][lane & 15][(lane >> 4) * 8]);
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int term = 0; term < 2; ++term) {
          uint32_t f[4];
          ldsm_x4(at + term * (kCombineRows * kPitch * 2) + 32 * k, f[0], f[1], f[2], f[3]);
#pragma unroll
          for (int j = 0; j < 4; ++j) mma_bf16(acc[j], f, u[k][j][0], u[k][j][1]);
        }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = (lane >> 2) + 8 * half;
        if (r < nr)
          *reinterpret_cast<uint4*>(out_row(r, kD) + 32 * warp + 8 * (lane & 3)) =
              make_uint4(pack_bf16(acc[0][2 * half], acc[0][2 * half + 1]), pack_bf16(acc[1][2 * half], acc[1][2 * half + 1]),
                         pack_bf16(acc[2][2 * half], acc[2][2 * half + 1]), pack_bf16(acc[3][2 * half], acc[3][2 * half + 1]));
      }
    }
    __syncthreads();                                            // weights and terms are free
  }
}

// What the host hands to a launcher: the argument block, the tensor maps, the launch shape.
struct Launch {
  Args a;
  CUtensorMap tmQ, tmUk, tmUv;
  int grid, smem;
};

}  // namespace f8mq

// One launcher per key rank (each its own translation unit); cudaErrorInvalidValue for a value rank that is not compiled in.
cudaError_t launch_f8_mq_rk32(const f8mq::Launch& l, cudaStream_t st);
cudaError_t launch_f8_mq_rk48(const f8mq::Launch& l, cudaStream_t st);
cudaError_t launch_f8_mq_rk64(const f8mq::Launch& l, cudaStream_t st);
cudaError_t launch_f8_mq_rk96(const f8mq::Launch& l, cudaStream_t st);
cudaError_t launch_f8_mq_rk128(const f8mq::Launch& l, cudaStream_t st);

}  // namespace stief
