// Attention of several causal query rows per head over the 8-bit floating-point cache (chunked prefill, speculative decode):
//     out_i = softmax(q_i' (c_k S_k)[0..p_i]^T / sqrt(128)) (c_v S_v)[0..p_i] U_v^T,   q_i' = q_i U_k,
// on the 5th-generation tensor cores, in the form of stief_mq.cuh: the same work units (sequence, KV head, 256 query rows in two
// tiles of 128), the same split of a long page range into parts, the same merge.  What the codes change:
//   operands   kind::f16 products want both operands in one 16-bit type, so every page is expanded once per CTA, for both
//              tiles, from codes to f16 (exact, one conversion per two codes), by warps of their own: they read the page's codes
//              from a ring that 1-D bulk copies fill and write the K and V blocks, swizzled as tcgen05.mma reads them, into the
//              ring of operands.  Value rows past the end of the sequence are written as zeros there, so that what
//              unspecified codes stand for (NaN) cannot reach the accumulator through 0 * x.
//   queries    Q' is rounded to f16 once (11 bits), each row first scaled by the power of two that brings its largest element to
//              2^11 .. 2^12: f16's range is no limit, and a row's factor goes into its exponents.
//   scales     powers of two.  The key scale joins a page's exponent factor.  The value scale 2^e joins the exponent itself: the
//              weight of a position is w = 2^(x + e - ref), ref going by the largest x + e of the row, so weights of pages
//              whose scales lie far apart keep their precision; the row sum takes w 2^-e.
//   weights    f16 (11 bits, where bf16 would leave 8), at most 2^15: the reference is moved when a row's largest has grown by
//              more than 2^8, and w = 2^7 at the reference.
// 512 threads, registers split by role (setmaxnreg):
//   warp 0        fetches the codes of the pages
//   warps 1, 2    MMA issue, one per tile (control flow and descriptors in uniform registers, stief_umma.cuh)
//   warps 4-11    softmax and epilogue, four per tile; thread = row = TMEM lane
//   warps 12-15   fill the ring of operands: expand the pages; raw queries, U_k and U_v come straight into it by TMA
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
constexpr int kStageBytes = 32768;               // one stage of the operand ring: a page's K and V, a raw query tile, or a basis
constexpr int kCtrlBytes = 1024;
constexpr int kMaxStages = 4, kMaxCodeStages = 8;
constexpr float kRescaleLog2 = 8.0f;             // move a row's reference when its largest exponent grew by more
constexpr float kHeadroomLog2 = 7.0f;            // weights are 2^7 at the reference: at most 2^15 in f16
constexpr int kPolyEvery = 4;                    // every fourth pair of exponentials as a polynomial (small ranks, see mq_attention_kernel)

struct Args {
  mq::Args m;                    // layer, batch, rows, outputs, parts; m.nst and m.qp_bytes as there, the pools in m.L are unused
  f8::Pools P;
  const __nv_bfloat16* q;        // read directly where the key side has no basis
  long long q_stride_b, q_stride_t;
  int n_code;                    // stages of the ring of codes
};

__host__ __device__ constexpr int code_stage_bytes(int rk, int rv) { return (kPage * (rk + rv) + f8::kScalesPerTile * 4 + 127) / 128 * 128; }

// instruction descriptors of kind::f16 with f16 operands (format 0) and fp32 accumulators; B K-major, or MN-major (bit 16)
__device__ __forceinline__ uint32_t idesc_f16_f32(int M, int N) { return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }
__device__ __forceinline__ uint32_t idesc_f16_f32_bmn(int M, int N) { return idesc_f16_f32(M, N) | (1u << 16); }

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
  constexpr int kCode = code_stage_bytes(RK, RV);
  const uint32_t ring = base;
  const uint32_t qp = ring + nst * kStageBytes;                 // Q' / O_down operands, one region per tile
  const uint32_t codes = qp + 2 * a.qp_bytes;
  const uint32_t ctrl = codes + n_code * kCode;
  uint8_t *qp_ptr = base_ptr + (qp - base), *codes_ptr = base_ptr + (codes - base), *ctrl_ptr = base_ptr + (ctrl - base);
  auto full_bar = [&](int s) { return ctrl + s * 8; };
  auto empty_bar = [&](int s) { return ctrl + (4 + s) * 8; };
  auto s_full = [&](int t, int i) { return ctrl + (8 + t * 2 + i) * 8; };
  auto p_full = [&](int t, int i) { return ctrl + (12 + t * 2 + i) * 8; };
  auto p_free = [&](int t, int i) { return ctrl + (16 + t * 2 + i) * 8; };
  auto qacc_full = [&](int t) { return ctrl + (20 + t) * 8; };
  auto qp_ready = [&](int t) { return ctrl + (22 + t) * 8; };
  auto o_full = [&](int t) { return ctrl + (24 + t) * 8; };
  auto od_ready = [&](int t) { return ctrl + (26 + t) * 8; };
  auto out_full = [&](int t) { return ctrl + (28 + t) * 8; };
  auto unit_done = [&](int t) { return ctrl + (30 + t) * 8; };
  auto code_full = [&](int s) { return ctrl + (32 + s) * 8; };
  auto code_empty = [&](int s) { return ctrl + (40 + s) * 8; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl_ptr + 48 * 8);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl_ptr + 48 * 8 + 4);
  volatile float2* page_scales = reinterpret_cast<volatile float2*>(ctrl_ptr + 50 * 8);     // [nst]: of the page in each operand stage

  const int G = a.L.G, Hkv = a.L.Hkv;
  const bool fold_k = a.L.U_k == nullptr, fold_v = a.L.U_v == nullptr;
  const int TT = kRows / G;                                     // query tokens per tile (rows from TT G on are not used)
  const Blocks bk = blocks_of(RK), bv = blocks_of(RV);
  const int n_units = ((a.n_q + 2 * TT - 1) / (2 * TT)) * a.Bt.B * Hkv * a.n_split;
  const bool backproj = !fold_v && a.n_split == 1;               // else the compressed (partial) result leaves the kernel
  int32_t* status = a.status;

  if (tid == 0) {
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(full_bar(s), 4);         // one arrival from each filling warp
      mbar_init(empty_bar(s), 2);        // one arrival from each tile's issuer
    }
    for (int s = 0; s < kMaxCodeStages; ++s) {
      mbar_init(code_full(s), 1);
      mbar_init(code_empty(s), 4);       // one arrival from each expanding warp
    }
    for (int t = 0; t < 2; ++t) {
      for (int i = 0; i < 2; ++i) {
        mbar_init(s_full(t, i), 1);
        mbar_init(p_full(t, i), 4);       // one arrival per softmax warp of the tile
        mbar_init(p_free(t, i), 1);
      }
      mbar_init(qacc_full(t), 1);
      mbar_init(qp_ready(t), 4);
      mbar_init(o_full(t), 1);
      mbar_init(od_ready(t), 4);
      mbar_init(out_full(t), 1);
      mbar_init(unit_done(t), 4);
    }
    *abort_flag = 0;
    mbar_fence_init();
  }
  launch_dependents();
  if (warp == 1) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), mq::kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  grid_dependency_wait();                                       // the setup above ran beside the kernel before; everything below reads its results

  // ring items of a unit ahead of its pages, and in all
  auto lead_of = [&](const mq::Unit& w) { return fold_k ? 0 : (w.np[0] > 0) + (w.np[1] > 0) + 1; };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");       // 512 x 128 registers at launch = 256 x 168 + 128 x 88 + 128 x 88
    if (warp == 0) {
      // ---------------------------------------------------------------------------------------- codes of the pages
      int cs = 0, use = 0;                                      // stage of the next page's codes, times it has been used
      for (int u = blockIdx.x; u < n_units; u += gridDim.x) {
        const mq::Unit w = mq::decode_unit(a, u, TT);
        if (!w.valid) continue;
        const int npmax = w.cnt;
        const int* bt = a.Bt.block_table + (size_t)w.b * a.Bt.max_pages;
        int ids = lane < npmax ? bt[w.p_lo + lane] : 0;
        for (int j0 = 0; j0 < npmax; j0 += 32) {
          const int nxt = j0 + 32 + lane < npmax ? bt[w.p_lo + j0 + 32 + lane] : 0;    // the next batch, a batch ahead
          const int cnt = min(32, npmax - j0);
          for (int jj = 0; jj < cnt; ++jj) {
            int pg = __shfl_sync(0xffffffffu, ids, jj);
            if (lane == 0) {
              if (pg < 0 || pg >= a.L.num_pages) {
                report(status, STIEF_ERR_BOUNDS);
                pg = 0;
              }
              if (use > 0) mbar_wait(code_empty(cs), (use - 1) & 1, abort_flag, status);
              const size_t tile = (size_t)pg * Hkv + w.h;
              const uint32_t dst = codes + cs * kCode;
              mbar_arrive_expect_tx(code_full(cs), kPage * (RK + RV) + f8::kScalesPerTile * 4);
              bulk_load_1d(dst, args.P.k_codes + tile * (kPage * RK), kPage * RK, code_full(cs));
              bulk_load_1d(dst + kPage * RK, args.P.v_codes + tile * (kPage * RV), kPage * RV, code_full(cs));
              bulk_load_1d(dst + kPage * (RK + RV), args.P.scales + tile * f8::kScalesPerTile, f8::kScalesPerTile * 4, code_full(cs));
              if (++cs == n_code) {
                cs = 0;
                ++use;
              }
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
      const uint32_t t_s = uniform(tmem_base) + mt * 256, t_o = t_s + 128;       // score buffers; Q' / O accumulator
      const uint32_t ring_u = uniform(ring), ctrl_u = uniform(ctrl), qp_u = uniform(qp) + mt * uniform(a.qp_bytes);
      auto bar = [&](int i) { return ctrl_u + i * 8; };                          // as numbered above
      const uint32_t id_qk = idesc_f16_f32(kRows, kPage), id_pv = idesc_f16_f32_bmn(kRows, RV);
      const uint32_t id_pj = idesc_bf16_f32_bmn(kRows, RK), id_bp = idesc_bf16_f32(kRows, kD);
      const uint32_t hi_k = desc_hi(desc_template(bk.layout, 16, 8 * bk.span)), hi_v = desc_hi(desc_template(bv.layout, 16, 8 * bv.span));
      const uint32_t hi_q = desc_hi(desc_template(2, 16, 1024));
      constexpr int nk = RK / 16, nv = RV / 16;
      // descriptor offset (in 16-byte units) of K step k of a K-major operand: inside a block 2 units per step, then the next block
      const int lgk = bk.bw == 64 ? 2 : bk.bw == 32 ? 1 : 0, lgv = bv.bw == 64 ? 2 : bv.bw == 32 ? 1 : 0;
      auto koff = [](int k, int lg, uint32_t blk) { return (uint32_t)(k >> lg) * blk + (uint32_t)(k & ((1 << lg) - 1)) * 2u; };
      const uint32_t qblk = (uint32_t)(kRows * bk.span) >> 4, kblk = (uint32_t)(kPage * bk.span) >> 4, oblk = (uint32_t)(kRows * bv.span) >> 4;
      const uint32_t pv_b = (uint32_t)(16 * bv.span) >> 4;                       // V page: 16 rows per K step
      const uint32_t dq = desc_lo(16, qp_u);                                     // this tile's Q' operand, and its O_down operand
      int st = 0, use = 0, kt = 0, pn = 0;
      const int nst_u = uniform(nst);
      auto consume = [&](uint32_t& addr, int& stage) {                           // next item of the ring, once it has landed
        mbar_wait_warp(bar(st), use & 1, abort_flag, status);
        addr = ring_u + st * kStageBytes;
        stage = st;
        if (++st == nst_u) {
          st = 0;
          ++use;
        }
      };
      auto drop = [&](int stage) {                                               // an item this tile has no use for
        if (lane == 0) mbar_arrive(bar(4 + stage));
        __syncwarp();
      };
      const bool dual = uniform(a.dual) != 0, fold_k_u = uniform((int)fold_k) != 0, backproj_u = uniform((int)backproj) != 0;
      for (int u = blockIdx.x; u < n_units; u += gridDim.x) {
        const mq::Unit w = mq::decode_unit(a, u, TT);
        if (uniform((int)w.valid) == 0) continue;
        const int wnp0 = uniform(w.np[0]), wnp1 = uniform(w.np[1]), npmax = uniform(w.cnt);
        const int np = mt ? wnp1 : wnp0;
        const bool active = np > 0;
        if (!fold_k_u) {
          uint32_t qa = 0, ua, tmp;
          int qs = 0, us, ts;
          if (wnp0 > 0) {                                                        // tile 0's raw queries
            if (mt == 0) consume(qa, qs);
            else { consume(tmp, ts); drop(ts); }
          }
          if (wnp1 > 0) {                                                        // tile 1's
            if (mt == 1) consume(qa, qs);
            else { consume(tmp, ts); drop(ts); }
          }
          consume(ua, us);
          if (active) {
            if (kt > 0) mbar_wait_warp(bar(30 + mt), (kt - 1) & 1, abort_flag, status);   // the tile's accumulator columns are free
            tc_fence_after();
            const uint32_t da = desc_lo(16, qa), db = desc_lo(kD * bk.span, ua);
#pragma unroll
            for (int k = 0; k < kD / 16; ++k)
              umma_ss(t_o, da + (uint32_t)(((k >> 2) * (kStageBytes / 2) + (k & 3) * 32) >> 4), hi_q, db + (uint32_t)(k * bk.span), hi_k, id_pj, k > 0 ? 1u : 0u);
            umma_commit_warp(bar(20 + mt));
            umma_commit_warp(bar(4 + qs));
            umma_commit_warp(bar(4 + us));
          } else {
            drop(us);
          }
        }
        if (active) mbar_wait_warp(bar(22 + mt), kt & 1, abort_flag, status);
        tc_fence_after();

        // jo counts this tile's own pages within the unit (every page it shares with the other tile, or every second page of
        // the range when the tiles run as two streams over the same rows)
        auto issue_pv = [&](int jo, uint32_t vaddr, int stage) {
          const int n = pn + jo;
          mbar_wait_warp(bar(12 + 2 * mt + (n & 1)), (n >> 1) & 1, abort_flag, status);
          tc_fence_after();
          const uint32_t pa = t_s + (n & 1) * 64;                                // P_n: f16 pairs in the score buffer's first 32 columns
          const uint32_t db = desc_lo(kPage * bv.span, vaddr);
#pragma unroll
          for (int k = 0; k < kPage / 16; ++k) umma_ts(t_o, pa + 8 * k, db + (uint32_t)k * pv_b, hi_v, id_pv, (jo > 0 || k > 0) ? 1u : 0u);
          umma_commit_warp(bar(16 + 2 * mt + (n & 1)));
          umma_commit_warp(bar(4 + stage));                                      // K and V of this page are no longer needed by this tile
        };
        uint32_t prev_v = 0;
        int prev_stage = 0, jo = 0;                                              // the page whose P V is still to be issued; own pages so far
        for (int j = 0; j < npmax; ++j) {
          uint32_t kaddr;
          int stage;
          consume(kaddr, stage);
          const bool mine = dual ? (j & 1) == mt : j < np;
          if (!mine) {
            drop(stage);
            continue;
          }
          const int n = pn + jo;
          if (n >= 2) mbar_wait_warp(bar(16 + 2 * mt + (n & 1)), ((n >> 1) - 1) & 1, abort_flag, status);   // P_(n-2), which sat in this buffer, has been consumed
          tc_fence_after();
          const uint32_t d_tmem = t_s + (n & 1) * 64, db = desc_lo(16, kaddr);
#pragma unroll
          for (int k = 0; k < nk; ++k) umma_ss(d_tmem, dq + koff(k, lgk, qblk), hi_k, db + koff(k, lgk, kblk), hi_k, id_qk, k > 0 ? 1u : 0u);
          umma_commit_warp(bar(8 + 2 * mt + (n & 1)));
          if (jo > 0) issue_pv(jo - 1, prev_v, prev_stage);
          prev_v = kaddr + kPage * RK * 2;
          prev_stage = stage;
          ++jo;
        }
        if (jo > 0) issue_pv(jo - 1, prev_v, prev_stage);
        if (active) umma_commit_warp(bar(24 + mt));
        if (backproj_u) {
          // OUT = O_down U_v^T with O_down handed over as two bf16 terms (value, then residual): two accumulating passes into the
          // tile's score columns, which are idle by now
          uint32_t ua;
          int us;
          consume(ua, us);
          if (active) {
            const uint32_t db = desc_lo(16, ua);
            for (int pass = 0; pass < 2; ++pass) {
              mbar_wait_warp(bar(26 + mt), pass, abort_flag, status);
              tc_fence_after();
#pragma unroll
              for (int k = 0; k < nv; ++k) umma_ss(t_s, dq + koff(k, lgv, oblk), hi_v, db + koff(k, lgv, oblk), hi_v, id_bp, (pass > 0 || k > 0) ? 1u : 0u);
              umma_commit_warp(bar(28 + mt));
            }
            umma_commit_warp(bar(4 + us));
          } else {
            drop(us);
          }
        }
        pn += np;
        kt += active;
      }
    }
  } else if (warp >= 12) {
    // ------------------------------------------------------------------------------------------ expansion of the pages
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    const int et = tid - 12 * 32;                               // 0 .. 127
    int st = 0, use = 0, cs = 0, cuse = 0;
    // All items of the operand ring are filled from here, in order (whoever waits for a stage has seen every earlier phase of its
    // barrier): raw queries and bases are TMA loads that one thread issues.
    auto acquire = [&]() {
      if (use > 0) mbar_wait(empty_bar(st), (use - 1) & 1, abort_flag, status);
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
          mbar_arrive_expect_tx(full_bar(st), bytes);
          issue(ring + st * kStageBytes, full_bar(st));
        } else {
          mbar_arrive(full_bar(st));
        }
      }
      advance();
    };
    if (et == 0) {
      if (!fold_k) {
        tma_prefetch_desc(&tmQ);
        tma_prefetch_desc(&tmUk);
      }
      if (backproj) tma_prefetch_desc(&tmUv);
    }
    for (int u = blockIdx.x; u < n_units; u += gridDim.x) {
      const mq::Unit w = mq::decode_unit(a, u, TT);
      if (!w.valid) continue;
      if (!fold_k) {
        for (int t = 0; t < 2; ++t) {
          if (w.np[t] == 0) continue;
          load((uint32_t)(TT * G) * kD * 2, [&](uint32_t dst, uint32_t bar) {
            tma_load_4d(dst, &tmQ, 0, w.h * G, w.tok0[t], w.b, bar);
            tma_load_4d(dst + kStageBytes / 2, &tmQ, 64, w.h * G, w.tok0[t], w.b, bar);
          });
        }
        load(kD * RK * 2, [&](uint32_t dst, uint32_t bar) {
          for (int i = 0; i < bk.nb; ++i) tma_load_3d(dst + i * kD * bk.span, &tmUk, i * bk.bw, 0, a.L.uk_stride ? w.h : 0, bar);
        });
      }
      for (int j = 0; j < w.cnt; ++j) {
        const int live = w.seq_len - (w.p_lo + j) * kPage;      // rows of the page that belong to the sequence (64 or more: all)
        mbar_wait(code_full(cs), cuse & 1, abort_flag, status);
        const uint8_t* src = codes_ptr + cs * kCode;
        constexpr int NK = (RK * 4 + 127) / 128, NV = (RV * 4 + 127) / 128;
        static_assert(NK <= 4 && NV <= 4, "pieces per thread");
        uint4 kq[NK], vq[NV];
#pragma unroll
        for (int i = 0; i < NK; ++i)
          if (RK % 32 == 0 || et + 128 * i < RK * 4) kq[i] = reinterpret_cast<const uint4*>(src)[et + 128 * i];
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (RV % 32 == 0 || et + 128 * i < RV * 4) vq[i] = reinterpret_cast<const uint4*>(src + kPage * RK)[et + 128 * i];
        float2 sc = make_float2(0.f, 0.f);
        if (et == 0) sc = *reinterpret_cast<const float2*>(src + kPage * (RK + RV));
        acquire();
        uint8_t* dst = base_ptr + st * kStageBytes;
        auto expand = [&](const uint4& q, uint4& lo, uint4& hi) {
          lo = make_uint4(f8::e4m3x2_to_f16x2(q.x & 0xffffu), f8::e4m3x2_to_f16x2(q.x >> 16), f8::e4m3x2_to_f16x2(q.y & 0xffffu), f8::e4m3x2_to_f16x2(q.y >> 16));
          hi = make_uint4(f8::e4m3x2_to_f16x2(q.z & 0xffffu), f8::e4m3x2_to_f16x2(q.z >> 16), f8::e4m3x2_to_f16x2(q.w & 0xffffu), f8::e4m3x2_to_f16x2(q.w >> 16));
        };
#pragma unroll
        for (int i = 0; i < NK; ++i) {
          const int piece = et + 128 * i, row = piece / (RK / 16), c = piece % (RK / 16) * 16;
          if (RK % 32 == 0 || piece < RK * 4) {
            uint4 lo, hi;
            expand(kq[i], lo, hi);
            *reinterpret_cast<uint4*>(dst + block_offset(bk, kPage, row, c)) = lo;
            *reinterpret_cast<uint4*>(dst + block_offset(bk, kPage, row, c + 8)) = hi;
          }
        }
        dst += kPage * RK * 2;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int piece = et + 128 * i, row = piece / (RV / 16), c = piece % (RV / 16) * 16;
          if (RV % 32 == 0 || piece < RV * 4) {
            uint4 lo, hi;
            expand(vq[i], lo, hi);
            if (row >= live) lo = hi = make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4*>(dst + block_offset(bv, kPage, row, c)) = lo;
            *reinterpret_cast<uint4*>(dst + block_offset(bv, kPage, row, c + 8)) = hi;
          }
        }
        if (et == 0) {
          page_scales[st].x = sc.x;
          page_scales[st].y = sc.y;
        }
        fence_proxy_async_smem();                               // generic writes -> visible to the tensor core's reads
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(full_bar(st));
          mbar_arrive(code_empty(cs));
        }
        advance();
        if (++cs == n_code) {
          cs = 0;
          ++cuse;
        }
      }
      if (backproj)
        load(kD * RV * 2, [&](uint32_t dst, uint32_t bar) {
          for (int i = 0; i < bv.nb; ++i) tma_load_3d(dst + i * kD * bv.span, &tmUv, i * bv.bw, 0, a.L.uv_stride ? w.h : 0, bar);
        });
    }
  } else {
    // ------------------------------------------------------------------------------------------ softmax / epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    const int t = (warp - 4) >> 2;                              // the tile this warp works for
    const int q4 = warp & 3;                                    // TMEM lane quarter this warp may access
    const int row = 32 * q4 + lane;                             // row of the tile = TMEM lane
    const uint32_t t_lane = tmem_base + ((uint32_t)(32 * q4) << 16) + t * 256;
    const uint32_t t_out = t_lane + 128;                        // Q' / O columns
    uint8_t* my_qp = qp_ptr + t * a.qp_bytes;
    const float c = kLog2e * rsqrtf((float)kD);                 // scores are scaled by 1/sqrt(d_h); exponent in base 2
    const int d_out = fold_v ? RV : kD;
    int kt = 0, pn = 0;
    int item = 0;                                               // ring items issued before the current unit
    auto arrive_warp = [&](uint32_t bar) {                      // after every lane's shared/TMEM accesses are ordered
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    for (int u = blockIdx.x; u < n_units; u += gridDim.x) {
      const mq::Unit w = mq::decode_unit(a, u, TT);
      if (!w.valid) continue;
      const int lead = lead_of(w);
      const int item0 = item + lead;
      item += lead + w.cnt + (backproj ? 1 : 0);
      if (w.np[t] == 0) continue;
      const int np = w.np[t];
      const int tok = w.tok0[t] + row / G, g = row - (row / G) * G;
      const bool row_valid = tok < w.q_len && row < TT * G;
      const int q_pos = w.q_start + min(tok, w.q_len - 1);      // rows past the end behave like the last valid token

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
            tmem_ld16(t_out + c0, *reinterpret_cast<uint32_t(*)[16]>(&x));
            tmem_ld_wait();
          }
        };
        if (!fold_k) {
          mbar_wait(qacc_full(t), kt & 1, abort_flag, status);
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
        c_row = f8::pow2(e) * c;
        for (int c0 = 0; c0 < RK; c0 += 16) {
          float x[16];
          piece(c0, x);
          uint32_t pk[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const __half2 v = __floats2half2_rn(x[2 * i] * norm, x[2 * i + 1] * norm);
            pk[i] = *reinterpret_cast<const uint32_t*>(&v);
          }
          *reinterpret_cast<uint4*>(my_qp + block_offset(bk, kRows, row, c0)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
          *reinterpret_cast<uint4*>(my_qp + block_offset(bk, kRows, row, c0 + 8)) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
        }
        fence_proxy_async_smem();
        tc_fence_before();
        arrive_warp(qp_ready(t));
      }

      float m_ref = -INFINITY, l = 0.f;                         // the largest exponent when the reference was last set; row sum
      int stg = (item0 + (a.dual ? t : 0)) % nst;               // operand stage of the next page
      for (int jo = 0; jo < np; ++jo) {
        const int j = a.dual ? 2 * jo + t : jo;                 // the page within the unit's range
        const int n = pn + jo, sb = n & 1;
        mbar_wait(s_full(t, sb), (n >> 1) & 1, abort_flag, status);
        tc_fence_after();
        uint32_t sv[64];
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld16(t_lane + sb * 64 + i * 16, *reinterpret_cast<uint32_t(*)[16]>(&sv[16 * i]));
        // written before the arrival that these scores' product waited for; the stage is not refilled before P is handed over
        const float ks = page_scales[stg].x, vs = page_scales[stg].y;
        stg += a.dual ? 2 : 1;
        while (stg >= nst) stg -= nst;
        tmem_ld_wait();
        float* s = reinterpret_cast<float*>(sv);
        const int p0 = (w.p_lo + j) * kPage;
        const bool edge = p0 + kPage - 1 > q_pos;
        if (edge) {                                             // a boundary page: positions after the row's own are masked
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (p0 + i > q_pos) s[i] = -INFINITY;
        }
        float mx0 = max3(s[0], s[1], s[2]), mx1 = max3(s[3], s[4], s[5]);     // two chains of three-input maxima
#pragma unroll
        for (int i = 6; i < 62; i += 4) {
          mx0 = max3(mx0, s[i], s[i + 1]);
          mx1 = max3(mx1, s[i + 2], s[i + 3]);
        }
        const float f = fmaxf(c_row * ks, 1e-37f);              // above zero: masked scores stay -inf
        const int ev = min(max((int)((__float_as_uint(vs) >> 23) & 255u) - 127, -126), 126);
        const float mx = fmaf(fmaxf(max3(mx0, s[62], s[63]), mx1), f, (float)ev);     // the rounded exponents are what the reference goes by
        if (jo == 0) {
          m_ref = mx;                                           // -inf when a part of a split range begins behind the row's position
        } else if (__any_sync(0xffffffffu, mx - m_ref > kRescaleLog2)) {
          mbar_wait(p_free(t, (n - 1) & 1), ((n - 1) >> 1) & 1, abort_flag, status);   // every earlier update of O is complete
          tc_fence_after();
          const bool grown = mx - m_ref > kRescaleLog2;         // a row's bits do not depend on its neighbours
          const float r = grown ? fast_exp2(m_ref - mx) : 1.f;
          l *= r;
          if (grown) m_ref = mx;
          for (int c0 = 0; c0 < RV; c0 += 16) {
            uint32_t v[16];
            tmem_ld16(t_out + c0, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * r);
            tmem_st16(t_out + c0, v);
          }
          tmem_st_wait();
        }
        const float ref = m_ref > -INFINITY ? m_ref - kHeadroomLog2 : 0.f;
        const uint64_t f2 = pack2(f, f), ev2 = pack2((float)ev, (float)ev), ref2 = pack2(-ref, -ref);
        uint64_t sum2 = pack2(0.f, 0.f);
        uint32_t pk[32];
        // Part of the pairs go to the FMA pipe as a polynomial where the exponentials set the pace (small ranks); it cannot
        // return an exact zero, so a page on which some row of the warp has masked positions takes the special-function unit.
        auto exponentials = [&](auto poly_tag) {
          constexpr bool kPoly = decltype(poly_tag)::value;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float x0, x1, e0, e1;
            unpack2(add2(fma2(pack2(s[2 * i], s[2 * i + 1]), f2, ev2), ref2), x0, x1);
            if (kPoly && (i % kPolyEvery) == 0) {
              exp2_pair_fma(pack2(fmaxf(x0, -125.f), fmaxf(x1, -125.f)), e0, e1);
            } else {
              e0 = fast_exp2(x0);
              e1 = fast_exp2(x1);
            }
            sum2 = add2(sum2, pack2(e0, e1));
            const __half2 v = __floats2half2_rn(e0, e1);
            pk[i] = *reinterpret_cast<const uint32_t*>(&v);
          }
        };
        if ((RK + RV <= 160) && !__any_sync(0xffffffffu, edge)) exponentials(std::true_type{});
        else exponentials(std::false_type{});
        {
          float a0, a1;
          unpack2(sum2, a0, a1);
          l = fmaf(a0 + a1, f8::pow2(-ev), l);
        }
        // P_n replaces the scores in TMEM: f16 pairs in the first 32 columns of the buffer, where the P V product reads its A operand
        tmem_st16(t_lane + sb * 64, *reinterpret_cast<uint32_t(*)[16]>(&pk[0]));
        tmem_st16(t_lane + sb * 64 + 16, *reinterpret_cast<uint32_t(*)[16]>(&pk[16]));
        tmem_st_wait();
        tc_fence_before();
        arrive_warp(p_full(t, sb));
      }

      // ---- epilogue of the unit
      mbar_wait(o_full(t), kt & 1, abort_flag, status);
      tc_fence_after();
      const float ref = m_ref - kHeadroomLog2;
      const float inv = 1.0f / l;
      __nv_bfloat16* orow = a.out + (size_t)w.b * a.out_stride_b + (size_t)tok * a.out_stride_t + (size_t)(w.h * G + g) * d_out;
      if (a.n_split > 1) {
        // partial result of this part of the page range: unnormalised mix, reference (base-2 units) and row sum
        const size_t prow = (((size_t)w.b * a.n_q + tok) * a.L.Hq + w.h * G + g) * a.n_parts + (a.dual ? 2 * w.split + t : w.split);
        for (int c0 = 0; c0 < RV; c0 += 16) {
          uint32_t v[16];
          tmem_ld16(t_out + c0, v);
          tmem_ld_wait();
          if (row_valid) {
            float4* dst = reinterpret_cast<float4*>(a.part_o + prow * RV + c0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              dst[i] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
          }
        }
        if (row_valid) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(ref, l);
      } else if (fold_v) {
        for (int c0 = 0; c0 < RV; c0 += 16) {
          uint32_t v[16], pk[8];
          tmem_ld16(t_out + c0, v);
          tmem_ld_wait();
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
            tmem_ld16(t_out + c0, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float x0 = __uint_as_float(v[2 * i]) * inv, x1 = __uint_as_float(v[2 * i + 1]) * inv;
              uint32_t hi, lo;
              split_bf16(x0, x1, hi, lo);
              pk[i] = pass ? lo : hi;
            }
            *reinterpret_cast<uint4*>(my_qp + block_offset(bv, kRows, row, c0)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            *reinterpret_cast<uint4*>(my_qp + block_offset(bv, kRows, row, c0 + 8)) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
          }
          fence_proxy_async_smem();
          tc_fence_before();
          arrive_warp(od_ready(t));
          mbar_wait(out_full(t), pass, abort_flag, status);     // the pass has read the operand (after the second: OUT is complete)
          tc_fence_after();
        }
        for (int c0 = 0; c0 < kD; c0 += 16) {
          uint32_t v[16], pk[8];
          tmem_ld16(t_lane + c0, v);
          tmem_ld_wait();
          pack16(v, 1.0f, pk);
          if (row_valid) {
            *reinterpret_cast<uint4*>(orow + c0) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            *reinterpret_cast<uint4*>(orow + c0 + 8) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
          }
        }
      }
      if (row_valid && a.out_lse && a.n_split == 1)
        a.out_lse[((size_t)w.b * a.n_q + tok) * a.L.Hq + w.h * G + g] = kLn2 * (ref + log2f(l));
      tc_fence_before();
      arrive_warp(unit_done(t));                                // the tile's TMEM columns and operand region are free
      pn += np;
      ++kt;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem_base, mq::kTmemCols);
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
