// Attention of a few causal query rows per head over the 8-bit floating-point cache (speculative decode: up to 64 rows of a KV head,
// tokens times query heads): the page loop of stief_f8_decode.cuh with 16 query rows per warp.  A tile of the tensor-core
// kernel (stief_f8_mq.cuh) would be mostly empty, and its expansion of the pages, not the memory, would set the pace (8 tokens
// over 4 x 32768 at 64/64: 127 us there).
//
// One CTA per (sequence, KV head, part of the page range).  With more than 16 rows, 2 or 4 warps read the same page, each for its 16
// rows, so a page is fetched once for all of them.
//   queries  Q' = q U_k on mma.sync (raw rows from global memory, U_k through shared memory), rounded to f16 once, each row scaled
//            by the power of two that brings its largest element to 2^11 .. 2^12
//   pages    as in the decode kernel: codes to f16 in registers, weights 2^(x + e - ref) with the value scale 2^e in the exponent,
//            O^T = V^T P^T with two groups of 8 rows as the columns of P^T
// The parts' mixes, sums and references are merged by f8_mq_combine_kernel.
//
// Measured with that kernel (4 x 32768 tokens, 32 query heads over 8, four parts): ranks 64/64 4 / 8 / 16 tokens 38 / 59 / 100 us, 128/128
// 8 tokens 100.  Two warps that read the same page convert it twice, which sets the pace from 32 rows on; 32 rows in one warp ran at 75 us where
// 16 in two ran at 68 (registers, half the warps to hide a page's chain), and the tensor-core kernel at 127.
#pragma once

#include "stief_f8_decode.cuh"
#include "stief_f8_mq.cuh"

namespace stief {
namespace f8rows {

using f8::PageTile;

constexpr int kMaxRows = 64;                     // query rows of a KV head
constexpr int kWarps = 8, kProducers = 4, kThreads = (kWarps + kProducers) * 32, kConsumers = kWarps * 32;
constexpr int kMaxStages = 32;

template <int RK, int RV>
struct Cfg {
  static constexpr int K_BYTES = PageTile<RK>::BYTES, V_BYTES = PageTile<RV>::BYTES, S_BYTES = f8::kScalesPerTile * 4;
  static constexpr int TX_BYTES = K_BYTES + V_BYTES + S_BYTES;
  static constexpr int STAGE_BYTES = (TX_BYTES + 1023) / 1024 * 1024;
  static constexpr int CTRL_BYTES = 1024;
  static constexpr int U_PITCH = RK * 2 + 16;              // bytes of a basis row in shared memory: ldmatrix reads eight of them without conflicts
  static_assert(4 * kWarps * 16 <= kMaxRows * (RK + 4), "the warps' references and sums fit where the queries were");
  static constexpr int Q_PITCH = RK + 4;                   // floats of a projected row
  static constexpr int MISC = CTRL_BYTES + kD * U_PITCH + kMaxRows * Q_PITCH * 4;
  static constexpr int BUDGET = 232448 - 1024 - MISC;
  // a multiple of the warps: a stage then has one lane's pages only, which sees every phase of its barriers
  static constexpr int NS = (BUDGET / STAGE_BYTES > kMaxStages ? kMaxStages : BUDGET / STAGE_BYTES) / kWarps * kWarps;
  static constexpr int SMEM_BYTES = 1024 + NS * STAGE_BYTES + MISC;
  static_assert(NS >= kWarps && kWarps % kProducers == 0, "a stage for each warp that has a page of its own, fetched by one producer");
  static_assert(kWarps * 16 * (RV + 4) * 4 <= NS * STAGE_BYTES, "the warps' results fit the ring once it is idle");
};

template <int RK, int RV>
__global__ void __launch_bounds__(kThreads, 1)
f8_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const f8mq::Args args) {
  using C = Cfg<RK, RV>;
  using TK = PageTile<RK>;
  using TV = PageTile<RV>;
  constexpr int NS = C::NS, NCK = TK::NC, NCV = TV::NC;
  const mq::Args& a = args.m;
  extern __shared__ uint8_t smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* ring_ptr = smem_raw + (ring - smem_u32(smem_raw));
  uint8_t* ctrl_ptr = ring_ptr + NS * C::STAGE_BYTES;
  const uint32_t ctrl = ring + NS * C::STAGE_BYTES;
  auto full_bar = [&](int s) { return ctrl + s * 8; };
  auto empty_bar = [&](int s) { return ctrl + (kMaxStages + s) * 8; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl_ptr + 2 * kMaxStages * 8);
  const uint32_t u_smem = ctrl + C::CTRL_BYTES;
  uint8_t* u_ptr = ctrl_ptr + C::CTRL_BYTES;
  float* qp = reinterpret_cast<float*>(u_ptr + kD * C::U_PITCH);

  launch_dependents();
  // warps per page: one for every 16 rows (rounded up to a power of two)
  const int G = a.L.G, Hkv = a.L.Hkv;
  const int lg = a.n_q * G <= 16 ? 0 : a.n_q * G <= 32 ? 1 : 2, groups = 1 << lg, lanes = kWarps >> lg;
  if (tid == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), groups);
    }
    *abort_flag = 0;
    mbar_fence_init();
  }
  __syncthreads();
  grid_dependency_wait();                                       // everything below reads the results of earlier kernels

  const int split = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  int ql = a.q_lens ? a.q_lens[b] : a.n_q;
  ql = min(max(ql, 0), a.n_q);
  const int len = a.Bt.seq_lens[b], q_start = len - ql;
  if (ql == 0) return;
  if (q_start < 0 || (len - 1) / kPage + 1 > a.Bt.max_pages) {  // fewer cached tokens than query rows, or a table too short
    if (tid == 0) report(a.status, STIEF_ERR_BOUNDS);
    return;
  }
  const int all = (len - 1) / kPage + 1;
  const int lo = (int)((long long)split * all / a.n_split), hi = (int)((long long)(split + 1) * all / a.n_split), np = hi - lo;
  if (np == 0) return;

  if (warp >= kWarps) {
    // ------------------------------------------------------------------ producer warps: page i of the CTA in stage i mod NS
    const int pw = warp - kWarps;
    if (lane == 0) {
      if constexpr (!TK::BULK) tma_prefetch_desc(&tmK);
      if constexpr (!TV::BULK) tma_prefetch_desc(&tmV);
    }
    int tbl = 0, win = -1;
    for (int i = pw; i < np; i += kProducers) {
      if ((i >> 5) != win) {                                    // block-table entries of a window of 32 pages, one per lane
        win = i >> 5;
        const int idx = lo + (win << 5) + lane;
        tbl = idx < hi ? a.Bt.block_table[(size_t)b * a.Bt.max_pages + idx] : 0;
      }
      int page = __shfl_sync(0xffffffffu, tbl, i & 31);
      if (page < 0 || page >= a.L.num_pages) {
        if (lane == 0) report(a.status, STIEF_ERR_BOUNDS);
        page = 0;
      }
      const int slot = i % NS, use = i / NS;
      if (lane == 0) {
        if (use > 0) mbar_wait(empty_bar(slot), (use - 1) & 1, abort_flag, a.status);
        const uint32_t st = ring + slot * C::STAGE_BYTES;
        const size_t tile = (size_t)page * Hkv + h;
        mbar_arrive_expect_tx(full_bar(slot), C::TX_BYTES);
        if constexpr (TK::BULK) bulk_load_1d(st, args.P.k_codes + tile * C::K_BYTES, C::K_BYTES, full_bar(slot));
        else tma_load_2d(st, &tmK, 0, (int)tile * TK::LINES, full_bar(slot));
        if constexpr (TV::BULK) bulk_load_1d(st + C::K_BYTES, args.P.v_codes + tile * C::V_BYTES, C::V_BYTES, full_bar(slot));
        else tma_load_2d(st + C::K_BYTES, &tmV, 0, (int)tile * TV::LINES, full_bar(slot));
        bulk_load_1d(st + C::K_BYTES + C::V_BYTES, args.P.scales + tile * f8::kScalesPerTile, C::S_BYTES, full_bar(slot));
      }
      __syncwarp();
    }
    return;
  }

  // ------------------------------------------------------------------ consumer warps: 16 rows of the pages of one lane
  const int gid = lane >> 2, tid4 = lane & 3, l7 = lane & 7, mat = lane >> 3;
  const int grp = warp & (groups - 1), pl = warp >> lg, n_rows = ql * G, row0 = 16 * grp;
  const __nv_bfloat16* Uk = a.L.U_k ? a.L.U_k + (size_t)h * a.L.uk_stride : nullptr;
  const int d_q = Uk ? kD : RK;
  auto q_row = [&](int row) {                                   // row = token * G + head of the group
    return args.q + (size_t)b * args.q_stride_b + (size_t)(row / G) * args.q_stride_t + (size_t)(h * G + row % G) * d_q;
  };

  // ---- Q' = q U_k: the lanes of a row group share its columns
  if (Uk) {
    uint32_t qa[8][4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = row0 + gid + 8 * e;
      const uint32_t* src = reinterpret_cast<const uint32_t*>(q_row(min(row, n_rows - 1))) + tid4;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        qa[ks][e] = row < n_rows ? __ldg(src + 8 * ks) : 0u;
        qa[ks][2 + e] = row < n_rows ? __ldg(src + 8 * ks + 4) : 0u;
      }
    }
    constexpr int kPieces = kD * RK / 8;                        // of 16 bytes
    for (int i = tid; i < kPieces; i += kConsumers) {
      const int d = i / (RK / 8), c = i % (RK / 8);
      *reinterpret_cast<uint4*>(u_ptr + d * C::U_PITCH + c * 16) = __ldg(reinterpret_cast<const uint4*>(Uk) + i);
    }
    bar1(kConsumers);
    for (int t = pl; t < RK / 8; t += lanes) {
      float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        uint32_t u[4];
        ldsm_x4_t(u_smem + (32 * kk + lane) * C::U_PITCH + t * 16, u[0], u[1], u[2], u[3]);
        mma_bf16(acc, qa[2 * kk], u[0], u[1]);
        mma_bf16(acc, qa[2 * kk + 1], u[2], u[3]);
      }
      *reinterpret_cast<float2*>(qp + (row0 + gid) * C::Q_PITCH + 8 * t + 2 * tid4) = make_float2(acc[0], acc[1]);
      *reinterpret_cast<float2*>(qp + (row0 + gid + 8) * C::Q_PITCH + 8 * t + 2 * tid4) = make_float2(acc[2], acc[3]);
    }
  } else {
    for (int i = tid; i < 16 * groups * (RK / 8); i += kConsumers) {
      const int row = i / (RK / 8), c = i % (RK / 8);
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      if (row < n_rows) w = __ldg(reinterpret_cast<const uint4*>(q_row(row)) + c);
      float* dst = qp + row * C::Q_PITCH + 8 * c;
      const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<float2*>(dst + 2 * e) = make_float2(bf16_lo(v[e]), bf16_hi(v[e]));
    }
  }
  bar1(kConsumers);

  // ---- A operand of the scores, in the order of channels in which the codes arrive: rows gid (e = 0) and gid + 8
  float fac[2];
  uint32_t qa[NCK][4];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float* src = qp + (row0 + gid + 8 * e) * C::Q_PITCH + 4 * tid4;
    float4 x[NCK];
    float top = 0.f;
#pragma unroll
    for (int ch = 0; ch < NCK; ++ch) {
      x[ch] = *reinterpret_cast<const float4*>(src + 16 * ch);
      top = fmaxf(top, fmaxf(fmaxf(fabsf(x[ch].x), fabsf(x[ch].y)), fmaxf(fabsf(x[ch].z), fabsf(x[ch].w))));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int ex = top > 0.f ? min(max((int)(__float_as_uint(top) >> 23) - 127, -112), 126) - 11 : 0;
    const float norm = f8::pow2(-ex);
    fac[e] = f8::pow2(ex) * (kLog2e * 0.08838834764831845f);
#pragma unroll
    for (int ch = 0; ch < NCK; ++ch) {
      qa[ch][e] = f8::pack_f16(x[ch].x * norm, x[ch].y * norm);
      qa[ch][2 + e] = f8::pack_f16(x[ch].z * norm, x[ch].w * norm);
    }
  }
  // first position that each of the thread's rows does not attend; the warp's smallest
  int end[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) end[e] = q_start + min((row0 + gid + 8 * e) / G, ql - 1) + 1;
  const int first_end = q_start + min(row0 / G, ql - 1) + 1;

  // addresses of the ldmatrix instructions that cover 16 tokens (as in the decode kernel)
  constexpr int LK = (2 * NCK + 3) / 4, LV = (2 * NCV + 3) / 4;
  uint32_t koff[LK], voff[LV];
#pragma unroll
  for (int i = 0; i < LK; ++i) {
    const int n = min(4 * i + mat, 2 * NCK - 1);
    koff[i] = TK::chunk(8 * (n / NCK) + l7, n % NCK);
  }
#pragma unroll
  for (int i = 0; i < LV; ++i) {
    const int n = min(4 * i + mat, 2 * NCV - 1);
    voff[i] = TV::chunk(8 * (n & 1) + l7, n >> 1);
  }

  float m[2] = {-INFINITY, -INFINITY}, em[2] = {0.f, 0.f}, l[2] = {0.f, 0.f}, n[2] = {f8::kNoSum, f8::kNoSum};      // as in the decode kernel
  float o[NCV][2][4];                                           // channels 16 i + 2 gid (+ 1) of rows 2 tid4, + 1, and of those 8 further
#pragma unroll
  for (int i = 0; i < NCV; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) o[i][e][0] = o[i][e][1] = o[i][e][2] = o[i][e][3] = 0.f;

  for (int i = pl; i < np; i += lanes) {
    const int slot = i % NS;
    mbar_wait(full_bar(slot), (i / NS) & 1, abort_flag, a.status);
    const uint32_t kt = ring + slot * C::STAGE_BYTES, vt = kt + C::K_BYTES;
    const int p0 = (lo + i) * kPage, live = len - p0;           // rows of the page that belong to the sequence (64 or more: all)
    float ks, vs;
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(ks), "=f"(vs) : "r"(vt + C::V_BYTES));

    // ---- scores: x[e][4 j + 2 u + c] is token 16 j + 8 u + 2 tid4 + c for row gid + 8 e
    float x[2][16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float s4[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) s4[u][0] = s4[u][1] = s4[u][2] = s4[u][3] = 0.f;
      uint32_t w[4 * LK];
#pragma unroll
      for (int q = 0; q < LK; ++q) {
        const uint32_t addr = kt + (koff[q] ^ TK::step(j)) + 16 * j * RK;
        if (2 * NCK - 4 * q >= 4) ldsm_x4(addr, w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
        else ldsm_x2(addr, w[4 * q], w[4 * q + 1]);
      }
#pragma unroll
      for (int n = 0; n < 2 * NCK; ++n) {
        uint32_t b0, b1;
        f8::expand4(w[n], b0, b1);
        f8::mma_f16(s4[n / NCK], qa[n % NCK][0], qa[n % NCK][1], qa[n % NCK][2], qa[n % NCK][3], b0, b1);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          x[0][4 * j + 2 * u + c] = s4[u][c];
          x[1][4 * j + 2 * u + c] = s4[u][2 + c];
        }
    }
    const float evf = f8::scale_exponent(vs);
    float above[2], tops[2];
    bool vanish[2], seldom = false;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float f = f8::score_factor(fac[e], ks);
#pragma unroll
      for (int t = 0; t < 16; ++t) x[e][t] = __fmul_rn(x[e][t], f);      // the rounded product is what the reference goes by
      if (p0 + kPage > first_end) {
#pragma unroll
        for (int t = 0; t < 16; ++t)
          if (p0 + 16 * (t >> 2) + 8 * ((t >> 1) & 1) + 2 * tid4 + (t & 1) >= end[e]) x[e][t] = -INFINITY;
      }
      float top = x[e][0];
#pragma unroll
      for (int t = 1; t < 16; ++t) top = fmaxf(top, x[e][t]);
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      tops[e] = top;
      const float beyond = top - m[e];
      above[e] = beyond + (evf - em[e]);
      vanish[e] = f8::may_vanish(beyond, above[e]);
      seldom |= above[e] > f8::kTopWeight || vanish[e] || top > n[e] + f8::kSumGrown;
    }
    if (__any_sync(0xffffffffu, seldom)) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const bool grown = above[e] > f8::kTopWeight;           // (a row that has seen nothing keeps -inf)
        const float alpha = grown ? fast_exp2(f8::kTopWeight - above[e]) : 1.f;
        const float a0 = __shfl_sync(0xffffffffu, alpha, 8 * tid4), a1 = __shfl_sync(0xffffffffu, alpha, 8 * tid4 + 4);
#pragma unroll
        for (int c = 0; c < NCV; ++c) {
          o[c][e][0] *= a0;
          o[c][e][1] *= a1;
          o[c][e][2] *= a0;
          o[c][e][3] *= a1;
        }
        if (grown) {
          m[e] = tops[e];
          em[e] = evf - f8::kTopWeight;
        }
        if (tops[e] > n[e] + f8::kSumGrown) {
          l[e] *= fast_exp2(n[e] - tops[e]);
          n[e] = tops[e];
        }
        if (vanish[e]) {
          float own = 0.f;
#pragma unroll
          for (int t = 0; t < 16; ++t) own += fast_exp2(x[e][t] - tops[e]);
          l[e] = fmaf(own, fast_exp2(tops[e] - n[e]), l[e]);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float ref = m[e] > -INFINITY ? m[e] : 0.f, shift = evf - em[e];
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        x[e][t] = fast_exp2((x[e][t] - ref) + shift);
        sum += x[e][t];
      }
      l[e] = fmaf(sum, above[e] < f8::kSumLow ? 0.f : fast_exp2((m[e] - n[e]) - shift), l[e]);
    }

    // ---- mix
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t p[2][2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        p[e][0] = f8::pack_f16(x[e][4 * j], x[e][4 * j + 1]);
        p[e][1] = f8::pack_f16(x[e][4 * j + 2], x[e][4 * j + 3]);
      }
      uint32_t w[4 * LV];
#pragma unroll
      for (int q = 0; q < LV; ++q) {
        const uint32_t addr = vt + (voff[q] ^ TV::step(j)) + 16 * j * RV;
        if (2 * NCV - 4 * q >= 4) ldsm_x4_t(addr, w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
        else f8::ldsm_x2_t(addr, w[4 * q], w[4 * q + 1]);
      }
      if (live < kPage) {                                       // rows past the end hold unspecified codes, NaN among them
        const int t0 = 16 * j + 2 * tid4;
        const uint32_t k0 = (t0 < live ? 0xffffu : 0u) | (t0 + 1 < live ? 0xffff0000u : 0u);
        const uint32_t k1 = (t0 + 8 < live ? 0xffffu : 0u) | (t0 + 9 < live ? 0xffff0000u : 0u);
#pragma unroll
        for (int n = 0; n < 2 * NCV; ++n) w[n] &= (n & 1) ? k1 : k0;
      }
#pragma unroll
      for (int c = 0; c < NCV; ++c) {
        uint32_t e0, d0, e1, d1;                                // even and odd channels, tokens 0-7 and 8-15 of the sixteen
        f8::expand4(__byte_perm(w[2 * c], 0u, 0x3120), e0, d0);
        f8::expand4(__byte_perm(w[2 * c + 1], 0u, 0x3120), e1, d1);
#pragma unroll
        for (int e = 0; e < 2; ++e) f8::mma_f16(o[c][e], e0, d0, e1, d1, p[e][0], p[e][1]);
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty_bar(slot));
  }

  // ------------------------------------------------------------------ merge the lanes of each row group, in the idle ring
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
    l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
  }
  bar1(kConsumers);                                             // every page has been consumed
  constexpr int WP = RV + 4;
  float* wo = reinterpret_cast<float*>(ring_ptr);               // [warp][16][WP]
  float* wm = qp;                                               // [warp][16], then the sums and their references
  float *wl = wm + kWarps * 16, *wn = wl + kWarps * 16, *we = wn + kWarps * 16;
#pragma unroll
  for (int c = 0; c < NCV; ++c)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      *reinterpret_cast<float2*>(wo + (warp * 16 + 8 * e + 2 * tid4) * WP + 16 * c + 2 * gid) = make_float2(o[c][e][0], o[c][e][2]);
      *reinterpret_cast<float2*>(wo + (warp * 16 + 8 * e + 2 * tid4 + 1) * WP + 16 * c + 2 * gid) = make_float2(o[c][e][1], o[c][e][3]);
    }
  if (tid4 == 0) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      wm[warp * 16 + gid + 8 * e] = m[e];
      wl[warp * 16 + gid + 8 * e] = l[e];
      wn[warp * 16 + gid + 8 * e] = n[e];
      we[warp * 16 + gid + 8 * e] = em[e];
    }
  }
  bar1(kConsumers);
  for (int idx = tid; idx < n_rows * (RV / 4); idx += kConsumers) {
    const int row = idx / (RV / 4), c = idx % (RV / 4), g = row >> 4, r = row & 15;
    float M = -INFINITY, E = 0.f, N = f8::kNoSum;
    for (int p = 0; p < lanes; ++p) {
      const int w = (p << lg) + g;
      if ((wm[w * 16 + r] - M) + (we[w * 16 + r] - E) > 0.f) {
        M = wm[w * 16 + r];
        E = we[w * 16 + r];
      }
      N = fmaxf(N, wn[w * 16 + r]);
    }
    float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
    float den = 0.f;
    for (int p = 0; p < lanes; ++p) {
      const int w = (p << lg) + g;
      const float mw = wm[w * 16 + r];
      if (mw == -INFINITY && wl[w * 16 + r] == 0.f) continue;   // a lane that the row attends nothing of (with scores that are all NaN the sum is NaN)
      const float f = fast_exp2((mw - M) + (we[w * 16 + r] - E));
      const float4 v = *reinterpret_cast<const float4*>(wo + (w * 16 + r) * WP + 4 * c);
      num.x = fmaf(v.x, f, num.x);
      num.y = fmaf(v.y, f, num.y);
      num.z = fmaf(v.z, f, num.z);
      num.w = fmaf(v.w, f, num.w);
      den = fmaf(wl[w * 16 + r], fast_exp2(wn[w * 16 + r] - N), den);
    }
    const float half = fast_exp2(0.5f * ((M - N) + E)), over = half / den;
    const size_t prow = (((size_t)b * a.n_q + row / G) * a.L.Hq + h * G + row % G) * a.n_parts + split;
    *reinterpret_cast<float4*>(a.part_o + prow * RV + 4 * c) = make_float4(num.x * half * over, num.y * half * over, num.z * half * over, num.w * half * over);
    if (c == 0) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(N, den);
  }
}

}  // namespace f8rows

// One launcher per key rank (in the decode kernel's translation units)
cudaError_t launch_f8_rows_rk32(const f8mq::Args& a, cudaStream_t st);
cudaError_t launch_f8_rows_rk48(const f8mq::Args& a, cudaStream_t st);
cudaError_t launch_f8_rows_rk64(const f8mq::Args& a, cudaStream_t st);
cudaError_t launch_f8_rows_rk96(const f8mq::Args& a, cudaStream_t st);
cudaError_t launch_f8_rows_rk128(const f8mq::Args& a, cudaStream_t st);

}  // namespace stief
