// Decode attention over the 8-bit floating-point cache, every rank: one query token per sequence,
//     out = softmax((q U_k) (c_k S_k)^T / sqrt(128)) (c_v S_v) U_v^T,   S_k, S_v one power of two per page and head,
// in the persistent split-T form of stief_decode.cuh (same partition of the batch's pages over the CTAs, same workspace, merge,
// combine and launch overlap).  Bound by memory: r_k + r_v bytes per cached (token, KV head) are read once.
//
// Every page of a CTA's range belongs to one of eight consumer warps, taken in turn; four producer warps fetch the pages into
// the warps' own ring stages (K tile, V tile, 16 bytes of scales).  A warp works through a page of 64 tokens alone:
//   scores  mma m16n8k16 f16: A = q' as two f16 terms (value and residual, rows 0-7 and 8-15: 22 significant bits), B = the key
//           codes.  ldmatrix leaves a thread four consecutive channels of one token in a register: two conversions
//           e4m3x2 -> f16x2 (exact) make them B fragments, the channels being contracted in that order on both sides.
//   softmax base 2, in registers.  The page's value scale is a power of two 2^e, so it joins the exponent: the weight of a
//           token is w = 2^(x + e - ref), x its score, ref the running maximum of x + e, in two parts (kTopWeight in stief_f8.cuh).
//           Weights of any two pages are thus right relative to each other's contribution, however far their scales lie
//           apart.  The row sum takes w 2^-e under a reference of its own.
//   mix     O^T = V^T P^T: the 16 channels of a 16-byte chunk are the 16 rows of A (ldmatrix.trans and a byte permutation
//           bring two tokens of one channel together; even channels in rows 0-7, odd ones in rows 8-15), B = the weights, in
//           the very registers that computed them.  Weights are rounded to f16 once, scaled by 2^15 so that the
//           rounding stays relative down to 2^-29 of the largest.
// With 64 tokens per warp and page a page's chain of dependent steps (load, product, maximum, exponential, product) is
// paid once per 8 KiB at ranks 64/64 and hidden behind seven other warps.
//
// Measured (32 query heads over 8): 4 x 32768 tokens 24 us at ranks 32/32, 28 at 48/64, 31 at 64/64 (4.4 TB/s; 26 where calls may overlap),
// 52 at 96/128, 60 at 128/128.  Every further 134 MB take 19 to 21 us (6.4 to 7.1 TB/s): what is left is 12 us from launch to the end
// of the combine, of which overlapped calls hide half.  1 x 1021 tokens: 10.3 us, 4.7 overlapped.
#pragma once

#include "stief_decode.cuh"
#include "stief_f8.cuh"
#include "stief_partition.cuh"

namespace stief {

struct F8DecodeArgs {
  LayerDev L;                    // bases and shape (the bf16 pool pointers are unused)
  f8::Pools P;
  BatchDev Bt;
  const __nv_bfloat16* q;        // [B][Hq][128, or r_k without key basis]
  float* partial_o;
  float* partial_lse;
  int* counters;
  // one section of the workspace, its control words and the epochs: as in DecodeArgs
  int* finished;
  int* units_done;
  unsigned epoch, prev_epoch;
  __nv_bfloat16* out;            // [B][Hq][128, or r_v without value basis]
  float* out_lse;
  int len_add;
  int QT;
  int wait_first;                // 1: no input may be read before the kernel that precedes this one has completed
  int32_t* status;
};

namespace f8 {

// A page tile in shared memory: 64 rows of R codes, one contiguous block of 64 R bytes in the pool.
//   R = 32, 64, 128: fetched as lines of 128 bytes under the 128-byte swizzle (4, 2, 1 rows a line), conflict-free for ldmatrix;
//   R = 48, 96:      one 1-D bulk copy, rows back to back: conflict-free at 48 bytes, a two-way conflict at 96.
template <int R>
struct PageTile {
  static constexpr bool BULK = R == 48 || R == 96;
  static constexpr int BYTES = kPage * R;
  static constexpr int LINES = BYTES / 128;
  static constexpr int NC = R / 16;                        // 16-byte chunks of a row
  // byte offset of chunk c of row t
  __host__ __device__ static __forceinline__ uint32_t chunk(int t, int c) {
    const uint32_t off = (uint32_t)(t * R + c * 16);
    return BULK ? off : off ^ (((off >> 7) & 7u) << 4);
  }
  // what chunk(t + 16 j, c) differs from chunk(t, c) by, t < 16: plus 16 j R, after this exclusive-or
  __host__ __device__ static constexpr uint32_t step(int j) { return BULK ? 0u : (((uint32_t)(16 * j * R) >> 7) & 7u) << 4; }
};

constexpr int kSegPadBytes = 288 * 1024;         // cache bytes one CTA streams in the time a segment start costs
__host__ __device__ __forceinline__ int seg_pad(int r_k, int r_v) { return kSegPadBytes / ((r_k + r_v) * kPage); }

template <int RK, int RV>
struct DecodeCfg8 {
  static constexpr int K_BYTES = PageTile<RK>::BYTES, V_BYTES = PageTile<RV>::BYTES, S_BYTES = kScalesPerTile * 4;
  static constexpr int TX_BYTES = K_BYTES + V_BYTES + S_BYTES;
  static constexpr int STAGE_BYTES = (TX_BYTES + 1023) / 1024 * 1024;       // stages keep the tiles' swizzle alignment
  static constexpr int NW = 8, NPW = 4, NT = NW * 32, THREADS = NT + NPW * 32;
  static constexpr int CTRL_BYTES = 1024;
  static constexpr int PREF_BYTES = ((kMaxBatch + 1) * 4 + 127) / 128 * 128;
  static constexpr int QP_BYTES = kGroupTile * kD * 4;
  static constexpr int ROWS_BYTES = kGroupTile * kD * 4;
  static constexpr int UNION_BYTES = ROWS_BYTES + NW * kGroupTile * kD * 4;
  static constexpr int MISC = CTRL_BYTES + PREF_BYTES + QP_BYTES + UNION_BYTES;
  static constexpr int RING_BUDGET = 232448 - 1024 - MISC;
  static constexpr int SPW = RING_BUDGET / (NW * STAGE_BYTES) > 4 ? 4 : RING_BUDGET / (NW * STAGE_BYTES);
  static constexpr int NS = NW * SPW;
  static constexpr int RING_BYTES = NS * STAGE_BYTES;
  static constexpr int SMEM_BYTES = 1024 + RING_BYTES + MISC;
  static_assert(K_BYTES % 1024 == 0 && V_BYTES % 1024 == 0, "both tiles keep the swizzle alignment");
  static_assert(SPW >= 1 && NS <= 32, "ring shape");
  static_assert((NW * 8 * RV + 4 * NW * 8) * 4 <= UNION_BYTES, "merge scratch must fit");
  static_assert(kCombineScratchFloats * 4 <= UNION_BYTES, "combine scratch must fit");
  static_assert(SMEM_BYTES <= 232448, "exceeds the 227 KiB shared memory of an SM");
};

// D += A(16x16, row) * B(16x8, col), f16 inputs, fp32 accumulate
// (not volatile: the compiler may move it past the loads around it)
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm_x2_t(uint32_t addr, uint32_t& r0, uint32_t& r1) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(r0), "=r"(r1) : "r"(addr));
}
template <int RK, int RV>
__global__ void __launch_bounds__(DecodeCfg8<RK, RV>::THREADS, 1)
decode_f8_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const F8DecodeArgs a) {
  using C = DecodeCfg8<RK, RV>;
  using TK = PageTile<RK>;
  using TV = PageTile<RV>;
  constexpr int NW = C::NW, NS = C::NS, SPW = C::SPW, NT = C::NT, NPW = C::NPW;
  constexpr int NCK = TK::NC, NCV = TV::NC;

  extern __shared__ uint8_t smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int c = blockIdx.x, n_cta = gridDim.x;

  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* ring_ptr = smem_raw + (ring - smem_u32(smem_raw));
  uint8_t* ctrl_ptr = ring_ptr + C::RING_BYTES;
  const uint32_t ctrl = ring + C::RING_BYTES;
  auto full_bar = [&](int s) { return ctrl + s * 8; };
  auto empty_bar = [&](int s) { return ctrl + (32 + s) * 8; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl_ptr + 64 * 8);
  volatile int* last_flag = abort_flag + 1;
  volatile int* section_free = abort_flag + 2;             // the workspace section's previous user is done
  volatile int* gate = abort_flag + 3;                     // thread 0's verdict for the segment at hand
  float* q_norm = reinterpret_cast<float*>(ctrl_ptr + 66 * 8);       // [8]: power of two that brings the row's largest q' to 2^11 .. 2^12
  float* q_fac = q_norm + 8;                                         // [8]: its inverse times log2(e) / sqrt(128)
  int* pref = reinterpret_cast<int*>(ctrl_ptr + C::CTRL_BYTES);
  float* qp = reinterpret_cast<float*>(ctrl_ptr + C::CTRL_BYTES + C::PREF_BYTES);
  float* un = reinterpret_cast<float*>(ctrl_ptr + C::CTRL_BYTES + C::PREF_BYTES + C::QP_BYTES);

  // The next kernel on the stream may take over each SM as soon as this grid's CTA leaves it.
  launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    *abort_flag = 0;
    *section_free = 0;
    *last_flag = 0;
    mbar_fence_init();
  }
  // Without the overlap flag everything from here on waits for the kernel before; the launch itself and the setup above did not.
  if (a.wait_first) grid_dependency_wait();
  const int pad = seg_pad(RK, RV);
  build_page_prefix(pref, a.Bt, a.len_add, pad, c == 0 ? a.status : nullptr);   // ends with __syncthreads

  const int B = a.Bt.B, Hkv = a.L.Hkv, QT = a.QT, G = a.L.G;
  const int upb = Hkv * QT;
  const int total = pref[B] * upb;
  const int P = pages_per_cta(total, n_cta);

  SegmentWalker walk;
  walk.init(pref, B, upb, pad, c, P, total);
  Segment seg;

  // ------------------------------------------------------------------ producer warps
  // Page i of the CTA goes to consumer warp i mod 8; producer warp i mod 4 fetches it (one issuing thread could not keep up
  // with small tiles).
  if (warp >= NW) {
    const int pw = warp - NW;
    if (lane == 0) {
      if constexpr (!TK::BULK) tma_prefetch_desc(&tmK);
      if constexpr (!TV::BULK) tma_prefetch_desc(&tmV);
    }
    // Consecutive launches take the workspace sections in turn; before the consumers write into this one its previous
    // user must be done, which the section's control word tells (decode_persistent_kernel does the same).
    auto look_at_section = [&]() {
      if (pw == 0 && lane == 0 && a.prev_epoch != 0u && *section_free == 0) {
        int seen;
        asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(a.finished) : "memory");
        if ((unsigned)seen == a.prev_epoch) *section_free = 1;
      }
    };
    look_at_section();
    int i_base = 0;            // pages of this CTA before the current segment
    while (walk.next(seg)) {
      const int h = seg.j / QT;
      const int npg = seg.p1 - seg.p0;
      int tbl = 0, win = -1;
      for (int k = (pw - i_base % NPW + NPW) % NPW; k < npg; k += NPW) {
        if ((k >> 5) != win) {                             // block-table entries of a window of 32 pages, one per lane
          win = k >> 5;
          const int idx = seg.p0 + (win << 5) + lane;
          tbl = (idx < seg.p1) ? a.Bt.block_table[(size_t)seg.b * a.Bt.max_pages + idx] : 0;
        }
        int page = __shfl_sync(0xffffffffu, tbl, k & 31);
        if (page < 0 || page >= a.L.num_pages) {
          if (lane == 0) report(a.status, STIEF_ERR_BOUNDS);
          page = 0;
        }
        const int i = i_base + k, kw = i / NW;             // the consumer warp's kw-th page
        const int slot = (i % NW) * SPW + kw % SPW, use = kw / SPW;
        if (lane == 0) {
          if (use > 0) mbar_wait(empty_bar(slot), (use - 1) & 1, abort_flag, a.status);
          const uint32_t st = ring + slot * C::STAGE_BYTES;
          const size_t tile = (size_t)page * Hkv + h;
          mbar_arrive_expect_tx(full_bar(slot), C::TX_BYTES);
          if constexpr (TK::BULK) bulk_load_1d(st, a.P.k_codes + tile * C::K_BYTES, C::K_BYTES, full_bar(slot));
          else tma_load_2d(st, &tmK, 0, (int)tile * TK::LINES, full_bar(slot));
          if constexpr (TV::BULK) bulk_load_1d(st + C::K_BYTES, a.P.v_codes + tile * C::V_BYTES, C::V_BYTES, full_bar(slot));
          else tma_load_2d(st + C::K_BYTES, &tmV, 0, (int)tile * TV::LINES, full_bar(slot));
          bulk_load_1d(st + C::K_BYTES + C::V_BYTES, a.P.scales + tile * kScalesPerTile, C::S_BYTES, full_bar(slot));
        }
        __syncwarp();
      }
      i_base += npg;
      look_at_section();
    }
    return;
  }

  // ------------------------------------------------------------------ consumer warps
  const int gid = lane >> 2, tid4 = lane & 3, l7 = lane & 7, mat = lane >> 3;

  // Addresses of the ldmatrix instructions that cover 16 tokens: matrix number n is (8 tokens, chunk): for keys
  // (n / NCK, n mod NCK), for values (n mod 2, n / 2), four matrices an instruction, the last one of two where 2 NC is not a
  // multiple of 4.
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

  int i_base = 0;              // pages of this CTA before the current segment
  int n_final = 0;             // units this CTA finalised (merged or zero-filled)

  while (walk.next(seg)) {
    const int b = seg.b, h = seg.j / QT, qt = seg.j % QT;
    const int npg = seg.p1 - seg.p0;
    const int ng = min(kGroupTile, G - qt * kGroupTile);
    const size_t head0 = (size_t)b * a.L.Hq + (size_t)h * G + (size_t)qt * kGroupTile;
    const int len = min(max(a.Bt.seq_lens[b] + a.len_add, 0), seg.npages * kPage);
    const int last_valid = len - (seg.npages - 1) * kPage;          // tokens in the sequence's last page (1..64)

    // ---- prologue: q' = q U_k for the unit's queries
    {
      float* rows = un;                  // [8][128] fp32
      float* red = un + kGroupTile * kD; // [NW][8][128]
      const __nv_bfloat16* Uk = a.L.U_k ? a.L.U_k + (size_t)h * a.L.uk_stride : nullptr;
      const int dk = Uk ? kD : RK;
      const uint32_t row_mask = (1u << ng) - 1u;
      BasisSlice<NW, RK> sk;
      if (Uk) sk.load(Uk, warp, lane);
      if (tid < kGroupTile * 16) {
        const int r = tid / 16, ch = tid % 16;
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (r < ng && 8 * ch < dk) w = __ldg(reinterpret_cast<const uint4*>(a.q + (head0 + r) * dk) + ch);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<float2*>(rows + tid * 8 + 2 * e) = make_float2(bf16_lo(ww[e]), bf16_hi(ww[e]));
      }
      bar1(NT);
      if (Uk) {
        sk.contract(rows, row_mask, red, warp, lane, kGroupTile);
        bar1(NT);
      }
      // warp r finishes row r: the sum of the shares, and the power of two that brings its largest value to 2^11 .. 2^12
      float top = 0.f;
      for (int j = lane; j < RK; j += 32) {
        const float x = ((row_mask >> warp) & 1u) ? (Uk ? warp_shares<NW>(red, warp, j, kGroupTile) : rows[warp * kD + j]) : 0.f;
        qp[warp * RK + j] = x;
        top = fmaxf(top, fabsf(x));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (lane == 0) {
        const int e = top > 0.f ? min(max((int)(__float_as_uint(top) >> 23) - 127, -112), 126) - 11 : 0;
        q_norm[warp] = pow2(-e);
        q_fac[warp] = pow2(e) * (kLog2e * 0.08838834764831845f);
      }
      bar1(NT);
    }
    const float fac = q_fac[gid];
    uint32_t qa[NCK][4];                                   // rows 0-7: value, rows 8-15: residual
    {
      const float norm = q_norm[gid];
#pragma unroll
      for (int ch = 0; ch < NCK; ++ch) {
        const float4 x = *reinterpret_cast<const float4*>(qp + gid * RK + 16 * ch + 4 * tid4);
        const float y[4] = {x.x * norm, x.y * norm, x.z * norm, x.w * norm};
        qa[ch][0] = pack_f16(y[0], y[1]);
        qa[ch][2] = pack_f16(y[2], y[3]);
        const float2 h0 = __half22float2(*reinterpret_cast<const __half2*>(&qa[ch][0])), h1 = __half22float2(*reinterpret_cast<const __half2*>(&qa[ch][2]));
        qa[ch][1] = pack_f16(y[0] - h0.x, y[1] - h0.y);
        qa[ch][3] = pack_f16(y[2] - h1.x, y[3] - h1.y);
      }
    }

    float m = -INFINITY, em = 0.f, l = 0.f, n = kNoSum;    // row gid: both parts of the reference, this thread's share of the sum, the sum's reference
    float o[NCV][4];                                       // channels 16 i + 2 gid, + 1 (o[.][0], [1] and [2], [3]) of queries 2 tid4, 2 tid4 + 1
#pragma unroll
    for (int i = 0; i < NCV; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

    for (int k = (warp - i_base % NW + NW) % NW; k < npg; k += NW) {
      const int kw = (i_base + k) / NW;
      const int slot = warp * SPW + kw % SPW;
      mbar_wait(full_bar(slot), (kw / SPW) & 1, abort_flag, a.status);
      const uint32_t kt = ring + slot * C::STAGE_BYTES, vt = kt + C::K_BYTES;
      const bool tail = (seg.p0 + k == seg.npages - 1) && (last_valid < kPage);
      float ks, vs;
      asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(ks), "=f"(vs) : "r"(vt + C::V_BYTES));

      // ---- scores: x[4 j + 2 u + e] is token 16 j + 8 u + 2 tid4 + e
      float x[16];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float s4[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) s4[u][0] = s4[u][1] = s4[u][2] = s4[u][3] = 0.f;
        uint32_t w[4 * LK];
#pragma unroll
        for (int i = 0; i < LK; ++i) {
          const uint32_t addr = kt + (koff[i] ^ TK::step(j)) + 16 * j * RK;
          if (2 * NCK - 4 * i >= 4) ldsm_x4(addr, w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
          else ldsm_x2(addr, w[4 * i], w[4 * i + 1]);
        }
#pragma unroll
        for (int n = 0; n < 2 * NCK; ++n) {
          uint32_t b0, b1;
          expand4(w[n], b0, b1);
          mma_f16(s4[n / NCK], qa[n % NCK][0], qa[n % NCK][1], qa[n % NCK][2], qa[n % NCK][3], b0, b1);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          x[4 * j + 2 * u] = s4[u][0] + s4[u][2];
          x[4 * j + 2 * u + 1] = s4[u][1] + s4[u][3];
        }
      }
      const float f = score_factor(fac, ks);
      const float evf = scale_exponent(vs);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = __fmul_rn(x[i], f);               // the rounded product is what the reference goes by
      if (tail) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (16 * (i >> 2) + 8 * ((i >> 1) & 1) + 2 * tid4 + (i & 1) >= last_valid) x[i] = -INFINITY;
      }

      // ---- online softmax
      float mx[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) mx[i] = fmaxf(x[i], x[i + 8]);
#pragma unroll
      for (int i = 0; i < 4; ++i) mx[i] = fmaxf(mx[i], mx[i + 4]);
      float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float beyond = top - m, above = beyond + (evf - em);       // (above: log2 of the page's largest weight; infinity: nothing seen before)
      const bool vanish = may_vanish(beyond, above);
      // seldom after a sequence's first pages: the references grow, or the page's weights may vanish in the sum
      if (__any_sync(0xffffffffu, above > kTopWeight || vanish || top > n + kSumGrown)) {
        const bool grown = above > kTopWeight;
        const float alpha = grown ? fast_exp2(kTopWeight - above) : 1.f;
        const float a0 = __shfl_sync(0xffffffffu, alpha, 8 * tid4), a1 = __shfl_sync(0xffffffffu, alpha, 8 * tid4 + 4);
#pragma unroll
        for (int i = 0; i < NCV; ++i) {
          o[i][0] *= a0;
          o[i][1] *= a1;
          o[i][2] *= a0;
          o[i][3] *= a1;
        }
        if (grown) {
          m = top;
          em = evf - kTopWeight;
        }
        if (top > n + kSumGrown) {
          l *= fast_exp2(n - top);
          n = top;
        }
        if (vanish) {
          float own = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) own += fast_exp2(x[i] - top);
          l = fmaf(own, fast_exp2(top - n), l);
        }
      }
      const float ref = m > -INFINITY ? m : 0.f, shift = evf - em;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[i] = fast_exp2((x[i] - ref) + shift);
        sum += x[i];
      }
      l = fmaf(sum, above < kSumLow ? 0.f : fast_exp2((m - n) - shift), l);

      // ---- mix
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t p0 = pack_f16(x[4 * j], x[4 * j + 1]), p1 = pack_f16(x[4 * j + 2], x[4 * j + 3]);
        uint32_t w[4 * LV];
#pragma unroll
        for (int i = 0; i < LV; ++i) {
          const uint32_t addr = vt + (voff[i] ^ TV::step(j)) + 16 * j * RV;
          if (2 * NCV - 4 * i >= 4) ldsm_x4_t(addr, w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
          else ldsm_x2_t(addr, w[4 * i], w[4 * i + 1]);
        }
        if (tail) {                                        // rows past the end hold unspecified codes, NaN among them
          const int t0 = 16 * j + 2 * tid4;
          const uint32_t k0 = (t0 < last_valid ? 0xffffu : 0u) | (t0 + 1 < last_valid ? 0xffff0000u : 0u);
          const uint32_t k1 = (t0 + 8 < last_valid ? 0xffffu : 0u) | (t0 + 9 < last_valid ? 0xffff0000u : 0u);
#pragma unroll
          for (int n = 0; n < 2 * NCV; ++n) w[n] &= (n & 1) ? k1 : k0;
        }
#pragma unroll
        for (int i = 0; i < NCV; ++i) {
          uint32_t e0, d0, e1, d1;                         // even and odd channels, tokens 0-7 and 8-15 of the sixteen
          expand4(__byte_perm(w[2 * i], 0u, 0x3120), e0, d0);
          expand4(__byte_perm(w[2 * i + 1], 0u, 0x3120), e1, d1);
          mma_f16(o[i], e0, d0, e1, d1, p0, p1);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(slot));
    }
    i_base += npg;

    // ------------------------------------------------------------------ merge the warps of this segment
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    float* wo = un;                      // [NW][8][RV]
    float* wm = wo + NW * 8 * RV;        // [NW][8]
    float* wl = wm + NW * 8;             // [NW][8]
    float* wn = wl + NW * 8;             // [NW][8]
    float* we = wn + NW * 8;             // [NW][8]
#pragma unroll
    for (int i = 0; i < NCV; ++i) {
      *reinterpret_cast<float2*>(wo + (warp * 8 + 2 * tid4) * RV + 16 * i + 2 * gid) = make_float2(o[i][0], o[i][2]);
      *reinterpret_cast<float2*>(wo + (warp * 8 + 2 * tid4 + 1) * RV + 16 * i + 2 * gid) = make_float2(o[i][1], o[i][3]);
    }
    if (tid4 == 0) {
      wm[warp * 8 + gid] = m;
      wl[warp * 8 + gid] = l;
      wn[warp * 8 + gid] = n;
      we[warp * 8 + gid] = em;
    }
    // Everything up to here only read inputs.  This section of the workspace may still be in use by its previous user when the
    // launch overlaps earlier kernels.  Thread 0 settles the question for the CTA before the barrier: yes if producer 0 saw
    // that user's epoch in the control word, else it looks once more itself; without a yes everyone waits for the
    // predecessor grid (which completes only after all before it).
    if (tid == 0) {
      int go = *section_free;
      if (go == 0 && a.prev_epoch != 0u) {
        int seen;
        asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(a.finished) : "memory");
        go = (unsigned)seen == a.prev_epoch;
        if (go) *section_free = 1;
      }
      *gate = go;
    }
    bar1(NT);
    const int u = b * upb + seg.j;
    const int slot_id = c + u;
    if (*gate == 0) grid_dependency_wait();
    // what each warp's mix counts for (in place of its reference) and what the row's is multiplied by: eight threads a row
    if (tid < 64) {
      const int w = tid & 7, gg = tid >> 3;
      const float mw = wm[w * 8 + gg], ew = we[w * 8 + gg], nw = wn[w * 8 + gg];
      float M = mw, E = ew, N = nw;
#pragma unroll
      for (int o1 = 1; o1 < 8; o1 <<= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, M, o1), e2 = __shfl_xor_sync(0xffffffffu, E, o1);
        const bool larger = (m2 - M) + (e2 - E) > 0.f;
        M = larger ? m2 : M;
        E = larger ? e2 : E;
        N = fmaxf(N, __shfl_xor_sync(0xffffffffu, N, o1));
      }
      float den = fast_exp2(nw - N) * wl[w * 8 + gg];
#pragma unroll
      for (int o1 = 1; o1 < 8; o1 <<= 1) den += __shfl_xor_sync(0xffffffffu, den, o1);
      const float half = fast_exp2(0.5f * ((M - N) + E));  // in two steps: it reaches beyond fp32's exponents where scales lie far apart
      wm[w * 8 + gg] = fast_exp2((mw - M) + (ew - E)) * half;
      if (w == 0) {
        wl[gg] = half / den;
        // a sum that is not a number weighs more than any other, so that it is not passed over where parts are joined
        if (gg < ng) __stcg(a.partial_lse + (size_t)slot_id * kGroupTile + gg, den == den ? (N + log2f(den)) * kLn2 : INFINITY);
      }
    }
    bar1(NT);
    for (int idx = tid; idx < ng * RV; idx += NT) {
      const int gg = idx / RV, j = idx % RV;
      float num = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) num = fmaf(wm[w * 8 + gg], wo[(w * 8 + gg) * RV + j], num);
      __stcg(a.partial_o + ((size_t)slot_id * kGroupTile + gg) * RV + j, num * wl[gg]);
    }

    // ------------------------------------------------------------------ the unit's last partial triggers the combine
    int first, last;
    unit_cta_span(pref, upb, pad, P, b, seg.j, &first, &last);
    const int nseg = last - first + 1;
    bar1(NT);                                              // the CTA's partial is written; a fence of one thread behind it covers all of it
    if (tid == 0) {
      int is_last = 1;
      if (nseg > 1) {
        __threadfence();
        const int prev = atomicAdd(a.counters + u, 1);
        is_last = (prev == nseg - 1);
        if (is_last) {
          a.counters[u] = 0;                               // leave the counter clean for the next call
          __threadfence();
        }
      }
      *last_flag = is_last;
    }
    bar1(NT);
    if (*last_flag) {
      combine_unit<RV>(a.L, b, h, qt, first + u, nseg, a.partial_o, a.partial_lse, a.out, a.out_lse, un, tid, NT);
      ++n_final;
    }
    bar1(NT);
  }

  // units of empty sequences get their zero rows from CTA (u mod n_cta)
  const int d_out = a.L.U_v ? kD : RV;
  for (int u = c; u < B * upb; u += n_cta) {
    const int b = u / upb, j = u % upb;
    if (pref[b + 1] != pref[b]) continue;
    const int h = j / QT, qt = j % QT;
    const int ng = min(kGroupTile, G - qt * kGroupTile);
    const size_t head0 = (size_t)b * a.L.Hq + (size_t)h * G + (size_t)qt * kGroupTile;
    for (int idx = tid; idx < ng * d_out; idx += NT) a.out[head0 * d_out + idx] = __float2bfloat16_rn(0.f);
    if (a.out_lse && tid < ng) a.out_lse[head0 + tid] = -INFINITY;
    ++n_final;
  }
  // Every unit is finalised by exactly one CTA (merged, or zero-filled).  The CTA that finalises the kernel's last unit
  // publishes the kernel's epoch: from then on this section of the workspace is free for its next user.  That CTA also
  // waits for the predecessor grid before it leaves, so that this grid never completes before an earlier one (stream
  // order stays transitive); the others leave at once and hand their SMs to the next kernel.
  if (n_final > 0) {
    bar1(NT);                                              // all of the CTA's reads of partials and writes of outputs are issued
    if (tid == 0) {
      __threadfence();
      const int before = atomicAdd(a.units_done, n_final);
      if (before + n_final == B * upb) {
        *a.units_done = 0;
        __threadfence();
        asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(a.finished), "r"((int)a.epoch) : "memory");
        grid_dependency_wait();
      }
    }
  }
}

}  // namespace f8

// One launcher per key rank (each its own translation unit); cudaErrorInvalidValue for a value rank that is not compiled in.
cudaError_t launch_f8_decode_rk32(const F8DecodeArgs& a, int n_cta, cudaStream_t st);
cudaError_t launch_f8_decode_rk48(const F8DecodeArgs& a, int n_cta, cudaStream_t st);
cudaError_t launch_f8_decode_rk64(const F8DecodeArgs& a, int n_cta, cudaStream_t st);
cudaError_t launch_f8_decode_rk96(const F8DecodeArgs& a, int n_cta, cudaStream_t st);
cudaError_t launch_f8_decode_rk128(const F8DecodeArgs& a, int n_cta, cudaStream_t st);

}  // namespace stief
