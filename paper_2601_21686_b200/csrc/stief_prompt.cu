// stief_prompt_attention: causal attention over packed prompts,  out_i = softmax(q_i K[0..i]^T / sqrt(128)) V[0..i]  inside each
// prompt, on tcgen05 with fp32 accumulators in TMEM.
//
// A row tile is 128 consecutive tokens of one query head; key blocks are 128 tokens, counted from the prompt's first token, so
// exactly the last block of a tile is the masked triangle.  The tiles of one (prompt, KV head) are numbered (token block, head
// of the group) and taken in PAIRS: two tiles use every K and V block that the CTA fetches, and with an even group both have the
// same length.
//
// What bounds it.  Per tile and block: 2 x 128^3 MACs, 1024 cycles of the tensor pipe (the score product, both operands in
// shared memory, takes 89 cycles per K = 16 step instead of 64: 8 KiB of operands at about 92 bytes a cycle), against 16384
// exponentials, 1024 cycles of the special-function units (16 per clock and SM).  A tile's chain is serial: scores ->
// softmax (about 1800 cycles: TMEM load 240, maximum 280, exponentials 1150, publication 100) -> P V -> next scores (about
// 1300 from the last P to the next S).  Two tiles half a period apart overlap one's softmax with the other's products; there is
// no TMEM for a third (512 columns: per tile 128 for S and 128 for O).  A quarter or an eighth of the exponentials as a
// polynomial on the FMA pipe, starting them from the previous block's maximum, and two threads per row were measured: each
// slower (polynomial 1/4: 596 against 535 us for four prompts of 4096; previous block's maximum: 571; two threads per row: 557
// against 469 us for one of 8192): what they add to the instruction stream costs more than the unit that they relieve.  So does
// publishing P at three quarters instead of the half (504 against 480 us), and keeping half of the row, the other loaded again, so
// that a polynomial share fits the registers (542 to 589 against 490 us).
//
// One persistent CTA per SM, 512 threads (128 registers each at launch, dealt out again by role):
//   warps 0-3, 4-7  softmax of tile 0 / 1: thread = row = TMEM lane, the block's 128 scores in registers
//   warps 8-11      epilogue of both tiles: O / l to global memory while the softmax warps are on the next item
//   warp 12         TMA producer: query tiles, then K_0, V_0, K_1, V_1, ... through a ring of four 32 KiB stages
//   warps 13, 14    MMA issue, a warp per tile:  O += P_j V_j, then S = Q K_(j+1)^T, both M = N = 128
// P_j (bf16 pairs, 64 columns) takes the place of S_j, from where the P V product reads it; the next S is issued behind that
// product by the same thread, so it cannot overtake it, and its completion implies the product's: the accumulator may then be
// rescaled without another wait.  The issuers take turns, step by step: left alone the tiles fall into step, both in the softmax
// and then both waiting for the tensor pipe (607 against 476 us for four prompts of 4096); one issuer for both spends the
// pipe's time on its own waits (565).
//
// The reference maximum of a row follows the true one only when that has grown by more than 2^8: the accumulator in TMEM is
// rescaled a few times per row instead of at every block.
//
// Measured (32 query heads over 8, TFLOP/s of the causal half): one prompt of 16384 tokens 1.95 to 2.00 ms = 1128 to 1100 call
// after call, at 1616 MHz under the power limit, and 1.76 ms = 1252 in bursts of five with pauses; four of 4096 546 us = 1007 and
// 490 us = 1122; the card's cuBLAS rates are 1709 in a burst and 1411 sustained.  One of 8192 under the profiler: tensor pipe
// 61 % and special-function units 61 % of their cycles, DRAM 130 MB (each input once), 38 % of the issue slots.  The factor per
// row that far scores need (stief_softmax.cuh) costs 1 to 2 %.
#include <cfloat>
#include <cstring>

#include "stief_host_util.h"
#include "stief_softmax.cuh"
#include "stief_umma.cuh"

namespace stief {
namespace prompt {

using namespace tc;

struct Args {
  int Hq, Hkv, G, B;
  int total;
  const int32_t* cu;
  long long out_stride;
  __nv_bfloat16* out;
  float* out_lse;
  int32_t* status;
};

constexpr int kThreads = 512;
constexpr int kRows = 128;                      // tokens of a tile, and of a key block
constexpr int kTileBytes = kRows * kD * 2;      // 32 KiB: a query tile, a K block, a V block
constexpr int kStages = 4;
constexpr int kHeadBytes = 11264;               // prompts (8192), barriers (512), row sums (2048); then the tiles
constexpr int kSmem = kHeadBytes + (2 + kStages) * kTileBytes;
static_assert(kSmem <= 232448, "227 KiB of shared memory per CTA");
constexpr int kTmemCols = 512;
constexpr float kRescaleLog2 = 8.0f;

struct Prompts {                                // in shared memory, in order of falling length
  int lo[kMaxBatch], len[kMaxBatch];
};
__device__ __forceinline__ int pairs_of(const Args& a, int len) { return len <= 0 ? 0 : (((len + kRows - 1) / kRows) * a.G + 1) >> 1; }

struct Item {
  int lo, len;                                  // first token and length of the prompt
  int kvh;
  int tok0[2], head[2], np[2];                  // per tile: first token within the prompt, query head, key blocks (0 = no tile)
  bool valid;
};

// Work items in order of falling length: level p holds pair p of every prompt that has one, for every KV head.  Items are
// dealt to the CTAs back and forth, so that all get nearly the same sum.  Every role walks the same list.
struct Walk {
  int round, p, cnt, base, next_pairs;
  __device__ __forceinline__ void start(const Args& a, const Prompts& ps) {
    round = 0;
    base = 0;
    cnt = 0;
    p = pairs_of(a, ps.len[0]);
    next_pairs = p;
    lower(a, ps);
  }
  __device__ __forceinline__ void lower(const Args& a, const Prompts& ps) {      // to the next level
    --p;
    while (cnt < a.B && next_pairs > p) {
      ++cnt;
      next_pairs = cnt < a.B ? pairs_of(a, ps.len[cnt]) : 0;
    }
  }
  __device__ __forceinline__ Item next(const Args& a, const Prompts& ps) {
    Item w;
    const int g = gridDim.x, c = blockIdx.x;
    const long long idx = (long long)round * g + ((round & 1) ? g - 1 - c : c);
    ++round;
    while (p >= 0 && idx >= (long long)base + (long long)cnt * a.Hkv) {
      base += cnt * a.Hkv;
      lower(a, ps);
    }
    w.valid = p >= 0;
    w.np[0] = w.np[1] = 0;
    if (!w.valid) return w;
    const int k = (int)(idx - base), b = k / a.Hkv;
    w.kvh = k % a.Hkv;
    w.lo = ps.lo[b];
    w.len = ps.len[b];
    const int nb = (w.len + kRows - 1) / kRows;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int x = 2 * p + t, tb = x / a.G;
      w.tok0[t] = tb * kRows;
      w.head[t] = w.kvh * a.G + x - tb * a.G;
      w.np[t] = tb < nb ? tb + 1 : 0;
    }
    return w;
  }
};

__global__ void __launch_bounds__(kThreads, 1)
prompt_attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                        const __grid_constant__ CUtensorMap tmV, const Args a) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  Prompts& ps = *reinterpret_cast<Prompts*>(smem);
  uint8_t* ctrl_ptr = smem + sizeof(Prompts);
  const uint32_t ctrl = smem_u32(ctrl_ptr);
  float2* sums = reinterpret_cast<float2*>(ctrl_ptr + 512);     // [tile][row] reference (base 2) and sum
  uint8_t* tiles_ptr = smem + kHeadBytes;
  const uint32_t q_smem = smem_u32(tiles_ptr), ring = q_smem + 2 * kTileBytes;
  auto full_bar = [&](int s) { return ctrl + s * 8; };
  auto empty_bar = [&](int s) { return ctrl + (8 + s) * 8; };
  auto q_full = [&](int t) { return ctrl + (16 + t) * 8; };
  auto q_empty = [&](int t) { return ctrl + (18 + t) * 8; };
  auto s_full = [&](int t) { return ctrl + (20 + t) * 8; };
  auto p_full = [&](int t, int half) { return ctrl + (22 + 2 * t + half) * 8; };
  auto o_full = [&](int t) { return ctrl + (26 + t) * 8; };
  auto o_free = [&](int t) { return ctrl + (28 + t) * 8; };
  auto sums_full = [&](int t) { return ctrl + (30 + t) * 8; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl_ptr + 34 * 8);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl_ptr + 34 * 8 + 4);
  int32_t* status = a.status;
  if (q_smem & 1023u) {                         // the swizzled tiles need it; dynamic shared memory starts there
    report(status, STIEF_ERR_CUDA);
    return;
  }

  if (tid == 0) {
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  // prompts in order of falling length (ties by number): the rank of each is a count over all
  int *lens = reinterpret_cast<int*>(tiles_ptr), *los = lens + kMaxBatch;
  for (int b = tid; b < a.B; b += kThreads) {
    const int lo = a.cu[b], hi = a.cu[b + 1];
    const bool ok = lo >= 0 && hi >= lo && hi <= a.total;      // else its boundaries are not usable
    if (!ok) report(status, STIEF_ERR_BOUNDS);
    lens[b] = ok ? hi - lo : 0;
    los[b] = lo;
  }
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 2);               // one arrival from each tile's issuer
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full(t), 1);
      mbar_init(q_empty(t), 1);
      mbar_init(s_full(t), 1);
      mbar_init(p_full(t, 0), 4);               // one arrival per softmax warp of the tile
      mbar_init(p_full(t, 1), 4);
      mbar_init(o_full(t), 1);
      mbar_init(ctrl + (32 + t) * 8, 1);        // whose turn it is to issue
      mbar_init(o_free(t), 4);                  // one arrival per epilogue warp
      mbar_init(sums_full(t), 4);
    }
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 12) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
  __syncthreads();
  for (int b = tid; b < a.B; b += kThreads) {
    const int mine = lens[b];
    int rank = 0;
    for (int i = 0; i < a.B; ++i) rank += lens[i] > mine || (lens[i] == mine && i < b);
    ps.lo[rank] = los[b];
    ps.len[rank] = mine;
  }
  fence_proxy_async_smem();                     // the scratch above becomes a target of TMA writes
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  Walk walk;
  if (warp >= 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");       // 512 x 128 registers at launch = 256 x 176 + 128 x 80 + 128 x 80
    if (warp == 12) {
      // ---------------------------------------------------------------------------------------- producer
      int st = 0, use = 0, nq[2] = {0, 0};
      auto put = [&](const CUtensorMap* tm, int tok, int head) {
        if (use > 0) mbar_wait(empty_bar(st), (use - 1) & 1, abort_flag, status);
        mbar_arrive_expect_tx(full_bar(st), kTileBytes);
        tma_load_4d(ring + st * kTileBytes, tm, 0, tok, 0, head, full_bar(st));
        if (++st == kStages) {
          st = 0;
          ++use;
        }
      };
      auto put_q = [&](const Item& w, int t) {
        if (w.np[t] == 0) return;
        if (nq[t] > 0) mbar_wait(q_empty(t), (nq[t] - 1) & 1, abort_flag, status);
        ++nq[t];
        mbar_arrive_expect_tx(q_full(t), kTileBytes);
        tma_load_4d(q_smem + t * kTileBytes, &tmQ, 0, w.lo + w.tok0[t], 0, w.head[t], q_full(t));
      };
      if (lane == 0) {
        walk.start(a, ps);
        for (Item w = walk.next(a, ps); w.valid; w = walk.next(a, ps)) {
          const int npmax = max(w.np[0], w.np[1]);
          put_q(w, 0);
          put(&tmK, w.lo, w.kvh);
          put_q(w, 1);
          put(&tmV, w.lo, w.kvh);
          for (int j = 1; j < npmax; ++j) {
            put(&tmK, w.lo + j * kRows, w.kvh);
            put(&tmV, w.lo + j * kRows, w.kvh);
          }
        }
      }
    } else if (warp < 15) {
      // ---------------------------------------------------------------------------------------- MMA issue, tile t
      // The whole warp runs the control flow, kept uniform (stief_umma.cuh); one elected lane issues.
      const int t = uniform(warp) - 13;
      const uint32_t tmem_u = uniform(tmem_base) + t * 256, q_u = uniform(q_smem) + t * kTileBytes, ring_u = uniform(ring), ctrl_u = uniform(ctrl);
      const uint32_t id_qk = idesc_bf16_f32(kRows, kRows), id_pv = idesc_bf16_f32_bmn(kRows, kD);
      const uint32_t hi = desc_hi(desc_template(2, 16, 1024));                 // 128-byte swizzle, 8-row groups 1024 bytes apart
      const uint32_t qa = desc_lo(16, q_u);
      int st = 0, use = 0, kt = 0, n = 0, turns = 0;
      bool mine = false;
      auto bar = [&](int i) { return ctrl_u + i * 8; };                        // as numbered above
      auto consume = [&](uint32_t& addr, int& stage) {
        mbar_wait_warp(bar(st), use & 1, abort_flag, status);
        addr = ring_u + st * kTileBytes;
        stage = st;
        if (++st == kStages) {
          st = 0;
          ++use;
        }
      };
      auto arrive = [&](int i) {
        if (lane == 0) mbar_arrive(bar(i));
        __syncwarp();
      };
      auto take_turn = [&]() {
        if (t) mbar_wait_warp(bar(33), turns & 1, abort_flag, status);
        else if (turns > 0) mbar_wait_warp(bar(32), (turns - 1) & 1, abort_flag, status);
        ++turns;
        mine = true;
      };
      auto pass_turn = [&]() {
        if (mine) arrive(33 - t);
        mine = false;
      };
      auto score = [&](uint32_t k_addr) {                                      // S = Q K^T; rows of 128 bytes, K-major
        const uint32_t ka = desc_lo(16, k_addr);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t off = (uint32_t)((k >> 2) * (kTileBytes / 2) + (k & 3) * 32) >> 4;
          umma_ss(tmem_u, qa + off, hi, ka + off, hi, id_qk, k > 0 ? 1u : 0u);
        }
        umma_commit_warp(bar(20 + t));
      };
      uint32_t k_addr = 0, v_addr = 0;
      int k_stage = 0, v_stage = 0, nq = 0;
      auto first_operands = [&]() {                                            // of an item's first score product
        mbar_wait_warp(bar(16 + t), nq & 1, abort_flag, status);
        ++nq;
        consume(k_addr, k_stage);
      };
      walk.start(a, ps);
      Item w = walk.next(a, ps);
      bool live = uniform((int)w.valid) != 0;
      int np0 = uniform(w.np[0]), np1 = uniform(w.np[1]);
      if (live && (t ? np1 : np0) > 0) {
        first_operands();
        score(k_addr);
        umma_commit_warp(bar(8 + k_stage));
        if ((t ? np1 : np0) == 1) umma_commit_warp(bar(18 + t));
      }
      while (live) {
        const int np = t ? np1 : np0, npmax = max(np0, np1);
        w = walk.next(a, ps);
        int nx = 0;                                                            // blocks of this tile in the next item
        for (int j = 0; j < npmax; ++j) {
          const bool last = j + 1 == npmax;
          if (last) {
            live = uniform((int)w.valid) != 0;
            np0 = uniform(w.np[0]);
            np1 = uniform(w.np[1]);
            nx = live ? (t ? np1 : np0) : 0;
          }
          // everything that the step's products need besides P is waited for ahead of it
          const bool own = j < np, more = j + 1 < np, cross = last && nx > 0;
          if (!own) {                                                          // blocks that only the other tile uses
            consume(k_addr, k_stage);
            arrive(8 + k_stage);
          }
          consume(v_addr, v_stage);
          if (!own) arrive(8 + v_stage);
          if (more) consume(k_addr, k_stage);
          else if (cross) first_operands();
          if (own) {
            if (j == 0 && kt > 0) mbar_wait_warp(bar(28 + t), (kt - 1) & 1, abort_flag, status);   // the epilogue has read the item before
          }
          take_turn();
          if (own) mbar_wait_warp(bar(22 + 2 * t), n & 1, abort_flag, status);
          tc_fence_after();
          if (own) {
            const uint32_t va = desc_lo(kRows * 128, v_addr);                  // O += P V; V MN-major, two halves of 64 channels
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              if (k == 4) {
                mbar_wait_warp(bar(23 + 2 * t), n & 1, abort_flag, status);
                tc_fence_after();
              }
              umma_ts(tmem_u + 128, tmem_u + 8 * k, va + (uint32_t)(k * 2048 >> 4), hi, id_pv, j > 0 || k > 0 ? 1u : 0u);
            }
            ++n;
            if (j == np - 1) umma_commit_warp(bar(26 + t));
          }
          if (more || cross) score(k_addr);
          pass_turn();
          if (own) umma_commit_warp(bar(8 + v_stage));
          if (more || cross) {
            umma_commit_warp(bar(8 + k_stage));
            if (more ? j + 2 == np : nx == 1) umma_commit_warp(bar(18 + t));
          }
        }
        kt += np > 0;
      }
    }
  } else if (warp >= 8) {
    // ------------------------------------------------------------------------------------------ epilogue of both tiles
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    const int q4 = warp & 3, row = 32 * q4 + lane;
    const uint32_t t_lane = tmem_base + ((uint32_t)(32 * q4) << 16) + 128;
    int kt[2] = {0, 0};
    walk.start(a, ps);
    Item w = walk.next(a, ps);
    while (w.valid) {
      const Item nx = walk.next(a, ps);                      // its boundaries are on the way meanwhile
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (w.np[t] == 0) continue;
        const int tok = w.tok0[t] + row;
        mbar_wait(sums_full(t), kt[t] & 1, abort_flag, status);
        const float2 ml = sums[t * kRows + row];
        mbar_wait(o_full(t), kt[t] & 1, abort_flag, status);
        ++kt[t];
        tc_fence_after();
        const bool row_valid = tok < w.len;
        if (w.tok0[t] + 32 * q4 < w.len) {
          const float inv = 1.0f / ml.y;
          __nv_bfloat16* orow = a.out + (size_t)(w.lo + tok) * a.out_stride + (size_t)w.head[t] * kD;
#pragma unroll
          for (int c0 = 0; c0 < kD; c0 += 32) {
            uint32_t v[32];
            tmem_ld32(t_lane + t * 256 + c0, v);
            tmem_ld_wait();
            if (row_valid) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint32_t k[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) k[e] = pack_bf16(__uint_as_float(v[8 * i + 2 * e]) * inv, __uint_as_float(v[8 * i + 2 * e + 1]) * inv);
                *reinterpret_cast<uint4*>(orow + c0 + 8 * i) = make_uint4(k[0], k[1], k[2], k[3]);
              }
            }
          }
          if (row_valid && a.out_lse) a.out_lse[(size_t)(w.lo + tok) * a.Hq + w.head[t]] = kLn2 * (ml.x + log2f(ml.y));
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(o_free(t));
      }
      w = nx;
    }
  } else {
    // ------------------------------------------------------------------------------------------ softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    const int t = warp >> 2, q4 = warp & 3, row = 32 * q4 + lane;
    const uint32_t t_s = tmem_base + ((uint32_t)(32 * q4) << 16) + t * 256, t_o = t_s + 128;
    const float c = kLog2e * rsqrtf((float)kD);
    int n = 0, kt = 0, item = 0;                                // blocks and items of this tile so far; ring items of both tiles
    auto arrive_warp = [&](uint32_t bar) {
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    walk.start(a, ps);
    Item w = walk.next(a, ps);
    while (w.valid) {
      const Item nx = walk.next(a, ps);
      const int item0 = item;
      item += 2 * max(w.np[0], w.np[1]);
      const int np = t ? w.np[1] : w.np[0], tok0 = t ? w.tok0[1] : w.tok0[0], len = w.len;
      w = nx;
      if (np == 0) continue;
      const bool warp_live = tok0 + 32 * q4 < len;
      float m_ref = 0.f, l = 0.f;
      float c_row = c;                                          // of the row's exponents
      for (int j = 0; j < np; ++j, ++n) {
        const int p0 = j * kRows;
        const bool diag = j == np - 1;
        mbar_wait(s_full(t), n & 1, abort_flag, status);
        tc_fence_after();
        if (p0 + kRows > len) {
          // rows behind the prompt's end: whatever they hold (another prompt's values, NaN) must not reach the accumulator
          // through 0 * x.  Both tiles zero them; the values are the same.
          const int idx = item0 + 2 * j + 1, stg = idx % kStages;
          mbar_wait(full_bar(stg), (idx / kStages) & 1, abort_flag, status);
          uint8_t* v = tiles_ptr + (2 + stg) * kTileBytes;
          const int dead = len - p0;
          for (int e = row; e < (kRows - dead) * 16; e += kRows)
            *reinterpret_cast<uint4*>(v + ((e >> 3) & 1) * (kTileBytes / 2) + (dead + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async_smem();
        }
        if (!warp_live) {                                       // none of the warp's rows exists
          arrive_warp(p_full(t, 0));
          arrive_warp(p_full(t, 1));
          continue;
        }
        uint32_t sv[128];
        float* s = reinterpret_cast<float*>(sv);
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld32(t_s + 32 * i, sv + 32 * i);
        tmem_ld_wait();
        if (diag) {
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i > row) s[i] = -INFINITY;
        }
        float mx;
        {
          float m[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
          for (int i = 4; i < 124; i += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = max3(m[e], s[i + 2 * e], s[i + 2 * e + 1]);
          mx = fmaxf(max3(max3(m[0], s[124], s[125]), m[1], m[2]), max3(m[3], s[126], s[127]));
        }
        if (j == 0) {
          m_ref = fmaxf(mx, -FLT_MAX);
          l = 0.f;
          c_row = exponent_scale(m_ref, c);
        } else if (const bool grown = (mx - m_ref) * c > kRescaleLog2; __any_sync(0xffffffffu, grown)) {
          const float f = grown ? reference_weight(m_ref, mx, c) : 1.0f;    // a row's bits do not depend on its neighbours
          if (grown) m_ref = mx;
          c_row = exponent_scale(m_ref, c);
          l *= f;
#pragma unroll 1
          for (int c0 = 0; c0 < kD; c0 += 16) {
            uint32_t v[16];
            tmem_ld16(t_o + c0, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
            tmem_st16(t_o + c0, v);
          }
        }
        const uint64_t c2 = pack2(c_row, c_row), neg2 = pack2(-m_ref * c_row, -m_ref * c_row);
        uint64_t sum[2] = {0ull, 0ull};                         // pairs of +0
#pragma unroll
        for (int h = 0; h < 2; ++h) {                           // 64 columns: probabilities as bf16 pairs over the scores
#pragma unroll
          for (int g = 2 * h; g < 2 * h + 2; ++g) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float x0, x1;
              unpack2(fma2(pack2(s[32 * g + 2 * i], s[32 * g + 2 * i + 1]), c2, neg2), x0, x1);
              const float e0 = fast_exp2(x0), e1 = fast_exp2(x1);
              sum[i & 1] = add2(sum[i & 1], pack2(e0, e1));
              pk[i] = pack_bf16(e0, e1);
            }
            tmem_st16(t_s + 16 * g, pk);
          }
          tmem_st_wait();
          tc_fence_before();
          arrive_warp(p_full(t, h));
        }
        float a0, a1;
        unpack2(add2(sum[0], sum[1]), a0, a1);
        l += a0 + a1;
      }
      // the row's reference and sum go to the epilogue warps; the words are free once they have taken the item before
      if (kt > 0) mbar_wait(o_free(t), (kt - 1) & 1, abort_flag, status);
      ++kt;
      sums[t * kRows + row] = make_float2(m_ref * c, l);
      arrive_warp(sums_full(t));
    }
  }

  if (*abort_flag) let_copies_land();           // a wait ran out: nobody has waited for the ring's last copies
  tc_fence_before();
  __syncthreads();
  if (warp == 12) tmem_dealloc(tmem_base, kTmemCols);
}

}  // namespace prompt
}  // namespace stief

using namespace stief;

extern "C" int stief_prompt_attention(int32_t Hq, int32_t Hkv, int32_t B, int32_t total_tokens, const int32_t* cu_seqlens, const uint16_t* q,
                                      int64_t q_stride_t, const uint16_t* k, int64_t k_stride_t, const uint16_t* v, int64_t v_stride_t,
                                      uint16_t* out, int64_t out_stride_t, float* out_lse, uint32_t flags, int32_t* status, void* stream) {
  if (Hq <= 0 || Hkv <= 0 || Hq % Hkv || B <= 0 || B > kMaxBatch || total_tokens < 0 || !cu_seqlens || flags != 0u) return STIEF_ERR_INVALID_ARG;
  if (total_tokens == 0) return STIEF_OK;
  if (!q || !k || !v || !out) return STIEF_ERR_INVALID_ARG;
  if (q_stride_t < (int64_t)Hq * kD || k_stride_t < (int64_t)Hkv * kD || v_stride_t < (int64_t)Hkv * kD || out_stride_t < (int64_t)Hq * kD ||
      q_stride_t % 8 || k_stride_t % 8 || v_stride_t % 8 || out_stride_t % 8)
    return STIEF_ERR_INVALID_ARG;
  if (!host::aligned(q, 16) || !host::aligned(k, 16) || !host::aligned(v, 16) || !host::aligned(out, 16)) return STIEF_ERR_INVALID_ARG;
  // items are counted in int: a pair of tiles per 256 rows of every query head, and one per (prompt, KV head) more
  const long long most = ((long long)total_tokens / prompt::kRows + B) * Hq + (long long)B * Hkv;
  if (most >= (1ll << 30)) return STIEF_ERR_INVALID_ARG;

  // [heads][2 halves of 64 channels][tokens][64]: one box is a tile as two swizzled blocks of 128 rows x 128 bytes
  CUtensorMap tm[3];
  auto tile_map = [&](CUtensorMap* m, const uint16_t* p, int64_t stride, int heads) {
    const unsigned long long dims[4] = {64ull, (unsigned long long)total_tokens, 2ull, (unsigned long long)heads};
    const unsigned long long strides[3] = {(unsigned long long)stride * 2, 128ull, 256ull};
    const unsigned box[4] = {64u, (unsigned)prompt::kRows, 2u, 1u};
    return encode_bf16_map(m, p, 4, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
  };
  if (!tile_map(&tm[0], q, q_stride_t, Hq) || !tile_map(&tm[1], k, k_stride_t, Hkv) || !tile_map(&tm[2], v, v_stride_t, Hkv)) return STIEF_ERR_CUDA;

  prompt::Args a;
  a.Hq = Hq; a.Hkv = Hkv; a.G = Hq / Hkv; a.B = B; a.total = total_tokens; a.cu = cu_seqlens;
  a.out_stride = out_stride_t; a.out = reinterpret_cast<__nv_bfloat16*>(out); a.out_lse = out_lse; a.status = status;
  static bool configured[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return STIEF_ERR_CUDA;
  if (!configured[dev]) {
    if (cudaFuncSetAttribute(prompt::prompt_attention_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, prompt::kSmem) != cudaSuccess) return STIEF_ERR_CUDA;
    configured[dev] = true;
  }
  const int sms = host::sm_count();
  prompt::prompt_attention_kernel<<<(int)(most < sms ? most : sms), prompt::kThreads, prompt::kSmem, static_cast<cudaStream_t>(stream)>>>(tm[0], tm[1], tm[2], a);
  return cudaGetLastError() == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}
