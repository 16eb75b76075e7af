// stief_prompt_attention: causal attention over packed prompts,  out_i = softmax(q_i K[0..i]^T / sqrt(128)) V[0..i]  inside each
// prompt, on tcgen05 with fp32 accumulators in TMEM.
//
// A row tile is 128 consecutive tokens of one query head; key blocks are 128 tokens, counted from the prompt's first token, so
// exactly the last block of a tile is the masked triangle.  The tiles of one (prompt, KV head) are numbered (token block, head
// of the group) and taken in PAIRS: two tiles use every K and V block that the CTA fetches, and with an even group both have the
// same length.  Operations per pair and block: 2 x 2 x 128 x 128 x 128 MACs, 2048 tensor cycles, against 2 x 16384
// exponentials, 2048 cycles of the special-function units (16 per clock and SM): both pipes are needed in full, so a part of
// the exponentials runs as a polynomial on the FMA pipe, and the two tiles alternate: while one tile's probabilities are made,
// the tensor pipe works on the other's two products.
//
// One persistent CTA per SM, 384 threads:
//   warps 0-3, 4-7  softmax and epilogue of tile 0 / 1: thread = row = TMEM lane, the block's 128 scores in registers
//   warp 8          TMA producer: query tiles, then K_0, V_0, K_1, V_1, ... through a ring of five 32 KiB stages
//   warps 9, 10     MMA issue, one warp per tile:  S = Q K_j^T, then O += P_j V_j, both M = N = 128
// TMEM (512 columns): per tile 128 for S and 128 for O.  P_j (bf16 pairs, 64 columns) takes the place of S_j, from where
// the P V product reads it; the next S is issued behind that product by the same thread, so it cannot overtake it, and its
// completion implies the product's: the accumulator may then be rescaled without another wait.
//
// The reference maximum of a row follows the true one only when that has grown by more than 2^8: the accumulator in TMEM is
// rescaled a few times per row instead of at every block.
#include <cstring>

#include "stief_host_util.h"
#include "stief_softmax.cuh"

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

constexpr int kThreads = 384;
constexpr int kRows = 128;                      // tokens of a tile, and of a key block
constexpr int kTileBytes = kRows * kD * 2;      // 32 KiB: a query tile, a K block, a V block
constexpr int kStages = 5;
constexpr int kHeadBytes = kMaxBatch * 2 + 1024;   // prompt order and barriers, ahead of the tiles
constexpr int kSmem = kHeadBytes + (2 + kStages) * kTileBytes;
static_assert(kSmem <= 232448, "227 KiB of shared memory per CTA");
constexpr int kTmemCols = 512;
constexpr float kRescaleLog2 = 8.0f;
constexpr int kPolyEvery = 4;                   // every fourth pair of exponentials runs on the FMA pipe

// Length of prompt b, or -1 when its boundaries are not usable
__device__ __forceinline__ int prompt_len(const Args& a, int b) {
  const int lo = a.cu[b], hi = a.cu[b + 1];
  return lo < 0 || hi < lo || hi > a.total ? -1 : hi - lo;
}
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
  __device__ __forceinline__ void start(const Args& a, const uint16_t* order) {
    round = 0;
    base = 0;
    cnt = 0;
    p = pairs_of(a, prompt_len(a, order[0]));
    next_pairs = p;
    lower(a, order);
  }
  __device__ __forceinline__ void lower(const Args& a, const uint16_t* order) {      // to the next level
    --p;
    while (cnt < a.B && next_pairs > p) {
      ++cnt;
      next_pairs = cnt < a.B ? pairs_of(a, prompt_len(a, order[cnt])) : 0;
    }
  }
  __device__ __forceinline__ Item next(const Args& a, const uint16_t* order) {
    Item w;
    const int g = gridDim.x, c = blockIdx.x;
    const long long idx = (long long)round * g + ((round & 1) ? g - 1 - c : c);
    ++round;
    while (p >= 0 && idx >= (long long)base + (long long)cnt * a.Hkv) {
      base += cnt * a.Hkv;
      lower(a, order);
    }
    w.valid = p >= 0;
    w.np[0] = w.np[1] = 0;
    if (!w.valid) return w;
    const int k = (int)(idx - base), b = order[k / a.Hkv];
    w.kvh = k % a.Hkv;
    w.lo = a.cu[b];
    w.len = a.cu[b + 1] - w.lo;
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
  uint16_t* order = reinterpret_cast<uint16_t*>(smem);
  uint8_t* ctrl_ptr = smem + kMaxBatch * 2;
  const uint32_t ctrl = smem_u32(ctrl_ptr);
  uint8_t* tiles_ptr = smem + kHeadBytes;
  const uint32_t q_smem = smem_u32(tiles_ptr), ring = q_smem + 2 * kTileBytes;
  auto full_bar = [&](int s) { return ctrl + s * 8; };
  auto empty_bar = [&](int s) { return ctrl + (8 + s) * 8; };
  auto q_full = [&](int t) { return ctrl + (16 + t) * 8; };
  auto q_empty = [&](int t) { return ctrl + (18 + t) * 8; };
  auto s_full = [&](int t) { return ctrl + (20 + t) * 8; };
  auto p_full = [&](int t, int half) { return ctrl + (22 + 2 * t + half) * 8; };
  auto o_full = [&](int t) { return ctrl + (26 + t) * 8; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl_ptr + 28 * 8);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl_ptr + 28 * 8 + 4);
  int32_t* status = a.status;
  if (q_smem & 1023u) {                         // the swizzled tiles need it; dynamic shared memory starts there
    report(status, STIEF_ERR_CUDA);
    return;
  }

  // prompts in order of falling length (ties by number): the rank of each is a count over all
  int* pairs = reinterpret_cast<int*>(tiles_ptr);
  for (int b = tid; b < a.B; b += kThreads) {
    const int len = prompt_len(a, b);
    if (len < 0) report(status, STIEF_ERR_BOUNDS);
    pairs[b] = pairs_of(a, len);
  }
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 2);               // one arrival from each tile's MMA warp
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full(t), 1);
      mbar_init(q_empty(t), 1);
      mbar_init(s_full(t), 1);
      mbar_init(p_full(t, 0), 4);               // one arrival per softmax warp of the tile
      mbar_init(p_full(t, 1), 4);
      mbar_init(o_full(t), 1);
    }
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 8) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
  __syncthreads();
  for (int b = tid; b < a.B; b += kThreads) {
    const int mine = pairs[b];
    int rank = 0;
    for (int i = 0; i < a.B; ++i) rank += pairs[i] > mine || (pairs[i] == mine && i < b);
    order[rank] = (uint16_t)b;
  }
  fence_proxy_async_smem();                     // the scratch above becomes a target of TMA writes
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  Walk walk;
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");       // 384 x 168 registers at launch = 256 x 208 + 128 x 88
    if (warp == 8) {
      // ---------------------------------------------------------------------------------------- producer
      if (lane == 0) {
        tma_prefetch_desc(&tmQ);
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmV);
      }
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
        walk.start(a, order);
        for (Item w = walk.next(a, order); w.valid; w = walk.next(a, order)) {
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
    } else if (warp < 11) {
      // ---------------------------------------------------------------------------------------- MMA issue, tile mt
      // The whole warp runs the control flow (descriptors stay in uniform registers); one lane issues.
      const bool leader = lane == 0;
      const int mt = __shfl_sync(0xffffffffu, warp, 0) - 9;
      const uint32_t tmem_u = __shfl_sync(0xffffffffu, tmem_base, 0);
      const uint32_t t_s = tmem_u + mt * 256, t_o = t_s + 128;
      const uint32_t id_qk = idesc_bf16_f32(kRows, kRows), id_pv = idesc_bf16_f32_bmn(kRows, kD);
      const uint64_t d_k = desc_template(2, 16, 1024);                         // rows of 128 bytes, K-major
      const uint64_t d_v = desc_template(2, kRows * 128, 1024);                // V block, MN-major: two halves of 64 channels
      const uint64_t dq = desc_at(d_k, q_smem + mt * kTileBytes);
      int st = 0, use = 0, kt = 0, n = 0;
      auto consume = [&](uint32_t& addr, int& stage) {
        mbar_wait(full_bar(st), use & 1, abort_flag, status);
        addr = ring + st * kTileBytes;
        stage = st;
        if (++st == kStages) {
          st = 0;
          ++use;
        }
      };
      auto koff = [](int k) { return (uint32_t)((k >> 2) * (kTileBytes / 2) + (k & 3) * 32) >> 4; };
      walk.start(a, order);
      for (Item w = walk.next(a, order); __shfl_sync(0xffffffffu, (int)w.valid, 0); w = walk.next(a, order)) {
        const int np0 = __shfl_sync(0xffffffffu, w.np[0], 0), np1 = __shfl_sync(0xffffffffu, w.np[1], 0);
        const int np = mt ? np1 : np0, npmax = max(np0, np1);
        if (np > 0) {
          mbar_wait(q_full(mt), kt & 1, abort_flag, status);
          ++kt;
        }
        for (int j = 0; j < npmax; ++j) {
          uint32_t addr;
          int stage;
          consume(addr, stage);
          if (j < np) {
            tc_fence_after();
            const uint64_t db = desc_at(d_k, addr);
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (leader) umma_bf16(t_s, dq + koff(k), db + koff(k), id_qk, k > 0 ? 1u : 0u);
            if (leader) {
              umma_commit(s_full(mt));
              umma_commit(empty_bar(stage));
              if (j == np - 1) umma_commit(q_empty(mt));
            }
          } else if (leader) {
            mbar_arrive(empty_bar(stage));
          }
          consume(addr, stage);
          if (j < np) {
            const uint64_t db = desc_at(d_v, addr);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              if ((k & 3) == 0) {
                mbar_wait(p_full(mt, k >> 2), n & 1, abort_flag, status);
                tc_fence_after();
              }
              if (leader) umma_bf16_ts(t_o, t_s + 8 * k, db + (uint32_t)(k * 2048 >> 4), id_pv, (j > 0 || k > 0) ? 1u : 0u);
            }
            ++n;
            if (leader) {
              umma_commit(empty_bar(stage));
              if (j == np - 1) umma_commit(o_full(mt));
            }
          } else if (leader) {
            mbar_arrive(empty_bar(stage));
          }
        }
      }
    }
  } else {
    // ------------------------------------------------------------------------------------------ softmax / epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int t = warp >> 2, q4 = warp & 3, row = 32 * q4 + lane;
    const uint32_t t_s = tmem_base + ((uint32_t)(32 * q4) << 16) + t * 256, t_o = t_s + 128;
    const float c = kLog2e * rsqrtf((float)kD);
    int n = 0, kt = 0, item = 0;                                // blocks and items of this tile so far; ring items of both tiles
    auto arrive_warp = [&](uint32_t bar) {
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    walk.start(a, order);
    for (Item w = walk.next(a, order); w.valid; w = walk.next(a, order)) {
      const int item0 = item;
      item += 2 * max(w.np[0], w.np[1]);
      const int np = w.np[t];
      if (np == 0) continue;
      const int tok = w.tok0[t] + row;
      const bool row_valid = tok < w.len, warp_live = w.tok0[t] + 32 * q4 < w.len;
      float m_ref = 0.f, l = 0.f;
      for (int j = 0; j < np; ++j, ++n) {
        const int p0 = j * kRows;
        const bool diag = j == np - 1;
        mbar_wait(s_full(t), n & 1, abort_flag, status);
        tc_fence_after();
        if (p0 + kRows > w.len) {
          // rows behind the prompt's end: whatever they hold (another prompt's values, NaN) must not reach the accumulator
          // through 0 * x.  Both tiles zero them; the values are the same.
          const int idx = item0 + 2 * j + 1, stg = idx % kStages;
          mbar_wait(full_bar(stg), (idx / kStages) & 1, abort_flag, status);
          uint8_t* v = tiles_ptr + (2 + stg) * kTileBytes;
          const int dead = w.len - p0;
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
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld32(t_s + 32 * i, sv + 32 * i);
        tmem_ld_wait();
        float* s = reinterpret_cast<float*>(sv);
        if (diag) {
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i > row) s[i] = -INFINITY;
        }
        float mx0 = max3(s[0], s[1], s[2]), mx1 = max3(s[3], s[4], s[5]);
#pragma unroll
        for (int i = 6; i < 126; i += 4) {
          mx0 = max3(mx0, s[i], s[i + 1]);
          mx1 = max3(mx1, s[i + 2], s[i + 3]);
        }
        const float mx = fmaxf(max3(mx0, s[126], s[127]), mx1);
        if (j == 0) {
          m_ref = fmaxf(mx, -1e30f);
          l = 0.f;
        } else if (const bool grown = (mx - m_ref) * c > kRescaleLog2; __any_sync(0xffffffffu, grown)) {
          const float f = grown ? fast_exp2((m_ref - mx) * c) : 1.0f;       // a row's bits do not depend on its neighbours
          if (grown) m_ref = mx;
          l *= f;
          for (int c0 = 0; c0 < kD; c0 += 32) {
            uint32_t v[32];
            tmem_ld32(t_o + c0, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
            tmem_st32(t_o + c0, v);
          }
          tmem_st_wait();
        }
        const uint64_t c2 = pack2(c, c), neg2 = pack2(-m_ref * c, -m_ref * c);
        uint64_t sum2 = pack2(0.f, 0.f);
        // 64 columns: probabilities as bf16 pairs over the scores.  The polynomial cannot return an exact zero, so the
        // masked block takes the special-function unit throughout.
        auto half_row = [&](int h, auto poly_tag) {
          constexpr bool kPoly = decltype(poly_tag)::value;
          uint32_t pk[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float x0, x1, e0, e1;
            unpack2(fma2(pack2(s[64 * h + 2 * i], s[64 * h + 2 * i + 1]), c2, neg2), x0, x1);
            if (kPoly && (i % kPolyEvery) == 0) {
              exp2_pair_fma(pack2(fmaxf(x0, -125.f), fmaxf(x1, -125.f)), e0, e1);
            } else {
              e0 = fast_exp2(x0);
              e1 = fast_exp2(x1);
            }
            sum2 = add2(sum2, pack2(e0, e1));
            pk[i] = pack_bf16(e0, e1);
          }
          tmem_st32(t_s + 32 * h, pk);
          tmem_st_wait();
          tc_fence_before();
          arrive_warp(p_full(t, h));
        };
        if (!diag) {
          half_row(0, std::true_type{});
          half_row(1, std::true_type{});
        } else {
          half_row(0, std::false_type{});
          half_row(1, std::false_type{});
        }
        float a0, a1;
        unpack2(sum2, a0, a1);
        l += a0 + a1;
      }
      // ---- epilogue: O / l
      mbar_wait(o_full(t), kt & 1, abort_flag, status);
      ++kt;
      tc_fence_after();
      if (warp_live) {
        const float inv = 1.0f / l;
        __nv_bfloat16* orow = a.out + (size_t)(w.lo + tok) * a.out_stride + (size_t)w.head[t] * kD;
        for (int c0 = 0; c0 < kD; c0 += 32) {
          uint32_t v[32];
          tmem_ld32(t_o + c0, v);
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
        if (row_valid && a.out_lse) a.out_lse[(size_t)(w.lo + tok) * a.Hq + w.head[t]] = kLn2 * (m_ref * c + log2f(l));
      }
      tc_fence_before();                                        // ordered before this tile's next P by the arrival that publishes it
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 8) tmem_dealloc(tmem_base, kTmemCols);
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
