// New tokens into the paged cache with the position rotation on the way: stief_rope_append (bf16 pools) and stief_f8_append
// (e4m3 pools with one scale for each page and head).  Per token x of head h at position p:
//     k_row = R_p(k) U_k[h],  v_row = v U_v[h],  q_out = R_p(q),    R_p: (a, b) -> (a cos - b sin, b cos + a sin) per channel pair.
//
// Every input is read once and every output written once, 11.6 flops a byte at 32 query heads, 8 KV heads and ranks 64/64:
// bound by memory, so the products run on mma.sync from registers (a tcgen05 tile would want the rotated rows in shared
// memory all the same, and its rate is not needed).
//
// One launch, two kinds of CTAs of 128 threads, all resident at once:
//   rows of the cache  a CTA belongs to one (head, side) and keeps its basis as B fragments in registers (warp w: the 8-column
//                      tiles w, w + 4, ...).  It walks the pages that the call touches: up to 64 rows of one page are loaded,
//                      rotated in fp32 and left in shared memory as bf16 terms (value and residuals: 2 terms keep 16 significant
//                      bits, far below the rounding to bf16; 3 keep fp32's 24, so that an e4m3 code is the one fp32 arithmetic
//                      gives; values and unrotated keys are bf16 already), multiplied, and leave through shared memory as one
//                      contiguous piece of the page.
//   queries            16 tokens x 8 heads at a time; a thread owns one eighth of a token's channels, so its cosines and sines
//                      serve all 8 heads.
//
// The 8-bit cache: a CTA sees all rows that a page receives, so the block's scale is settled in one exchange between its
// warps: the larger of the scale that the page's older rows have and the least power of two that holds the new rows.  When it
// grows, the same CTA moves the older rows' codes.
#include "stief_f8.cuh"
#include "stief_host_util.h"

namespace stief {
namespace rope {

constexpr int kThreads = 128;
constexpr int kRowBytes = kD * 2;                 // a row in shared memory: 16 chunks of 16 bytes, chunk c at place c ^ (row & 7)
constexpr int kTermBytes = kPage * kRowBytes;
constexpr int kTokQ = 16, kHeadsQ = 8;            // tokens and heads of a query unit
constexpr int kMaxPlace = 1 << 30;                // places in the cache end here

struct Args {
  LayerDev L;                    // bf16 pools: k_pool, v_pool
  f8::Pools P;                   // 8-bit pools
  BatchDev Bt;
  const __nv_bfloat16 *q, *k, *v;
  long long q_stride, k_stride, v_stride, qo_stride;
  __nv_bfloat16* q_out;
  const int32_t* cu;
  const int32_t* positions;
  int total, ends_at_len;
  const float* table;            // [max_pos][rot]; rot = 0: no rotation
  int max_pos, rot, interleaved;
  int n_kv, per_slot;            // CTAs for the cache's rows: per_slot for each (head, side); the others are for the queries
  int32_t* status;
};

// The sequences of a call, in shared memory: first packed token, tokens, place of the first token, prefix sums of touched pages.
struct Sequences {
  int *cu, *n, *start, *pref;
};
__device__ __forceinline__ Sequences sequences_at(uint8_t* p, int B) {
  Sequences s;
  s.cu = reinterpret_cast<int*>(p);
  s.n = s.cu + B;
  s.start = s.n + B;
  s.pref = s.start + B;
  return s;
}
constexpr int sequences_bytes(int B) { return (4 * B + 1) * 4; }

// Called by all threads; ends with a barrier.
__device__ __forceinline__ void load_sequences(const Sequences& s, const Args& a) {
  const int B = a.Bt.B;
  for (int b = threadIdx.x; b < B; b += kThreads) {
    const int lo = a.cu[b], hi = a.cu[b + 1], len = a.Bt.seq_lens[b];
    const bool in_order = lo >= 0 && hi >= lo && hi <= a.total;
    int n = in_order ? hi - lo : 0;
    const int start = a.ends_at_len ? len - n : len;
    if (!in_order || len < 0 || start < 0 || start > kMaxPlace - n) {
      if (blockIdx.x == 0) report(a.status, STIEF_ERR_BOUNDS);
      n = 0;
    }
    s.cu[b] = lo;
    s.n[b] = n;
    s.start[b] = n > 0 ? start : 0;
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    int carry = 0;
    for (int base = 0; base < B; base += 32) {
      const int b = base + lane;
      const int v = b < B && s.n[b] > 0 ? (s.start[b] % kPage + s.n[b] + kPage - 1) / kPage : 0;
      int x = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += t;
      }
      if (b < B) s.pref[b + 1] = carry + x;
      carry += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) s.pref[0] = 0;
  }
  __syncthreads();
}

// the largest i in 0 .. n - 1 with first[i] <= x (0 if there is none)
__device__ __forceinline__ int last_at_most(const int* first, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// A thread's eighth of a row: two chunks of 8 channels that hold 8 pairs (slots below rot / 16), or that are not turned.
struct Eighth {
  int c0, c1;
  bool turned;
};
__device__ __forceinline__ Eighth eighth_of(int j, int rot, int interleaved) {
  Eighth e;
  const int nr = rot >> 4;
  e.turned = j < nr;
  if (interleaved) {
    e.c0 = 2 * j;
    e.c1 = 2 * j + 1;
  } else {
    e.c0 = e.turned ? j : 2 * j;                  // rot / 8 + 2 (j - rot / 16) = 2 j
    e.c1 = e.turned ? j + nr : 2 * j + 1;
  }
  return e;
}

__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8]) {
  x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
  x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// 8 cosines and 8 sines of slot j
__device__ __forceinline__ void load_angles(const Args& a, int pos, int j, float (&cs)[8], float (&sn)[8]) {
  const float4* row = reinterpret_cast<const float4*>(a.table + (size_t)pos * a.rot);
  const int half4 = a.rot >> 3;                    // float4 pieces of the cosines
  const float4 c0 = __ldg(row + 2 * j), c1 = __ldg(row + 2 * j + 1), s0 = __ldg(row + half4 + 2 * j), s1 = __ldg(row + half4 + 2 * j + 1);
  cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w; cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
  sn[0] = s0.x; sn[1] = s0.y; sn[2] = s0.z; sn[3] = s0.w; sn[4] = s1.x; sn[5] = s1.y; sn[6] = s1.z; sn[7] = s1.w;
}
__device__ __forceinline__ void turn(float& x, float& y, float c, float s) {
  const float t = fmaf(x, c, -y * s);
  y = fmaf(y, c, x * s);
  x = t;
}
__device__ __forceinline__ void turn_eighth(float (&x)[8], float (&y)[8], const float (&cs)[8], const float (&sn)[8], int interleaved) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      turn(x[2 * i], x[2 * i + 1], cs[i], sn[i]);
      turn(y[2 * i], y[2 * i + 1], cs[4 + i], sn[4 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(x[i], y[i], cs[i], sn[i]);
  }
}

// ---------------------------------------------------------------------------------------------
// queries
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void turn_queries(const Args& a, const Sequences& s, int cta, int n_cta) {
  const int groups = (a.L.Hq + kHeadsQ - 1) / kHeadsQ;
  const long long units = (long long)((a.total + kTokQ - 1) / kTokQ) * groups;
  const int j = threadIdx.x & 7;
  const Eighth e = eighth_of(j, a.rot, a.interleaved);
  for (long long u = cta; u < units; u += n_cta) {
    const int tok = (int)(u / groups) * kTokQ + (threadIdx.x >> 3), h0 = (int)(u % groups) * kHeadsQ;
    if (tok >= a.total) continue;
    const int b = last_at_most(s.cu, a.Bt.B, tok);
    if (tok < s.cu[b] || tok - s.cu[b] >= s.n[b]) continue;          // a token of no sequence
    const int pos = a.positions ? a.positions[tok] : s.start[b] + tok - s.cu[b];
    if (a.rot && (pos < 0 || pos >= a.max_pos)) {
      report(a.status, STIEF_ERR_BOUNDS);
      continue;
    }
    float cs[8], sn[8];
    if (e.turned) load_angles(a, pos, j, cs, sn);
    const uint4* src = reinterpret_cast<const uint4*>(a.q + (size_t)tok * a.q_stride);
    uint4* dst = reinterpret_cast<uint4*>(a.q_out + (size_t)tok * a.qo_stride);
#pragma unroll
    for (int g = 0; g < kHeadsQ; g += 4) {
      uint4 w0[4], w1[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (h0 + g + i < a.L.Hq) {
          w0[i] = src[(h0 + g + i) * 16 + e.c0];
          w1[i] = src[(h0 + g + i) * 16 + e.c1];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (h0 + g + i < a.L.Hq) {
          if (e.turned) {
            float x[8], y[8];
            unpack8(w0[i], x);
            unpack8(w1[i], y);
            turn_eighth(x, y, cs, sn, a.interleaved);
            w0[i] = pack8(x);
            w1[i] = pack8(y);
          }
          dst[(h0 + g + i) * 16 + e.c0] = w0[i];
          dst[(h0 + g + i) * 16 + e.c1] = w1[i];
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// rows of the cache
// ---------------------------------------------------------------------------------------------
// NT: 8-column tiles of a warp at most (rank 32: 1, 48 and 64: 2, 96: 3, 128: 4)
template <int NT, bool F8>
__device__ __forceinline__ void append_rows(const Args& a, const Sequences& s, uint8_t* smem, int* row_ok, float* tops) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tid4 = lane & 3;
  const int slot = blockIdx.x / a.per_slot, part = blockIdx.x - slot * a.per_slot;
  const int h = slot >> 1, side = slot & 1;
  const int R = side ? a.L.r_v : a.L.r_k;
  const __nv_bfloat16* Ub = side ? a.L.U_v : a.L.U_k;
  const __nv_bfloat16* U = Ub ? Ub + (size_t)h * (side ? a.L.uv_stride : a.L.uk_stride) : nullptr;
  const int d_in = U ? kD : R;
  const int rot = side ? 0 : a.rot;
  // a side without basis is stored as it is: in bf16 the first term is all of it
  const int n_terms = rot == 0 || (!F8 && !U) ? 1 : F8 ? 3 : 2;
  const __nv_bfloat16* X = side ? a.v : a.k;
  const long long stride = side ? a.v_stride : a.k_stride;
  const uint32_t tile = smem_u32(smem);
  const int pages = s.pref[a.Bt.B];
  if (part >= pages) return;

  // ---- the basis as B fragments: tile t = warp + 4 i, k-step ks: rows 16 ks + 2 tid4, + 1 (and + 8, + 9) of column 8 t + gid
  uint32_t uf[NT][8][2];
  if (U) {
    const int rowb = R * 2;
    for (int i = tid; i < kD * R / 8; i += kThreads) {
      const uint4 w = __ldg(reinterpret_cast<const uint4*>(U) + i);
      reinterpret_cast<uint4*>(smem)[i] = w;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int t = min(warp + 4 * i, R / 8 - 1);                          // a warp without a tile repeats the last (its results are not used)
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        ldsm_x4_t(tile + (32 * kk + lane) * rowb + t * 16, uf[i][2 * kk][0], uf[i][2 * kk][1], uf[i][2 * kk + 1][0], uf[i][2 * kk + 1][1]);
    }
    __syncthreads();
  }

  for (int it = part; it < pages; it += a.per_slot) {
    const int b = last_at_most(s.pref, a.Bt.B, it);                        // empty sequences repeat a prefix: the last one is meant
    const int start = s.start[b], n = s.n[b];
    const int pi = start / kPage + it - s.pref[b];
    const int place0 = max(start, pi * kPage), m = min(start + n, pi * kPage + kPage) - place0;
    const int slot0 = place0 & (kPage - 1), tok0 = s.cu[b] + place0 - start;
    int page = -1;
    if (pi < a.Bt.max_pages) page = a.Bt.block_table[(size_t)b * a.Bt.max_pages + pi];
    if (page < 0 || page >= a.L.num_pages) {                               // the same for every thread
      if (tid == 0) report(a.status, STIEF_ERR_BOUNDS);
      continue;
    }
    const size_t tile_id = (size_t)page * a.L.Hkv + h;
    float s_old = 0.f;
    if (F8 && slot0 > 0) s_old = a.P.scales[tile_id * f8::kScalesPerTile + side];

    // ---- rows into shared memory, rotated, as bf16 terms
    bool any = false;
#pragma unroll
    for (int i = 0; i < kPage * 8 / kThreads; ++i) {
      const int u = tid + i * kThreads, row = u >> 3, j = u & 7;
      if (row >= m) continue;
      const int tok = tok0 + row;
      const Eighth e = eighth_of(j, rot, a.interleaved);
      const uint4* src = reinterpret_cast<const uint4*>(X + (size_t)tok * stride + (size_t)h * d_in);
      uint4 w0 = make_uint4(0u, 0u, 0u, 0u), w1 = w0;
      if (e.c0 * 8 < d_in) w0 = __ldg(src + e.c0);
      if (e.c1 * 8 < d_in) w1 = __ldg(src + e.c1);
      bool ok = true;
      if (a.rot) {                                                         // values too: a token outside the table is not stored at all
        const int pos = a.positions ? a.positions[tok] : place0 + row;
        ok = pos >= 0 && pos < a.max_pos;
        if (ok && e.turned) {
          float cs[8], sn[8], x[8], y[8];
          load_angles(a, pos, j, cs, sn);
          unpack8(w0, x);
          unpack8(w1, y);
          turn_eighth(x, y, cs, sn, a.interleaved);
          w0 = pack8(x);
          w1 = pack8(y);
          if (n_terms > 1) {
            uint4 r0 = w0, r1 = w1;
            for (int term = 1; term < n_terms; ++term) {
              float p[8];
              unpack8(r0, p);
#pragma unroll
              for (int c = 0; c < 8; ++c) x[c] -= p[c];
              unpack8(r1, p);
#pragma unroll
              for (int c = 0; c < 8; ++c) y[c] -= p[c];
              r0 = pack8(x);
              r1 = pack8(y);
              uint8_t* dst = smem + term * kTermBytes + row * kRowBytes;
              *reinterpret_cast<uint4*>(dst + ((e.c0 ^ (row & 7)) << 4)) = r0;
              *reinterpret_cast<uint4*>(dst + ((e.c1 ^ (row & 7)) << 4)) = r1;
            }
          }
        } else if (n_terms > 1) {
          for (int term = 1; term < n_terms; ++term) {
            uint8_t* dst = smem + term * kTermBytes + row * kRowBytes;
            *reinterpret_cast<uint4*>(dst + ((e.c0 ^ (row & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4*>(dst + ((e.c1 ^ (row & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
      }
      *reinterpret_cast<uint4*>(smem + row * kRowBytes + ((e.c0 ^ (row & 7)) << 4)) = w0;
      *reinterpret_cast<uint4*>(smem + row * kRowBytes + ((e.c1 ^ (row & 7)) << 4)) = w1;
      if (j == 0) {
        row_ok[row] = ok;
        if (!ok) report(a.status, STIEF_ERR_BOUNDS);
      }
      any |= ok;
    }
    if (!__syncthreads_or(any)) continue;

    // ---- products, the smallest term first
    float acc[kPage / 16][NT][4];
#pragma unroll
    for (int mt = 0; mt < kPage / 16; ++mt) {
#pragma unroll
      for (int i = 0; i < NT; ++i) acc[mt][i][0] = acc[mt][i][1] = acc[mt][i][2] = acc[mt][i][3] = 0.f;
      if (mt * 16 < m && U) {
        const int row = 16 * mt + (lane & 15);
        for (int term = n_terms - 1; term >= 0; --term) {
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            uint32_t af[4];
            ldsm_x4(tile + term * kTermBytes + row * kRowBytes + (((2 * ks + (lane >> 4)) ^ (row & 7)) << 4), af[0], af[1], af[2], af[3]);
#pragma unroll
            for (int i = 0; i < NT; ++i) mma_bf16(acc[mt][i], af, uf[i][ks][0], uf[i][ks][1]);
          }
        }
      } else if (mt * 16 < m) {                                            // no basis: the rows themselves
        for (int term = n_terms - 1; term >= 0; --term) {
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            const int t = warp + 4 * i;
            if (t >= R / 8) continue;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int row = 16 * mt + gid + 8 * e;
              const uint32_t w = *reinterpret_cast<const uint32_t*>(smem + term * kTermBytes + row * kRowBytes + ((t ^ (row & 7)) << 4) + 4 * tid4);
              acc[mt][i][2 * e] += bf16_lo(w);
              acc[mt][i][2 * e + 1] += bf16_hi(w);
            }
          }
        }
      }
    }

    // ---- the block's scale
    float scale = 1.f, inv = 1.f;
    if constexpr (F8) {
      float top = 0.f;
#pragma unroll
      for (int mt = 0; mt < kPage / 16; ++mt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = 16 * mt + gid + 8 * e;
          if (row < m && row_ok[row]) {
#pragma unroll
            for (int i = 0; i < NT; ++i) {
              if (warp + 4 * i < R / 8) {
                const float x = fabsf(acc[mt][i][2 * e]), y = fabsf(acc[mt][i][2 * e + 1]);
                top = fmaxf(top, fmaxf(x <= 3.402823466e38f ? x : 0.f, y <= 3.402823466e38f ? y : 0.f));   // NaN and infinities leave the scale alone
              }
            }
          }
        }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (lane == 0) tops[warp] = top;
      __syncthreads();                                                     // also: every warp has read its operands
      top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
      scale = fmaxf(f8::scale_for(top), s_old);
      inv = 1.f / scale;                                                   // exact for a power of two
      if (slot0 > 0 && scale != s_old) {                                   // the page's older rows move to the larger scale
        const float ratio = s_old * inv;
        uint4* old = reinterpret_cast<uint4*>((side ? a.P.v_codes : a.P.k_codes) + tile_id * kPage * R);
        for (int i = tid; i < slot0 * R / 16; i += kThreads) {
          uint4 w = old[i];
          uint32_t* p = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float2 x = f8::e4m3x2_to_float2(p[c] & 0xffffu), y = f8::e4m3x2_to_float2(p[c] >> 16);
            p[c] = f8::pack_e4m3(x.x * ratio, x.y * ratio, y.x * ratio, y.y * ratio);
          }
          old[i] = w;
        }
      }
      if (tid == 0) a.P.scales[tile_id * f8::kScalesPerTile + side] = scale;
    } else {
      __syncthreads();
    }

    // ---- results through shared memory: rows back to back, as they lie in the page
    constexpr int kElt = F8 ? 1 : 2;
#pragma unroll
    for (int mt = 0; mt < kPage / 16; ++mt) {
      if (mt * 16 >= m) break;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int t = warp + 4 * i;
        if (t < R / 8) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int row = 16 * mt + gid + 8 * e, col = 8 * t + 2 * tid4;
            if constexpr (F8)
              *reinterpret_cast<uint16_t*>(smem + row * R + col) = (uint16_t)f8::pack_e4m3(acc[mt][i][2 * e] * inv, acc[mt][i][2 * e + 1] * inv, 0.f, 0.f);
            else
              *reinterpret_cast<uint32_t*>(smem + (row * R + col) * 2) = pack_bf16(acc[mt][i][2 * e], acc[mt][i][2 * e + 1]);
          }
        }
      }
    }
    __syncthreads();
    {
      const int per_row = R * kElt / 16;
      uint8_t* pool = F8 ? (side ? a.P.v_codes : a.P.k_codes) : reinterpret_cast<uint8_t*>(side ? a.L.v_pool : a.L.k_pool);
      uint4* dst = reinterpret_cast<uint4*>(pool + (tile_id * kPage + slot0) * R * kElt);
      for (int i = tid; i < m * per_row; i += kThreads)
        if (row_ok[i / per_row]) dst[i] = reinterpret_cast<const uint4*>(smem)[i];
    }
    __syncthreads();                                                       // the tile and row_ok are free
  }
}

template <int NT, bool F8>
__global__ void __launch_bounds__(kThreads, NT > 2 ? 3 : 4)
append_rotated_kernel(const Args a) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int row_ok[kPage];
  __shared__ float tops[4];
  const int tile_bytes = F8 ? 3 * kTermBytes : 2 * kTermBytes;
  const Sequences s = sequences_at(smem + tile_bytes, a.Bt.B);
  load_sequences(s, a);
  if ((int)blockIdx.x >= a.n_kv) {
    turn_queries(a, s, blockIdx.x - a.n_kv, gridDim.x - a.n_kv);
    return;
  }
  append_rows<NT, F8>(a, s, smem, row_ok, tops);
}

template <int NT, bool F8>
cudaError_t launch(Args a, cudaStream_t st) {
  auto kern = append_rotated_kernel<NT, F8>;
  const int smem = (F8 ? 3 : 2) * kTermBytes + sequences_bytes(a.Bt.B);
  static bool configured[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!configured[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (F8 ? 3 : 2) * kTermBytes + sequences_bytes(kMaxBatch));
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  const int resident = host::sm_count() * (NT > 2 ? 3 : 4), slots = 2 * a.L.Hkv;
  const long long few = a.total < a.Bt.B ? a.total : a.Bt.B;
  const long long pages = a.total / kPage + 2 * few < a.total ? a.total / kPage + 2 * few : a.total;      // pages touched, at most
  long long per_slot = (resident * 9 / 20) / slots;
  per_slot = per_slot < 1 ? 1 : per_slot > pages ? pages : per_slot;
  a.per_slot = (int)per_slot;
  a.n_kv = slots * a.per_slot;
  long long n_q = 0;
  if (a.q) {
    n_q = (long long)((a.total + kTokQ - 1) / kTokQ) * ((a.L.Hq + kHeadsQ - 1) / kHeadsQ);
    const long long left = resident - a.n_kv > resident / 4 ? resident - a.n_kv : resident / 4;
    if (n_q > left) n_q = left;
  }
  kern<<<(unsigned)(a.n_kv + n_q), kThreads, smem, st>>>(a);
  return cudaGetLastError();
}

template <bool F8>
cudaError_t launch_rank(const Args& a, cudaStream_t st) {
  const int r = a.L.r_k > a.L.r_v ? a.L.r_k : a.L.r_v;
  return r <= 32 ? launch<1, F8>(a, st) : r <= 64 ? launch<2, F8>(a, st) : r <= 96 ? launch<3, F8>(a, st) : launch<4, F8>(a, st);
}

bool rank_ok(int r) { return r == 32 || r == 48 || r == 64 || r == 96 || r == 128; }

// What both calls refuse; fills everything of `a` but the pools.
template <class Layer>
int fill(Args& a, const Layer* layer, const stief_batch* batch, const stief_rotation* rotation, const uint16_t* q, int64_t q_stride_t,
         const uint16_t* k, int64_t k_stride_t, const uint16_t* v, int64_t v_stride_t, int32_t total_tokens, const int32_t* cu_seqlens,
         const int32_t* positions, int32_t ends_at_len, uint16_t* q_out, int64_t q_out_stride_t, int32_t* status) {
  using host::aligned;
  if (!layer || layer->Hq <= 0 || layer->Hkv <= 0 || layer->Hq % layer->Hkv != 0 || layer->num_pages <= 0) return STIEF_ERR_INVALID_ARG;
  if (layer->d != kD || !rank_ok(layer->r_k) || !rank_ok(layer->r_v)) return STIEF_ERR_UNSUPPORTED;
  const int rc = host::check_batch(batch);
  if (rc != STIEF_OK) return rc;
  if (!k || !v || !cu_seqlens || total_tokens < 0 || (q == nullptr) != (q_out == nullptr) || (q && !rotation) || ends_at_len < 0 || ends_at_len > 1) return STIEF_ERR_INVALID_ARG;
  const long long dk = layer->U_k ? kD : layer->r_k, dv = layer->U_v ? kD : layer->r_v;
  if (k_stride_t < layer->Hkv * dk || v_stride_t < layer->Hkv * dv || k_stride_t % 8 || v_stride_t % 8 || !aligned(k, 16) || !aligned(v, 16))
    return STIEF_ERR_INVALID_ARG;
  if (q && (q_stride_t < (long long)layer->Hq * kD || q_out_stride_t < (long long)layer->Hq * kD || q_stride_t % 8 || q_out_stride_t % 8 ||
            !aligned(q, 16) || !aligned(q_out, 16) || (q == q_out && q_stride_t != q_out_stride_t)))
    return STIEF_ERR_INVALID_ARG;
  if ((layer->U_k && !aligned(layer->U_k, 128)) || (layer->U_v && !aligned(layer->U_v, 128)) || layer->uk_head_stride < 0 || layer->uv_head_stride < 0 ||
      layer->uk_head_stride % 8 || layer->uv_head_stride % 8 || !aligned(cu_seqlens, 4) || !aligned(positions, 4))
    return STIEF_ERR_INVALID_ARG;
  a.rot = 0;
  a.table = nullptr;
  a.max_pos = a.interleaved = 0;
  if (rotation) {
    if (!rotation->table || !aligned(rotation->table, 16) || rotation->max_pos <= 0 || rotation->rot_dim < 16 || rotation->rot_dim > kD ||
        rotation->rot_dim % 16 || rotation->interleaved < 0 || rotation->interleaved > 1)
      return STIEF_ERR_INVALID_ARG;
    if (dk != kD) return STIEF_ERR_UNSUPPORTED;                           // compressed keys cannot be rotated any more
    a.table = rotation->table;
    a.max_pos = rotation->max_pos;
    a.rot = rotation->rot_dim;
    a.interleaved = rotation->interleaved;
  }
  a.L.Hq = layer->Hq; a.L.Hkv = layer->Hkv; a.L.G = layer->Hq / layer->Hkv; a.L.r_k = layer->r_k; a.L.r_v = layer->r_v; a.L.num_pages = layer->num_pages;
  a.L.U_k = reinterpret_cast<const __nv_bfloat16*>(layer->U_k); a.L.uk_stride = layer->uk_head_stride;
  a.L.U_v = reinterpret_cast<const __nv_bfloat16*>(layer->U_v); a.L.uv_stride = layer->uv_head_stride;
  a.L.k_pool = a.L.v_pool = nullptr;
  a.P = f8::Pools{nullptr, nullptr, nullptr};
  a.Bt = host::to_dev(batch);
  a.q = reinterpret_cast<const __nv_bfloat16*>(q);
  a.k = reinterpret_cast<const __nv_bfloat16*>(k);
  a.v = reinterpret_cast<const __nv_bfloat16*>(v);
  a.q_stride = q_stride_t; a.k_stride = k_stride_t; a.v_stride = v_stride_t; a.qo_stride = q_out_stride_t;
  a.q_out = reinterpret_cast<__nv_bfloat16*>(q_out);
  a.cu = cu_seqlens;
  a.positions = positions;
  a.total = total_tokens;
  a.ends_at_len = ends_at_len;
  a.status = status;
  return STIEF_OK;
}

}  // namespace rope
}  // namespace stief

using namespace stief;

extern "C" int stief_rope_append(const stief_layer* layer, const stief_batch* batch, const stief_rotation* rotation, const uint16_t* q,
                                 int64_t q_stride_t, const uint16_t* k, int64_t k_stride_t, const uint16_t* v, int64_t v_stride_t,
                                 int32_t total_tokens, const int32_t* cu_seqlens, const int32_t* positions, int32_t ends_at_len,
                                 uint16_t* q_out, int64_t q_out_stride_t, int32_t* status, void* stream) {
  rope::Args a;
  const int rc = rope::fill(a, layer, batch, rotation, q, q_stride_t, k, k_stride_t, v, v_stride_t, total_tokens, cu_seqlens, positions,
                            ends_at_len, q_out, q_out_stride_t, status);
  if (rc != STIEF_OK) return rc;
  if (!layer->k_pool || !layer->v_pool || !host::aligned(layer->k_pool, 128) || !host::aligned(layer->v_pool, 128)) return STIEF_ERR_INVALID_ARG;
  if (total_tokens == 0) return STIEF_OK;
  a.L.k_pool = reinterpret_cast<__nv_bfloat16*>(layer->k_pool);
  a.L.v_pool = reinterpret_cast<__nv_bfloat16*>(layer->v_pool);
  return rope::launch_rank<false>(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}

extern "C" int stief_f8_append(const stief_f8layer* layer, const stief_batch* batch, const stief_rotation* rotation, const uint16_t* q,
                               int64_t q_stride_t, const uint16_t* k, int64_t k_stride_t, const uint16_t* v, int64_t v_stride_t,
                               int32_t total_tokens, const int32_t* cu_seqlens, const int32_t* positions, int32_t ends_at_len,
                               uint16_t* q_out, int64_t q_out_stride_t, int32_t* status, void* stream) {
  rope::Args a;
  const int rc = rope::fill(a, layer, batch, rotation, q, q_stride_t, k, k_stride_t, v, v_stride_t, total_tokens, cu_seqlens, positions,
                            ends_at_len, q_out, q_out_stride_t, status);
  if (rc != STIEF_OK) return rc;
  if (!layer->k_codes || !layer->v_codes || !layer->scales || !host::aligned(layer->k_codes, 128) || !host::aligned(layer->v_codes, 128) ||
      !host::aligned(layer->scales, 16))
    return STIEF_ERR_INVALID_ARG;
  if (total_tokens == 0) return STIEF_OK;
  a.P = f8::Pools{layer->k_codes, layer->v_codes, layer->scales};
  return rope::launch_rank<true>(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}
