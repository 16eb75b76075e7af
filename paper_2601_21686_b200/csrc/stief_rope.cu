// New tokens into the paged cache with the position rotation on the way: stief_rope_append (bf16 pools) and stief_f8_append
// (e4m3 pools with one scale for each page and head).  Per token x of head h at position p:
//     k_row = R_p(k) U_k[h],  v_row = v U_v[h],  q_out = R_p(q),    R_p: (a, b) -> (a cos - b sin, b cos + a sin) per channel pair.
//
// Every input is read once and every output written once, 11.6 flops a byte at 32 query heads, 8 KV heads and ranks 64/64:
// bound by memory, so the products run on mma.sync from registers (a tcgen05 tile would want the rotated rows in shared
// memory all the same, and its rate is not needed).
//
// One launch, two kinds of CTAs of 256 threads, all resident at once:
//   rows of the cache  a CTA belongs to one (head, side) and keeps its basis as B fragments in registers (warp w: the 8-column
//                      tiles w and w + 8).  It walks tiles of 64 row slots: up to 64 rows of one page, or fewer rows of several
//                      pages (a decode batch has one row in each).  Rows arrive by cp.async a tile ahead, are rotated in fp32 and
//                      left in shared memory as bf16 terms (value and residuals: 2 terms keep 16 significant bits, far below
//                      the rounding to bf16; 3 keep fp32's 24, so that an e4m3 code is the one fp32 arithmetic gives;
//                      values and unrotated keys are bf16 already), multiplied, and leave through shared memory as
//                      contiguous pieces of the pages.
//   queries            32 tokens x 8 heads at a time; a thread owns one eighth of a token's channels, so its cosines and sines
//                      serve all 8 heads.
//
// The 8-bit cache: a tile holds all rows that a page receives, so the block's scale is settled in one exchange between the
// CTA's warps: the larger of the scale that the page's older rows have and the least power of two that holds the new rows.  When it
// grows, the same CTA moves the older rows' codes.
//
// Measured (32 query heads over 8; 17600 tokens of 8 prompts): bf16 64/64 98 us (3.9 TB/s of inputs and outputs), 128/128 118;
// 8-bit 32/32 117, 64/64 118, 96/128 144, 128/32 156.  One token 5.5 to 6.2 us, 64 sequences of one token 6.7 and (8-bit) 8.8.  What
// bounds the large calls is the chain of a tile (rotate, multiply, settle the scale, stage) with two CTAs per SM to hide it, not the
// memory; its rounds of a 96-channel 8-bit key tile take 1300 (raw rows), 2700, 5600, 1800 and 2400 cycles.
#include <type_traits>

#include "stief_f8.cuh"
#include "stief_host_util.h"

namespace stief {
namespace rope {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kRowBytes = kD * 2;                 // a row in shared memory: 16 chunks of 16 bytes, chunk c at place c ^ (row & 7)
constexpr int kTermBytes = kPage * kRowBytes;
constexpr int kTokQ = kThreads / 8, kHeadsQ = 8;            // tokens and heads of a query unit
constexpr int kRotateUnroll = 2;
constexpr int kResident = 2;                      // CTAs of an SM
// Of the CTAs that are resident together: for rows of the cache; the others turn queries (17600 prompt tokens, 0.7 / 0.75 / 0.8 / 0.85:
// bf16 64/64 97 / 98 / 104 / 120 us, 8-bit 96/128 170 / 162 / 144 / 151)
constexpr double kRowsShare = 0.75, kRowsShareF8 = 0.8;
constexpr int kMaxPlace = 1 << 30;                // places in the cache end here

// raw rows and up to three terms (8-bit cache), or two
template <bool F8>
constexpr int tile_bytes() { return (F8 ? 4 : 3) * kTermBytes; }

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
  int per_key, per_value;        // CTAs for the cache's rows: per_key for each head's keys, per_value for its values; the others are
                                 // for the queries
  int32_t* status;
};

// The sequences of a call, in shared memory: first packed token, tokens, place of the first token, prefix sums of touched pages.
struct Sequences {
  int *cu, *n, *start, *pref, *most;             // most: the largest number of tokens
};
__device__ __forceinline__ Sequences sequences_at(uint8_t* p, int B) {
  Sequences s;
  s.cu = reinterpret_cast<int*>(p);
  s.n = s.cu + B;
  s.start = s.n + B;
  s.pref = s.start + B;
  s.most = s.pref + B + 1;
  return s;
}
constexpr int sequences_bytes(int B) { return (4 * B + 2) * 4; }

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
    int carry = 0, most = 0;
    for (int base = 0; base < B; base += 32) {
      const int b = base + lane;
      const int v = b < B && s.n[b] > 0 ? (s.start[b] % kPage + s.n[b] + kPage - 1) / kPage : 0;
      if (b < B) most = max(most, s.n[b]);
      int x = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += t;
      }
      if (b < B) s.pref[b + 1] = carry + x;
      carry += __shfl_sync(0xffffffffu, x, 31);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) {
      s.pref[0] = 0;
      *s.most = most;
    }
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
  const long long units = ((long long)a.total + kTokQ - 1) / kTokQ * groups;
  const int j = threadIdx.x & 7;
  const Eighth e = eighth_of(j, a.rot, a.interleaved);
  for (long long u = cta; u < units; u += n_cta) {
    const int tok = (int)(u / groups) * kTokQ + (threadIdx.x >> 3), h0 = (int)(u % groups) * kHeadsQ;
    if (tok >= a.total) continue;
    // all rows of the unit are on their way while the token's sequence is looked for and its angles are fetched
    const uint4* src = reinterpret_cast<const uint4*>(a.q + (size_t)tok * a.q_stride) + h0 * 16;
    uint4* dst = reinterpret_cast<uint4*>(a.q_out + (size_t)tok * a.qo_stride) + h0 * 16;
    uint4 w0[kHeadsQ], w1[kHeadsQ];
#pragma unroll
    for (int i = 0; i < kHeadsQ; ++i) {
      if (h0 + i < a.L.Hq) {
        w0[i] = src[i * 16 + e.c0];
        w1[i] = src[i * 16 + e.c1];
      }
    }
    const int b = last_at_most(s.cu, a.Bt.B, tok);
    if (tok < s.cu[b] || tok - s.cu[b] >= s.n[b]) continue;          // a token of no sequence
    const int pos = a.positions ? a.positions[tok] : s.start[b] + tok - s.cu[b];
    if (pos < 0 || pos >= a.max_pos) {
      report(a.status, STIEF_ERR_BOUNDS);
      continue;
    }
    float cs[8], sn[8];
    if (e.turned) load_angles(a, pos, j, cs, sn);
#pragma unroll
    for (int i = 0; i < kHeadsQ; ++i) {
      if (h0 + i < a.L.Hq) {
        if (e.turned) {
          float x[8], y[8];
          unpack8(w0[i], x);
          unpack8(w1[i], y);
          turn_eighth(x, y, cs, sn, a.interleaved);
          w0[i] = pack8(x);
          w1[i] = pack8(y);
        }
        dst[i * 16 + e.c0] = w0[i];
        dst[i * 16 + e.c1] = w1[i];
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// rows of the cache
// ---------------------------------------------------------------------------------------------
// What a tile knows of each of its pages (a "touch": the rows that one page receives)
struct Touch {
  int tok0, m;                   // first packed token, rows (0: nothing to do)
  int place0;                    // place of the first row in the sequence
  int page;
  float old;                     // 8-bit cache: the page's scale, if it holds older rows (else 0)
};
struct TileState {
  Touch touch[3][kPage];         // of this tile, of the next, and of the one before, whose rows may still be on their way out
  int row_ok[kPage];
  alignas(16) float tops[kWarps][kPage];          // largest magnitude of each row, by warp
  float top[kPage], inverse[kPage], half_top[2];
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint32_t row_chunk(int row, int chunk) { return row * kRowBytes + ((chunk ^ (row & 7)) << 4); }

// NT: 8-column tiles of a warp at most (ranks up to 64: 1, above: 2)
template <int NT, bool F8>
__device__ __forceinline__ void append_rows(const Args& a, const Sequences& s, uint8_t* smem, TileState& ts) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tid4 = lane & 3;
  const int n_key = a.per_key * a.L.Hkv;
  const int side = (int)blockIdx.x >= n_key, at = side ? blockIdx.x - n_key : blockIdx.x, per_slot = side ? a.per_value : a.per_key;
  const int h = at / per_slot, part = at - h * per_slot;
  const int R = side ? a.L.r_v : a.L.r_k;
  const __nv_bfloat16* Ub = side ? a.L.U_v : a.L.U_k;
  const __nv_bfloat16* U = Ub ? Ub + (size_t)h * (side ? a.L.uv_stride : a.L.uk_stride) : nullptr;
  const int d_in = U ? kD : R;
  const int rot = side ? 0 : a.rot;
  // a side without basis is stored as it is: in bf16 the first term is all of it
  const int n_terms = rot == 0 || (!F8 && !U) ? 1 : F8 ? 3 : 2;
  const __nv_bfloat16* X = side ? a.v : a.k;
  const long long stride = side ? a.v_stride : a.k_stride;
  uint8_t* pool = F8 ? (side ? a.P.v_codes : a.P.k_codes) : reinterpret_cast<uint8_t*>(side ? a.L.v_pool : a.L.k_pool);

  // A page has as many row slots as the longest sequence needs (a power of two), and a tile takes so many pages that there are no
  // more tiles than CTAs, as far as its slots go
  const int touches = s.pref[a.Bt.B];
  int lg = 0;
  while ((1 << lg) < min(*s.most, kPage)) ++lg;
  const int cap = 1 << lg, group = min(kPage >> lg, max(1, (touches + per_slot - 1) / per_slot)), tiles = (touches + group - 1) / group;
  const int slots = group << lg;
  if (part >= tiles) return;

  auto find_touches = [&](int tile, int buf) {                             // threads 0 .. group - 1
    if (tid >= group) return;
    Touch t = {0, 0, 0, -1, 0.f};
    const int it = tile * group + tid;
    if (it < touches) {
      const int b = last_at_most(s.pref, a.Bt.B, it);                      // empty sequences repeat a prefix: the last one is meant
      const int start = s.start[b], n = s.n[b];
      const int pi = start / kPage + it - s.pref[b];
      t.place0 = max(start, pi * kPage);
      t.m = min(start + n, pi * kPage + kPage) - t.place0;
      t.tok0 = s.cu[b] + t.place0 - start;
      if (pi < a.Bt.max_pages) t.page = a.Bt.block_table[(size_t)b * a.Bt.max_pages + pi];
      if (t.page < 0 || t.page >= a.L.num_pages) {
        report(a.status, STIEF_ERR_BOUNDS);
        t.m = 0;
      } else if (F8 && (t.place0 & (kPage - 1)) != 0) {
        t.old = a.P.scales[((size_t)t.page * a.L.Hkv + h) * f8::kScalesPerTile + side];
      }
    }
    ts.touch[buf][tid] = t;
  };
  // Shared memory: the raw rows, then the terms.  With one term the rows are multiplied as they arrive: two tiles take turns.
  const uint32_t base = smem_u32(smem);
  auto raw_at = [&](int n) { return n_terms == 1 ? (n & 1) * kTermBytes : 0; };
  const int term0 = kTermBytes;                                            // n_terms > 1: where the terms lie
  // Results on their way out: rows back to back, the 16-byte pieces of a row exchanged so that the eight rows that a store
  // instruction writes lie in different banks
  const int row_bytes = R * (F8 ? 1 : 2);
  const int swz_shift = row_bytes % 128 == 0 ? 0 : row_bytes % 64 == 0 ? 1 : 2, swz_mask = row_bytes % 128 == 0 ? 7 : row_bytes % 64 == 0 ? 3 : row_bytes == 48 ? 0 : 1;
  auto staged = [&](int row, int byte) { return row * row_bytes + (byte ^ (((row >> swz_shift) & swz_mask) << 4)); };
  const bool single = group == 1;                                          // one page per tile: its rows lie behind one another, here and there
  auto fetch = [&](int buf, int raw) {
    const int row0 = tid >> 4, chunk = tid & 15;
    if (chunk < d_in / 8) {
      if (single) {
        const Touch& t = ts.touch[buf][0];
        const __nv_bfloat16* src = X + (size_t)(t.tok0 + row0) * stride + (size_t)h * d_in + chunk * 8;
        uint32_t dst = base + raw + row_chunk(row0, chunk);                // a multiple of eight rows on: the same place in its group of eight
        for (int row = row0; row < t.m; row += kThreads / 16, src += (kThreads / 16) * stride, dst += (kThreads / 16) * kRowBytes) cp_async16(dst, src);
      } else {
        for (int slot = row0; slot < slots; slot += kThreads / 16) {
          const Touch& t = ts.touch[buf][slot >> lg];
          const int row = slot & (cap - 1);
          if (row < t.m) cp_async16(base + raw + row_chunk(slot, chunk), X + (size_t)(t.tok0 + row) * stride + (size_t)h * d_in + chunk * 8);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  // ---- the basis as B fragments: tile t = warp + 4 i, k-step ks: rows 16 ks + 2 tid4, + 1 (and + 8, + 9) of column 8 t + gid
  uint32_t uf[NT][8][2];
  find_touches(part, 0);
  if (U) {
    const int rowb = R * 2;
    for (int i = tid; i < kD * R / 8; i += kThreads) reinterpret_cast<uint4*>(smem)[i] = __ldg(reinterpret_cast<const uint4*>(U) + i);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int t = min(warp + kWarps * i, R / 8 - 1);                          // a warp without a tile repeats the last (its results are not used)
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        ldsm_x4_t(base + (32 * kk + lane) * rowb + t * 16, uf[i][2 * kk][0], uf[i][2 * kk][1], uf[i][2 * kk + 1][0], uf[i][2 * kk + 1][1]);
    }
  }
  __syncthreads();
  fetch(0, raw_at(0));

  int n = 0, buf = 0;
  for (int tile = part; tile < tiles; tile += per_slot, ++n) {
    const Touch* touch = ts.touch[buf];
    const int next = buf == 2 ? 0 : buf + 1;
    find_touches(tile + per_slot, next);                                   // past the last tile: touches without rows
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    const int raw = raw_at(n);
    const int operand = n_terms > 1 ? term0 : raw;

    // ---- which rows are real (values too: a token outside the table is not stored at all)
    auto position = [&](int slot, bool& ok) {                              // of the token in a slot
      const Touch& t = touch[slot >> lg];
      const int row = slot & (cap - 1);
      ok = slot < slots && row < t.m;
      if (!ok || !a.rot) return 0;
      const int pos = a.positions ? a.positions[t.tok0 + row] : t.place0 + row;
      ok = pos >= 0 && pos < a.max_pos;
      return pos;
    };
    bool missing = false;                                                  // a row of a page that is not to be stored
    if (tid < kPage) {
      bool ok;
      position(tid, ok);
      ts.row_ok[tid] = ok;
      missing = !ok && tid < slots && (tid & (cap - 1)) < touch[tid >> lg].m;
      if (missing) report(a.status, STIEF_ERR_BOUNDS);
    }
    // ---- rotation: raw rows -> terms; an eighth of a row at a time
    if (rot) {
      const int j = tid & 7;
      const Eighth e = eighth_of(j, rot, a.interleaved);
#pragma unroll kRotateUnroll
      for (int i = 0; i < kPage * 8 / kThreads; ++i) {
        const int slot = (tid >> 3) + i * (kThreads / 8);
        bool ok;
        const int pos = position(slot, ok);
        if (ok) {
          float cs[8], sn[8];
          if (e.turned) load_angles(a, pos, j, cs, sn);
          float x[8], y[8];
          uint4 *p0 = reinterpret_cast<uint4*>(smem + raw + row_chunk(slot, e.c0)), *p1 = reinterpret_cast<uint4*>(smem + raw + row_chunk(slot, e.c1));
          unpack8(*p0, x);
          unpack8(*p1, y);
          if (e.turned) turn_eighth(x, y, cs, sn, a.interleaved);
          if (n_terms == 1) {                                              // no basis: in place
            *p0 = pack8(x);
            *p1 = pack8(y);
          } else {
            uint8_t *d0 = smem + term0 + row_chunk(slot, e.c0), *d1 = smem + term0 + row_chunk(slot, e.c1);
#pragma unroll
            for (int term = 0; term < (F8 ? 3 : 2); ++term) {
              const uint4 r0 = pack8(x), r1 = pack8(y);
              *reinterpret_cast<uint4*>(d0 + term * kTermBytes) = r0;
              *reinterpret_cast<uint4*>(d1 + term * kTermBytes) = r1;
              float p[8];
              unpack8(r0, p);
#pragma unroll
              for (int c = 0; c < 8; ++c) x[c] -= p[c];
              unpack8(r1, p);
#pragma unroll
              for (int c = 0; c < 8; ++c) y[c] -= p[c];
            }
          }
        }
      }
    }
    // one page, all of its rows: the common case of prompts (a page outside the pool has no rows, and nothing of it is addressed)
    const bool whole = single && !__syncthreads_or(missing || touch[0].m == 0);
    if (!single) __syncthreads();
    fetch(next, raw_at(n + 1));

    // ---- products, the smallest term first
    float acc[kPage / 16][NT][4];
    const int rows = group == 1 ? touch[0].m : slots;                      // slots behind hold nothing
#pragma unroll
    for (int mt = 0; mt < kPage / 16; ++mt)
#pragma unroll
      for (int i = 0; i < NT; ++i) acc[mt][i][0] = acc[mt][i][1] = acc[mt][i][2] = acc[mt][i][3] = 0.f;
    // row tiles side by side, so that their chains overlap: all four, or the first alone (a decode batch)
    auto products = [&](auto tiles_tag, uint32_t from) {
      constexpr int MT = decltype(tiles_tag)::value;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        uint32_t af[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) ldsm_x4(from + row_chunk(16 * mt + (lane & 15), 2 * ks + (lane >> 4)), af[mt][0], af[mt][1], af[mt][2], af[mt][3]);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < NT; ++i) mma_bf16(acc[mt][i], af[mt], uf[i][ks][0], uf[i][ks][1]);
      }
    };
#pragma unroll 1
    for (int term = n_terms - 1; term >= 0; --term) {
      if (U) {
        const uint32_t from = base + operand + term * kTermBytes;
        if (rows > 16) products(std::integral_constant<int, kPage / 16>{}, from);
        else products(std::integral_constant<int, 1>{}, from);
      } else {                                                             // no basis: the rows themselves
#pragma unroll
        for (int mt = 0; mt < kPage / 16; ++mt)
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            const int t = warp + kWarps * i;
            if (mt * 16 >= rows || t >= R / 8) continue;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t w = *reinterpret_cast<const uint32_t*>(smem + operand + term * kTermBytes + row_chunk(16 * mt + gid + 8 * e, t) + 4 * tid4);
              acc[mt][i][2 * e] += bf16_lo(w);
              acc[mt][i][2 * e + 1] += bf16_hi(w);
            }
          }
      }
    }

    // ---- scales of the pages
    bool odd = false;                                                      // NaN or infinities among this thread's values
    float whole_inverse = 1.f;
    if constexpr (F8) {
      float row_top[kPage / 16][2], most = 0.f;
      const int last = single ? touch[0].m : kPage;
#pragma unroll
      for (int mt = 0; mt < kPage / 16; ++mt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = 0.f, sum = 0.f;
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            if (warp + kWarps * i < R / 8) {
              const float x = acc[mt][i][2 * e], y = acc[mt][i][2 * e + 1];
              top = fmaxf(top, fmaxf(fabsf(x), fabsf(y)));
              sum += (x - x) + (y - y);                                    // NaN if one of them is not finite
            }
          }
          if (sum != 0.f) {
            odd = true;
            top = 0.f;
#pragma unroll
            for (int i = 0; i < NT; ++i)
              if (warp + kWarps * i < R / 8) {                                  // they leave the scale alone
                const float x = fabsf(acc[mt][i][2 * e]), y = fabsf(acc[mt][i][2 * e + 1]);
                top = fmaxf(top, fmaxf(x <= 3.402823466e38f ? x : 0.f, y <= 3.402823466e38f ? y : 0.f));
              }
          }
          row_top[mt][e] = top;
          if (16 * mt + gid + 8 * e < last) most = fmaxf(most, top);
        }
      // the larger of the new rows' scale and the one of the page's older rows, which move to it when it grows: a warp per page
      auto settle = [&](const Touch& t, float scale) {
        const int held = t.place0 & (kPage - 1);
        if (held > 0 && scale != t.old) {
          const float ratio = t.old / scale;
          uint4* codes = reinterpret_cast<uint4*>(pool + ((size_t)t.page * a.L.Hkv + h) * kPage * R);
          for (int i = lane; i < held * R / 16; i += 32) {
            uint4 w = codes[i];
            uint32_t* p = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float2 x = f8::e4m3x2_to_float2(p[c] & 0xffffu), y = f8::e4m3x2_to_float2(p[c] >> 16);
              p[c] = f8::pack_e4m3(x.x * ratio, x.y * ratio, y.x * ratio, y.y * ratio);
            }
            codes[i] = w;
          }
        }
        if (lane == 0) a.P.scales[((size_t)t.page * a.L.Hkv + h) * f8::kScalesPerTile + side] = scale;
      };
      if (whole) {                                                         // one exchange; every thread then knows the scale
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (lane == 0) ts.tops[0][warp] = most;
        __syncthreads();                                                   // also: every warp has read its operands
        const float4 t0 = *reinterpret_cast<const float4*>(&ts.tops[0][0]), t1 = *reinterpret_cast<const float4*>(&ts.tops[0][4]);
        most = fmaxf(fmaxf(fmaxf(t0.x, t0.y), fmaxf(t0.z, t0.w)), fmaxf(fmaxf(t1.x, t1.y), fmaxf(t1.z, t1.w)));
        const float scale = fmaxf(f8::scale_for(most), touch[0].old);
        whole_inverse = 1.f / scale;                                       // exact for a power of two
        if (warp == kWarps - 1) settle(touch[0], scale);
      } else {
#pragma unroll
        for (int mt = 0; mt < kPage / 16; ++mt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = row_top[mt][e];
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            if (tid4 == 0) ts.tops[warp][16 * mt + gid + 8 * e] = top;
          }
        __syncthreads();                                                   // also: every warp has read its operands
        if (tid < kPage) {                                                 // thread = row slot; a page without a real row ends below zero
          float top = ts.row_ok[tid] ? 0.f : -1.f;
          for (int w = 0; w < kWarps; ++w) top = ts.row_ok[tid] ? fmaxf(top, ts.tops[w][tid]) : top;
          for (int o = 1; o < cap && o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          if (cap == kPage) {
            if (lane == 0) ts.half_top[warp] = top;
          } else if ((tid & (cap - 1)) == 0) {
            ts.top[tid >> lg] = top;
          }
        }
        __syncthreads();
        for (int g = warp; g < group; g += kWarps) {
          const float top = cap == kPage ? fmaxf(ts.half_top[0], ts.half_top[1]) : ts.top[g];
          if (touch[g].m == 0 || top < 0.f) continue;
          const float scale = fmaxf(f8::scale_for(top), touch[g].old);
          if (lane == 0) ts.inverse[g] = 1.f / scale;
          settle(touch[g], scale);
        }
        __syncthreads();
      }
      if (odd) {                                                           // infinities become NaN, as which they are stored
#pragma unroll
        for (int mt = 0; mt < kPage / 16; ++mt)
#pragma unroll
          for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (!(fabsf(acc[mt][i][c]) <= 3.402823466e38f)) acc[mt][i][c] = __uint_as_float(0x7fc00000u);
      }
    } else {
      __syncthreads();
    }

    // ---- results through shared memory: rows back to back, as they lie in their page
    uint8_t* stage = smem + operand;
#pragma unroll
    for (int mt = 0; mt < kPage / 16; ++mt) {
      if (mt * 16 >= rows) break;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = 16 * mt + gid + 8 * e;
        float inv = 1.f;
        if constexpr (F8) inv = whole ? whole_inverse : ts.inverse[row >> lg];       // (of pages without rows: not used)
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          if (warp + kWarps * i < R / 8) {
            const float x = acc[mt][i][2 * e] * inv, y = acc[mt][i][2 * e + 1] * inv;
            if constexpr (F8) {
              const uint32_t w = __nv_cvt_float2_to_fp8x2(make_float2(x, y), __NV_SATFINITE, __NV_E4M3);
              *reinterpret_cast<uint16_t*>(stage + staged(row, 8 * (warp + kWarps * i) + 2 * tid4)) = (uint16_t)w;
            } else {
              *reinterpret_cast<uint32_t*>(stage + staged(row, 16 * (warp + kWarps * i) + 4 * tid4)) = pack_bf16(x, y);
            }
          }
        }
      }
    }
    __syncthreads();
    const int per_row = row_bytes / 16;
    const uint32_t recip = 65536u / per_row + 1;                           // i / per_row of i < 1024
    uint4* whole_dst = whole ? reinterpret_cast<uint4*>(pool + (((size_t)touch[0].page * a.L.Hkv + h) * kPage + (touch[0].place0 & (kPage - 1))) * row_bytes) : nullptr;
    for (int i = tid; i < rows * per_row; i += kThreads) {
      const int slot = (i * recip) >> 16, piece = i - slot * per_row;
      const uint4 w = *reinterpret_cast<const uint4*>(stage + staged(slot, piece * 16));
      if (whole) {
        whole_dst[i] = w;
      } else if (ts.row_ok[slot]) {
        const Touch& t = touch[slot >> lg];
        uint4* dst = reinterpret_cast<uint4*>(pool + (((size_t)t.page * a.L.Hkv + h) * kPage + ((t.place0 + (slot & (cap - 1))) & (kPage - 1))) * row_bytes);
        dst[piece] = w;
      }
    }
    buf = next;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <int NT, bool F8>
__global__ void __launch_bounds__(kThreads, kResident)
append_rotated_kernel(const Args a) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ TileState ts;
  launch_dependents();
  grid_dependency_wait();
  const Sequences s = sequences_at(smem + tile_bytes<F8>(), a.Bt.B);
  load_sequences(s, a);
  const int n_kv = (a.per_key + a.per_value) * a.L.Hkv;
  if ((int)blockIdx.x >= n_kv) turn_queries(a, s, blockIdx.x - n_kv, gridDim.x - n_kv);
  else append_rows<NT, F8>(a, s, smem, ts);
}

template <int NT, bool F8>
cudaError_t launch(Args a, cudaStream_t st) {
  auto kern = append_rotated_kernel<NT, F8>;
  const int smem = tile_bytes<F8>() + sequences_bytes(a.Bt.B);
  static bool configured[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!configured[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, tile_bytes<F8>() + sequences_bytes(kMaxBatch));
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  // CTAs that are resident together, in shares by the time that rows of keys, values and queries take; no more than there are
  // pages to touch
  const int resident = host::sm_count() * kResident, Hkv = a.L.Hkv;
  const long long few = a.total < a.Bt.B ? a.total : a.Bt.B;
  const long long pages = a.total / kPage + 2 * few < a.total ? a.total / kPage + 2 * few : a.total;
  // what a tile takes, by side and rank (in thousands of cycles, two CTAs on an SM): rotation and the residual terms on top of the product
  const double key = F8 ? 16 + a.L.r_k / 10.0 : 9 + a.L.r_k / 13.0, value = F8 ? 9 + a.L.r_v / 13.0 : 5 + a.L.r_v / 16.0;
  auto share = [&](double cost) {
    const long long n = (long long)(resident * (F8 ? kRowsShareF8 : kRowsShare) * cost / (key + value) / Hkv);
    return (int)(n < 1 ? 1 : n > pages ? pages : n);
  };
  a.per_key = share(key);
  a.per_value = share(value);
  const int n_kv = (a.per_key + a.per_value) * Hkv;
  long long n_q = 0;
  if (a.q) {
    n_q = ((long long)a.total + kTokQ - 1) / kTokQ * ((a.L.Hq + kHeadsQ - 1) / kHeadsQ);
    const long long left = resident - n_kv > resident / 16 ? resident - n_kv : resident / 16;      // (many heads: more CTAs than are resident)
    if (n_q > left) n_q = left;
  }
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = host::after_previous(attr, dim3((unsigned)(n_kv + n_q)), kThreads, smem, st);
  return cudaLaunchKernelEx(&cfg, kern, a);
}

template <bool F8>
cudaError_t launch_rank(const Args& a, cudaStream_t st) {
  const int r = a.L.r_k > a.L.r_v ? a.L.r_k : a.L.r_v;
  return r <= 64 ? launch<1, F8>(a, st) : launch<2, F8>(a, st);
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
