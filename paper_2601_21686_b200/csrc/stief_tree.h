// Arguments of the tree attention kernels, and the checks of the entry point.
#pragma once

#include "stief_host_util.h"

namespace stief {
namespace tree {

constexpr int kMaxNodes = STIEF_TREE_MAX_NODES;
// query rows of a work unit: two tiles of 128, or one that both hold
__host__ __device__ constexpr int unit_rows_of(int r_k) { return r_k <= 64 ? 256 : 128; }
constexpr int kPad = 3;                    // start-up cost of a unit, in blocks of 128 positions

struct Args {
  LayerDev L;
  BatchDev Bt;
  const __nv_bfloat16* q;                  // [B][n_q][Hq][d_q]
  long long q_stride_b, q_stride_t;        // elements
  int n_q;
  const int32_t* n_nodes;                  // [B] or NULL = n_q
  const uint32_t* mask;                    // [B][n_q][mask_words]
  int mask_words;
  __nv_bfloat16* out;                      // [B][n_q][Hq][d_out]
  long long out_stride_b, out_stride_t;
  float* out_lse;                          // [B][n_q][Hq] or NULL
  int32_t* status;
  // planning and workspace (see carve)
  int n_cta, max_units, unit_rows;         // CTAs; units per (sequence, KV head) at most; rows of a unit
  int nst;                                 // ring stages
  int q_regions;                           // Q' regions in shared memory: value and remainder, for each tile where a unit may have over 128 rows
  __nv_bfloat16* qp;                       // [2][B][Hkv][n_q G][r_k]  projected queries and their remainders, rows (node, head of the group)
  float* part_o;                           // [(n_cta + units)][2 tiles][r_v / 4][128 lanes] float4
  float* part_ml;                          // [(n_cta + units)][2 tiles][128] float2: reference (a score), sum
};

// Workspace: a segment is found by (CTA + unit), so there are at most n_cta + units of them
inline size_t carve(void* base, int B, int n_q, int Hq, int Hkv, int r_k, int r_v, Args* a) {
  const int G = Hq / Hkv, rows = n_q * G, n_cta = host::sm_count();
  const int unit_rows = unit_rows_of(r_k), max_units = (rows + unit_rows - 1) / unit_rows;
  const size_t slots = 2 * ((size_t)n_cta + (size_t)B * Hkv * max_units);
  uint8_t* p = static_cast<uint8_t*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    uint8_t* at = p + off;
    off += host::align_up(bytes, 128);
    return at;
  };
  uint8_t* qp = take((size_t)B * Hkv * rows * r_k * 4);
  uint8_t *po = take(slots * 128 * r_v * 4), *ml = take(slots * 128 * 8);
  if (a) {
    a->n_cta = n_cta;
    a->max_units = max_units;
    a->unit_rows = unit_rows;
    a->qp = reinterpret_cast<__nv_bfloat16*>(qp);
    a->part_o = reinterpret_cast<float*>(po);
    a->part_ml = reinterpret_cast<float*>(ml);
  }
  return off;
}


inline int check(const stief_layer* l, const stief_batch* batch, const uint16_t* q, int64_t q_stride_b, int64_t q_stride_t, int32_t n_q,
                 const int32_t* n_nodes, const uint32_t* mask, int32_t mask_words, void* workspace, size_t workspace_bytes, uint16_t* out,
                 int64_t out_stride_b, int64_t out_stride_t, float* out_lse, uint32_t flags, int32_t* status, Args* a) {
  if (!l || !q || !out || !mask || flags != 0u) return STIEF_ERR_INVALID_ARG;
  const int rc = host::check_batch(batch);
  if (rc != STIEF_OK) return rc;
  if (l->Hq <= 0 || l->Hkv <= 0 || l->Hq % l->Hkv || l->num_pages <= 0 || !l->k_pool || !l->v_pool) return STIEF_ERR_INVALID_ARG;
  if (n_q <= 0 || mask_words < (n_q + 31) / 32) return STIEF_ERR_INVALID_ARG;
  auto rank_ok = [](int r) { return r == 32 || r == 48 || r == 64 || r == 96 || r == 128; };
  if (l->d != kD || !rank_ok(l->r_k) || !rank_ok(l->r_v) || n_q > kMaxNodes) return STIEF_ERR_UNSUPPORTED;
  const long long q_row = (long long)l->Hq * (l->U_k ? kD : l->r_k), o_row = (long long)l->Hq * (l->U_v ? kD : l->r_v);
  if (q_stride_t < q_row || q_stride_b < q_row || q_stride_t % 8 || q_stride_b % 8 || out_stride_t < o_row || out_stride_b < o_row ||
      out_stride_t % 8 || out_stride_b % 8)                     // sequences or tokens outermost
    return STIEF_ERR_INVALID_ARG;
  if (!host::aligned(q, 16) || !host::aligned(out, 16) || !host::aligned(l->k_pool, 128) || !host::aligned(l->v_pool, 128) ||
      (l->U_k && !host::aligned(l->U_k, 16)) || (l->U_v && !host::aligned(l->U_v, 16)) || l->uk_head_stride % 8 ||
      l->uv_head_stride % 8 || l->uk_head_stride < 0 || l->uv_head_stride < 0)
    return STIEF_ERR_INVALID_ARG;
  if ((long long)l->num_pages * l->Hkv * kPage >= (1ll << 31)) return STIEF_ERR_INVALID_ARG;   // pool rows are counted in int
  // rows of the projected queries and positions of the work axis are counted in int
  const long long rows = (long long)n_q * (l->Hq / l->Hkv), units = (long long)batch->B * l->Hkv * ((rows + 127) / 128);
  if ((long long)batch->B * l->Hkv * rows >= (1ll << 30) || units * (batch->max_pages_per_seq / 2 + 1 + kPad) >= (1ll << 31) ||
      (units + host::sm_count()) * 256 >= (1ll << 31))
    return STIEF_ERR_INVALID_ARG;
  if (!workspace || !host::aligned(workspace, 128)) return STIEF_ERR_INVALID_ARG;
  if (workspace_bytes < stief_tree_workspace_bytes(batch->B, n_q, l->Hq, l->Hkv, l->r_v)) return STIEF_ERR_WORKSPACE;
  a->L.Hq = l->Hq; a->L.Hkv = l->Hkv; a->L.G = l->Hq / l->Hkv; a->L.r_k = l->r_k; a->L.r_v = l->r_v; a->L.num_pages = l->num_pages;
  a->L.U_k = reinterpret_cast<const __nv_bfloat16*>(l->U_k); a->L.uk_stride = l->uk_head_stride;
  a->L.U_v = reinterpret_cast<const __nv_bfloat16*>(l->U_v); a->L.uv_stride = l->uv_head_stride;
  a->L.k_pool = reinterpret_cast<__nv_bfloat16*>(l->k_pool); a->L.v_pool = reinterpret_cast<__nv_bfloat16*>(l->v_pool);
  a->Bt = host::to_dev(batch);
  a->q = reinterpret_cast<const __nv_bfloat16*>(q);
  a->q_stride_b = q_stride_b; a->q_stride_t = q_stride_t;
  a->n_q = n_q;
  a->n_nodes = n_nodes;
  a->mask = mask;
  a->mask_words = mask_words;
  a->out = reinterpret_cast<__nv_bfloat16*>(out);
  a->out_stride_b = out_stride_b; a->out_stride_t = out_stride_t;
  a->out_lse = out_lse;
  a->status = status;
  carve(workspace, batch->B, n_q, l->Hq, l->Hkv, l->r_k, l->r_v, a);   // (the size asked for is the widest keys': r_k is no argument there)
  return STIEF_OK;
}

}  // namespace tree
}  // namespace stief
