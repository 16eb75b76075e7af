// Attention over the compressed cache in 8-bit floating point: argument checks and launches of stief_f8_decode_attention and
// stief_f8_mq_attention.
#include <algorithm>

#include "stief_f8_decode.cuh"
#include "stief_f8_mq.cuh"
#include "stief_f8_rows.cuh"
#include "stief_host_util.h"

namespace stief {
namespace {

using namespace host;

bool f8_rank_ok(int r) { return r == 32 || r == 48 || r == 64 || r == 96 || r == 128; }

int check_f8layer(const stief_f8layer* l) {
  if (!l || l->Hq <= 0 || l->Hkv <= 0 || l->Hq % l->Hkv != 0 || l->num_pages <= 0) return STIEF_ERR_INVALID_ARG;
  if (l->d != kD || !f8_rank_ok(l->r_k) || !f8_rank_ok(l->r_v)) return STIEF_ERR_UNSUPPORTED;
  if (!l->k_codes || !l->v_codes || !l->scales || !aligned(l->k_codes, 128) || !aligned(l->v_codes, 128) || !aligned(l->scales, 16))
    return STIEF_ERR_INVALID_ARG;
  if ((l->U_k && !aligned(l->U_k, 128)) || (l->U_v && !aligned(l->U_v, 128)) || l->uk_head_stride < 0 || l->uv_head_stride < 0 ||
      l->uk_head_stride % 64 || l->uv_head_stride % 64)
    return STIEF_ERR_INVALID_ARG;
  if ((long long)l->num_pages * l->Hkv * 192 >= (1ll << 31)) return STIEF_ERR_INVALID_ARG;       // TMA row coordinates stay in int
  return STIEF_OK;
}

LayerDev f8layer_to_dev(const stief_f8layer* l) {
  LayerDev d;
  d.Hq = l->Hq; d.Hkv = l->Hkv; d.G = l->Hq / l->Hkv; d.r_k = l->r_k; d.r_v = l->r_v; d.num_pages = l->num_pages;
  d.U_k = reinterpret_cast<const __nv_bfloat16*>(l->U_k); d.uk_stride = l->uk_head_stride;
  d.U_v = reinterpret_cast<const __nv_bfloat16*>(l->U_v); d.uv_stride = l->uv_head_stride;
  d.k_pool = nullptr; d.v_pool = nullptr;
  return d;
}

constexpr int kMqRows = 128;

}  // namespace
}  // namespace stief

using namespace stief;

extern "C" int stief_f8_decode_attention(const stief_f8layer* layer, const stief_batch* batch, const uint16_t* q, int32_t len_add,
                                         void* workspace, size_t workspace_bytes, int32_t num_parts, uint16_t* out, float* out_lse,
                                         uint32_t flags, int32_t* status, void* stream) {
  if (flags & ~STIEF_DECODE_OVERLAP_PREVIOUS) return STIEF_ERR_INVALID_ARG;
  int rc = check_f8layer(layer);
  if (rc) return rc;
  rc = check_batch(batch);
  if (rc) return rc;
  if (!q || !aligned(q, 16) || !workspace || !aligned(workspace, 128) || !out || !aligned(out, 16)) return STIEF_ERR_INVALID_ARG;
  if (len_add < 0 || len_add > 1 || num_parts < 0 || num_parts > 65535) return STIEF_ERR_INVALID_ARG;
  const int n_cta = resolve_parts(num_parts), QT = query_tiles(layer->Hq, layer->Hkv);
  if ((long long)batch->B * (batch->max_pages_per_seq + f8::seg_pad(layer->r_k, layer->r_v)) * layer->Hkv * QT >= (1ll << 31)) return STIEF_ERR_INVALID_ARG;
  const Workspace w = carve(workspace, batch->B, layer->Hq, layer->Hkv, layer->r_v, n_cta, workspace_bytes);
  if (w.bytes > workspace_bytes) return STIEF_ERR_WORKSPACE;
  F8DecodeArgs a;
  a.L = f8layer_to_dev(layer);
  a.P = f8::Pools{layer->k_codes, layer->v_codes, layer->scales};
  a.Bt = to_dev(batch);
  a.q = reinterpret_cast<const __nv_bfloat16*>(q);
  const bool ov = (flags & STIEF_DECODE_OVERLAP_PREVIOUS) != 0 && n_cta >= sm_count();   // full grids only (see run_decode)
  const WorkspaceTurn turn = take_workspace_turn(workspace);
  a.partial_o = w.partial_o[turn.section]; a.partial_lse = w.partial_lse[turn.section]; a.counters = w.counters[turn.section];
  a.finished = w.control + turn.section;
  a.units_done = w.control + kWorkspaceSections + turn.section;
  a.epoch = turn.epoch;
  a.prev_epoch = ov ? turn.prev_epoch : 0u;
  a.out = reinterpret_cast<__nv_bfloat16*>(out);
  a.out_lse = out_lse;
  a.len_add = len_add;
  a.QT = QT;
  a.wait_first = !ov;
  a.status = status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaErrorInvalidValue;
  switch (layer->r_k) {
    case 32: e = launch_f8_decode_rk32(a, n_cta, st); break;
    case 48: e = launch_f8_decode_rk48(a, n_cta, st); break;
    case 64: e = launch_f8_decode_rk64(a, n_cta, st); break;
    case 96: e = launch_f8_decode_rk96(a, n_cta, st); break;
    case 128: e = launch_f8_decode_rk128(a, n_cta, st); break;
  }
  return e == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}

extern "C" int32_t stief_f8_mq_num_splits(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t max_pages_per_seq) {
  if (B <= 0 || n_q <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || max_pages_per_seq <= 0) return 0;
  const int G = Hq / Hkv;
  if (G > kMqRows) return 0;
  if (n_q > 65535) return 1;                                                            // calls of more rows are not split
  const int TT = kMqRows / G;
  const long long base = ((long long)n_q + 2 * TT - 1) / (2 * TT) * B * Hkv;            // units without splitting
  const long long most = std::min(32ll, std::max(1ll, (long long)max_pages_per_seq / 4));   // at least a few pages per part
  if ((long long)n_q * G <= f8rows::kMaxRows)                                           // few rows have a kernel of their own for split ranges
    return (int32_t)std::min(most, std::max(2ll, sm_count() / base));
  // Microseconds as measured, within a fifth: a round of units costs 10 and 2.25 for two pages (tiles of the same rows share a unit's
  // pages); joined parts cost 12, 0.4 per thousand rows and part and 0.3 for each part of a row.  One sequence, ranks 64/64, 1 / 2 / 4
  // parts: 512 tokens over 8192 136 / 94 / 107, 2048 over 4096 132 / 190 / -, 256 over 4096 72 / 53 / 41.  The constants are those of 64/64
  // for all ranks, and every sequence counts as long as the longest that the caller names.
  double best = 0.;
  long long s = 1;
  for (long long i = 1; i <= most; ++i) {
    const double parts = (double)(i > 1 && n_q <= TT ? 2 * i : i), rounds = (double)((base * i + sm_count() - 1) / sm_count());
    const double us = rounds * (10. + 2.25 * (max_pages_per_seq / 2 + max_pages_per_seq % 2) / parts) + (i > 1 ? 12. + (4e-4 * B * n_q * Hq + 0.3) * parts : 0.);
    if (i == 1 || us < best) {
      best = us;
      s = i;
    }
  }
  return (int32_t)s;
}

extern "C" size_t stief_f8_mq_workspace_bytes(int32_t B, int32_t n_q, int32_t Hq, int32_t r_v, int32_t num_splits) {
  return stief_mq_workspace_bytes(B, n_q, Hq, r_v, num_splits);
}

// Joins the parts of a call.  Tiles of fewer than 16 rows where those would leave SMs without work.
template <int RV>
static cudaError_t launch_combine(const mq::Args& a, cudaStream_t st) {
  const long long rows = (long long)a.n_q * a.L.G, heads = (long long)a.L.Hkv * a.Bt.B;
  int tile = f8mq::kCombineRows;
  while (tile > 4 && (rows + tile - 1) / tile * heads < 2 * sm_count()) tile /= 2;
  const long long tiles = (rows + tile - 1) / tile, most = std::max(1ll, 4ll * sm_count() / heads);     // one wave, four to an SM
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = after_previous(attr, dim3((unsigned)(tiles < most ? tiles : most), a.L.Hkv, a.Bt.B), f8mq::kCombineThreads, 0, st);
  return cudaLaunchKernelEx(&cfg, f8mq::f8_mq_combine_kernel<RV>, a, tile);
}

extern "C" int stief_f8_mq_attention(const stief_f8layer* layer, const stief_batch* batch, const uint16_t* q, int64_t q_stride_b,
                                     int64_t q_stride_t, int32_t n_q, const int32_t* q_lens, void* workspace, size_t workspace_bytes,
                                     int32_t num_splits, uint16_t* out, int64_t out_stride_b, int64_t out_stride_t, float* out_lse,
                                     uint32_t flags, int32_t* status, void* stream) {
  if (!layer || !q || !out || flags != 0u || num_splits < 1 || num_splits > 32 || n_q <= 0) return STIEF_ERR_INVALID_ARG;
  int rc = check_batch(batch);
  if (rc) return rc;
  rc = check_f8layer(layer);
  if (rc) return rc;
  if (num_splits > 1) {
    if (!workspace || !aligned(workspace, 128)) return STIEF_ERR_INVALID_ARG;
    if (workspace_bytes < stief_f8_mq_workspace_bytes(batch->B, n_q, layer->Hq, layer->r_v, num_splits) || n_q > 65535) return STIEF_ERR_WORKSPACE;
  }
  const int G = layer->Hq / layer->Hkv;
  if (G > kMqRows) return STIEF_ERR_UNSUPPORTED;
  const long long dk = layer->U_k ? kD : layer->r_k, dv = layer->U_v ? kD : layer->r_v;
  const long long q_row = layer->Hq * dk, o_row = layer->Hq * dv;
  if (q_stride_t < q_row || q_stride_b < q_row || q_stride_t % 8 || q_stride_b % 8 || out_stride_t < o_row || out_stride_b < o_row ||
      out_stride_t % 8 || out_stride_b % 8 || !aligned(q, 16) || !aligned(out, 16))
    return STIEF_ERR_INVALID_ARG;
  const int RK = layer->r_k, RV = layer->r_v, TT = kMqRows / G;
  const bool fold_k = !layer->U_k, fold_v = !layer->U_v;
  const long long n_units = ((long long)n_q + 2 * TT - 1) / (2 * TT) * batch->B * layer->Hkv * num_splits;
  if (n_q > (1 << 30) || n_units >= (1ll << 31) - 65536) return STIEF_ERR_INVALID_ARG;      // a CTA counts past the last by a grid's worth
  f8mq::Launch L = {};
  const tc::Blocks bk = tc::blocks_of(RK), bv = tc::blocks_of(RV);
  const unsigned long long nq = n_q, Hq = layer->Hq, B = batch->B;
  if (!fold_k) {
    const unsigned long long dims[4] = {(unsigned long long)kD, Hq, nq, B};
    const unsigned long long strides[3] = {kD * 2, (unsigned long long)q_stride_t * 2, (unsigned long long)q_stride_b * 2};
    const unsigned box[4] = {64u, (unsigned)G, (unsigned)TT, 1u};
    if (!encode_bf16_map(&L.tmQ, q, 4, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B)) return STIEF_ERR_CUDA;
  }
  auto basis_map = [&](CUtensorMap* tm, const void* U, long long head_stride, int R, const tc::Blocks& b) {
    const unsigned long long nh = head_stride ? (unsigned long long)layer->Hkv : 1ull;
    const unsigned long long dims[3] = {(unsigned long long)R, (unsigned long long)kD, nh};
    const unsigned long long strides[2] = {(unsigned long long)R * 2, (unsigned long long)(head_stride ? head_stride : (long long)kD * R) * 2};
    const unsigned box[3] = {(unsigned)b.bw, (unsigned)kD, 1u};
    return encode_bf16_map(tm, U, 3, dims, strides, box, b.span == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : b.span == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B);
  };
  if (!fold_k && !basis_map(&L.tmUk, layer->U_k, layer->uk_head_stride, RK, bk)) return STIEF_ERR_CUDA;
  if (!fold_v && !basis_map(&L.tmUv, layer->U_v, layer->uv_head_stride, RV, bv)) return STIEF_ERR_CUDA;
  mq::Args& a = L.a.m;
  a.L = f8layer_to_dev(layer);
  a.Bt = to_dev(batch);
  a.q_lens = q_lens;
  a.n_q = n_q;
  a.out = reinterpret_cast<__nv_bfloat16*>(out);
  a.out_stride_b = out_stride_b;
  a.out_stride_t = out_stride_t;
  a.out_lse = out_lse;
  a.status = status;
  a.n_split = num_splits;
  const bool few = num_splits > 1 && (long long)n_q * G <= f8rows::kMaxRows;       // a tensor-core tile would be mostly empty
  a.dual = (!few && num_splits > 1 && n_q <= TT) ? 1 : 0;        // the second tile would have no rows of its own
  a.n_parts = num_splits * (1 + a.dual);
  a.part_o = num_splits > 1 ? static_cast<float*>(workspace) : nullptr;
  a.part_ml = a.part_o ? a.part_o + (size_t)batch->B * n_q * layer->Hq * a.n_parts * RV : nullptr;
  a.qp_bytes = f8mq::kRows * 2 * (fold_v ? RK : (RK > RV ? RK : RV));
  L.a.P = f8::Pools{layer->k_codes, layer->v_codes, layer->scales};
  L.a.q = reinterpret_cast<const __nv_bfloat16*>(q);
  L.a.q_stride_b = q_stride_b;
  L.a.q_stride_t = q_stride_t;
  // Shared memory: as many operand stages as fit beside four slots of codes (at 128/128 four: two blocks), the rest holds codes,
  // which is what keeps the memory busy.
  const int stage = f8mq::stage_bytes(RK, RV), slot = f8mq::slot_bytes(RK, RV), room = mq::kSmemLimit - 1024 - 2 * a.qp_bytes - f8mq::kCtrlBytes;
  a.nst = (room - f8mq::kMinCodeSlots * slot) / stage;
  if (a.nst > f8mq::kMaxStages) a.nst = f8mq::kMaxStages;
  L.a.n_code = (room - a.nst * stage) / slot;
  if (L.a.n_code > f8mq::kMaxCodeSlots) L.a.n_code = f8mq::kMaxCodeSlots;
  if (a.nst < f8mq::kMinStages || L.a.n_code < f8mq::kMinCodeSlots) return STIEF_ERR_UNSUPPORTED;
  L.smem = 1024 + 2 * a.qp_bytes + f8mq::kCtrlBytes + a.nst * stage + L.a.n_code * slot;
  L.grid = (int)(n_units < sm_count() ? n_units : sm_count());
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaErrorInvalidValue;
  switch (RK) {
    case 32: e = few ? launch_f8_rows_rk32(L.a, st) : launch_f8_mq_rk32(L, st); break;
    case 48: e = few ? launch_f8_rows_rk48(L.a, st) : launch_f8_mq_rk48(L, st); break;
    case 64: e = few ? launch_f8_rows_rk64(L.a, st) : launch_f8_mq_rk64(L, st); break;
    case 96: e = few ? launch_f8_rows_rk96(L.a, st) : launch_f8_mq_rk96(L, st); break;
    case 128: e = few ? launch_f8_rows_rk128(L.a, st) : launch_f8_mq_rk128(L, st); break;
  }
  if (e == cudaSuccess && num_splits > 1) {
    switch (RV) {
      case 32: e = launch_combine<32>(a, st); break;
      case 48: e = launch_combine<48>(a, st); break;
      case 64: e = launch_combine<64>(a, st); break;
      case 96: e = launch_combine<96>(a, st); break;
      case 128: e = launch_combine<128>(a, st); break;
    }
  }
  return e == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}
