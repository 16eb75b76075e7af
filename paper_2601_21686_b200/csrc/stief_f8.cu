// Attention over the compressed cache in 8-bit floating point: argument checks and launches of stief_f8_decode_attention and
// stief_f8_mq_attention.
#include "stief_f8_decode.cuh"
#include "stief_host_util.h"

namespace stief {
namespace f8 {

struct SimpleArgs {
  LayerDev L;
  Pools P;
  BatchDev Bt;
  const __nv_bfloat16* q;
  long long q_b, q_t;
  int n_q, len_add;
  const int32_t* q_lens;
  __nv_bfloat16* out;
  long long o_b, o_t;
  float* out_lse;
  int32_t* status;
};

// One block per (token, query head, sequence): a pass over the pages with the running maximum and sum of the softmax.
__global__ void __launch_bounds__(128)
f8_rows_kernel(const SimpleArgs a) {
  __shared__ float qp[kD], p[kPage], od[kD], red[4];
  const int i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int h = hq / a.L.G, RK = a.L.r_k, RV = a.L.r_v;
  int ql = a.q_lens ? a.q_lens[b] : a.n_q;
  ql = min(max(ql, 0), a.n_q);
  if (i >= ql) return;
  const int len = a.Bt.seq_lens[b] + a.len_add;
  const bool fold_k = a.L.U_k == nullptr, fold_v = a.L.U_v == nullptr;
  if ((a.q_lens || a.n_q > 1) && len < ql || (len + kPage - 1) / kPage > a.Bt.max_pages) {
    if (tid == 0) report(a.status, STIEF_ERR_BOUNDS);
    return;
  }
  const int n = max(0, len - ql + i + 1);
  const __nv_bfloat16* qr = a.q + b * a.q_b + i * a.q_t + (long long)hq * (fold_k ? RK : kD);
  if (tid < RK) {
    float x = 0.f;
    if (fold_k) x = __bfloat162float(qr[tid]);
    else
      for (int d = 0; d < kD; ++d) x = fmaf(__bfloat162float(qr[d]), __bfloat162float(a.L.U_k[(size_t)h * a.L.uk_stride + d * RK + tid]), x);
    qp[tid] = x * 0.08838834764831845f;
  }
  __syncthreads();
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int pg = 0; pg * kPage < n; ++pg) {
    int page = a.Bt.block_table[(size_t)b * a.Bt.max_pages + pg];
    if (page < 0 || page >= a.L.num_pages) {
      if (tid == 0) report(a.status, STIEF_ERR_BOUNDS);
      page = 0;
    }
    const size_t tile = (size_t)page * a.L.Hkv + h;
    const int cnt = min(kPage, n - pg * kPage);
    if (tid < kPage) {
      float s = 0.f;
      const uint8_t* k = a.P.k_codes + (tile * kPage + tid) * RK;
      for (int c = 0; c < RK; c += 2) {
        const float2 x = e4m3x2_to_float2(*reinterpret_cast<const uint16_t*>(k + c));
        s = fmaf(qp[c + 1], x.y, fmaf(qp[c], x.x, s));
      }
      p[tid] = tid < cnt ? s * a.P.scales[tile * kScalesPerTile] : -INFINITY;
    }
    __syncthreads();
    float top = m;
    for (int t = 0; t < cnt; ++t) top = fmaxf(top, p[t]);
    const float f = __expf(m - top), vs = a.P.scales[tile * kScalesPerTile + 1];
    m = top;
    l *= f;
    o *= f;
    for (int t = 0; t < cnt; ++t) {
      const float w = __expf(p[t] - m);
      l += w;
      if (tid < RV) o = fmaf(w * vs, e4m3x2_to_float2(a.P.v_codes[(tile * kPage + t) * RV + tid]).x, o);
    }
    __syncthreads();
  }
  if (tid < RV) od[tid] = l > 0.f ? o / l : 0.f;
  __syncthreads();
  const int d_out = fold_v ? RV : kD;
  if (tid < d_out) {
    float x = 0.f;
    if (fold_v) x = od[tid];
    else
      for (int c = 0; c < RV; ++c) x = fmaf(od[c], __bfloat162float(a.L.U_v[(size_t)h * a.L.uv_stride + tid * RV + c]), x);
    a.out[b * a.o_b + i * a.o_t + (long long)hq * d_out + tid] = __float2bfloat16_rn(x);
  }
  if (tid == 0 && a.out_lse) a.out_lse[((size_t)b * a.n_q + i) * a.L.Hq + hq] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace f8

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
  a.status = status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaErrorInvalidValue;
  switch (layer->r_k) {
    case 32: e = launch_f8_decode_rk32(a, n_cta, ov, st); break;
    case 48: e = launch_f8_decode_rk48(a, n_cta, ov, st); break;
    case 64: e = launch_f8_decode_rk64(a, n_cta, ov, st); break;
    case 96: e = launch_f8_decode_rk96(a, n_cta, ov, st); break;
    case 128: e = launch_f8_decode_rk128(a, n_cta, ov, st); break;
  }
  return e == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}

extern "C" int32_t stief_f8_mq_num_splits(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t max_pages_per_seq) {
  if (B <= 0 || n_q <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || max_pages_per_seq <= 0) return 0;
  const int G = Hq / Hkv;
  if (G > kMqRows) return 0;
  const int TT = kMqRows / G;
  const long long base = ((long long)n_q + 2 * TT - 1) / (2 * TT) * B * Hkv;            // units without splitting
  long long s = sm_count() / base;                                                      // parts so that the units about fill the GPU
  if (s > 32) s = 32;
  if (s > max_pages_per_seq / 4) s = max_pages_per_seq / 4;                             // at least a few pages per part
  return (int32_t)(s < 1 ? 1 : s);
}

extern "C" size_t stief_f8_mq_workspace_bytes(int32_t B, int32_t n_q, int32_t Hq, int32_t r_v, int32_t num_splits) {
  return stief_mq_workspace_bytes(B, n_q, Hq, r_v, num_splits);
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
  f8::SimpleArgs a;
  a.L = f8layer_to_dev(layer);
  a.P = f8::Pools{layer->k_codes, layer->v_codes, layer->scales};
  a.Bt = to_dev(batch);
  a.q = reinterpret_cast<const __nv_bfloat16*>(q);
  a.q_b = q_stride_b;
  a.q_t = q_stride_t;
  a.n_q = n_q;
  a.len_add = 0;
  a.q_lens = q_lens;
  a.out = reinterpret_cast<__nv_bfloat16*>(out);
  a.o_b = out_stride_b;
  a.o_t = out_stride_t;
  a.out_lse = out_lse;
  a.status = status;
  f8::f8_rows_kernel<<<dim3(n_q, layer->Hq, batch->B), 128, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}
