// stief_tree_attention: attention of a tree of drafted tokens over the compressed cache.
#include "stief_host_util.h"
#include "stief_tree.h"

namespace stief {
namespace tree {

constexpr int kThreads = 128;

// One block per (node, query head, sequence).  A thread scores one position of each run of 128 and then owns one
// channel of the mix; the running maximum and sum are block-wide.
__global__ void __launch_bounds__(kThreads) tree_attention_kernel(const Args a) {
  __shared__ float qs[kD], qp[kD], ps[kThreads], red[4], od[kD];
  const int node = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int RK = a.L.r_k, RV = a.L.r_v, h = hq / a.L.G;
  const int ctx = a.Bt.seq_lens[b];
  int n = a.n_nodes ? a.n_nodes[b] : a.n_q;
  n = min(max(n, 0), a.n_q);
  if (node >= n) return;
  if (ctx < 0 || ((long long)ctx + n + kPage - 1) / kPage > a.Bt.max_pages) {
    if (tid == 0) report(a.status, STIEF_ERR_BOUNDS);
    return;
  }
  const bool fold_k = a.L.U_k == nullptr, fold_v = a.L.U_v == nullptr;
  const int dq = fold_k ? RK : kD, d_out = fold_v ? RV : kD;
  const __nv_bfloat16* q = a.q + (size_t)b * a.q_stride_b + (size_t)node * a.q_stride_t + (size_t)hq * dq;
  if (tid < dq) qs[tid] = __bfloat162float(q[tid]);
  __syncthreads();
  if (tid < RK) {
    float s = 0.f;
    if (fold_k) s = qs[tid];
    else
      for (int d = 0; d < kD; ++d) s = fmaf(qs[d], __bfloat162float(a.L.U_k[(size_t)h * a.L.uk_stride + d * RK + tid]), s);
    qp[tid] = s;
  }
  __syncthreads();
  const uint32_t* mask = a.mask + ((size_t)b * a.n_q + node) * a.mask_words;
  float m = -INFINITY, l = 0.f, o = 0.f;
  const float c = kLog2e * rsqrtf((float)kD);
  auto row = [&](int t) -> long long {
    const int page = a.Bt.block_table[(size_t)b * a.Bt.max_pages + t / kPage];
    if (page < 0 || page >= a.L.num_pages) {
      report(a.status, STIEF_ERR_BOUNDS);
      return -1;
    }
    return ((long long)page * a.L.Hkv + h) * kPage + t % kPage;
  };
  for (int t0 = 0; t0 < ctx + n; t0 += kThreads) {
    const int t = t0 + tid;
    float s = -INFINITY;
    bool seen = t < ctx;
    if (t >= ctx && t < ctx + n) seen = (mask[(t - ctx) / 32] >> ((t - ctx) % 32)) & 1;
    if (seen) {
      const long long r = row(t);
      s = 0.f;
      if (r >= 0)
        for (int j = 0; j < RK; ++j) s = fmaf(qp[j], __bfloat162float(a.L.k_pool[r * RK + j]), s);
      s *= c;
    }
    float mx = s;
    for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    if (tid % 32 == 0) red[tid / 32] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float m_new = fmaxf(m, mx), base = m_new == -INFINITY ? 0.f : m_new;
    const float p = seen ? exp2f(s - base) : 0.f, f = exp2f(m - base);
    ps[tid] = p;
    float sum = p;
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    __syncthreads();
    if (tid % 32 == 0) red[tid / 32] = sum;
    __syncthreads();
    l = l * f + red[0] + red[1] + red[2] + red[3];
    m = m_new;
    if (tid < RV) {
      o *= f;
      for (int i = 0; i < kThreads && t0 + i < ctx + n; ++i)
        if (ps[i] != 0.f) {
          const long long r = row(t0 + i);
          if (r >= 0) o = fmaf(ps[i], __bfloat162float(a.L.v_pool[r * RV + tid]), o);
        }
    }
    __syncthreads();
  }
  if (tid < RV) od[tid] = l > 0.f ? o / l : 0.f;
  __syncthreads();
  if (tid < d_out) {
    float s = 0.f;
    if (fold_v) s = od[tid];
    else
      for (int j = 0; j < RV; ++j) s = fmaf(od[j], __bfloat162float(a.L.U_v[(size_t)h * a.L.uv_stride + tid * RV + j]), s);
    a.out[(size_t)b * a.out_stride_b + (size_t)node * a.out_stride_t + (size_t)hq * d_out + tid] = __float2bfloat16_rn(s);
  }
  if (tid == 0 && a.out_lse) a.out_lse[((size_t)b * a.n_q + node) * a.L.Hq + hq] = l > 0.f ? kLn2 * (m + log2f(l)) : -INFINITY;
}

}  // namespace tree
}  // namespace stief

using namespace stief;

extern "C" size_t stief_tree_workspace_bytes(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t r_v) {
  if (B <= 0 || n_q <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || r_v <= 0) return 0;
  return 128;
}

extern "C" int stief_tree_attention(const stief_layer* layer, const stief_batch* batch, const uint16_t* q, int64_t q_stride_b,
                                    int64_t q_stride_t, int32_t n_q, const int32_t* n_nodes, const uint32_t* tree_mask,
                                    int32_t mask_words, void* workspace, size_t workspace_bytes, uint16_t* out, int64_t out_stride_b,
                                    int64_t out_stride_t, float* out_lse, uint32_t flags, int32_t* status, void* stream) {
  tree::Args a;
  const int rc = tree::check(layer, batch, q, q_stride_b, q_stride_t, n_q, n_nodes, tree_mask, mask_words, workspace, workspace_bytes, out,
                             out_stride_b, out_stride_t, out_lse, flags, status, &a);
  if (rc != STIEF_OK) return rc;
  tree::tree_attention_kernel<<<dim3(n_q, layer->Hq, batch->B), tree::kThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}
