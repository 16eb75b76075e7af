// stief_prompt_attention: causal attention over packed prompts.
#include "stief_host_util.h"

namespace stief {
namespace prompt {

struct Args {
  int Hq, Hkv, B;
  int total;
  const int32_t* cu;
  const __nv_bfloat16 *q, *k, *v;
  long long q_stride, k_stride, v_stride, out_stride;
  __nv_bfloat16* out;
  float* out_lse;
  int32_t* status;
};

constexpr int kThreads = 128;

// One block per (token of the longest prompt, query head, sequence)
__global__ void __launch_bounds__(kThreads) prompt_attention_kernel(const Args a) {
  __shared__ float qs[kD], ps[kThreads], red[4];
  const int row = blockIdx.x, hq = blockIdx.y, tid = threadIdx.x, h = hq / (a.Hq / a.Hkv);
  int b = 0;
  for (; b < a.B; ++b) {
    const int lo = a.cu[b], hi = a.cu[b + 1];
    if (lo < 0 || hi < lo || hi > a.total) {
      if (tid == 0) report(a.status, STIEF_ERR_BOUNDS);
      continue;
    }
    if (row >= lo && row < hi) break;
  }
  if (b == a.B) return;
  const int lo = a.cu[b];
  qs[tid] = __bfloat162float(a.q[(size_t)row * a.q_stride + (size_t)hq * kD + tid]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o = 0.f;
  const float c = kLog2e * rsqrtf((float)kD);
  for (int t0 = lo; t0 <= row; t0 += kThreads) {
    const int t = t0 + tid;
    float s = -INFINITY;
    if (t <= row) {
      s = 0.f;
      for (int d = 0; d < kD; ++d) s = fmaf(qs[d], __bfloat162float(a.k[(size_t)t * a.k_stride + (size_t)h * kD + d]), s);
      s *= c;
    }
    float mx = s;
    for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    if (tid % 32 == 0) red[tid / 32] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float m_new = fmaxf(m, mx), p = exp2f(s - m_new), f = exp2f(m - m_new);
    ps[tid] = p;
    float sum = p;
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    __syncthreads();
    if (tid % 32 == 0) red[tid / 32] = sum;
    __syncthreads();
    l = l * f + red[0] + red[1] + red[2] + red[3];
    m = m_new;
    o *= f;
    for (int i = 0; i < kThreads && t0 + i <= row; ++i) o = fmaf(ps[i], __bfloat162float(a.v[(size_t)(t0 + i) * a.v_stride + (size_t)h * kD + tid]), o);
    __syncthreads();
  }
  a.out[(size_t)row * a.out_stride + (size_t)hq * kD + tid] = __float2bfloat16_rn(o / l);
  if (tid == 0 && a.out_lse) a.out_lse[(size_t)row * a.Hq + hq] = kLn2 * (m + log2f(l));
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
  prompt::Args a;
  a.Hq = Hq; a.Hkv = Hkv; a.B = B; a.total = total_tokens; a.cu = cu_seqlens;
  a.q = reinterpret_cast<const __nv_bfloat16*>(q); a.k = reinterpret_cast<const __nv_bfloat16*>(k); a.v = reinterpret_cast<const __nv_bfloat16*>(v);
  a.q_stride = q_stride_t; a.k_stride = k_stride_t; a.v_stride = v_stride_t; a.out_stride = out_stride_t;
  a.out = reinterpret_cast<__nv_bfloat16*>(out); a.out_lse = out_lse; a.status = status;
  if (Hq > 65535) return STIEF_ERR_INVALID_ARG;
  prompt::prompt_attention_kernel<<<dim3(total_tokens, Hq), prompt::kThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}
