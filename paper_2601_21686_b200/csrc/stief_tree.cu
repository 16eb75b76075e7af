// stief_tree_attention: the projection of the queries and the joining of the partial results (the kernel between them
// is in stief_tree.cuh), argument checks, tensor maps and launches.
#include "stief_tree.cuh"

namespace stief {
namespace tree {

// ---------------------------------------------------------------------------------------------
// project_kernel: q' = q U_k for 16 rows (node, head of the group) of one (sequence, KV head).  A group of r_k threads owns
// the columns for a share of the rows; a row of U_k is read by neighbouring threads, the queries are broadcast from shared
// memory.  128 r_k MACs per row, next to 2 T (r_k + r_v) of the attention.
// ---------------------------------------------------------------------------------------------
constexpr int kSmallThreads = 128, kSmallRows = 16;

template <int RK>
__global__ void __launch_bounds__(kSmallThreads) project_kernel(const Args a) {
  constexpr int kGroups = kSmallThreads / RK, kPer = kSmallRows / kGroups;
  __shared__ __align__(16) float x[kD][kSmallRows];
  launch_dependents();
  const int h = blockIdx.y, b = blockIdx.z, G = a.L.G, rows = a.n_q * G, r0 = blockIdx.x * kSmallRows;
  const int n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.n_q) : a.n_q;
  if (r0 >= n * G) return;
  const bool fold = a.L.U_k == nullptr;
  const int dq = fold ? RK : kD;
  const int live = min(kSmallRows, n * G - r0);
  __nv_bfloat16* dst = a.qp + (((size_t)b * a.L.Hkv + h) * rows + r0) * RK;
  auto src = [&](int r) {
    const int node = (r0 + r) / G, g = r0 + r - node * G;
    return a.q + (size_t)b * a.q_stride_b + (size_t)node * a.q_stride_t + (size_t)(h * G + g) * dq;
  };
  if (fold) {                                                   // the queries arrive projected: rows are only packed
    for (int e = threadIdx.x; e < live * (RK / 8); e += kSmallThreads)
      reinterpret_cast<uint4*>(dst)[e] = reinterpret_cast<const uint4*>(src(e / (RK / 8)))[e % (RK / 8)];
    return;
  }
  for (int e = threadIdx.x; e < kSmallRows * (kD / 8); e += kSmallThreads) {
    const int r = e % kSmallRows, d = e / kSmallRows * 8;
    const uint4 v = r < live ? reinterpret_cast<const uint4*>(src(r))[d / 8] : make_uint4(0u, 0u, 0u, 0u);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[d + 2 * i][r] = bf16_lo(w[i]);
      x[d + 2 * i + 1][r] = bf16_hi(w[i]);
    }
  }
  __syncthreads();
  const int grp = threadIdx.x / RK, j = threadIdx.x - grp * RK;
  if (grp >= kGroups) return;
  const __nv_bfloat16* U = a.L.U_k + (size_t)h * a.L.uk_stride + j;
  float acc[kPer] = {};
#pragma unroll 8
  for (int d = 0; d < kD; ++d) {
    const float u = __bfloat162float(U[d * RK]);
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
      const float4 q = *reinterpret_cast<const float4*>(&x[d][grp * kPer + i]);
      acc[i] = fmaf(q.x, u, acc[i]);
      acc[i + 1] = fmaf(q.y, u, acc[i + 1]);
      acc[i + 2] = fmaf(q.z, u, acc[i + 2]);
      acc[i + 3] = fmaf(q.w, u, acc[i + 3]);
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (grp * kPer + i < live) dst[(grp * kPer + i) * RK + j] = __float2bfloat16_rn(acc[i]);
}

// ---------------------------------------------------------------------------------------------
// combine_kernel: 16 rows of one (sequence, KV head).  The segments of the rows' unit follow from the running costs; each left
// one partial result per tile that had a block.
// ---------------------------------------------------------------------------------------------
template <int RV>
__global__ void __launch_bounds__(kSmallThreads) combine_kernel(const Args a) {
  __shared__ __align__(16) float od[RV][kSmallRows];
  __shared__ float lse[kSmallRows];
  grid_dependency_wait();
  const int h = blockIdx.y, b = blockIdx.z, G = a.L.G, r0 = blockIdx.x * kSmallRows;
  const Seq s = sequence(a, b);
  const int live = min(kSmallRows, s.n * G - r0);
  if (live <= 0) return;
  const int unit = r0 / kUnitRows, rows = min(s.n * G - unit * kUnitRows, kUnitRows), in_unit = r0 - unit * kUnitRows;
  const bool dual = rows <= kRows;
  const int tile = dual ? 0 : in_unit / kRows, row0 = in_unit - tile * kRows;
  const int total = a.prefix[a.Bt.B], n = cta_count(a, total);
  const int first = a.prefix[b] + (h * s.units + unit) * (s.blocks + kPad) + kPad, end = first + s.blocks;     // real blocks
  // the CTA whose range holds position p is the last one that starts at or before it
  auto owner = [&](int p) { return (int)((((long long)p + 1) * n - 1) / total); };
  const int c0 = owner(first), c1 = owner(end - 1);
  const int slot0 = (b * a.L.Hkv + h) * a.max_units + unit;
  auto blocks_of_cta = [&](int i) { return min(end, range_start(i + 1, n, total)) - max(first, range_start(i, n, total)); };
  for (int e = threadIdx.x; e < kSmallRows * (RV / 4); e += kSmallThreads) {
    const int r = e % kSmallRows, c4 = e / kSmallRows;
    if (r >= live) continue;
    const size_t at = (size_t)row0 + r;
    auto ml = [&](size_t slot) { return reinterpret_cast<const float2*>(a.part_ml)[slot * a.slot_rows + at]; };
    auto parts = [&](auto use) {
      for (int i = c0; i <= c1; ++i) {
        const int cnt = blocks_of_cta(i);
        const size_t slot = (size_t)(i + slot0) * 2;
        if (cnt <= 0) continue;
        use(slot + tile);
        if (dual && cnt > 1) use(slot + 1);
      }
    };
    float M = -INFINITY, den = 0.f;
    parts([&](size_t slot) { M = fmaxf(M, ml(slot).x); });
    float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
    parts([&](size_t slot) {
      const float2 x = ml(slot);
      const float w = fast_exp2(x.x - M);
      const float4 o = reinterpret_cast<const float4*>(a.part_o)[(slot * (RV / 4) + c4) * a.slot_rows + at];
      den = fmaf(x.y, w, den);
      num.x = fmaf(o.x, w, num.x);
      num.y = fmaf(o.y, w, num.y);
      num.z = fmaf(o.z, w, num.z);
      num.w = fmaf(o.w, w, num.w);
    });
    const float inv = den > 0.f ? 1.0f / den : 0.f;             // a row that saw nothing: zeros
    od[4 * c4][r] = num.x * inv;
    od[4 * c4 + 1][r] = num.y * inv;
    od[4 * c4 + 2][r] = num.z * inv;
    od[4 * c4 + 3][r] = num.w * inv;
    if (c4 == 0) lse[r] = den > 0.f ? kLn2 * (M + log2f(den)) : -INFINITY;
  }
  __syncthreads();
  auto where = [&](int r, int& node, int& hq) {
    node = (r0 + r) / G;
    hq = h * G + r0 + r - node * G;
  };
  if (a.out_lse && threadIdx.x < live) {
    int node, hq;
    where(threadIdx.x, node, hq);
    a.out_lse[((size_t)b * a.n_q + node) * a.L.Hq + hq] = lse[threadIdx.x];
  }
  const bool fold = a.L.U_v == nullptr;
  const int d_out = fold ? RV : kD, d = threadIdx.x;
  if (d >= d_out) return;
  float acc[kSmallRows] = {};
  if (fold) {
#pragma unroll
    for (int r = 0; r < kSmallRows; ++r) acc[r] = od[d][r];
  } else {                                                      // one output channel per thread: row d of U_v
    const uint4* U = reinterpret_cast<const uint4*>(a.L.U_v + (size_t)h * a.L.uv_stride + (size_t)d * RV);
#pragma unroll 2
    for (int c8 = 0; c8 < RV / 8; ++c8) {
      const uint4 u = U[c8];
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float uv = i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
#pragma unroll
        for (int r = 0; r < kSmallRows; r += 4) {
          const float4 o = *reinterpret_cast<const float4*>(&od[c8 * 8 + i][r]);
          acc[r] = fmaf(o.x, uv, acc[r]);
          acc[r + 1] = fmaf(o.y, uv, acc[r + 1]);
          acc[r + 2] = fmaf(o.z, uv, acc[r + 2]);
          acc[r + 3] = fmaf(o.w, uv, acc[r + 3]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kSmallRows; ++r)
    if (r < live) {
      int node, hq;
      where(r, node, hq);
      a.out[(size_t)b * a.out_stride_b + (size_t)node * a.out_stride_t + (size_t)hq * d_out + d] = __float2bfloat16_rn(acc[r]);
    }
}

cudaError_t launch_project(const Args& a, dim3 grid, cudaStream_t st) {
  switch (a.L.r_k) {
    case 32: project_kernel<32><<<grid, kSmallThreads, 0, st>>>(a); break;
    case 48: project_kernel<48><<<grid, kSmallThreads, 0, st>>>(a); break;
    case 64: project_kernel<64><<<grid, kSmallThreads, 0, st>>>(a); break;
    case 96: project_kernel<96><<<grid, kSmallThreads, 0, st>>>(a); break;
    case 128: project_kernel<128><<<grid, kSmallThreads, 0, st>>>(a); break;
    default: return cudaErrorInvalidValue;
  }
  return cudaGetLastError();
}

cudaError_t launch_combine(const Args& a, dim3 grid, cudaStream_t st) {
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = after_previous(attr, grid, kSmallThreads, 0, st);
  switch (a.L.r_v) {
    case 32: return cudaLaunchKernelEx(&cfg, combine_kernel<32>, a);
    case 48: return cudaLaunchKernelEx(&cfg, combine_kernel<48>, a);
    case 64: return cudaLaunchKernelEx(&cfg, combine_kernel<64>, a);
    case 96: return cudaLaunchKernelEx(&cfg, combine_kernel<96>, a);
    case 128: return cudaLaunchKernelEx(&cfg, combine_kernel<128>, a);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace tree
}  // namespace stief

using namespace stief;

extern "C" size_t stief_tree_workspace_bytes(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t r_v) {
  if (B <= 0 || n_q <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || r_v <= 0) return 0;
  return tree::carve(nullptr, B, n_q, Hq, Hkv, 128, r_v, nullptr);
}

extern "C" int stief_tree_attention(const stief_layer* layer, const stief_batch* batch, const uint16_t* q, int64_t q_stride_b,
                                    int64_t q_stride_t, int32_t n_q, const int32_t* n_nodes, const uint32_t* tree_mask,
                                    int32_t mask_words, void* workspace, size_t workspace_bytes, uint16_t* out, int64_t out_stride_b,
                                    int64_t out_stride_t, float* out_lse, uint32_t flags, int32_t* status, void* stream) {
  tree::Launch L;
  tree::Args& a = L.a;
  const int rc = tree::check(layer, batch, q, q_stride_b, q_stride_t, n_q, n_nodes, tree_mask, mask_words, workspace, workspace_bytes, out,
                             out_stride_b, out_stride_t, out_lse, flags, status, &a);
  if (rc != STIEF_OK) return rc;
  const int RK = layer->r_k, RV = layer->r_v, G = layer->Hq / layer->Hkv;
  const tc::Blocks bk = tc::blocks_of(RK), bv = tc::blocks_of(RV);
  auto rows_map = [](CUtensorMap* tm, const void* p, int R, unsigned long long rows, unsigned box_rows, const tc::Blocks& b) {
    const unsigned long long dims[2] = {(unsigned long long)R, rows};
    const unsigned long long strides[1] = {(unsigned long long)R * 2};
    const unsigned box[2] = {(unsigned)b.bw, box_rows};
    return encode_bf16_map(tm, p, 2, dims, strides, box,
                           b.span == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : b.span == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B);
  };
  const unsigned long long pool_rows = (unsigned long long)layer->num_pages * layer->Hkv * kPage;
  if (!rows_map(&L.tmQ, a.qp, RK, (unsigned long long)batch->B * layer->Hkv * n_q * G, tree::kRows, bk) ||
      !rows_map(&L.tmK, layer->k_pool, RK, pool_rows, kPage, bk) || !rows_map(&L.tmV, layer->v_pool, RV, pool_rows, kPage, bv))
    return STIEF_ERR_CUDA;
  const int fixed = tree::kHeadBytes + 2 * tree::kRows * RK * 2, stage = kPage * (RK + RV) * 2;
  a.nst = (tree::kSmemLimit - fixed) / stage;
  if (a.nst > tree::kMaxStages) a.nst = tree::kMaxStages;
  L.smem = fixed + a.nst * stage;
  L.grid = a.n_cta;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const dim3 small((unsigned)((n_q * G + tree::kSmallRows - 1) / tree::kSmallRows), (unsigned)layer->Hkv, (unsigned)batch->B);
  cudaError_t e = tree::launch_project(a, small, st);
  if (e == cudaSuccess) switch (RK) {
      case 32: e = launch_tree_rk32(L, st); break;
      case 48: e = launch_tree_rk48(L, st); break;
      case 64: e = launch_tree_rk64(L, st); break;
      case 96: e = launch_tree_rk96(L, st); break;
      default: e = launch_tree_rk128(L, st); break;
    }
  if (e == cudaSuccess) e = tree::launch_combine(a, small, st);
  return e == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}
