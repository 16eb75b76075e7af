// stief_tree_attention: the projection of the queries and the joining of the partial results (the kernel between them
// is in stief_tree.cuh), argument checks, tensor maps and launches.
#include "stief_tree.cuh"

namespace stief {
namespace tree {

constexpr int kSmallThreads = 128, kSmallRows = 16;

// ---------------------------------------------------------------------------------------------
// project_kernel: q' = q U_k for 16 rows (node, head of the group) of one (sequence, KV head), by mma.sync (16 rows are too few
// for a tcgen05 tile).  Its time is the latency of its loads, so all of them are issued before the first is used.
// ---------------------------------------------------------------------------------------------
template <int RK>
__global__ void __launch_bounds__(kSmallThreads) project_kernel(const Args a) {
  constexpr int kQRow = kD + 8, kURow = RK + 8;                 // padded rows: ldmatrix without bank conflicts
  __shared__ __align__(16) __nv_bfloat16 xq[kSmallRows * kQRow];
  __shared__ __align__(16) __nv_bfloat16 xu[kD * kURow];
  launch_dependents();
  const int h = blockIdx.y, b = blockIdx.z, G = a.L.G, rows = a.n_q * G, r0 = blockIdx.x * kSmallRows;
  const int n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.n_q) : a.n_q;
  const bool fold = a.L.U_k == nullptr;
  const int dq = fold ? RK : kD;
  const int live = min(kSmallRows, n * G - r0);
  __nv_bfloat16* dst = a.qp + (((size_t)b * a.L.Hkv + h) * rows + r0) * RK;
  __nv_bfloat16* rem = dst + (size_t)a.Bt.B * a.L.Hkv * rows * RK;
  auto src = [&](int r) {
    const int node = (r0 + r) / G, g = r0 + r - node * G;
    return reinterpret_cast<const uint4*>(a.q + (size_t)b * a.q_stride_b + (size_t)node * a.q_stride_t + (size_t)(h * G + g) * dq);
  };
  if (fold) {                                                   // the queries arrive projected: rows are only packed
    for (int e = threadIdx.x; e < live * (RK / 8); e += kSmallThreads) reinterpret_cast<uint4*>(dst)[e] = src(e / (RK / 8))[e % (RK / 8)];
    return;
  }
  constexpr int kULoads = kD * (RK / 8) / kSmallThreads;
  uint4 u[kULoads], q[2];
  const uint4* U = reinterpret_cast<const uint4*>(a.L.U_k + (size_t)h * a.L.uk_stride);
#pragma unroll
  for (int i = 0; i < kULoads; ++i) u[i] = U[i * kSmallThreads + threadIdx.x];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = i * kSmallThreads + threadIdx.x;
    q[i] = e / 16 < live ? src(e / 16)[e % 16] : make_uint4(0u, 0u, 0u, 0u);
  }
  if (live <= 0) return;
#pragma unroll
  for (int i = 0; i < kULoads; ++i) {
    const int e = i * kSmallThreads + threadIdx.x;
    *reinterpret_cast<uint4*>(xu + e / (RK / 8) * kURow + e % (RK / 8) * 8) = u[i];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = i * kSmallThreads + threadIdx.x;
    *reinterpret_cast<uint4*>(xq + e / 16 * kQRow + e % 16 * 8) = q[i];
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int p = warp; p < RK / 16; p += kSmallThreads / 32) {    // 16 columns at a time
    float acc[2][4] = {};
#pragma unroll
    for (int k = 0; k < kD; k += 16) {
      uint32_t A[4], b0, b1, b2, b3;
      ldsm_x4(smem_u32(xq + (lane & 15) * kQRow + k + (lane >> 4) * 8), A[0], A[1], A[2], A[3]);
      ldsm_x4_t(smem_u32(xu + (k + (lane & 15)) * kURow + p * 16 + (lane >> 4) * 8), b0, b1, b2, b3);
      mma_bf16(acc[0], A, b0, b1);
      mma_bf16(acc[1], A, b2, b3);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = (lane >> 2) + 8 * i;
        uint32_t v, x;
        split_bf16(acc[t][2 * i], acc[t][2 * i + 1], v, x);
        if (r < live) {
          *reinterpret_cast<uint32_t*>(dst + r * RK + p * 16 + t * 8 + (lane & 3) * 2) = v;
          *reinterpret_cast<uint32_t*>(rem + r * RK + p * 16 + t * 8 + (lane & 3) * 2) = x;
        }
      }
  }
}

// ---------------------------------------------------------------------------------------------
// combine_kernel: 16 rows of one (sequence, KV head).  The segments of the rows' unit follow from the running costs and the CTAs'
// ranges; each left one partial result.  All its time is the latency of loads, hence the many threads for 16 rows: the
// weights of all parts are found first, then every thread sums four channels of a row over a share of the parts.  The back-projection runs on mma.sync with the joined rows as bf16 value + remainder (16
// significant bits) and U_v fetched before the wait for the kernel that makes the parts.
// ---------------------------------------------------------------------------------------------
constexpr int kPartChunk = 256;                                 // parts whose weights are held at a time

template <int RV, int kJoinThreads>
__global__ void __launch_bounds__(kJoinThreads) combine_kernel(const Args a) {
  constexpr int kWarps = kJoinThreads / 32, kTiles = 16 / kWarps;          // 8 output channels per warp and step
  constexpr int kRow = RV + 8, kGroups = kJoinThreads / kSmallRows, kItems = kSmallRows * RV / 4;
  constexpr int kSplit = kJoinThreads / kItems > 0 ? kJoinThreads / kItems : 1, kPer = (kItems + kJoinThreads - 1) / kJoinThreads;
  __shared__ __align__(16) __nv_bfloat16 hi[kSmallRows * kRow], lo[kSmallRows * kRow];
  __shared__ float weight[kPartChunk][kSmallRows];
  __shared__ int slot_of[kPartChunk];
  __shared__ float red[kJoinThreads / 32][kSmallRows];
  __shared__ float4 share[kSplit > 1 ? (kSplit - 1) * kItems : 1];
  __shared__ int start_of[kPartChunk], cost_of[2][kJoinThreads / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = blockIdx.y, b = blockIdx.z, G = a.L.G, r0 = blockIdx.x * kSmallRows;
  const bool fold = a.L.U_v == nullptr;
  uint32_t u[kTiles][RV / 16][2];                               // B fragments of this warp's output channels
  if (!fold) {
    const __nv_bfloat16* U = a.L.U_v + (size_t)h * a.L.uv_stride + (size_t)(warp * 8 + (lane >> 2)) * RV + (lane & 3) * 2;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int k = 0; k < RV / 16; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) u[t][k][i] = *reinterpret_cast<const uint32_t*>(U + t * kWarps * 8 * RV + k * 16 + i * 8);
  }
  // what the partition says, found again from the lengths while the kernel before still runs
  const Seq s = sequence(a, b);
  const int live = min(kSmallRows, s.n * G - r0);
  if (live <= 0) {                                              // a grid none of whose blocks waited could end before the kernel
    grid_dependency_wait();                                     // ahead of it, which reads lengths and counts: what follows on
    return;                                                     // the stream may write them
  }
  int before = 0, all = 0;                                      // running cost up to this sequence, and of all
  for (int i = tid; i < a.Bt.B; i += kJoinThreads) {
    const int cost = sequence_cost(a, sequence(a, i));
    all += cost;
    before += i < b ? cost : 0;
  }
  before = __reduce_add_sync(0xffffffffu, before);
  all = __reduce_add_sync(0xffffffffu, all);
  if (lane == 0) {
    cost_of[0][warp] = before;
    cost_of[1][warp] = all;
  }
  __syncthreads();
  int total = 0;
  before = 0;
#pragma unroll
  for (int i = 0; i < kJoinThreads / 32; ++i) {
    before += cost_of[0][i];
    total += cost_of[1][i];
  }
  const int unit = r0 / a.unit_rows, rows = min(s.n * G - unit * a.unit_rows, a.unit_rows), in_unit = r0 - unit * a.unit_rows;
  const bool dual = rows <= kRows;
  const int tile = dual ? 0 : in_unit / kRows, row0 = in_unit - tile * kRows;
  const int n = cta_count(a, total);
  const int first = before + (h * s.units + unit) * (s.blocks + kPad) + kPad, end = first + s.blocks;     // real blocks
  // the CTA whose range holds position p is the last one that starts at or before it
  auto owner = [&](int p) { return (int)((((long long)p + 1) * n - 1) / total); };
  const int c0 = owner(first), c1 = owner(end - 1);
  for (int i = tid; i <= c1 + 1 - c0 && i < kPartChunk; i += kJoinThreads) start_of[i] = range_start(c0 + i, n, total);
  __syncthreads();
  // Every CTA from the first to the last has a block of the unit, and so a part of tile 0 (or of the rows' own tile, when the
  // tiles hold different rows); tile 1 has one too where it had a block, else tile 0's part stands in with weight 0.
  const int parts = (dual ? 2 : 1) * (c1 - c0 + 1), slot0 = (c0 + (b * a.L.Hkv + h) * a.max_units + unit) * 2;
  auto part_slot = [&](int p, bool& there) {
    there = true;
    if (!dual) return slot0 + 2 * p + tile;
    const int i = p >> 1, lo = i + 1 < kPartChunk ? start_of[i] : range_start(c0 + i, n, total), hi = i + 1 < kPartChunk ? start_of[i + 1] : range_start(c0 + i + 1, n, total);
    there = !(p & 1) || min(end, hi) - max(first, lo) > 1;
    return slot0 + p - (there ? 0 : 1);
  };
  const int r = tid % kSmallRows, grp = tid / kSmallRows, at = row0 + min(r, live - 1);
  auto over_groups = [&](float v, auto join) {                  // over the threads that share a row
    v = join(v, __shfl_xor_sync(0xffffffffu, v, 16));
    __syncthreads();
    if (lane < kSmallRows) red[warp][lane] = v;
    __syncthreads();
#pragma unroll
    for (int i = 1; i < kJoinThreads / 32; ++i) v = join(i > 1 ? v : red[0][r], red[i][r]);
    return v;
  };
  grid_dependency_wait();
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + at;
  const float c = kLog2e * rsqrtf((float)kD);
  float M = -INFINITY;
  for (int p = grp; p < parts; p += kGroups) {
    bool there;
    M = fmaxf(M, ml[(size_t)part_slot(p, there) * kRows].x);
  }
  M = over_groups(M, [](float x, float y) { return fmaxf(x, y); });
  float den = 0.f;
  float4 num[kPer] = {};
  const int share_i = kSplit > 1 ? tid / kItems : 0;
  auto item_of = [&](int i) { return kSplit > 1 ? tid % kItems : tid + i * kJoinThreads; };       // (four channels, row), the row fastest
  for (int p0 = 0; p0 < parts; p0 += kPartChunk) {
    if (p0) __syncthreads();                                    // the weights of the chunk before have been read
    const int cnt = min(parts - p0, kPartChunk);
    for (int p = grp; p < cnt; p += kGroups) {
      bool there;
      const int slot = part_slot(p0 + p, there);
      const float2 x = ml[(size_t)slot * kRows];
      const float w = there ? reference_weight(x.x, M, c) : 0.f;
      if (r == 0) slot_of[p] = slot;
      den = fmaf(x.y, w, den);
      weight[p][r] = w;
    }
    __syncthreads();
    if (share_i < kSplit) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int item = item_of(i), ir = item % kSmallRows, c4 = item / kSmallRows;
        if (item >= kItems) continue;
        const float4* po = reinterpret_cast<const float4*>(a.part_o) + (size_t)c4 * kRows + row0 + min(ir, live - 1);
#pragma unroll 8
        for (int p = share_i; p < cnt; p += kSplit) {           // neighbouring threads, neighbouring rows
          const float w = weight[p][ir];
          const float4 o = po[(size_t)slot_of[p] * (RV / 4) * kRows];
          num[i].x = fmaf(o.x, w, num[i].x);
          num[i].y = fmaf(o.y, w, num[i].y);
          num[i].z = fmaf(o.z, w, num[i].z);
          num[i].w = fmaf(o.w, w, num[i].w);
        }
      }
    }
  }
  den = over_groups(den, [](float x, float y) { return x + y; });
  if (kSplit > 1 && share_i > 0 && share_i < kSplit) share[(share_i - 1) * kItems + item_of(0)] = num[0];
  auto where = [&](int row, int& node, int& hq) {
    node = (r0 + row) / G;
    hq = h * G + r0 + row - node * G;
  };
  if (a.out_lse && grp == 0 && r < live) {
    int node, hq;
    where(r, node, hq);
    a.out_lse[((size_t)b * a.n_q + node) * a.L.Hq + hq] = den > 0.f ? kLn2 * (__fmul_rn(M, c) + log2f(den)) : -INFINITY;
  }
  __syncthreads();
  if (share_i == 0) {
    const float inv = den > 0.f ? 1.0f / den : 0.f;             // (an item's row is r: items and threads are multiples of 16) no part of a row: zeros
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int item = item_of(i), c4 = item / kSmallRows;
      if (item >= kItems) continue;
#pragma unroll
      for (int k = 0; k + 1 < kSplit; ++k) {
        const float4 o = share[k * kItems + item];
        num[i].x += o.x;
        num[i].y += o.y;
        num[i].z += o.z;
        num[i].w += o.w;
      }
      uint32_t v[2], x[2];
      split_bf16(num[i].x * inv, num[i].y * inv, v[0], x[0]);
      split_bf16(num[i].z * inv, num[i].w * inv, v[1], x[1]);
      *reinterpret_cast<uint2*>(hi + r * kRow + c4 * 4) = make_uint2(v[0], v[1]);
      *reinterpret_cast<uint2*>(lo + r * kRow + c4 * 4) = make_uint2(x[0], x[1]);
    }
  }
  __syncthreads();
  if (fold) {
    for (int e = tid; e < live * (RV / 2); e += kJoinThreads) {
      const int row = e / (RV / 2), c = e % (RV / 2) * 2;
      const uint32_t v = *reinterpret_cast<const uint32_t*>(hi + row * kRow + c);
      int node, hq;
      where(row, node, hq);
      *reinterpret_cast<uint32_t*>(a.out + (size_t)b * a.out_stride_b + (size_t)node * a.out_stride_t + (size_t)hq * RV + c) = v;
    }
    return;
  }
  float acc[kTiles][4] = {};
#pragma unroll
  for (int k = 0; k < RV / 16; ++k) {
    uint32_t A[4], B[4];
    ldsm_x4(smem_u32(hi + (lane & 15) * kRow + k * 16 + (lane >> 4) * 8), A[0], A[1], A[2], A[3]);
    ldsm_x4(smem_u32(lo + (lane & 15) * kRow + k * 16 + (lane >> 4) * 8), B[0], B[1], B[2], B[3]);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      mma_bf16(acc[t], A, u[t][k][0], u[t][k][1]);
      mma_bf16(acc[t], B, u[t][k][0], u[t][k][1]);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (lane >> 2) + 8 * i;
    if (row >= live) continue;
    int node, hq;
    where(row, node, hq);
    __nv_bfloat16* o = a.out + (size_t)b * a.out_stride_b + (size_t)node * a.out_stride_t + (size_t)hq * kD + warp * 8 + (lane & 3) * 2;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) *reinterpret_cast<uint32_t*>(o + t * kWarps * 8) = pack_bf16(acc[t][2 * i], acc[t][2 * i + 1]);
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

// A unit's parts are as many as the CTAs that share it.  Few units (one long sequence with few heads) mean many parts, which
// 512 threads load faster (two tiles of up to 148 CTAs); many units mean many blocks, of which 128 threads let all run at once
// (16 sequences, 8 heads, 26 nodes: 20 us with 512 threads).
template <int RV>
cudaError_t launch_combine_rv(const Args& a, dim3 grid, cudaStream_t st) {
  cudaLaunchAttribute attr[1];
  const bool many = (long long)a.Bt.B * a.L.Hkv * a.max_units * 8 < a.n_cta;
  const cudaLaunchConfig_t cfg = host::after_previous(attr, grid, many ? 512 : 128, 0, st);
  return many ? cudaLaunchKernelEx(&cfg, combine_kernel<RV, 512>, a) : cudaLaunchKernelEx(&cfg, combine_kernel<RV, 128>, a);
}

cudaError_t launch_combine(const Args& a, dim3 grid, cudaStream_t st) {
  switch (a.L.r_v) {
    case 32: return launch_combine_rv<32>(a, grid, st);
    case 48: return launch_combine_rv<48>(a, grid, st);
    case 64: return launch_combine_rv<64>(a, grid, st);
    case 96: return launch_combine_rv<96>(a, grid, st);
    case 128: return launch_combine_rv<128>(a, grid, st);
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
  const unsigned long long q_rows = 2ull * batch->B * layer->Hkv * n_q * G;      // values, then remainders
  if (!rows_map(&L.tmQ, a.qp, RK, q_rows, tree::kRows, bk) || !rows_map(&L.tmQ32, a.qp, RK, q_rows, 32u, bk) ||
      !rows_map(&L.tmK, layer->k_pool, RK, pool_rows, kPage, bk) || !rows_map(&L.tmV, layer->v_pool, RV, pool_rows, kPage, bv))
    return STIEF_ERR_CUDA;
  a.q_regions = n_q * G > tree::kRows && a.unit_rows > tree::kRows ? 4 : 2;
  const int fixed = tree::kHeadBytes + tree::join_bytes(RV) + a.q_regions * tree::kRows * RK * 2, stage = tree::kBlock * (RK + RV) * 2;
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
