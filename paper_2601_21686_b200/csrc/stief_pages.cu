// Page operations of the paged cache: taking pages (stief_pages_reserve), forking, reordering and freeing sequences
// (stief_pages_fork), copying pages (stief_pages_copy) and moving the accepted rows of a drafted tree to the end of the
// committed context (stief_tree_accept).  Every other entry point only READS the block table; these write it.
//
// The paging state lives on the device and nothing here needs the host: a page is free when its reference count is
// zero, and the lowest free page is always taken first, so the result does not depend on the order in which threads
// run (the only atomics add to integer reference counts).  A page that two sequences share is always full: rows are
// only ever appended behind a sequence's last row, so a shared page is never written.
#include <climits>

#include "stief_host_util.h"

namespace stief {
namespace pages {

struct TableDev {
  int B, max_pages, num_pages;
  int* block_table;
  int* seq_lens;
  int* counts;
  int* refs;
};

constexpr int kPoolsPerLaunch = 128;          // 2 KiB of kernel parameters
struct Pools {
  void* base[kPoolsPerLaunch];
  long long bytes[kPoolsPerLaunch];           // of one page
};

// Workspace of stief_pages_fork: nothing in it survives a call
struct ForkWork {
  int* rows;                                  // [B][max_pages] the new table rows of slots that change
  int* lens;                                  // [B] new lengths
  int* counts;                                // [B] new page counts, -1 = the slot does not change
  int* wants;                                 // [B] 1 = the slot needs a page of its own for its partial last page
  int* src;                                   // [B] page copies to make ...
  int* dst;
  int* n_pairs;                               // ... and how many
};

__host__ __device__ inline size_t fork_ints(long long B, long long max_pages) { return (size_t)(B * max_pages + 5 * B + 32); }

__device__ __forceinline__ ForkWork carve_fork(int* w, int B, int max_pages) {
  ForkWork f;
  f.n_pairs = w;
  f.lens = w + 32;
  f.counts = f.lens + B;
  f.wants = f.counts + B;
  f.src = f.wants + B;
  f.dst = f.src + B;
  f.rows = f.dst + B;
  return f;
}

// Exclusive prefix sum over a block of 1024 threads (32 warps); `total` is the same for all threads
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();                            // warp_sums of an earlier call have been read
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int s = warp_sums[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, s, d);
      if (lane >= d) s += y;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  total = warp_sums[31];
  return x - v + (warp ? warp_sums[warp - 1] : 0);
}

constexpr int kScanThreads = 1024;
// Calls take(rank, page) for the `want` lowest free pages (ranks 0, 1, ...); returns how many there are, up to `want`.
// One block of 1024 threads; four reference counts per thread and step.
template <typename F>
__device__ __forceinline__ int lowest_free_pages(const TableDev& t, int want, int* warp_sums, F take) {
  int found = 0;
  for (int p0 = 0; p0 < t.num_pages && found < want; p0 += 4 * kScanThreads) {
    const int p = p0 + 4 * (int)threadIdx.x;
    bool free_[4];
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      free_[i] = p + i < t.num_pages && __ldcg(t.refs + p + i) == 0;      // the atomics of this kernel went to L2
      n += free_[i];
    }
    int total, rank = found + block_scan(n, warp_sums, total);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (free_[i]) {
        if (rank < want) take(rank, p + i);
        ++rank;
      }
    found += total;
  }
  return min(found, want);
}

// ---------------------------------------------------------------------------------------------
// reserve: one block
// ---------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kScanThreads)
reserve_kernel(const TableDev t, const int* extra, int extra_all, int32_t* status) {
  __shared__ int warp_sums[32];
  __shared__ int pref[kMaxBatch + 1];
  const int b = threadIdx.x;
  int need = 0, have = 0;
  if (b < t.B) {
    have = t.counts[b];
    const int len = t.seq_lens[b], add = extra ? extra[b] : extra_all;
    if (have < 0 || have > t.max_pages || len < 0 || add < 0) {
      report(status, STIEF_ERR_BOUNDS);
    } else {
      const long long pages = ((long long)len + add + kPage - 1) / kPage;
      if (pages > t.max_pages) report(status, STIEF_ERR_BOUNDS);          // such a sequence gets nothing
      else need = max(0, (int)pages - have);
    }
  }
  int total;
  const int at = block_scan(need, warp_sums, total);
  pref[b] = at;                                                            // kMaxBatch == kScanThreads
  if (b == 0) pref[kMaxBatch] = total;
  __syncthreads();
  if (total == 0) return;
  const int got = lowest_free_pages(t, total, warp_sums, [&](int rank, int page) {
    int lo = 0, hi = t.B - 1;                                              // the last slot whose first rank is <= rank
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (pref[mid] <= rank) lo = mid;
      else hi = mid - 1;
    }
    t.block_table[(size_t)lo * t.max_pages + t.counts[lo] + rank - pref[lo]] = page;
    t.refs[page] = 1;
  });
  __syncthreads();                                                         // counts are read above, written below
  if (b < t.B && need > 0) {
    t.counts[b] = have + min(max(got - at, 0), need);
    if (got - at < need) report(status, STIEF_ERR_NO_PAGES);
  }
}

// ---------------------------------------------------------------------------------------------
// fork, in three launches (two for a small table): rows and reference counts (a block per slot), pages for the copies (one
// block), the copies and the new state.  The kernel boundaries are the two grid-wide barriers that the permutation needs.
// ---------------------------------------------------------------------------------------------
constexpr int kRowThreads = 256;

// One slot's new row, by `width` threads of number `lane`; any(x): whether x holds in one of them
template <typename Any>
__device__ __forceinline__ void fork_row(const TableDev& t, const ForkWork& f, const int* parent, int32_t* status, int b, int lane, int width, Any any) {
  auto parent_of = [&](int s) {                                            // an id outside the batch: the slot stays as it is
    const int p = parent[s];
    return p < -1 || p >= t.B ? s : p;
  };
  const int p = parent_of(b);
  if (lane == 0 && p != parent[b]) report(status, STIEF_ERR_BOUNDS);
  if (p == b) {
    if (lane == 0) {
      f.counts[b] = -1;
      f.wants[b] = 0;
    }
    return;
  }
  // the parent's pages go to ONE heir: the parent itself if it stays, else its lowest-numbered child
  int earlier = p < 0;
  if (p >= 0) {
    earlier = parent_of(p) == p;
    for (int s = lane; s < b; s += width) earlier |= parent_of(s) == p;
  }
  const bool heir = !any(earlier);
  int len = 0, have = 0, full = 0, part = 0, keep = 0;
  if (p >= 0) {
    len = t.seq_lens[p];
    have = t.counts[p];
    if (len < 0 || have < 0 || have > t.max_pages || (len + kPage - 1ll) / kPage > have) {
      if (lane == 0) report(status, STIEF_ERR_BOUNDS);                     // such a parent is taken for an empty sequence
      len = have = 0;
    }
    full = len / kPage;
    part = len % kPage > 0;
    keep = heir ? have : full;
  }
  const int* from = t.block_table + (size_t)max(p, 0) * t.max_pages;
  int* to = f.rows + (size_t)b * t.max_pages;
  for (int i = lane; i < keep; i += width) {
    const int page = from[i];
    to[i] = page;
    if (page >= 0 && page < t.num_pages) atomicAdd(&t.refs[page], 1);
    else report(status, STIEF_ERR_BOUNDS);
  }
  const int old = min(max(t.counts[b], 0), t.max_pages);
  for (int i = lane; i < old; i += width) {
    const int page = t.block_table[(size_t)b * t.max_pages + i];
    if (page >= 0 && page < t.num_pages) atomicSub(&t.refs[page], 1);
  }
  if (lane == 0) {
    const int copied = part && !heir ? from[full] : -1;
    const bool ok = copied >= 0 && copied < t.num_pages;
    if (part && !heir && !ok) report(status, STIEF_ERR_BOUNDS);
    f.lens[b] = part && !heir && !ok ? full * kPage : len;
    f.counts[b] = keep;
    f.wants[b] = ok;
    f.src[b] = copied;
  }
}

__global__ void __launch_bounds__(kRowThreads)
fork_rows_kernel(const TableDev t, const int* parent, int* work, int32_t* status) {
  launch_dependents();
  const ForkWork f = carve_fork(work, t.B, t.max_pages);
  fork_row(t, f, parent, status, blockIdx.x, threadIdx.x, kRowThreads, [](int x) { return __syncthreads_or(x); });
}

// Pages for the copies; with kRows the rows before them too, a warp per slot: one launch fewer where the table is small
template <bool kRows>
__global__ void __launch_bounds__(kScanThreads)
fork_pages_kernel(const TableDev t, const int* parent, int* work, int32_t* status) {
  __shared__ int warp_sums[32];
  __shared__ int got_page[kMaxBatch];
  launch_dependents();
  const ForkWork f = carve_fork(work, t.B, t.max_pages);
  if (!kRows) grid_dependency_wait();                                      // the rows are made by the launch before
  if (kRows) {
    for (int b = threadIdx.x >> 5; b < t.B; b += kScanThreads / 32)
      fork_row(t, f, parent, status, b, threadIdx.x & 31, 32, [](int x) { return __any_sync(0xffffffffu, x); });
    __threadfence();
    __syncthreads();
  }
  const int b = threadIdx.x;
  const int wants = b < t.B ? f.wants[b] : 0, src = wants ? f.src[b] : 0;
  int total;
  const int rank = block_scan(wants, warp_sums, total);
  int got = 0;
  if (total) got = lowest_free_pages(t, total, warp_sums, [&](int r, int page) { got_page[r] = page; });
  __syncthreads();                                                         // src[] is rewritten in compact form below
  if (wants) {
    const int n = f.counts[b];
    if (rank < got) {
      const int page = got_page[rank];
      t.refs[page] = 1;
      f.rows[(size_t)b * t.max_pages + n] = page;
      f.counts[b] = n + 1;
      f.src[rank] = src;
      f.dst[rank] = page;
    } else {                                                               // no page left: the child ends at its last full page
      report(status, STIEF_ERR_NO_PAGES);
      f.lens[b] = n * kPage;
    }
  }
  if (b == 0) f.n_pairs[0] = got;
}

constexpr int kCopyThreads = 256, kCopyChunk = kCopyThreads * 16 * 4;      // 16 KiB per block and step
// One chunk of one page, four 16-byte loads in flight per thread
__device__ __forceinline__ void copy_chunk(char* base, long long bytes, int src, int dst, long long at) {
  const char* s = base + (size_t)src * bytes;
  char* d = base + (size_t)dst * bytes;
  uint4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long o = at + ((long long)i * kCopyThreads + threadIdx.x) * 16;
    if (o < bytes) v[i] = *reinterpret_cast<const uint4*>(s + o);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long o = at + ((long long)i * kCopyThreads + threadIdx.x) * 16;
    if (o < bytes) *reinterpret_cast<uint4*>(d + o) = v[i];
  }
}

// Items (pair, pool, chunk), the chunk fastest, dealt to the blocks in turn
__device__ __forceinline__ void copy_items(const Pools& pools, int n_pools, int chunks, int num_pages, const int* src, const int* dst, int n, int32_t* status) {
  const long long per_pair = (long long)n_pools * chunks, items = per_pair * n;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int pair = (int)(it / per_pair), rest = (int)(it - pair * per_pair), pool = rest / chunks;
    const long long at = (long long)(rest - pool * chunks) * kCopyChunk;
    if (at >= pools.bytes[pool]) continue;
    const int s = src[pair], d = dst[pair];
    if (s < 0 || s >= num_pages || d < 0 || d >= num_pages) {
      if (threadIdx.x == 0) report(status, STIEF_ERR_BOUNDS);
      continue;
    }
    if (s != d) copy_chunk(static_cast<char*>(pools.base[pool]), pools.bytes[pool], s, d, at);
  }
}

__global__ void __launch_bounds__(kCopyThreads)
fork_copy_kernel(const TableDev t, const __grid_constant__ Pools pools, int n_pools, int chunks, int commit, const int* work) {
  const ForkWork f = carve_fork(const_cast<int*>(work), t.B, t.max_pages);
  grid_dependency_wait();
  if (commit)
    for (int b = blockIdx.x; b < t.B; b += gridDim.x) {
      const int n = f.counts[b];
      if (n < 0) continue;
      for (int i = threadIdx.x; i < n; i += kCopyThreads) t.block_table[(size_t)b * t.max_pages + i] = f.rows[(size_t)b * t.max_pages + i];
      if (threadIdx.x == 0) {
        t.seq_lens[b] = f.lens[b];
        t.counts[b] = n;
      }
    }
  copy_items(pools, n_pools, chunks, t.num_pages, f.src, f.dst, f.n_pairs[0], nullptr);
}

__global__ void __launch_bounds__(kCopyThreads)
copy_kernel(const __grid_constant__ Pools pools, int n_pools, int chunks, int num_pages, const int* src, const int* dst, int n, int32_t* status) {
  copy_items(pools, n_pools, chunks, num_pages, src, dst, n, status);
}

// ---------------------------------------------------------------------------------------------
// accept: row accepted[b][j] of the drafted nodes -> position seq_lens[b] + j, in every pool.  A block takes one
// (pool, KV head, sequence).  The node list is strictly increasing, so accepted[j] >= j: a batch of rows is read before
// it is written, and what it overwrites (rows below its own end) no later batch reads.
// ---------------------------------------------------------------------------------------------
constexpr int kAcceptThreads = 128;
struct RowPools {
  void* base[kPoolsPerLaunch];
  int rank[kPoolsPerLaunch];
};

__global__ void __launch_bounds__(kAcceptThreads)
accept_kernel(const __grid_constant__ RowPools pools, const BatchDev Bt, int Hkv, int num_pages, const int* accepted, int max_accept,
              const int* n_accepted, int32_t* status) {
  const int pool = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int n = n_accepted[b], len = Bt.seq_lens[b];
  const int* nodes = accepted + (size_t)b * max_accept;
  const int* bt = Bt.block_table + (size_t)b * Bt.max_pages;
  auto page_of = [&](long long pos) {
    const long long i = pos / kPage;
    const int page = pos >= 0 && pos <= INT_MAX && i < Bt.max_pages ? bt[i] : -1;     // positions are ints below
    return page >= 0 && page < num_pages ? page : -1;
  };
  int bad = n < 0 || n > max_accept || len < 0;
  if (!bad)
    for (int j = threadIdx.x; j < n; j += kAcceptThreads) {
      const int node = nodes[j];
      bad |= node < 0 || (j > 0 && nodes[j - 1] >= node);
      bad |= page_of((long long)len + node) < 0 || page_of((long long)len + j) < 0;
    }
  if (__syncthreads_or(bad)) {                                             // the same answer in every block of the sequence: it keeps its rows
    if (threadIdx.x == 0) report(status, STIEF_ERR_BOUNDS);
    return;
  }
  const int r8 = pools.rank[pool] / 8;                                     // 16-byte pieces of a row
  uint4* base = static_cast<uint4*>(pools.base[pool]);
  auto row = [&](int pos) { return base + (((size_t)page_of(pos) * Hkv + h) * kPage + pos % kPage) * r8; };
  const int total = n * r8;
  for (int e0 = 0; e0 < total; e0 += 4 * kAcceptThreads) {
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = e0 + i * kAcceptThreads + threadIdx.x;
      if (e < total) v[i] = row(len + nodes[e / r8])[e % r8];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = e0 + i * kAcceptThreads + threadIdx.x;
      if (e < total) row(len + e / r8)[e % r8] = v[i];
    }
    __syncthreads();
  }
}

__global__ void advance_by_kernel(int32_t* seq_lens, const int32_t* deltas, int B) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < B) seq_lens[i] += deltas[i];
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
int check_table(const stief_page_table* t, TableDev* d) {
  if (!t || t->B <= 0 || t->B > kMaxBatch || t->max_pages_per_seq <= 0 || t->num_pages <= 0) return STIEF_ERR_INVALID_ARG;
  if (!t->block_table || !t->seq_lens || !t->page_counts || !t->ref_counts) return STIEF_ERR_INVALID_ARG;
  if (t->num_pages > (1 << 30) || (long long)t->B * t->max_pages_per_seq > (1 << 30)) return STIEF_ERR_INVALID_ARG;   // sums of pages are ints
  d->B = t->B;
  d->max_pages = t->max_pages_per_seq;
  d->num_pages = t->num_pages;
  d->block_table = t->block_table;
  d->seq_lens = t->seq_lens;
  d->counts = t->page_counts;
  d->refs = t->ref_counts;
  return STIEF_OK;
}

int check_pools(const stief_page_pool* pools, int n) {
  if (n < 0 || (n > 0 && !pools)) return STIEF_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i)
    if (!pools[i].base || !host::aligned(pools[i].base, 16) || pools[i].page_bytes <= 0 || pools[i].page_bytes % 16) return STIEF_ERR_INVALID_ARG;
  return STIEF_OK;
}

// Fills `out` with pools [first, first + n); returns the chunks of the largest page
int take_pools(const stief_page_pool* pools, int first, int n, Pools* out) {
  long long most = 0;
  for (int i = 0; i < n; ++i) {
    out->base[i] = pools[first + i].base;
    out->bytes[i] = pools[first + i].page_bytes;
    if (out->bytes[i] > most) most = out->bytes[i];
  }
  return (int)((most + kCopyChunk - 1) / kCopyChunk);
}

// Up to so many table entries one block finds the new rows as fast as a block per slot does, and a launch is saved (48 entries:
// 8.1 -> 6.5 us for the whole call; 1088 entries: 26.7 -> 30.6 us)
constexpr int kFewEntries = 256;

// A pool that is listed twice (layers that share a cache) would have its rows moved twice.  An insertion into a table of
// addresses while it is small (32 layers: 0.3 us), comparisons of all pairs beyond.
bool pools_differ(const stief_layer* layers, int n) {
  constexpr unsigned kSlots = 1024;
  const void* seen[kSlots] = {};
  auto pool = [&](int i) { return (const void*)(i & 1 ? layers[i >> 1].v_pool : layers[i >> 1].k_pool); };
  if (n > (int)kSlots / 4) {
    for (int i = 0; i < 2 * n; ++i)
      for (int j = 0; j < i; ++j)
        if (pool(i) == pool(j)) return false;
    return true;
  }
  for (int i = 0; i < 2 * n; ++i) {
    unsigned at = (unsigned)((reinterpret_cast<uintptr_t>(pool(i)) >> 7) * 0x9E3779B97F4A7C15ull >> 54);
    for (; seen[at]; at = (at + 1) % kSlots)
      if (seen[at] == pool(i)) return false;
    seen[at] = pool(i);
  }
  return true;
}

int copy_grid(long long items) {
  const long long most = (long long)host::sm_count() * 8;                  // eight blocks of 256 threads fill an SM
  return (int)(items < 1 ? 1 : items < most ? items : most);
}

}  // namespace pages
}  // namespace stief

using namespace stief;
using namespace stief::pages;

extern "C" size_t stief_pages_workspace_bytes(int32_t B, int32_t max_pages_per_seq) {
  if (B <= 0 || B > kMaxBatch || max_pages_per_seq <= 0) return 0;
  return host::align_up(fork_ints(B, max_pages_per_seq) * sizeof(int), 128);
}

extern "C" int stief_pages_reserve(const stief_page_table* table, const int32_t* extra, int32_t extra_all, int32_t* status, void* stream) {
  TableDev t;
  const int rc = check_table(table, &t);
  if (rc != STIEF_OK) return rc;
  if (!extra && extra_all < 0) return STIEF_ERR_INVALID_ARG;
  reserve_kernel<<<1, kScanThreads, 0, static_cast<cudaStream_t>(stream)>>>(t, extra, extra_all, status);
  return cudaGetLastError() == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}

extern "C" int stief_pages_fork(const stief_page_table* table, const stief_page_pool* pools_host, int32_t n_pools, const int32_t* parent,
                                void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
  TableDev t;
  int rc = check_table(table, &t);
  if (rc == STIEF_OK) rc = check_pools(pools_host, n_pools);
  if (rc != STIEF_OK) return rc;
  if (!parent || !workspace || !host::aligned(workspace, 128)) return STIEF_ERR_INVALID_ARG;
  if (workspace_bytes < stief_pages_workspace_bytes(t.B, t.max_pages)) return STIEF_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int* work = static_cast<int*>(workspace);
  cudaLaunchAttribute attr[1];                                             // each launch starts while the one before it ends
  if ((long long)t.B * t.max_pages <= kFewEntries) {
    fork_pages_kernel<true><<<1, kScanThreads, 0, st>>>(t, parent, work, status);
  } else {
    fork_rows_kernel<<<t.B, kRowThreads, 0, st>>>(t, parent, work, status);
    const cudaLaunchConfig_t cfg = host::after_previous(attr, dim3(1), kScanThreads, 0, st);
    if (cudaLaunchKernelEx(&cfg, fork_pages_kernel<false>, t, parent, work, status) != cudaSuccess) return STIEF_ERR_CUDA;
  }
  int first = 0;
  do {
    Pools p;
    const int n = n_pools - first < kPoolsPerLaunch ? n_pools - first : kPoolsPerLaunch;
    const int chunks = take_pools(pools_host, first, n, &p);
    long long items = (long long)t.B * n * chunks;
    if (items < t.B) items = t.B;
    const cudaLaunchConfig_t cfg = host::after_previous(attr, dim3(copy_grid(items)), kCopyThreads, 0, st);
    if (cudaLaunchKernelEx(&cfg, fork_copy_kernel, t, p, n, chunks, (int)(first == 0), (const int*)work) != cudaSuccess) return STIEF_ERR_CUDA;
    first += n;
  } while (first < n_pools);
  return cudaGetLastError() == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}

extern "C" int stief_pages_copy(const stief_page_pool* pools_host, int32_t n_pools, int32_t num_pages, const int32_t* src,
                                const int32_t* dst, int32_t n, int32_t* status, void* stream) {
  const int rc = check_pools(pools_host, n_pools);
  if (rc != STIEF_OK) return rc;
  if (n_pools <= 0 || num_pages <= 0 || n < 0 || (n > 0 && (!src || !dst))) return STIEF_ERR_INVALID_ARG;
  if (n == 0) return STIEF_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  for (int first = 0; first < n_pools; first += kPoolsPerLaunch) {
    Pools p;
    const int m = n_pools - first < kPoolsPerLaunch ? n_pools - first : kPoolsPerLaunch;
    const int chunks = take_pools(pools_host, first, m, &p);
    copy_kernel<<<copy_grid((long long)n * m * chunks), kCopyThreads, 0, st>>>(p, m, chunks, num_pages, src, dst, n, status);
  }
  return cudaGetLastError() == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}

extern "C" int stief_tree_accept(const stief_layer* layers_host, int32_t n_layers, const stief_batch* batch, const int32_t* accepted,
                                 int32_t max_accept, const int32_t* n_accepted, int32_t* status, void* stream) {
  const int rc = host::check_batch(batch);
  if (rc != STIEF_OK) return rc;
  if (!layers_host || n_layers <= 0 || !accepted || !n_accepted || max_accept <= 0) return STIEF_ERR_INVALID_ARG;
  const int Hkv = layers_host[0].Hkv, num_pages = layers_host[0].num_pages;
  if (Hkv <= 0 || Hkv > 65535 || num_pages <= 0) return STIEF_ERR_INVALID_ARG;
  for (int i = 0; i < n_layers; ++i) {
    const stief_layer& l = layers_host[i];
    if (l.Hkv != Hkv || l.num_pages != num_pages || !l.k_pool || !l.v_pool || !host::aligned(l.k_pool, 128) || !host::aligned(l.v_pool, 128))
      return STIEF_ERR_INVALID_ARG;
    for (int r : {l.r_k, l.r_v})
      if (r != 32 && r != 48 && r != 64 && r != 96 && r != 128) return STIEF_ERR_UNSUPPORTED;
  }
  if (!pools_differ(layers_host, n_layers)) return STIEF_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  for (int first = 0; first < n_layers; first += kPoolsPerLaunch / 2) {
    const int n = n_layers - first < kPoolsPerLaunch / 2 ? n_layers - first : kPoolsPerLaunch / 2;
    RowPools p;
    for (int i = 0; i < n; ++i) {
      p.base[2 * i] = layers_host[first + i].k_pool;
      p.rank[2 * i] = layers_host[first + i].r_k;
      p.base[2 * i + 1] = layers_host[first + i].v_pool;
      p.rank[2 * i + 1] = layers_host[first + i].r_v;
    }
    accept_kernel<<<dim3(2 * n, Hkv, batch->B), kAcceptThreads, 0, st>>>(p, host::to_dev(batch), Hkv, num_pages, accepted, max_accept, n_accepted, status);
  }
  return cudaGetLastError() == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}

extern "C" int stief_advance_seq_lens_by(int32_t* seq_lens, const int32_t* deltas, int32_t B, void* stream) {
  if (!seq_lens || !deltas || B <= 0) return STIEF_ERR_INVALID_ARG;
  advance_by_kernel<<<(B + 127) / 128, 128, 0, static_cast<cudaStream_t>(stream)>>>(seq_lens, deltas, B);
  return cudaGetLastError() == cudaSuccess ? STIEF_OK : STIEF_ERR_CUDA;
}
