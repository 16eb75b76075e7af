// Instantiations of the decode kernel, and of the one for a few query rows, over the 8-bit floating-point cache for one key
// rank (STIEF_RK, given on the command line) and every value rank.  Compiled once per key rank so the build parallelises.
#include "stief_f8_decode.cuh"
#include "stief_f8_rows.cuh"
#include "stief_host_util.h"
#include "stief_kernels.h"

#ifndef STIEF_RK
#error "compile with -DSTIEF_RK=<key rank>"
#endif

namespace stief {

// The pool as lines of 128 bytes; one box is a page tile.
template <int R>
static bool lines_map(CUtensorMap* tm, const void* pool, unsigned long long tiles) {
  const unsigned long long dims[2] = {128ull, tiles * f8::PageTile<R>::LINES}, strides[1] = {128ull};
  const unsigned box[2] = {128u, (unsigned)f8::PageTile<R>::LINES};
  return encode_u8_map(tm, pool, 2, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int RK, int RV>
static cudaError_t launch_one(const F8DecodeArgs& a, int n_cta, cudaStream_t st) {
  using C = f8::DecodeCfg8<RK, RV>;
  auto kern = f8::decode_f8_kernel<RK, RV>;
  static bool configured[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    // Every rank pair asks for the same (largest) carve-out: a kernel whose carve-out differs from its predecessor's cannot enter
    // an SM before that SM has drained, which would undo the overlap of consecutive layers.
    e = cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  const unsigned long long tiles = (unsigned long long)a.L.num_pages * a.L.Hkv;
  CUtensorMap tmK = {}, tmV = {};
  if (!f8::PageTile<RK>::BULK && !lines_map<RK>(&tmK, a.P.k_codes, tiles)) return cudaErrorInvalidValue;
  if (!f8::PageTile<RV>::BULK && !lines_map<RV>(&tmV, a.P.v_codes, tiles)) return cudaErrorInvalidValue;
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = host::after_previous(attr, dim3(n_cta), C::THREADS, C::SMEM_BYTES, st);
  return cudaLaunchKernelEx(&cfg, kern, tmK, tmV, a);
}

template <int RK, int RV>
static cudaError_t launch_rows(const f8mq::Args& a, cudaStream_t st) {
  using C = f8rows::Cfg<RK, RV>;
  auto kern = f8rows::f8_rows_kernel<RK, RV>;
  static bool configured[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!configured[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  const unsigned long long tiles = (unsigned long long)a.m.L.num_pages * a.m.L.Hkv;
  CUtensorMap tmK = {}, tmV = {};
  if (!f8::PageTile<RK>::BULK && !lines_map<RK>(&tmK, a.P.k_codes, tiles)) return cudaErrorInvalidValue;
  if (!f8::PageTile<RV>::BULK && !lines_map<RV>(&tmV, a.P.v_codes, tiles)) return cudaErrorInvalidValue;
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = host::after_previous(attr, dim3(a.m.n_split, a.m.L.Hkv, a.m.Bt.B), f8rows::kThreads, C::SMEM_BYTES, st);
  return cudaLaunchKernelEx(&cfg, kern, tmK, tmV, a);
}

#define STIEF_CAT_(a, b) a##b
#define STIEF_CAT(a, b) STIEF_CAT_(a, b)

cudaError_t STIEF_CAT(launch_f8_decode_rk, STIEF_RK)(const F8DecodeArgs& a, int n_cta, cudaStream_t st) {
  switch (a.L.r_v) {
    case 32: return launch_one<STIEF_RK, 32>(a, n_cta, st);
    case 48: return launch_one<STIEF_RK, 48>(a, n_cta, st);
    case 64: return launch_one<STIEF_RK, 64>(a, n_cta, st);
    case 96: return launch_one<STIEF_RK, 96>(a, n_cta, st);
    case 128: return launch_one<STIEF_RK, 128>(a, n_cta, st);
    default: return cudaErrorInvalidValue;
  }
}

cudaError_t STIEF_CAT(launch_f8_rows_rk, STIEF_RK)(const f8mq::Args& a, cudaStream_t st) {
  switch (a.m.L.r_v) {
    case 32: return launch_rows<STIEF_RK, 32>(a, st);
    case 48: return launch_rows<STIEF_RK, 48>(a, st);
    case 64: return launch_rows<STIEF_RK, 64>(a, st);
    case 96: return launch_rows<STIEF_RK, 96>(a, st);
    case 128: return launch_rows<STIEF_RK, 128>(a, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace stief
