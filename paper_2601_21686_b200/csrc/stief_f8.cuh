// The compressed cache in 8-bit floating point (e4m3, one power-of-two scale for each page, KV head and side): what its
// kernels share.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "stief_common.cuh"

namespace stief {
namespace f8 {

constexpr int kLowest = -100, kHighest = 119;    // exponents of a scale: codes times scales stay within fp32's and bf16's range
// Weights and row sums of the attention kernels.  A weight is w = 2^((x - M) + (e - E)), x the score and 2^e the page's value scale.  The
// reference stays in two parts, M a score and E by the exponent of a scale: with far scores (beyond 2^24 fp32 holds not even all
// integers) a sum of both would lose e and the headroom, where x - M is exact next to the largest.  (M, E) is moved when a weight would
// exceed 2^kTopWeight, which is in the range of f16.
// The sum of a row wants 2^x, and e may differ by 219 from page to page, so the sum l has a reference of its own, N, that goes by
// scores alone: l counts 2^(x - N).  N is set to a page's largest score where that lies more than kSumGrown above it, so with pages of
// 64 rows l stays below 2^(6 + 16) a page.  A page adds its sum of weights times 2^((M - N) + (E - e)).  Where its largest weight lies below 2^kSumLow,
// they may vanish in the sum: it then takes exponentials that go by the page's own largest (in the mix, whose f16 weights end at 2^-24,
// the page is nothing), unless its scores lie kSumSeen below M, which is in the sum: even 2^25 positions are nothing to that.  So scores
// alone, however far apart, do not lead there.
constexpr float kNoSum = -3.402823466e38f;       // N before anything was seen
constexpr float kTopWeight = 15.f, kSumGrown = 16.f, kSumLow = -80.f, kSumSeen = -72.f;
__device__ __forceinline__ bool may_vanish(float beyond, float above) { return above < kSumLow && beyond > kSumSeen; }       // x - M, log2 of a weight

// e of a scale 2^e, as a float and without a conversion, which would take a turn on the pipe of the exponentials
__device__ __forceinline__ float scale_exponent(float scale) { return __uint_as_float(0x4b000000u | ((__float_as_uint(scale) >> 23) & 255u)) - 8388735.f; }
// What turns a product of normalised queries and codes into a score.  Large queries over large scales leave fp32's range: a score is
// then infinite, but that of a row of zeros stays zero.
__device__ __forceinline__ float score_factor(float row, float scale) { return fminf(row * scale, 3.402823466e38f); }

constexpr int kScalesPerTile = 4;                // floats of a (page, head): key scale, value scale, two unused (16 bytes, one bulk copy)

// The layer as the attention kernels see it: LayerDev's pool pointers are unused.
struct Pools {
  uint8_t* k_codes;      // [pages][Hkv][64][r_k]
  uint8_t* v_codes;      // [pages][Hkv][64][r_v]
  float* scales;         // [pages][Hkv][kScalesPerTile]
};

__host__ __device__ __forceinline__ float pow2(int e) {        // 2^e, e in -126 .. 127
  const uint32_t u = (uint32_t)(e + 127) << 23;
#ifdef __CUDA_ARCH__
  return __uint_as_float(u);
#else
  union { uint32_t i; float f; } x;
  x.i = u;
  return x.f;
#endif
}

// The least power of two s with top <= 448 s (448 = 1.75 * 2^8), within the range that scales have.  top is finite and >= 0.
__device__ __forceinline__ float scale_for(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);      // a mantissa above 1.75 takes the next one
  return pow2(min(max(e, kLowest), kHighest));                 // subnormal tops end at the lowest too
}

// Four values as e4m3, rounded to nearest even; NaN and infinities become NaN, values beyond the range its largest value.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  auto nan_if_inf = [](float x) { return fabsf(x) <= 3.402823466e38f ? x : __uint_as_float(0x7fc00000u); };
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(nan_if_inf(a), nan_if_inf(b)), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(nan_if_inf(c), nan_if_inf(d)), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// Two e4m3 codes (bits [0, 16) of w) as two f16: exact, NaN stays NaN
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 p;\n\tcvt.u16.u32 p, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, p;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t w) {
  const uint32_t r = e4m3x2_to_f16x2(w);
  return __half22float2(*reinterpret_cast<const __half2*>(&r));
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// four codes -> two f16 pairs
__device__ __forceinline__ void expand4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 p, q;\n\tmov.b32 {p, q}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, p;\n\tcvt.rn.f16x2.e4m3x2 %1, q;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}

}  // namespace f8
}  // namespace stief
