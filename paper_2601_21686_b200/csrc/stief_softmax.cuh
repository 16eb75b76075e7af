// Softmax arithmetic of the tensor-core attention kernels: packed fp32 pairs, exponentials on the FMA pipe, rounding of a
// row to bf16 pairs, and wide TMEM accesses.
#pragma once

#include "stief_tc.cuh"

namespace stief {
namespace tc {

// packed fp32 pairs (sm_100): one instruction for two lanes of arithmetic
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// 2^x for a pair of x in [-125, 16] on the FMA pipe: x = n + f with n = rint(x) (the 1.5 * 2^23 trick leaves n in the low
// mantissa bits of t), 2^f by a cubic fitted to [-0.5, 0.5] (relative error 7.5e-5, far below the bf16 rounding of
// the probabilities), 2^n by adding n to the exponent field.  For the multi-query kernel (stief_mq.cuh): the special-function pipe
// does 16 ex2 per clock and SM, which at 64 of them per score row and page is its tightest unit, and a quarter of them go here.
// The prompt and tree kernels use no share of it: they were slower with one.
__device__ __forceinline__ void exp2_pair_fma(uint64_t x2, float& e0, float& e1) {
  const uint64_t magic = pack2(12582912.f, 12582912.f), neg_magic = pack2(-12582912.f, -12582912.f);
  const uint64_t t = add2(x2, magic);
  const uint64_t n = add2(t, neg_magic);
  const uint64_t f = fma2(n, pack2(-1.f, -1.f), x2);
  uint64_t q = fma2(f, pack2(0.05517145f, 0.05517145f), pack2(0.24261084f, 0.24261084f));
  q = fma2(q, f, pack2(0.69326097f, 0.69326097f));
  q = fma2(q, f, pack2(0.99992812f, 0.99992812f));
  float t0, t1, q0, q1;
  unpack2(t, t0, t1);
  unpack2(q, q0, q1);
  e0 = __int_as_float(__float_as_int(q0) + (__float_as_int(t0) << 23));
  e1 = __int_as_float(__float_as_int(q1) + (__float_as_int(t1) << 23));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Exponents are (s - m) c for scores s and a row's reference m, as one fma(s, c, -(m c)).  That rounds m c, which does no harm as
// long as it is the rounded product that counts as the reference (below, and in the row's log-sum-exp): up to kFarScore it
// moves the exponents of a row by at most 16, all alike.  Much beyond, it would be more than an exponent holds.  But there
// neighbouring scores lie at least 256 apart, so that all but the largest weigh nothing: any factor near c will do, and with a
// power of two m c is exact.
constexpr float kFarScore = 4294967296.f;                       // 2^32
__device__ __forceinline__ float exponent_scale(float m, float c) { return fabsf(m) > kFarScore ? 0.125f : c; }
// 2^((m - M) c): what a sum with reference m counts for next to one with a larger reference, M
__device__ __forceinline__ float reference_weight(float m, float M, float c) {
  const float cM = exponent_scale(M, c);
  return fast_exp2(__fsub_rn(__fmul_rn(m, cM), __fmul_rn(M, cM)));
}

// 16 fp32 values of a row -> 8 packed bf16 words
__device__ __forceinline__ void pack16(const uint32_t (&v)[16], float scale, uint32_t (&w)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = pack_bf16(__uint_as_float(v[2 * i]) * scale, __uint_as_float(v[2 * i + 1]) * scale);
}

// 32 consecutive 32-bit columns of this thread's TMEM lane
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr)
      : "memory");
}
}  // namespace tc
}  // namespace stief
