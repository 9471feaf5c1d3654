// The cap of scores, c tanh(x / c), for the bf16 attention kernels; the result is in units of the exponent (times log2 e).
#pragma once

#include "packed.cuh"
#include "tc_common.cuh"

namespace samkv {
namespace tc {

// x by `in` = scale / c to y, the result by `out` = c log2(e).  Up to |y| = 1, where heads spend their
// time, tanh(y) = y P(y^2), P the polynomial of degree 5 with the least relative error on [0, 1]: 2^-20.4 with its evaluation
// in fp32.  It runs on the FMA pipe, two values an instruction; an exponential and a reciprocal would take twice the time of
// the softmax's own exponentials on the special-function pipe, and serve larger scores, in the chunks that hold some.
constexpr float kTanh0 = 0.9999994136f, kTanh1 = -0.3332904230f, kTanh2 = 0.1328143324f, kTanh3 = -0.0516056571f,
                kTanh4 = 0.0167430969f, kTanh5 = -0.0030670534f;
__device__ __forceinline__ float cap_one(float x, float in, float out) {
  const float y = x * in, z = y * y;
  float q = fmaf(kTanh5 * out, z, kTanh4 * out);
  q = fmaf(q, z, kTanh3 * out);
  q = fmaf(q, z, kTanh2 * out);
  q = fmaf(q, z, kTanh1 * out);
  q = fmaf(q, z, kTanh0 * out);
  const float e = fast_exp2(y * (2.f * kLog2e));                   // (infinite and 0 give the ends)
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.f));
  return z <= 1.f ? y * q : fmaf(-2.f * out, r, out);
}
// Whether one of the scores is outside the polynomial's range (NaN is not).
template <int kN>
__device__ __forceinline__ bool beyond(const float* x, float in) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < kN; i += 2) top = fmaxf(fmaxf(top, fabsf(x[i])), fabsf(x[i + 1]));
  return !(top * in <= 1.f);
}
// cap_one of scores that are not beyond the range, two at a time: the same bits.
template <int kN>
__device__ __forceinline__ void cap_pairs(float* x, float in, float out) {
  const f2 in2 = both(in), c0 = both(kTanh0 * out), c1 = both(kTanh1 * out), c2 = both(kTanh2 * out), c3 = both(kTanh3 * out),
           c4 = both(kTanh4 * out), c5 = both(kTanh5 * out);
#pragma unroll
  for (int i = 0; i < kN; i += 2) {
    const f2 y = mul2(join2(x[i], x[i + 1]), in2), z = mul2(y, y);
    f2 q = fma2(c5, z, c4);
    q = fma2(q, z, c3);
    q = fma2(q, z, c2);
    q = fma2(q, z, c1);
    q = fma2(q, z, c0);
    const float2 r = split2(mul2(y, q));
    x[i] = r.x;
    x[i + 1] = r.y;
  }
}

}  // namespace tc
}  // namespace samkv
