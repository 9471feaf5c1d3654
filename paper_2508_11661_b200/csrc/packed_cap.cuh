// The cap of scores, c tanh(x / c), for the bf16 attention kernels; the result is in units of the exponent (times log2 e).
#pragma once

#include "packed.cuh"
#include "tc_common.cuh"

namespace samkv {
namespace tc {

// x by `in` = scale / c to y, the result by `out` = c log2(e).  Up to |y| = 1, where heads spend their time, tanh(y) = y P(y^2),
// P the polynomial of degree 5 with the least relative error on [0, 1]: 2^-20.6, with its scaled coefficients and its evaluation
// in fp32 2^-20.3, with the roundings of `in`, `out` and y 2^-20.1 (the fp32 kernels' tanhf is good to 2^-23).  It runs on the
// FMA pipe, two values an instruction; an exponential and a reciprocal would take twice the time of the softmax's own
// exponentials on the special-function pipe, and serve larger scores, in the chunks that hold some.
struct Cap {
  float2 c[6];                 // P's coefficients times out, each twice
  float in, out;               // out 0: no cap
};
inline Cap make_cap(float softcap, float scale) {
  static const float kTanh[6] = {0.9999994136f, -0.3332904230f, 0.1328143324f, -0.0516056571f, 0.0167430969f, -0.0030670534f};
  Cap cap = {};
  if (softcap > 0.f) {
    cap.in = scale / softcap;
    cap.out = softcap * kLog2e;
    for (int i = 0; i < 6; ++i) cap.c[i] = {kTanh[i] * cap.out, kTanh[i] * cap.out};
  }
  return cap;
}
__device__ __forceinline__ f2 pair_of(const float2& v) { return *reinterpret_cast<const f2*>(&v); }
__device__ __forceinline__ float cap_one(float x, const Cap& cap) {
  const float y = x * cap.in, z = y * y;
  float q = fmaf(cap.c[5].x, z, cap.c[4].x);
  q = fmaf(q, z, cap.c[3].x);
  q = fmaf(q, z, cap.c[2].x);
  q = fmaf(q, z, cap.c[1].x);
  q = fmaf(q, z, cap.c[0].x);
  const float e = fast_exp2(y * (2.f * kLog2e));                   // (infinite and 0 give the ends)
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.f));
  return z <= 1.f ? y * q : fmaf(-2.f * cap.out, r, cap.out);
}
// Whether one of the scores is outside the polynomial's range (NaN is not).
template <int kN>
__device__ __forceinline__ bool beyond(const float* x, const Cap& cap) {
  float top[4] = {0.f, 0.f, 0.f, 0.f};         // (side by side: one chain through 32 scores takes longer than their products)
#pragma unroll
  for (int i = 0; i < kN; i += 2) top[i / 2 % 4] = fmaxf(fmaxf(top[i / 2 % 4], fabsf(x[i])), fabsf(x[i + 1]));
  return !(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * cap.in <= 1.f);
}
// cap_one of scores that are not beyond the range, two at a time: the same bits.
template <int kN>
__device__ __forceinline__ void cap_pairs(float* x, const Cap& cap) {
  const f2 in2 = both(cap.in);
#pragma unroll
  for (int i = 0; i < kN; i += 2) {
    const f2 y = mul2(join2(x[i], x[i + 1]), in2), z = mul2(y, y);
    f2 q = fma2(pair_of(cap.c[5]), z, pair_of(cap.c[4]));
    q = fma2(q, z, pair_of(cap.c[3]));
    q = fma2(q, z, pair_of(cap.c[2]));
    q = fma2(q, z, pair_of(cap.c[1]));
    q = fma2(q, z, pair_of(cap.c[0]));
    const float2 r = split2(mul2(y, q));
    x[i] = r.x;
    x[i + 1] = r.y;
  }
}

}  // namespace tc
}  // namespace samkv
