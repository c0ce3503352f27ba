// SiLU to within 2^-21 of the value, GELU 2^-19.7 (2^-18.8 at -13, by its power's constant), GELU_TANH 2^-20.5 around zero and 2^-16 far
// down, where its argument's roundings are that; on all bf16 and fp16 numbers 2^-22.9, 2^-20.9 and 2^-18.1.  activation.h's GELU has 2^-22
// around zero and 2^-16.4 at -13.  For results that are rounded to 16 bits (by 2^-8 and 2^-11): an epilogue of 8192 x 8192 of them takes
// 17 to 25 us by card with SiLU, 28 to 38 with GELU, 24 to 34 with GELU_TANH; activation.h's, with branches for far arguments and
// divisions good to the last place, 87, 57 and 65 on the first.
#pragma once
#include "activation.h"

namespace cct {
namespace {

// exp2(-s c) as m 2^k, m near one; `rest`: what s is short of.
struct Power {
  float m;
  int k;
};
__device__ __forceinline__ Power power(float s, float c, float rest) {
  const float k = __builtin_rintf(-s * c);
  return {__builtin_amdgcn_exp2f(__builtin_fmaf(-rest, c, __builtin_fmaf(-s, c, -k))), (int)fminf(k, 4096.f)};
}

constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596299e-8f / 1.44269504f;  // log2(e), and the part it is short of it by
// z / (1 + exp(-z)).  Beyond 2^64 the one adds nothing: the rest of the power comes last, so that nothing overflows on the way.  (Far
// down, where k has no fraction, m may be anything: the result is 0 for all of them.)
__device__ __forceinline__ float silu_near(float z) {
  const float s = fminf(z, 100.f);
  const Power e = power(s, kLog2e, s * kLog2eRest);
  const int k = min(e.k, 64);
  return __builtin_ldexpf(z * __builtin_amdgcn_rcpf(1.f + __builtin_ldexpf(e.m, k)), k - e.k);
}
// The same of its argument: at -20 it is 0 (from -9 on the factor is below fp32's normal numbers, of which z's few digits more are left).
__device__ __forceinline__ float gelu_tanh_near(float z) {
  const float v = fminf(fmaxf(z, -20.f), 20.f), s = v * __builtin_fmaf(v * v, 2.f * kTanhC * kTanhD, 2.f * kTanhC);
  const Power e = power(s, kLog2e, s * kLog2eRest);
  const int k = min(e.k, 64);
  return z * __builtin_ldexpf(__builtin_amdgcn_rcpf(1.f + __builtin_ldexpf(e.m, k)), k - e.k);
}

// z Phi(z).  With a = |z| and t = 1 / (1 + 0.31 a), Phi(-a) = exp(-a^2 / 2) t G(t), G the polynomial of degree 7 that is closest to it,
// relative, over 0 <= a <= 20 (within 1.7e-7; a least-squares fit reweighted by its own errors, to the function in 64 bits).  One of
// degree 6 is within 1.3e-6, 2^-19.4 of GELU, and takes as long.
__device__ __forceinline__ float gelu_near(float z) {
  constexpr float G[] = {0.123655595f, 0.124079123f, 0.107661881f,  0.110446729f,
                         -0.0154997231f, 0.155677781f, -0.141939357f, 0.0359180607f};
  const float a = fminf(__builtin_fabsf(z), 20.f), s = a * a;
  const Power e = power(s, 0.721347520f, __builtin_fmaf(a, a, -s));
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.31f, 1.f));
  float q = G[7];
#pragma unroll
  for (int i = 6; i >= 0; --i) q = __builtin_fmaf(q, t, G[i]);
  q = __builtin_ldexpf(q * t * e.m, e.k);
  return z * (z < 0.f ? q : 1.f - q);
}

template <int N>
__device__ __forceinline__ void activate_near(int act, float (&z)[N]) {
  if (act == CCT_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = silu_near(z[e]);
  } else if (act == CCT_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = gelu_near(z[e]);
  } else if (act == CCT_ACT_GELU_TANH) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = gelu_tanh_near(z[e]);
  } else {
    activate<false>(act, z, z);
  }
}

}  // namespace
}  // namespace cct
