// Activations of the feed-forward operators and their derivatives, in fp32.
#pragma once
#include <type_traits>

#include "cct_internal.h"

namespace cct {
namespace {

// 1 / (1 + exp(-a)) as the product q c.  Below a = -87 it is no normal number, and from -88.7 on exp(-a) overflows, while what
// it is multiplied by keeps the products normal: far down q is exp(a + 32) (the sum is exact, and 1 + exp(a) is 1) and c is
// exp(-32), which is multiplied by last; elsewhere c is 1.  LOW: that can be.  A thread asks for all its values at once: one by
// one it cost an epilogue of 14 million SiLUs 1.6 of 34 us.
struct Logistic {
  float q, c;
};
template <bool LOW>
__device__ __forceinline__ Logistic logistic(float a) {
  const bool far = LOW && a < -64.f;
  const float e = expf(far ? a + 32.f : -a);
  return {far ? e : 1.f / (1.f + e), far ? 1.26641655e-14f : 1.f};
}
constexpr float kSiluLow = -64.f, kGeluTanhLow = -8.75f;  // the latter's logistic function is taken at -62 there
template <int N, class F>
__device__ __forceinline__ void with_low(const float (&z)[N], float low, F f) {
  float least = z[0];
#pragma unroll
  for (int e = 1; e < N; ++e) least = fminf(least, z[e]);
  if (least < low)
    f(std::true_type());
  else
    f(std::false_type());
}

constexpr float kSqrtHalf = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kTanhC = 0.79788456080286536f, kTanhD = 0.044715f;

// act(z) for several values, or act(z) u: one uniform branch for all of them
template <bool GATE, int N>
__device__ __forceinline__ void activate(int act, float (&z)[N], const float (&u)[N]) {
  auto gate = [&](float v, int e) { return GATE ? v * u[e] : v; };
  switch (act) {
    case CCT_ACT_RELU:
#pragma unroll
      for (int e = 0; e < N; ++e) z[e] = gate(z[e] < 0.f ? 0.f : z[e], e);  // NaN stays
      break;
    case CCT_ACT_SILU:
      with_low(z, kSiluLow, [&](auto low) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const Logistic s = logistic<decltype(low)::value>(z[e]);
          z[e] = gate(z[e] * s.q, e) * s.c;
        }
      });
      break;
    case CCT_ACT_GELU:  // erfc, not 1 + erf: the left tail keeps its digits
#pragma unroll
      for (int e = 0; e < N; ++e) z[e] = gate(z[e] * (0.5f * erfcf(-kSqrtHalf * z[e])), e);
      break;
    case CCT_ACT_GELU_TANH:  // (1 + tanh(a)) / 2 is the logistic function of 2 a
      with_low(z, kGeluTanhLow, [&](auto low) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const Logistic s = logistic<decltype(low)::value>(2.f * kTanhC * (z[e] + kTanhD * z[e] * z[e] * z[e]));
          z[e] = gate(z[e] * s.q, e) * s.c;
        }
      });
      break;
    default:
#pragma unroll
      for (int e = 0; e < N; ++e) z[e] = gate(z[e], e);
  }
}

// v act'(z), and w act(z) if BOTH
template <bool BOTH, int N>
__device__ __forceinline__ void activate_back(int act, const float (&z)[N], float (&v)[N], float (&w)[N]) {
  switch (act) {
    case CCT_ACT_RELU:
#pragma unroll
      for (int e = 0; e < N; ++e) {
        v[e] *= z[e] > 0.f ? 1.f : 0.f;
        if (BOTH) w[e] *= z[e] < 0.f ? 0.f : z[e];
      }
      break;
    case CCT_ACT_SILU:
      with_low(z, kSiluLow, [&](auto low) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const Logistic s = logistic<decltype(low)::value>(z[e]);
          v[e] = v[e] * (s.q * (1.f + z[e] * (1.f - s.q * s.c))) * s.c;
          if (BOTH) w[e] = w[e] * (z[e] * s.q) * s.c;
        }
      });
      break;
    case CCT_ACT_GELU:
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float phi = 0.5f * erfcf(-kSqrtHalf * z[e]);
        v[e] *= phi + z[e] * (kInvSqrt2Pi * expf(-0.5f * z[e] * z[e]));
        if (BOTH) w[e] *= z[e] * phi;
      }
      break;
    case CCT_ACT_GELU_TANH:
      with_low(z, kGeluTanhLow, [&](auto low) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float z2 = z[e] * z[e];
          const Logistic s = logistic<decltype(low)::value>(2.f * kTanhC * (z[e] + kTanhD * z[e] * z2));
          const float slope = 2.f * s.q * (1.f - s.q * s.c);  // 0 where z2 overflows: no infinity times 0
          v[e] = v[e] * (s.q + (slope == 0.f ? 0.f : z[e] * slope * (kTanhC * (1.f + 3.f * kTanhD * z2)))) * s.c;
          if (BOTH) w[e] = w[e] * (z[e] * s.q) * s.c;
        }
      });
      break;
    default:
      if (BOTH)
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] *= z[e];
  }
}

inline bool activation_known(int act) { return act >= CCT_ACT_NONE && act <= CCT_ACT_GELU_TANH; }

}  // namespace
}  // namespace cct
