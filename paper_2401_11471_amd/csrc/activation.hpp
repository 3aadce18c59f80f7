// The activations and their derivatives, shared by the kernels that apply one
// (activations with 8-bit checkpoints, group norm, gated feed-forward block).
#pragma once

#include "act8.hpp"

#include <type_traits>

namespace lrcnn {
namespace act8 {

#ifdef __HIPCC__
// 1 / (1 + exp(-x)), exp(-x) = 2^(-x log2 e)
__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * x));
}
// f(u) and f'(u). An argument beyond +-100 counts as +-100 in the factors that
// are then 0 or 1 (so that an infinity takes the function's limit); NaN stays.
// LEAN: the same numbers with minimum and maximum, which drop a NaN that the other factor
// has as well: fewer instructions, for kernels that they bound. Those that memory
// bounds gain or lose by the kind and keep the first form (16000 x 4096 bf16, backward from
// checkpoints: silu 108 us, LEAN 115; tanh form 120 and 110).
// gelu: u Phi(u), Phi(-|u|) = exp(-u^2/2) R(|u|), R the Mills ratio over
// sqrt(2 pi), here t P(t) with t = 1 / (1 + 0.3 |u|) and P of degree 7 fitted
// over [0, 14] to 1.5e-7 of R (4.4e-7 as evaluated in float32). The exponential's
// argument is rounded to float32, which adds some u^2 2^-25 of the value (1.4e-6
// at -5, 8e-6 at -13); that of the other two likewise. Below -87, where 1 / (1 +
// exp(-u)) is subnormal, silu is 0. tanh form: u s(2 k (u + 0.044715 u^3)), k =
// sqrt(2 / pi).
template <int KIND, bool LEAN = false>
__device__ __forceinline__ void activate(float u, float &f, float &df) {
  if constexpr (KIND == LRCNN_ACT_NONE) {
    f = u, df = 1.f;
    return;
  }
  if constexpr (KIND == LRCNN_ACT_RELU) {
    f = u > 0.f || u != u ? u : 0.f;
    df = u > 0.f ? 1.f : u != u ? u : 0.f;
    return;
  }
  const float lo = LEAN ? fmaxf(u, -100.f) : u < -100.f ? -100.f : u;
  const float x = LEAN ? u : lo > 100.f ? 100.f : lo;
  if constexpr (KIND == LRCNN_ACT_SILU) {
    const float s = sigmoid(x);
    f = lo * s;
    const float t = LEAN ? fminf(f, 100.f) : x * s;
    df = s + t * (1.f - s);
  } else if constexpr (KIND == LRCNN_ACT_GELU) {
    const float z = fabsf(x);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, z, 1.f));
    const float e = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    float p = 0.03567478433251381f;
    p = fmaf(p, t, -0.15720312297344208f);
    p = fmaf(p, t, 0.2063535749912262f);
    p = fmaf(p, t, -0.053683701902627945f);
    p = fmaf(p, t, 0.12856166064739227f);
    p = fmaf(p, t, 0.09991348534822464f);
    p = fmaf(p, t, 0.12075395882129669f);
    p = fmaf(p, t, 0.11962930113077164f);
    const float q = e * (t * p);
    const float phi = x < 0.f ? q : 1.f - q;
    f = lo * phi;
    df = fmaf(LEAN ? fminf(lo, 100.f) : x, 0.3989422804f * e, phi);
  } else {
    constexpr float k2 = 1.5957691216f, b = 0.044715f;
    const float s = sigmoid(k2 * x * fmaf(b, x * x, 1.f));
    const float c = LEAN ? fminf(lo, 100.f) : x;
    f = lo * s;
    df = s + c * s * (1.f - s) * k2 * fmaf(3.f * b, c * c, 1.f);
  }
}
#endif  // __HIPCC__

// f(an integral constant of the kind)
template <typename F>
int by_kind(int32_t kind, F &&f) {
  switch (kind) {
    case LRCNN_ACT_RELU: return f(std::integral_constant<int, LRCNN_ACT_RELU>());
    case LRCNN_ACT_GELU: return f(std::integral_constant<int, LRCNN_ACT_GELU>());
    case LRCNN_ACT_GELU_TANH: return f(std::integral_constant<int, LRCNN_ACT_GELU_TANH>());
    case LRCNN_ACT_SILU: return f(std::integral_constant<int, LRCNN_ACT_SILU>());
  }
  return refuse(LRCNN_EINVAL, "unknown activation");
}
template <typename F>
int by_kind_or_none(int32_t kind, F &&f) {
  if (kind == LRCNN_ACT_NONE) return f(std::integral_constant<int, LRCNN_ACT_NONE>());
  return by_kind(kind, f);
}

}  // namespace act8
}  // namespace lrcnn
