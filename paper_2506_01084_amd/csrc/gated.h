// The gated feed-forward block, F = act(G) * U, on the device: the activations, their slopes and what either direction stores (gfx950).
#pragma once

#include "logits_common.h"

namespace z2z_gated {

using z2z_logits::pack_bf16;

// act(x) = x Phi, and its slope: SiLU, Phi = 1 / (1 + e^-x), slope Phi + x Phi (1 - Phi); GELU, Phi the normal distribution's, slope Phi + x phi.
// GELU's erf as in gelu_erf, whose exponential e^(-x^2 / 2) is the density's, too.  (Reciprocals to the last bit but one, far inside the rounding of what is stored.)
struct Act {
  float value, slope;
};
__device__ __forceinline__ Act act_and_slope(float x, int act) {
  if (act == Z2Z_ACT_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-x)), v = x * p;
    return Act{v, fmaf(v, 1.0f - p, p)};
  }
  const float z = fabsf(x) * 0.70710678f, e = __expf(-z * z);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.0f));
  const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
  const float p = 0.5f * (1.0f + copysignf(1.0f - poly * e, x));
  return Act{x * p, fmaf(x * 0.3989422804f, e, p)};
}
__device__ __forceinline__ float act_of(float x, int act) { return act_and_slope(x, act).value; }

__device__ __forceinline__ uint2 pack4(const float (&x)[4]) { return uint2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])}; }
// Four columns of F out of fp32 sums.
__device__ __forceinline__ uint2 hidden4(const float (&g)[4], const float (&u)[4], int act) {
  float f[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = act_of(g[e], act) * u[e];
  return pack4(f);
}

// Four columns of the gradients dG = dF U act'(G) and dU = dF act(G), and of F once more, from dF and from G and U as the forward pass kept them, all fp32.
// (Kept in bf16 the two roundings would be half of the gradients' error: 3.5e-3 of their norm instead of 2.4e-3, of which the rounding of
// what is returned is 1.7e-3.  16411 rows, d_ff = 5504: 0.36 GB more to write and to read, KEPT_COST.)
struct Slopes4 {
  uint2 dg, du, f;
};
__device__ __forceinline__ Slopes4 slopes4(const float (&df)[4], const float4& g4, const float4& u4, int act) {
  const float g[4] = {g4.x, g4.y, g4.z, g4.w}, u[4] = {u4.x, u4.y, u4.z, u4.w};
  float dg[4], du[4], f[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const Act a = act_and_slope(g[e], act);
    dg[e] = df[e] * u[e] * a.slope;
    du[e] = df[e] * a.value;
    f[e] = a.value * u[e];
  }
  return Slopes4{pack4(dg), pack4(du), pack4(f)};
}

}  // namespace z2z_gated
