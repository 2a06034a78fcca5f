// The gated feed-forward block, F = act(G) * U, on the device: the activations, their slopes and what either direction stores (gfx950).
#pragma once

#include "logits_common.h"

namespace z2z_gated {

using z2z_logits::pack_bf16;

// act(x) = x Phi, and its slope: SiLU, Phi = 1 / (1 + e^-x), slope Phi + x Phi (1 - Phi); GELU, Phi the normal distribution's, slope Phi + x phi.
// Phi(-|x|) = e^(-x^2 / 2) t P(t), t = 1 / (1 + 0.361 |x|): that form keeps the tail's relative size, and e^(-x^2 / 2) is the density's, too.  P was fitted (least largest
// relative error over |x| <= 13.2, by linear programming over Chebyshev polynomials): 6.7e-7 off, with fp32 arithmetic 1e-6 up to |x| = 3 and (1 + x^2 / 2) 2^-23 more
// beyond, from the exponent.  (With gelu_erf's five coefficients, 1.5e-7 off in erf itself, Phi(-4.5) is 0.5 % off, Phi(-5) 5 %, and nothing is left of Phi(-6).)
// Reciprocals to the last bit but one, far inside the rounding of what is stored.
struct Act {
  float value, slope;
};
__device__ __forceinline__ Act act_and_slope(float x, int act) {
  if (act == Z2Z_ACT_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-x)), v = x * p;
    return Act{v, fmaf(v, 1.0f - p, p)};
  }
  const float e = __expf(-0.5f * x * x), t = __builtin_amdgcn_rcpf(fmaf(0.361f, fabsf(x), 1.0f));
  const float poly = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.0479777418f, -0.18152748f), 0.181000054f), 0.0261784457f), 0.140125394f), 0.142130584f), 0.144115597f);
  const float tail = t * poly, p = x < 0.f ? tail * e : fmaf(-tail, e, 1.0f);
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

// What the backward pass is given of an element: a = act(G) and s = U act'(G), by which dF is multiplied, with 15 bits of fraction (2^-16 off at most), and F.  Three matrices
// one behind the other in one buffer of 8 bytes an element: F in bf16, an operand of products in both directions; the upper halves of a and s, 4 bytes; the next
// bytes of either, 2.  (G and U in bf16 would be half of the gradients' error, 3.5e-3 of their norm instead of 2.3e-3, of which the rounding of what is returned is
// 1.7e-3.  In fp32 the backward pass's epilogue read and wrote 14 bytes an element, with the matrix cores waiting, instead of 10, and formed exponentials
// again: 16411 rows, d = 2048, d_ff = 5504 556 us for dF, 463 now, and 700 for the first product, 664.)
//
// Or, in a buffer of 4 bytes an element, G and U with 16 bits each, of which the backward pass forms those three matrices first.  Sign, then 0, 5 bits of exponent and 9
// of fraction for magnitudes from 2^-16 to 2^16 (2^-10 off at most), or 1, 8 bits of exponent and 6 of fraction for all others (2^-7; zeros, infinities and NaN stay
// what they are).  (bf16, with 2^-8 for all, doubles what these add to the gradients' error: 2.3e-3 of their norm to 3.5e-3.)
__device__ __forceinline__ uint32_t rounded24(float x) {
  const uint32_t u = __float_as_uint(x);
  // (the sum carries a fraction of ones into the exponent, as it should; not a NaN's into the sign, nor the largest number's into an infinity)
  return (u & 0x7FFFFFFFu) < 0x7F7FFF80u ? u + 0x80u : u;
}
// Four columns of F out of fp32 sums, and what else is kept of them (element `at` of the matrices is the first).
__device__ __forceinline__ uint2 hidden_and_kept4(const float (&g)[4], const float (&u)[4], int act, uint4* hi, uint2* lo) {
  float f[4];
  uint32_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const Act x = act_and_slope(g[e], act);
    f[e] = x.value * u[e];
    const uint32_t a = rounded24(x.value), s = rounded24(x.slope * u[e]);
    h[e] = __builtin_amdgcn_perm(s, a, 0x07060302u);
    l[e] = __builtin_amdgcn_perm(s, a, 0x0C0C0501u);
  }
  *hi = uint4{h[0], h[1], h[2], h[3]};
  *lo = uint2{l[0] | l[1] << 16, l[2] | l[3] << 16};
  return pack4(f);
}

// A number in 16 bits, as above.
constexpr uint32_t kNear = 111u << 9;        // 2^-16: exponent and 9 bits of fraction of the least number with the finer step
__device__ __forceinline__ uint32_t code16(float x) {
  const uint32_t u = __float_as_uint(x), size = u & 0x7FFFFFFFu, near = (size + 0x2000u) >> 14;
  // (the largest numbers stay below the infinity, a NaN stays one without its payload)
  const uint32_t far = size < 0x7F800000u ? min((size + 0x10000u) >> 17, 0x3FBFu) : size == 0x7F800000u ? 0x3FC0u : 0x3FE0u;
  return (near - kNear < 0x4000u ? near - kNear : 0x4000u | far) | (u >> 16 & 0x8000u);
}
__device__ __forceinline__ float of_code16(uint32_t c) {
  const uint32_t m = c & 0x3FFFu;
  return __uint_as_float((c & 0x4000u ? m << 17 : (m + kNear) << 14) | (c & 0x8000u) << 16);
}
__device__ __forceinline__ uint4 pairs4(const float (&g)[4], const float (&u)[4]) {
  return uint4{code16(g[0]) | code16(u[0]) << 16, code16(g[1]) | code16(u[1]) << 16, code16(g[2]) | code16(u[2]) << 16, code16(g[3]) | code16(u[3]) << 16};
}

// Four columns of F, of which element `at` is the first, and what is kept beside them.
__device__ __forceinline__ uint2 hidden_and_keep4(const float (&g)[4], const float (&u)[4], int act, const z2z_ffn_kept& kept, size_t at) {
  if (kept.lo) return hidden_and_kept4(g, u, act, reinterpret_cast<uint4*>(kept.hi + at), reinterpret_cast<uint2*>(kept.lo + at));
  if (kept.hi) *reinterpret_cast<uint4*>(kept.hi + at) = pairs4(g, u);
  return hidden4(g, u, act);
}

// Four columns of the gradients dG = dF U act'(G) and dU = dF act(G), from dF and what the forward pass kept.
struct Slopes4 {
  uint2 dg, du;
};
__device__ __forceinline__ Slopes4 slopes4(const float (&df)[4], const uint4& hi, const uint2& lo) {
  const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[2] = {lo.x, lo.y};
  float dg[4], du[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    du[e] = df[e] * __uint_as_float(__builtin_amdgcn_perm(h[e], l[e >> 1], e & 1 ? 0x0504020Cu : 0x0504000Cu));
    dg[e] = df[e] * __uint_as_float(__builtin_amdgcn_perm(h[e], l[e >> 1], e & 1 ? 0x0706030Cu : 0x0706010Cu));
  }
  return Slopes4{pack4(dg), pack4(du)};
}

}  // namespace z2z_gated
