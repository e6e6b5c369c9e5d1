// The activations and their slopes in f32, as compress, the gradients and the linear layers compute them.
#pragma once

#include "train.hpp"

namespace ginex {

// exp and 1/x: the library's and the division for f32; for results of 8 or 11 bits the instructions (1 unit each, and
// exp's argument is rounded once more: off by |x| 2^-24), without which 16-bit rows are bound by the vector unit.  1/x is 0
// where it would be below 2^-126: of silu that is x < -87, whose value is below 2^-119.
template <bool FINE>
__device__ __forceinline__ float exp_of(float x) {
  return FINE ? expf(x) : __builtin_amdgcn_exp2f(x * 1.44269504f);
}
template <bool FINE>
__device__ __forceinline__ float inverse(float x) {
  return FINE ? 1.f / x : __builtin_amdgcn_rcpf(x);
}

// Phi(-|x|) = erfc(z) / 2, z = |x| / sqrt 2, with bell = exp(-x^2 / 2):  exp(z^2) erfc(z) / 2 = t Q(t), t = 1 / (1 + a z),
// is smooth on all of [0, 1] (t by the instruction, also in f32: 1 unit); Q is a polynomial fitted to the least relative error here (weighted least squares at
// Chebyshev's points): 6e-9 of degree 10 for f32, 7e-7 of degree 7 for 16 bits.  One exponential serves Phi and its slope;
// erfcf took 363 instead of 300 us (gelu, 820 000 x 256 f32).
template <bool FINE>
__device__ __forceinline__ float tail(float x, float bell) {
  if (FINE) {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.282842712f, 1.f));
    float q = -1.460759161e-02f;
    q = fmaf(q, t, 7.022352350e-02f);
    q = fmaf(q, t, -1.177639811e-01f);
    q = fmaf(q, t, 6.878112558e-02f);
    q = fmaf(q, t, -2.344789024e-02f);
    q = fmaf(q, t, 4.195833894e-02f);
    q = fmaf(q, t, 5.950411182e-02f);
    q = fmaf(q, t, 8.586964844e-02f);
    q = fmaf(q, t, 1.038068641e-01f);
    q = fmaf(q, t, 1.128379301e-01f);
    q = fmaf(q, t, 1.128379174e-01f);
    return q * t * bell;
  }
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.325269119f, 1.f));
  float q = 3.385725232e-02f;
  q = fmaf(q, t, -1.133149230e-01f);
  q = fmaf(q, t, 8.459589749e-02f);
  q = fmaf(q, t, 2.630502449e-02f);
  q = fmaf(q, t, 9.342400306e-02f);
  q = fmaf(q, t, 1.155909210e-01f);
  q = fmaf(q, t, 1.297786344e-01f);
  q = fmaf(q, t, 1.297635293e-01f);
  return q * t * bell;
}

template <int ACT, bool FINE>
__device__ __forceinline__ float activated(float x) {
  if (ACT == GINEX_ACT_RELU) return x < 0.f ? 0.f : x;
  if (ACT == GINEX_ACT_SILU) return FINE ? x / (1.f + exp_of<FINE>(-x)) : x * inverse<FINE>(1.f + exp_of<FINE>(-x));
  if (ACT == GINEX_ACT_GELU) {
    const float below = tail<FINE>(x, exp_of<FINE>(-0.5f * x * x));
    return x * (x < 0.f ? below : 1.f - below);
  }
  return x;
}

// dy f'(x)
template <int ACT, bool FINE>
__device__ __forceinline__ float sloped(float x, float dy) {
  if (ACT == GINEX_ACT_RELU) return x > 0.f ? dy : (x <= 0.f ? 0.f : x);
  if (ACT == GINEX_ACT_SILU) {
    const float sigma = inverse<FINE>(1.f + exp_of<FINE>(-x));
    return dy * (sigma * fmaf(x, 1.f - sigma, 1.f));
  }
  const float bell = exp_of<FINE>(-0.5f * x * x), below = tail<FINE>(x, bell);
  return dy * fmaf(x * bell, 0.39894228040143268f, x < 0.f ? below : 1.f - below);
}

// The activation that all lanes have.
template <bool FINE>
__device__ __forceinline__ float activated_by(int32_t activation, float x) {
  switch (activation) {
    case GINEX_ACT_RELU: return activated<GINEX_ACT_RELU, FINE>(x);
    case GINEX_ACT_SILU: return activated<GINEX_ACT_SILU, FINE>(x);
    case GINEX_ACT_GELU: return activated<GINEX_ACT_GELU, FINE>(x);
  }
  return x;
}

}  // namespace ginex
