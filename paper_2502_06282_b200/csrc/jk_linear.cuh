// jk_linear: what its kernels share.
#pragma once

#include "jk_mx8.cuh"

struct lin_args {
  int rows, n_out, n_in, act;
  const void *x, *w, *w_up;
  const uint8_t *x_scale, *w_scale, *w_up_scale;
  const void *bias, *bias_up, *residual;
  void* out;
  uint8_t* out_scale;
  long long x_stride, r_stride, o_stride;
  int k_tiles_in, k_tiles_out;             // scale tiles along n_in and n_out
  int out_type;
};

// z -> act(z) [* up] in f32.  SiLU and GELU by the library's exponential and erfc: accurate to a few
// units of f32, which the f32 outputs show.
__device__ __forceinline__ float lin_act(float z, int act) {
  if (act == JK_ACT_SILU) return z / (1.f + expf(-z));
  if (act == JK_ACT_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);
  return z;
}

// The tensor-core kernels' form (their epilogue is bound by fetching its instructions: everything short, in loops of
// 8 values): SiLU by the approximate exponential and reciprocal, within 2^-18; GELU by
// erfc(x) = t exp(-x^2 + P(t)), t = 1 / (1 + x / 2), x >= 0.  P for outputs of 16 and 8 bits: the polynomial of degree 5
// that makes the largest relative error over 0 .. 10 smallest (7.6e-6, found by reweighted least squares on log erfc;
// 2^-16 with the roundings of the exponent, a 2^-7th of what bf16 rounds).  P for f32 outputs: that of degree 9 of Press et
// al., Numerical Recipes, 2nd ed., 6.2 (1.2e-7; 2^-18 with the exponent's roundings).
__device__ __forceinline__ float lin_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lin_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
#define LIN_LOG2E 1.4426950408889634f
template <bool F32> __device__ __forceinline__ float lin_gelu(float v) {
  const float a = fabsf(v), t = lin_rcp(fmaf(0.35355339059327376f, a, 1.f));     // x = |v| / sqrt 2
  float q;                                                                       // (exponents of 2)
  if (F32) {
    q = LIN_LOG2E * 0.17087277f;
    q = fmaf(q, t, LIN_LOG2E * -0.82215223f);
    q = fmaf(q, t, LIN_LOG2E * 1.48851587f);
    q = fmaf(q, t, LIN_LOG2E * -1.13520398f);
    q = fmaf(q, t, LIN_LOG2E * 0.27886807f);
    q = fmaf(q, t, LIN_LOG2E * -0.18628806f);
    q = fmaf(q, t, LIN_LOG2E * 0.09678418f);
    q = fmaf(q, t, LIN_LOG2E * 0.37409196f);
    q = fmaf(q, t, LIN_LOG2E * 1.00002368f);
    q = fmaf(q, t, LIN_LOG2E * -1.26551223f);
  } else {
    q = LIN_LOG2E * 0.22879023753f;
    q = fmaf(q, t, LIN_LOG2E * -0.70919065294f);
    q = fmaf(q, t, LIN_LOG2E * 0.47449294008f);
    q = fmaf(q, t, LIN_LOG2E * 0.25444333415f);
    q = fmaf(q, t, LIN_LOG2E * 1.01801351084f);
    q = fmaf(q, t, LIN_LOG2E * -1.26654175576f);
  }
  q = fmaf(a * a, -0.5f * LIN_LOG2E, q);
  const float e = t * lin_exp2(q);
  return v * (v <= 0.f ? 0.5f * e : fmaf(-0.5f, e, 1.f));                        // Phi(v) = erfc(-v / sqrt 2) / 2
}
template <int N> __device__ __forceinline__ void lin_act_all(float (&v)[N], int act, bool f32) {
  if (act == JK_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] *= lin_rcp(1.f + lin_exp2(-LIN_LOG2E * v[j]));
  } else if (act == JK_ACT_GELU && f32) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = lin_gelu<true>(v[j]);
  } else if (act == JK_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = lin_gelu<false>(v[j]);
  }
}
