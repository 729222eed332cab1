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

// The tensor-core kernels' form for many values: SiLU by the fast exponential and quotient, GELU by
// erfc(x) = t exp(-x^2 + P(t)), t = 1 / (1 + x / 2), x >= 0 (Chebyshev fit of Press et al., Numerical
// Recipes, 2nd ed., 6.2: relative error 1.2e-7 everywhere); both within 2^-19 of the value where it is not
// far below the rounding of what they are stored in.
__device__ __forceinline__ float lin_erfc(float x) {
  const float z = fabsf(x), t = __fdividef(1.f, fmaf(0.5f, z, 1.f));
  float q = 0.17087277f;
  q = fmaf(q, t, -0.82215223f);
  q = fmaf(q, t, 1.48851587f);
  q = fmaf(q, t, -1.13520398f);
  q = fmaf(q, t, 0.27886807f);
  q = fmaf(q, t, -0.18628806f);
  q = fmaf(q, t, 0.09678418f);
  q = fmaf(q, t, 0.37409196f);
  q = fmaf(q, t, 1.00002368f);
  q = fmaf(q, t, -1.26551223f);
  const float e = t * __expf(fmaf(-z, z, q));
  return x >= 0.f ? e : 2.f - e;
}
template <int N> __device__ __forceinline__ void lin_act_all(float (&v)[N], int act) {
  if (act == JK_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = __fdividef(v[j], 1.f + __expf(-v[j]));
  } else if (act == JK_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = 0.5f * v[j] * lin_erfc(-0.70710678118654752f * v[j]);
  }
}
