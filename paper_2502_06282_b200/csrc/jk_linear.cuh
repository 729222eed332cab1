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
