// Paged 8-bit KV cache: argument checks, quantisation and addressing shared by its kernels.
#pragma once

#include <cuda_fp8.h>

#include "jk_common.cuh"

#define PAGED_MAX_SEQS 1024
#define PAGED_MAX_POOL (1 << 24)     // pages
#define PAGED_OK 0                   // scratch[PAGED_OK]: 1 when the plan of the running call holds
#define PAGED_N_MOVED 1              // scratch[PAGED_N_MOVED]: pages that jk_paged_compact moves
#define PAGED_LISTS 64               // three lists of n_pages entries start here

// JK_OK when the descriptor can be used with this context.
int jk_paged_check(const jk_ctx* ctx, const jk_paged* c);

#ifdef __CUDACC__
// The smallest power of two s >= 2^-32 with amax <= 448 s: 448 = 1.75 * 2^8, so for amax = m 2^k,
// 1 <= m < 2, the exponent is k - 8 or, where m > 1.75, k - 7.
__device__ __forceinline__ int paged_scale_exp(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int k = (int)(b >> 23) - 127;
  const int e = k - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < -32 ? -32 : e;
}
__device__ __forceinline__ float paged_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// |x| where it counts for the scale: infinities and NaN do not.
__device__ __forceinline__ float paged_mag(float x) {
  const float a = fabsf(x);
  return a <= 3.402823466e38f ? a : 0.f;
}
__device__ __forceinline__ uint32_t paged_pack4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}
__device__ __forceinline__ float2 paged_unpack2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// 16 consecutive elements
template <typename T> __device__ __forceinline__ void paged_load16(const T* p, float (&o)[16]) {
  constexpr int VN = jk_vec<T>::N;
#pragma unroll
  for (int i = 0; i < 16 / VN; ++i) {
    float v[VN];
    jk_vec<T>::load(p + i * VN, v);
#pragma unroll
    for (int j = 0; j < VN; ++j) o[i * VN + j] = v[j];
  }
}
#endif
