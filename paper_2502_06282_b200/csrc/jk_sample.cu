// jk_sample: temperature, top-k, top-p and min-p over rows of logits, the draw of a token and the filtered
// rows (the sampled form of arXiv 2502.06282, Sec. 2.1 steps 2-3, draws with a temperature only).
//
// One block per row.  Logits are compared through their ordered 32-bit image (larger logit = larger
// unsigned integer).  Every filter is a prefix of (logit descending, index ascending), so the kept set
// is a threshold on the image plus a number of tokens equal to the threshold, lowest index first.
// Both thresholds (by count for top-k, by weight for top-p) are found by bisection over the image's
// bits: 32 passes over the row, which lies in L2.  Weights are formed and summed in double
// precision.
#include <math.h>

#include "jk_common.cuh"

#define SMP_THREADS 1024

// Larger value, larger image; NaN like -inf, +inf like the largest float.
__device__ __forceinline__ uint32_t smp_key(float z) {
  if (z != z) z = -INFINITY;
  if (z == INFINITY) z = 3.402823466e38f;
  if (z == 0.f) z = 0.f;                                 // -0 and +0 are one value
  const uint32_t b = __float_as_uint(z);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float smp_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}
#define SMP_NOTHING 0x007fffffu                          // the image of -inf

struct smp_scratch {
  double d[33];
  int i[33];
};

__device__ __forceinline__ double smp_sum_d(double v, smp_scratch& s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (lane == 0) s.d[warp] = v;
  __syncthreads();
  double t = 0.0;
  for (int w = 0; w < SMP_THREADS / 32; ++w) t += s.d[w];
  return t;
}
__device__ __forceinline__ int smp_sum_i(int v, smp_scratch& s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (lane == 0) s.i[warp] = v;
  __syncthreads();
  int t = 0;
  for (int w = 0; w < SMP_THREADS / 32; ++w) t += s.i[w];
  return t;
}

template <typename T>
__global__ void __launch_bounds__(SMP_THREADS) k_sample(
    const T* __restrict__ logits, long long stride, int V, const float* __restrict__ temperature,
    const int32_t* __restrict__ top_k, const float* __restrict__ top_p, const float* __restrict__ min_p,
    const float* __restrict__ u, int32_t* __restrict__ out_tok, float* __restrict__ out_logits) {
  __shared__ smp_scratch S;
  __shared__ unsigned s_max;
  __shared__ int s_first;
  __shared__ double s_before[SMP_THREADS];
  __shared__ int s_ties[SMP_THREADS];
  jk_pdl_wait();
  jk_pdl_trigger();
  const int r = blockIdx.x, tid = threadIdx.x;
  const T* z = logits + (size_t)r * stride;
  float* out = out_logits ? out_logits + (size_t)r * V : nullptr;
  if (tid == 0) { s_max = 0u; s_first = 0x7fffffff; }
  __syncthreads();
  unsigned mx = 0u;
  for (int i = tid; i < V; i += SMP_THREADS) mx = max(mx, smp_key(jk_to_float(z[i])));
  atomicMax(&s_max, mx);
  __syncthreads();
  const unsigned kmax = s_max;
  if (kmax <= SMP_NOTHING) {                             // nothing but -inf
    if (out) for (int i = tid; i < V; i += SMP_THREADS) out[i] = -INFINITY;
    if (out_tok && tid == 0) out_tok[r] = -1;
    return;
  }
  const float zmax = smp_value(kmax);
  const float temp = temperature ? temperature[r] : 1.f;
  if (!(temp > 0.f)) {                                   // greedy
    for (int i = tid; i < V; i += SMP_THREADS)
      if (smp_key(jk_to_float(z[i])) == kmax) { atomicMin(&s_first, i); break; }
    __syncthreads();
    if (out) for (int i = tid; i < V; i += SMP_THREADS) out[i] = i == s_first ? 0.f : -INFINITY;
    if (out_tok && tid == 0) out_tok[r] = s_first;
    return;
  }
  const double inv_t = 1.0 / (double)temp;
  auto weight = [&](uint32_t key) { return exp(((double)smp_value(key) - (double)zmax) * inv_t); };
  auto count_from = [&](uint32_t k0) {                   // tokens with image >= k0
    int n = 0;
    for (int i = tid; i < V; i += SMP_THREADS) n += smp_key(jk_to_float(z[i])) >= k0;
    return smp_sum_i(n, S);
  };
  auto mass_from = [&](uint32_t k0) {
    double m = 0.0;
    for (int i = tid; i < V; i += SMP_THREADS) {
      const uint32_t k = smp_key(jk_to_float(z[i]));
      if (k >= k0) m += weight(k);
    }
    return smp_sum_d(m, S);
  };
  // top-k: threshold image and how many of the tokens equal to it stay
  uint32_t thr = SMP_NOTHING + 1;
  int ties = V;
  const int k = top_k ? top_k[r] : 0;
  if (k > 0 && k < V && count_from(thr) > k) {
    uint32_t v = 0u;
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
      if (count_from(v | bit) >= k) v |= bit;
    thr = v;
    ties = k - (v == 0xffffffffu ? 0 : count_from(v + 1));
  }
  // top-p: among those, the largest threshold that holds top_p of their weight
  const float p = top_p ? top_p[r] : 1.f;
  if (p < 1.f) {
    const double above = mass_from(thr + 1);
    const int equal = min(ties, count_from(thr) - count_from(thr + 1));
    const double target = (double)p * (above + equal * weight(thr));
    if (above >= target && above > 0.0) {
      uint32_t v = 0u;
      for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
        if ((v | bit) <= kmax && mass_from(v | bit) >= target) v |= bit;
      thr = max(v, thr + 1);
    }
    if (thr > kmax) thr = kmax;
    const double need = (target - mass_from(thr + 1)) / weight(thr);
    const int n = need <= 1.0 ? 1 : (need >= (double)V ? V : (int)ceil(need));
    ties = above >= target && above > 0.0 ? n : min(ties, n);
  }
  // min-p: a bound on the logit itself
  const float mp = min_p ? min_p[r] : 0.f;
  const double bound = mp > 0.f ? fmin(0.0, (double)temp * log((double)mp)) : -INFINITY;
  auto keeps = [&](uint32_t key) { return key >= thr && (double)smp_value(key) - (double)zmax >= bound; };
  // every thread owns a run of the row: ties before it, then kept weight before it
  const int per = (V + SMP_THREADS - 1) / SMP_THREADS;
  const int i0 = min(V, tid * per), i1 = min(V, i0 + per);
  int nt = 0;
  for (int i = i0; i < i1; ++i) nt += smp_key(jk_to_float(z[i])) == thr;
  s_ties[tid] = nt;
  __syncthreads();
  if (tid == 0) {
    int run = 0;
    for (int j = 0; j < SMP_THREADS; ++j) { const int x = s_ties[j]; s_ties[j] = run; run += x; }
  }
  __syncthreads();
  const int t0 = s_ties[tid];
  const float ft = temp;
  double mine = 0.0;
  int at = t0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t key = smp_key(jk_to_float(z[i]));
    const bool keep = keeps(key) && (key != thr || at++ < ties);
    if (keep) mine += weight(key);
    if (out) out[i] = keep ? fmaxf(-3.402823466e38f, fminf(3.402823466e38f, smp_value(key) / ft)) : -INFINITY;
  }
  if (!out_tok) return;
  s_before[tid] = mine;
  __syncthreads();
  double total = 0.0, before = 0.0;
  for (int j = 0; j < SMP_THREADS; ++j) {
    if (j == tid) before = total;
    total += s_before[j];
  }
  const double goal = (double)u[r] * total;
  // the run in which the cumulative weight passes the goal; the last kept token if rounding lets none
  if (mine > 0.0) {
    double run = before;
    int last = -1;
    at = t0;
    for (int i = i0; i < i1; ++i) {
      const uint32_t key = smp_key(jk_to_float(z[i]));
      const bool keep = keeps(key) && (key != thr || at++ < ties);
      if (!keep) continue;
      last = i;
      run += weight(key);
      if (run > goal) break;
    }
    if (before <= goal && before + mine > goal) atomicMin(&s_first, last);
  }
  __syncthreads();
  if (s_first == 0x7fffffff) {
    __shared__ int s_last;
    if (tid == 0) s_last = -1;
    __syncthreads();
    at = t0;
    for (int i = i0; i < i1; ++i) {
      const uint32_t key = smp_key(jk_to_float(z[i]));
      if (keeps(key) && (key != thr || at++ < ties)) atomicMax(&s_last, i);
    }
    __syncthreads();
    if (tid == 0) s_first = s_last;
    __syncthreads();
  }
  if (tid == 0) out_tok[r] = s_first;
}

extern "C" int jk_sample(jk_ctx* ctx, void* stream, int32_t rows, const void* logits, int32_t logits_dtype,
                         int64_t row_stride, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, const float* u, int32_t* out_tok,
                         float* out_logits) {
  if (!ctx || !logits || (!out_tok && !out_logits) || (out_tok && !u)) return JK_ERR_NULL;
  if (logits_dtype != JK_F32 && logits_dtype != JK_BF16) return JK_ERR_DTYPE;
  const int V = ctx->cfg.vocab;
  if (rows < 1 || row_stride < V) return JK_ERR_SHAPE;
  if ((uintptr_t)logits % jk_elem_size(logits_dtype)) return JK_ERR_ALIGN;
  const void* words[] = {temperature, top_k, top_p, min_p, u, out_tok, out_logits};
  for (const void* p : words)
    if ((uintptr_t)p & 3) return JK_ERR_ALIGN;
  cudaStream_t st = (cudaStream_t)stream;
  JK_PROF(ctx, st, JK_ST_SAMPLE);
  if (logits_dtype == JK_BF16)
    jk_launch_pdl(k_sample<__nv_bfloat16>, dim3(rows), dim3(SMP_THREADS), 0, st,
                  (const __nv_bfloat16*)logits, (long long)row_stride, V, temperature, top_k, top_p,
                  min_p, u, out_tok, out_logits);
  else
    jk_launch_pdl(k_sample<float>, dim3(rows), dim3(SMP_THREADS), 0, st, (const float*)logits,
                  (long long)row_stride, V, temperature, top_k, top_p, min_p, u, out_tok, out_logits);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}
