// jk_linear: argument checks, and the kernel on CUDA cores (f32 contexts; every type while the
// tensor path is off).
#include "jk_linear.cuh"

int jk_tma_available(jk_ctx* ctx);                                             // jk_gemm_tc.cu
int jk_linear_tc(jk_ctx* ctx, cudaStream_t st, const lin_args& a, bool mx);    // jk_linear_tc.cu
int jk_linear_pair(jk_ctx* ctx, cudaStream_t st, const lin_args& a, bool mx);  // jk_linear_pair.cu
int jk_linear_tc_pays(jk_ctx* ctx, const lin_args& a, bool mx, bool* pays);    // jk_linear_tc.cu

// ------------------------------------------------------------------------------------------ operands
// Four consecutive elements of a row as f32; element types: float, bf16, uint8_t (mx8 codes, k a
// multiple of 4, so one scale covers them).
__device__ __forceinline__ float4 lin_load4(const float* row, int k, const uint8_t*, size_t, int) {
  return *reinterpret_cast<const float4*>(row + k);
}
__device__ __forceinline__ float4 lin_load4(const __nv_bfloat16* row, int k, const uint8_t*, size_t, int) {
  const uint2 v = *reinterpret_cast<const uint2*>(row + k);
  return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                     __uint_as_float(v.y & 0xffff0000u));
}
__device__ __forceinline__ float4 lin_load4(const uint8_t* row, int k, const uint8_t* scale, size_t r, int k_tiles) {
  const uint32_t v = *reinterpret_cast<const uint32_t*>(row + k);
  const float s = paged_pow2((int)scale[mx_scale_at(r, k >> 5, k_tiles)] - 127);
  const float2 a = paged_unpack2(v), b = paged_unpack2(v >> 16);
  return make_float4(a.x * s, a.y * s, b.x * s, b.y * s);
}

// ------------------------------------------------------------------------------------------ CUDA cores
// A value's way out: row r, output n, from a group of lanes that hold a scale block of 32 outputs, `n_own` consecutive
// ones each.  Every lane of the warp calls it.
template <typename T, int OWN>
__device__ __forceinline__ void lin_out(const lin_args& a, const float (&y)[OWN], int r, int n) {
  constexpr int LANES = 32 / OWN;
  const bool row_live = r < a.rows;
  float v[OWN];
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    v[i] = y[i];
    if (a.residual && row_live && n + i < a.n_out) v[i] += jk_to_float(((const T*)a.residual)[(size_t)r * a.r_stride + n + i]);
  }
  if (a.out_type == JK_ROWS_MX8) {                     // n_out is a multiple of 32: a block is live as a whole
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < OWN; ++i) m = fmaxf(m, paged_mag(v[i]));
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (!row_live || n >= a.n_out) return;
    const int e = paged_scale_exp(m);
    const float inv = paged_pow2(-e);
#pragma unroll
    for (int i = 0; i < OWN; ++i)
      ((uint8_t*)a.out)[(size_t)r * a.n_out + n + i] = (uint8_t)__nv_cvt_float_to_fp8(v[i] * inv, __NV_SATFINITE, __NV_E4M3);
    if ((n & 31) == 0) a.out_scale[mx_scale_at(r, n >> 5, a.k_tiles_out)] = (uint8_t)(e + 127);
    return;
  }
  if (!row_live) return;
#pragma unroll
  for (int i = 0; i < OWN; ++i)
    if (n + i < a.n_out) {
      if (a.out_type == JK_ROWS_F32) ((float*)a.out)[(size_t)r * a.o_stride + n + i] = v[i];
      else ((T*)a.out)[(size_t)r * a.o_stride + n + i] = jk_from_float<T>(v[i]);
    }
}
template <typename T> __device__ __forceinline__ float lin_bias(const void* b, int n, int n_out) {
  return b && n < n_out ? jk_to_float(((const T*)b)[n]) : 0.f;
}

// Eight sums over the warp's lanes at once, 9 exchanges instead of 40: at each of three steps a lane hands on half of what it
// holds and takes the other half's partner.  Lane l returns the sum of value 4 (l >> 4 & 1) + 2 (l >> 3 & 1) + (l >> 2 & 1).
__device__ __forceinline__ float warp_sums8(float (&v)[8], int lane) {
#pragma unroll
  for (int h = 4; h > 0; h >>= 1) {
    const bool up = lane & (h * 4);
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const float give = up ? v[i] : v[i + h], keep = up ? v[i + h] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, h * 4);
    }
  }
  v[0] += __shfl_xor_sync(0xffffffffu, v[0], 2);
  return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
}

// Few rows: a warp owns OUTS weight rows (gated: of w and of w_up) and up to 8 rows of x, its lanes go along k: every
// weight is read once from memory, x comes from the caches.  Bound by latency at the sizes it is taken for, and, at one
// weight row a warp, by x on its way from the caches.
#define LR_ROWS 8
template <typename TX, typename T, bool GATED, int OUTS>
__global__ void __launch_bounds__(256, 2) k_linear_rows(const lin_args a) {
  jk_pdl_wait();
  jk_pdl_trigger();
  constexpr int W = OUTS * (1 + GATED);
  const int lane = threadIdx.x & 31, n = (blockIdx.x * 8 + (threadIdx.x >> 5)) * OUTS, r0 = blockIdx.y * LR_ROWS;
  if (n >= a.n_out) return;
  float acc[W][LR_ROWS];
#pragma unroll
  for (int i = 0; i < W; ++i)
#pragma unroll
    for (int j = 0; j < LR_ROWS; ++j) acc[i][j] = 0.f;
  const int last = OUTS > 1 ? min(n + OUTS, a.n_out) - 1 : n;
  const TX *w0 = (const TX*)a.w + (size_t)n * a.n_in, *w1 = (const TX*)a.w + (size_t)last * a.n_in;
  const TX* u0 = GATED ? (const TX*)a.w_up + (size_t)n * a.n_in : nullptr;
  static_assert(OUTS <= 2 && (OUTS == 1 || !GATED), "two outputs, plain ones");
#pragma unroll (OUTS == 1 ? 4 : 2)
  for (int k = lane * 4; k < a.n_in; k += 128) {
    float4 w[W];
    w[0] = lin_load4(w0, k, a.w_scale, n, a.k_tiles_in);
    if (GATED) w[W - 1] = lin_load4(u0, k, a.w_up_scale, n, a.k_tiles_in);
    if (OUTS > 1) w[W - 1] = lin_load4(w1, k, a.w_scale, last, a.k_tiles_in);
#pragma unroll
    for (int j = 0; j < LR_ROWS; ++j)
      if (r0 + j < a.rows) {
        const float4 x = lin_load4((const TX*)a.x + (size_t)(r0 + j) * a.x_stride, k, a.x_scale, r0 + j, a.k_tiles_in);
#pragma unroll
        for (int i = 0; i < W; ++i)
          acc[i][j] += fmaf(x.x, w[i].x, fmaf(x.y, w[i].y, fmaf(x.z, w[i].z, x.w * w[i].w)));
      }
  }
  const int r = r0 + 4 * (lane >> 4 & 1) + 2 * (lane >> 3 & 1) + (lane >> 2 & 1);
#pragma unroll
  for (int i = 0; i < OUTS; ++i) {
    const float z = warp_sums8(acc[i], lane), zu = GATED ? warp_sums8(acc[W - OUTS + i], lane) : 0.f;
    if ((lane & 3) || r >= a.rows || n + i >= a.n_out) continue;
    float y = lin_act(z + lin_bias<T>(a.bias, n + i, a.n_out), a.act);
    if (GATED) y *= zu + lin_bias<T>(a.bias_up, n + i, a.n_out);
    if (a.residual) y += jk_to_float(((const T*)a.residual)[(size_t)r * a.r_stride + n + i]);
    if (a.out_type == JK_ROWS_F32) ((float*)a.out)[(size_t)r * a.o_stride + n + i] = y;
    else ((T*)a.out)[(size_t)r * a.o_stride + n + i] = jk_from_float<T>(y);
  }
}

// The rest: a block makes ROWS rows times 128 weight rows (gated: 64 of w and 64 of w_up, the two of an output in one
// thread), 8 columns and ROWS / 16 rows a thread, k in steps of 16 through two buffers of shared memory, the next
// step's loads on their way while one is multiplied.  The sum of 32 products is formed by itself and then added,
// which keeps long sums within a few units of f32.  Where the tiles are few, `split` blocks of a cluster share one along
// k and each finishes every split-th part of its rows from all their sums.
// Two products an instruction (fma.rn.f32x2): one each spent two thirds of the issue slots and left the multipliers idle.
#define LB_N 128
#define LB_K 16
__device__ __forceinline__ uint64_t lb_pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t lb_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ void lb_add(float& a, float& b, uint64_t p) {
  float x, y;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p));
  a += x;
  b += y;
}
template <typename TX, typename T, bool GATED, int ROWS>
__global__ void __launch_bounds__(256) k_linear_block(const lin_args a, int split) {
  constexpr int RT = ROWS / 16, OUTS = GATED ? 64 : 128;
  constexpr int RING = 2 * LB_K * (LB_N + 4 + ROWS + 4), SUMS = ROWS <= 64 ? ROWS * LB_N : 0;
  __shared__ __align__(16) float s_mem[RING > SUMS ? RING : SUMS];
  float (*s_w)[LB_K][LB_N + 4] = reinterpret_cast<float (*)[LB_K][LB_N + 4]>(s_mem);
  float (*s_x)[LB_K][ROWS + 4] = reinterpret_cast<float (*)[LB_K][ROWS + 4]>(s_mem + 2 * LB_K * (LB_N + 4));
  jk_pdl_wait();
  jk_pdl_trigger();
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int rank = blockIdx.x % split, n0 = blockIdx.x / split * OUTS, r0 = blockIdx.y * ROWS;
  const int lr = threadIdx.x >> 2, lk = (threadIdx.x & 3) * 4;         // loading: rows lr, lr + 64, four elements
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  float4 pw[2], px[(ROWS + 63) / 64];
  auto ask = [&](int k0) {
    const bool in = k0 + lk < a.n_in;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = n0 + lr + (GATED ? 0 : 64 * h);
      const bool up = GATED && h;
      pw[h] = in && n < a.n_out ? lin_load4((const TX*)(up ? a.w_up : a.w) + (size_t)n * a.n_in, k0 + lk,
                                            up ? a.w_up_scale : a.w_scale, n, a.k_tiles_in) : zero;
    }
#pragma unroll
    for (int h = 0; h < (ROWS + 63) / 64; ++h) {
      const int r = lr + 64 * h;
      px[h] = in && r < ROWS && r0 + r < a.rows
                  ? lin_load4((const TX*)a.x + (size_t)(r0 + r) * a.x_stride, k0 + lk, a.x_scale, r0 + r, a.k_tiles_in) : zero;
    }
  };
  auto put = [&](int b) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float v[4] = {pw[h].x, pw[h].y, pw[h].z, pw[h].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) s_w[b][lk + i][lr + 64 * h] = v[i];
    }
#pragma unroll
    for (int h = 0; h < (ROWS + 63) / 64; ++h)
      if (lr + 64 * h < ROWS) {
        const float v[4] = {px[h].x, px[h].y, px[h].z, px[h].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) s_x[b][lk + i][lr + 64 * h] = v[i];
      }
  };
  float acc[RT][8];
  uint64_t part[RT][4];                    // of outputs 2 j and 2 j + 1
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[i][2 * j] = acc[i][2 * j + 1] = 0.f;
      part[i][j] = 0;
    }
  const int all = (a.n_in + LB_K - 1) / LB_K, s0 = (int)((long long)all * rank / split);
  const int steps = (int)((long long)all * (rank + 1) / split) - s0;
  ask(s0 * LB_K);
  put(0);
  __syncthreads();
  for (int s = 0; s < steps; ++s) {
    const int b = s & 1;
    if (s + 1 < steps) ask((s0 + s + 1) * LB_K);
#pragma unroll
    for (int k = 0; k < LB_K; ++k) {
      float x[RT];
      const float4 w0 = *reinterpret_cast<const float4*>(&s_w[b][k][tx * 4]), w1 = *reinterpret_cast<const float4*>(&s_w[b][k][64 + tx * 4]);
      const uint64_t w[4] = {lb_pair(w0.x, w0.y), lb_pair(w0.z, w0.w), lb_pair(w1.x, w1.y), lb_pair(w1.z, w1.w)};
      if constexpr (RT >= 4) {
#pragma unroll
        for (int i = 0; i < RT; i += 4)
          *reinterpret_cast<float4*>(&x[i]) = *reinterpret_cast<const float4*>(&s_x[b][k][ty * RT + i]);
      } else {
#pragma unroll
        for (int i = 0; i < RT; ++i) x[i] = s_x[b][k][ty * RT + i];
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const uint64_t xx = lb_pair(x[i], x[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) part[i][j] = lb_fma(xx, w[j], part[i][j]);
      }
    }
    if ((s & 1) || s + 1 == steps) {
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) { lb_add(acc[i][2 * j], acc[i][2 * j + 1], part[i][j]); part[i][j] = 0; }
    }
    if (s + 1 < steps) put(b ^ 1);
    __syncthreads();
  }
  if constexpr (SUMS > 0) {
    if (split > 1) {
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<float4*>(&s_mem[(ty * RT + i) * LB_N + 64 * h + tx * 4]) =
              make_float4(acc[i][4 * h], acc[i][4 * h + 1], acc[i][4 * h + 2], acc[i][4 * h + 3]);
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
      const int lane = threadIdx.x & 31;
      for (int r = rank + split * (threadIdx.x >> 5); r < ROWS; r += split * 8) {
        float z[4] = {0.f, 0.f, 0.f, 0.f}, zu[4] = {0.f, 0.f, 0.f, 0.f};
        const int at = r * LB_N + (GATED ? (lane & 15) : lane) * 4;
        for (int i = 0; i < split; ++i) {                // in the order of k
          const float* o = jk_cluster_map(&s_mem[at], i);
          const float4 v = *reinterpret_cast<const float4*>(o);
          z[0] += v.x; z[1] += v.y; z[2] += v.z; z[3] += v.w;
          if (GATED) {
            const float4 u = *reinterpret_cast<const float4*>(o + 64);
            zu[0] += u.x; zu[1] += u.y; zu[2] += u.z; zu[3] += u.w;
          }
        }
        // (gated: the upper lanes hold what the lower ones do, and nothing to write)
        const int n = GATED && lane >= 16 ? a.n_out : n0 + lane * 4;
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[j] = lin_act(z[j] + lin_bias<T>(a.bias, n + j, a.n_out), a.act);
          if (GATED) y[j] *= zu[j] + lin_bias<T>(a.bias_up, n + j, a.n_out);
        }
        lin_out<T, 4>(a, y, r0 + r, n);
      }
      __syncwarp();                        // (lin_out lets lanes without an output go)
      asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
      return;
    }
  }
  // a thread has outputs tx * 4 .. + 3 (and 64 on, or their gate's partners): eight neighbouring lanes a scale block
#pragma unroll
  for (int h = 0; h < (GATED ? 1 : 2); ++h) {
    const int n = n0 + 64 * h + tx * 4;
    float bias[4], bias_up[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bias[j] = lin_bias<T>(a.bias, n + j, a.n_out);
      bias_up[j] = GATED ? lin_bias<T>(a.bias_up, n + j, a.n_out) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y[j] = lin_act(acc[i][4 * h + j] + bias[j], a.act);
        if (GATED) y[j] *= acc[i][4 + j] + bias_up[j];
      }
      lin_out<T, 4>(a, y, r0 + ty * RT + i, n);
    }
  }
}

// Up to 16 rows, while a scale block's outputs need not meet: warps of outputs, of two each where there are more than the SMs
// hold at a time (16 x 1928 x 4250 31.2 us with one, 17.8 with two, 1 x 4096 x 4096 15.0 and 12.3, 5 x 8192 x 8192 80
// and 86, 16 x 512 x 512 2.5 and 3.0; gated, where two are four rows of weights, 5.8 and 9.1 for 16 x 1376 x 512).  Up to 32, blocks of 32 rows with up to 8 to
// a tile.  Else blocks of 128 or of 64 rows, the latter with 1 to 8 to a tile, by what the SM with the most of them needs:
// a step of 16 along k takes a block of 128 rows 1.63 us, one of 64 rows 1.13 us alone on its SM and 0.98 next to another.
// Measured in f32, us, with 128 rows / 64 / 64 shared by 2: 1024 x 4096 x 4096 837 / 992 / 872, 256 x 4096 x 4096 417 / 289 /
// 257, 313 x 9352 x 3456 gated 1803 / 1151 / 1143; the whole range against CUDA 12.9's library, which makes the products
// alone: 16 x 1376 x 512 gated 5.8 (31), 60 x 4096 x 4096 68 (88), 1024 x 4096 x 4096 837 (626).
template <typename TX, typename T>
static void launch_cc(cudaStream_t st, const lin_args& a, int sms) {
  const bool gated = a.w_up != nullptr;
  if (a.rows <= 2 * LR_ROWS && a.out_type != JK_ROWS_MX8) {
    const int y = (a.rows + LR_ROWS - 1) / LR_ROWS, outs = !gated && (long long)a.n_out * y >= 16ll * sms ? 2 : 1;
    const dim3 grid((unsigned)((a.n_out + 8 * outs - 1) / (8 * outs)), (unsigned)y);
    jk_launch_pdl(gated ? k_linear_rows<TX, T, true, 1> : outs == 2 ? k_linear_rows<TX, T, false, 2> : k_linear_rows<TX, T, false, 1>,
                  grid, dim3(256), 0, st, a);
    return;
  }
  const int outs = gated ? LB_N / 2 : LB_N, n_tiles = (a.n_out + outs - 1) / outs, all = (a.n_in + LB_K - 1) / LB_K;
  int R = 32, split = 1;                   // (shares of 8 steps at least)
  if (a.rows <= 32) {
    const long long tiles = n_tiles;
    while (split < 8 && tiles * split * 2 <= 4ll * sms && all >= 16 * split) split *= 2;
  } else {
    const auto most = [&](int rows, int s) { return ((long long)n_tiles * ((a.rows + rows - 1) / rows) * s + sms - 1) / sms; };
    double best = 1.63 * most(128, 1) * all;
    R = 128;
    for (int s = 1; s <= 8 && (s == 1 || all >= 8 * s); s *= 2) {
      const long long n = most(64, s);
      const double us = (n == 1 ? 1.13 : 0.98 * n) * ((all + s - 1) / s) + (s > 1 ? 3 + 2 * s : 0);
      if (us < best) { best = us; R = 64; split = s; }
    }
  }
  const dim3 grid((unsigned)(n_tiles * split), (unsigned)((a.rows + R - 1) / R));
  auto k = R == 128 ? (gated ? k_linear_block<TX, T, true, 128> : k_linear_block<TX, T, false, 128>)
           : R == 64 ? (gated ? k_linear_block<TX, T, true, 64> : k_linear_block<TX, T, false, 64>)
                     : (gated ? k_linear_block<TX, T, true, 32> : k_linear_block<TX, T, false, 32>);
  jk_launch_pdl_cluster(k, grid, dim3(256), (unsigned)split, 0, st, a, split);
}

// ------------------------------------------------------------------------------------------ host side
extern "C" int jk_linear(jk_ctx* ctx, void* stream, const jk_linear_op* op, int32_t rows, const void* x,
                         const uint8_t* x_scale, int64_t x_stride, const void* residual, int64_t residual_stride,
                         void* out, int32_t out_type, uint8_t* out_scale, int64_t out_stride) {
  if (!ctx || !op || !x || !out || !op->w) return JK_ERR_NULL;
  const bool mx = op->operands == JK_ROWS_MX8;
  if (!mx && op->operands != JK_ROWS_T) return JK_ERR_DTYPE;
  if (out_type != JK_ROWS_T && out_type != JK_ROWS_F32 && out_type != JK_ROWS_MX8) return JK_ERR_DTYPE;
  if (mx && (!x_scale || !op->w_scale || (op->w_up && !op->w_up_scale))) return JK_ERR_NULL;
  if (out_type == JK_ROWS_MX8 && !out_scale) return JK_ERR_NULL;
  if (op->act < JK_ACT_NONE || op->act > JK_ACT_GELU || (op->bias_up && !op->w_up)) return JK_ERR_SHAPE;
  const int64_t N = op->n_out, K = op->n_in, most = (int64_t)1 << 31;
  if (rows < 1 || rows > (1 << 20) || N < 1 || N > (1 << 20) || K < 1 || K > (1 << 17) || K % (mx ? MX_BLOCK : 8))
    return JK_ERR_SHAPE;
  if (out_type == JK_ROWS_MX8 && N % MX_BLOCK) return JK_ERR_SHAPE;
  if (x_stride == 0) x_stride = K;
  if (residual_stride == 0) residual_stride = N;
  if (out_stride == 0) out_stride = N;
  if (x_stride < K || residual_stride < N || out_stride < N || x_stride > most || residual_stride > most ||
      out_stride > most || (mx && x_stride != K) || (out_type == JK_ROWS_MX8 && out_stride != N))
    return JK_ERR_SHAPE;
  const size_t es = jk_elem_size(ctx->cfg.dtype), xs = mx ? 1 : es;
  const size_t os = out_type == JK_ROWS_MX8 ? 1 : out_type == JK_ROWS_F32 ? 4 : es;
  const void* ptrs[] = {x, x_scale, op->w, op->w_scale, op->bias, op->w_up, op->w_up_scale, op->bias_up, residual,
                        out, out_scale};
  for (const void* p : ptrs)
    if (!jk_aligned16(p)) return JK_ERR_ALIGN;
  if ((x_stride * xs) % 16) return JK_ERR_ALIGN;
  // what is written must not be read as well, but for the residual in place
  const size_t sc_w = mx ? jk_row_scale_bytes(N, K) : 0, sc_x = mx ? jk_row_scale_bytes(rows, K) : 0;
  const void* in[] = {x, x_scale, op->w, op->w_scale, op->bias, op->w_up, op->w_up_scale, op->bias_up, residual};
  const size_t in_b[] = {((size_t)(rows - 1) * x_stride + K) * xs, sc_x, (size_t)(N * K) * xs, sc_w, (size_t)N * es,
                         (size_t)(N * K) * xs, sc_w, (size_t)N * es,
                         ((size_t)(rows - 1) * residual_stride + N) * es};
  const size_t row_b[] = {(size_t)K * xs, (size_t)N * es}, apart[] = {(size_t)x_stride * xs, (size_t)residual_stride * es};
  const size_t out_b = ((size_t)(rows - 1) * out_stride + N) * os;
  const size_t sc_o = out_type == JK_ROWS_MX8 ? jk_row_scale_bytes(rows, N) : 0;
  for (int i = 0; i < 9; ++i) {
    const bool in_place = i == 8 && out == residual && os == es && out_stride == residual_stride;
    const bool written = i == 0 || i == 8 ? jk_rows_overlap(out, rows, N * os, out_stride * os, in[i], rows, row_b[i / 8], apart[i / 8])
                                          : jk_overlap(out, out_b, in[i], in_b[i]);
    if ((written && !in_place) || (sc_o && jk_overlap(out_scale, sc_o, in[i], in_b[i])))
      return JK_ERR_SHAPE;
  }
  if (sc_o && jk_overlap(out, out_b, out_scale, sc_o)) return JK_ERR_SHAPE;
  lin_args a;
  memset(&a, 0, sizeof(a));
  a.rows = rows; a.n_out = (int)N; a.n_in = (int)K; a.act = op->act;
  a.x = x; a.w = op->w; a.w_up = op->w_up;
  a.x_scale = x_scale; a.w_scale = op->w_scale; a.w_up_scale = op->w_up_scale;
  a.bias = op->bias; a.bias_up = op->bias_up; a.residual = residual;
  a.out = out; a.out_scale = out_scale; a.out_type = out_type;
  a.x_stride = x_stride; a.r_stride = residual_stride; a.o_stride = out_stride;
  a.k_tiles_in = mx_k_tiles(K); a.k_tiles_out = mx_k_tiles(N);
  if (!ctx->ws) return JK_ERR_WORKSPACE;
  int rc = jk_ensure_device_info(ctx);
  if (rc != JK_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (ctx->tensor_path && ctx->cfg.dtype == JK_BF16 && jk_tma_available(ctx)) {
    // Of the kernel that streams weights past few rows and that for many rows the one with the lower cost.  Measured, us,
    // 4096 inputs in bf16: 4096 outputs, 64 rows 10.7 against 21.5, 256 rows 16.2 / 24.1, 512 rows 22.0 / 25.2; 1024
    // outputs, 512 rows 14.3 / 21.4; 6144 outputs, 512 rows 31.9 / 30.4; in 8 bits 4096 outputs, 256 rows 13.3 / 16.6, 512
    // rows 15.9 / 17.2, 768 rows 20.4 / 18.3.
    bool few;
    if ((rc = jk_linear_tc_pays(ctx, a, mx, &few)) != JK_OK) return rc;
    return few ? jk_linear_tc(ctx, st, a, mx) : jk_linear_pair(ctx, st, a, mx);
  }
  JK_PROF(ctx, st, JK_ST_LINEAR);
  if (ctx->cfg.dtype == JK_F32) {
    if (mx) launch_cc<uint8_t, float>(st, a, ctx->sm_count);
    else launch_cc<float, float>(st, a, ctx->sm_count);
  } else {
    if (mx) launch_cc<uint8_t, __nv_bfloat16>(st, a, ctx->sm_count);
    else launch_cc<__nv_bfloat16, __nv_bfloat16>(st, a, ctx->sm_count);
  }
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}
