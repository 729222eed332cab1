// jk_linear: argument checks, and the kernel on CUDA cores (f32 contexts; every type while the
// tensor path is off).
#include "jk_linear.cuh"

int jk_tma_available(jk_ctx* ctx);                                             // jk_gemm_tc.cu
int jk_linear_tc(jk_ctx* ctx, cudaStream_t st, const lin_args& a, bool mx);    // jk_linear_tc.cu
int jk_linear_pair(jk_ctx* ctx, cudaStream_t st, const lin_args& a, bool mx);  // jk_linear_pair.cu
struct lt_params;
struct lp_params;
double jk_linear_tc_plan(const lin_args& a, bool mx, int sms, lt_params* out);
double jk_linear_pair_plan(const lin_args& a, bool mx, int sms, lp_params* out);

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
// Block = 32 outputs x 32 rows, 8 warps: a lane owns an output, a warp four rows, so that a
// warp holds the 32 outputs of a scale block.  k runs in steps of 32 through shared memory; a step's sum is
// formed by itself and then added, which keeps long sums within a few units of f32.
#define LS_B 32
template <typename TX, typename T, bool GATED>
__global__ void __launch_bounds__(256) k_linear_cc(const lin_args a) {
  __shared__ float s_w[1 + GATED][LS_B][LS_B + 1];
  __shared__ __align__(16) float s_x[LS_B][LS_B];
  jk_pdl_wait();
  jk_pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n0 = blockIdx.x * LS_B, r0 = blockIdx.y * LS_B;
  const int lr = threadIdx.x >> 3, lk = (threadIdx.x & 7) * 4;        // loading: a row, four elements
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  float acc[4] = {0.f, 0.f, 0.f, 0.f}, acc_up[4] = {0.f, 0.f, 0.f, 0.f};
  const TX* xr = (const TX*)a.x + (size_t)(r0 + lr) * a.x_stride;
  const TX* wr = (const TX*)a.w + (size_t)(n0 + lr) * a.n_in;
  const TX* ur = GATED ? (const TX*)a.w_up + (size_t)(n0 + lr) * a.n_in : nullptr;
  const bool x_live = r0 + lr < a.rows, w_live = n0 + lr < a.n_out;
  for (int k0 = 0; k0 < a.n_in; k0 += LS_B) {
    const bool in = k0 + lk < a.n_in;
    const float4 xv = x_live && in ? lin_load4(xr, k0 + lk, a.x_scale, r0 + lr, a.k_tiles_in) : zero;
    const float4 wv = w_live && in ? lin_load4(wr, k0 + lk, a.w_scale, n0 + lr, a.k_tiles_in) : zero;
    float4 uv = zero;
    if (GATED && w_live && in) uv = lin_load4(ur, k0 + lk, a.w_up_scale, n0 + lr, a.k_tiles_in);
    __syncthreads();
    *reinterpret_cast<float4*>(&s_x[lr][lk]) = xv;
    s_w[0][lk][lr] = wv.x; s_w[0][lk + 1][lr] = wv.y; s_w[0][lk + 2][lr] = wv.z; s_w[0][lk + 3][lr] = wv.w;
    if (GATED) {
      s_w[GATED][lk][lr] = uv.x; s_w[GATED][lk + 1][lr] = uv.y;
      s_w[GATED][lk + 2][lr] = uv.z; s_w[GATED][lk + 3][lr] = uv.w;
    }
    __syncthreads();
    float part[4] = {0.f, 0.f, 0.f, 0.f}, part_up[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < LS_B; k += 4) {
      float w[4], u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = s_w[0][k + i][lane];
        if (GATED) u[i] = s_w[GATED][k + i][lane];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 x4 = *reinterpret_cast<const float4*>(&s_x[warp * 4 + j][k]);
        const float xs[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          part[j] = fmaf(xs[i], w[i], part[j]);
          if (GATED) part_up[j] = fmaf(xs[i], u[i], part_up[j]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[j] += part[j];
      if (GATED) acc_up[j] += part_up[j];
    }
  }
  const int n = n0 + lane;
  const bool live = n < a.n_out;
  const float b = live && a.bias ? jk_to_float(((const T*)a.bias)[n]) : 0.f;
  const float bu = GATED && live && a.bias_up ? jk_to_float(((const T*)a.bias_up)[n]) : 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = r0 + warp * 4 + j;
    if (r >= a.rows) break;
    float y = lin_act(acc[j] + b, a.act);
    if (GATED) y *= acc_up[j] + bu;
    if (live && a.residual) y += jk_to_float(((const T*)a.residual)[(size_t)r * a.r_stride + n]);
    if (a.out_type == JK_ROWS_MX8) {                   // n_out is a multiple of 32: the warp is all live
      const int e = paged_scale_exp(jk_warp_max(paged_mag(y)));
      const float v = y * paged_pow2(-e);
      ((uint8_t*)a.out)[(size_t)r * a.n_out + n] = (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3);
      if (lane == 0) a.out_scale[mx_scale_at(r, n0 >> 5, a.k_tiles_out)] = (uint8_t)(e + 127);
    } else if (live && a.out_type == JK_ROWS_F32) {
      ((float*)a.out)[(size_t)r * a.o_stride + n] = y;
    } else if (live) {
      ((T*)a.out)[(size_t)r * a.o_stride + n] = jk_from_float<T>(y);
    }
  }
}

template <typename TX, typename T>
static void launch_cc(cudaStream_t st, const lin_args& a) {
  const dim3 grid((unsigned)((a.n_out + LS_B - 1) / LS_B), (unsigned)((a.rows + LS_B - 1) / LS_B));
  if (a.w_up) jk_launch_pdl(k_linear_cc<TX, T, true>, grid, dim3(256), 0, st, a);
  else jk_launch_pdl(k_linear_cc<TX, T, false>, grid, dim3(256), 0, st, a);
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
  const size_t out_b = ((size_t)(rows - 1) * out_stride + N) * os;
  const size_t sc_o = out_type == JK_ROWS_MX8 ? jk_row_scale_bytes(rows, N) : 0;
  for (int i = 0; i < 9; ++i) {
    const bool in_place = i == 8 && out == residual && os == es && out_stride == residual_stride;
    if ((jk_overlap(out, out_b, in[i], in_b[i]) && !in_place) || (sc_o && jk_overlap(out_scale, sc_o, in[i], in_b[i])))
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
    // Few rows: the kernel that streams weights past them, while the rows fit one tile (256, gated 128) and by the
    // costs that the two kernels give.  Measured, us, 4096 x 4096 in bf16: 64 rows 12.4 against 21.5, 128 rows 16.1 / 22.0,
    // 256 rows 25.0 / 22.2; in 8 bits 128 rows 13.5 / 17.3, 192 rows 19.1 / 17.4; 1376 x 512: 60 rows 7.2 / 8.8.
    const bool few = rows <= (op->w_up ? 128 : 256) &&
                     jk_linear_tc_plan(a, mx, ctx->sm_count, nullptr) <= jk_linear_pair_plan(a, mx, ctx->sm_count, nullptr);
    return few ? jk_linear_tc(ctx, st, a, mx) : jk_linear_pair(ctx, st, a, mx);
  }
  JK_PROF(ctx, st, JK_ST_LINEAR);
  if (ctx->cfg.dtype == JK_F32) {
    if (mx) launch_cc<uint8_t, float>(st, a);
    else launch_cc<float, float>(st, a);
  } else {
    if (mx) launch_cc<uint8_t, __nv_bfloat16>(st, a);
    else launch_cc<__nv_bfloat16, __nv_bfloat16>(st, a);
  }
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}
