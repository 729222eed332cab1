// RMS norm with the residual's addition (T and / or 8-bit output), and rows to 8 bits.
//
//   s = x + delta, y = s / sqrt(mean(s^2) + eps) * weight
//
// One pass: a block keeps a row's f32 sums s in registers between the reduction of s^2 and the output,
// so x and delta are read once and every output is written once.  A thread
// holds pieces of 8 consecutive elements; four neighbouring lanes make a scale block of 32, whose
// largest element takes two shuffles.
//
// Bound by memory: 8191 rows of 8192 with sum and 8-bit rows, 472 MB in 75 to 83 us (6.3 to 5.7 TB/s); 240 rows of 4096 2.8 us and
// one row 1.8 us, replayed from a graph, are a launch, a chain of two loads and a reduction.
#include "jk_mx8.cuh"

// ------------------------------------------------------------------------------------------ pieces
// 8 consecutive elements of T as f32, and back
template <typename T> struct piece;
template <> struct piece<__nv_bfloat16> {
  uint4 r;
  __device__ __forceinline__ void fill(bool one) {
    const uint32_t w = one ? 0x3f803f80u : 0x80008000u;
    r = make_uint4(w, w, w, w);
  }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ float at(int i) const {
    const uint32_t w = i < 2 ? r.x : i < 4 ? r.y : i < 6 ? r.z : r.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[8]) {
    uint4 o;
    uint32_t* w = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = o;
  }
};
template <> struct piece<float> {
  float4 a, b;
  __device__ __forceinline__ void fill(bool one) {
    const float w = one ? 1.f : -0.f;
    a = b = make_float4(w, w, w, w);
  }
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ float at(int i) const {
    return i == 0 ? a.x : i == 1 ? a.y : i == 2 ? a.z : i == 3 ? a.w : i == 4 ? b.x : i == 5 ? b.y : i == 6 ? b.z : b.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
};

// A piece's 8 codes and, by the first of the four lanes that share the block, its scale byte.
// Every lane of the warp calls it (dead lanes with zeros).
__device__ __forceinline__ void mx_store_piece(const float (&v)[8], bool live, uint8_t* codes, uint8_t* scale) {
  float amax = 0.f;                        // (a maximum leaves NaN out by itself; infinities are rare)
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
  if (__any_sync(0xffffffffu, amax > 3.402823466e38f)) {
    amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, paged_mag(v[i]));
  }
  amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
  amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
  if (!live) return;
  const int e = paged_scale_exp(amax);
  const float inv = paged_pow2(-e);
  uint2 o;
  o.x = paged_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
  o.y = paged_pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
  *reinterpret_cast<uint2*>(codes) = o;
  if ((threadIdx.x & 3) == 0) *scale = (uint8_t)(e + 127);
}

// ------------------------------------------------------------------------------------------ the norm
// A block takes rows blockIdx.x, + gridDim.x, ...; a thread holds P pieces of a row, blockDim.x * 8 elements apart.
// With AHEAD the next row is asked for before the block meets over the present one, so that loads are always
// on their way, and the weights stay in registers.
template <typename T, int P> struct norm_row {
  piece<T> a[P], b[P];
  // (pieces past the row, and a delta that is not given, stay -0, which leaves every x what it is)
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      a[p].fill(false);
      b[p].fill(false);
    }
  }
  __device__ __forceinline__ void ask(const T* x, const T* delta, size_t at, int n, int step) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = threadIdx.x * 8 + p * step;
      if (c < n) {
        a[p].load(x + at + c);
        if (delta) b[p].load(delta + at + c);
      }
    }
  }
};
template <typename T, int P, bool AHEAD>
__global__ void __launch_bounds__(AHEAD ? 512 : 1024, AHEAD && P < 4 ? 2 : 1) k_add_norm(
    const T* x, const T* delta, const T* __restrict__ weight, int rows, int n, float eps, T* out_sum, T* out,
    uint8_t* codes, uint8_t* scales, int k_tiles) {
  __shared__ float red[2][32];
  jk_pdl_wait();
  jk_pdl_trigger();
  const int step = blockDim.x * 8, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  norm_row<T, P> next;
  piece<T> w[P];
  next.clear();
#pragma unroll
  for (int p = 0; p < P; ++p) w[p].fill(true);
  if (AHEAD) {
    next.ask(x, delta, (size_t)blockIdx.x * n, n, step);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = threadIdx.x * 8 + p * step;
      if (weight && c < n) w[p].load(weight + c);
    }
  }
  int turn = 0;
  for (int row = blockIdx.x; row < rows; row += (int)gridDim.x, turn ^= 1) {
    const size_t at = (size_t)row * n;
    if (!AHEAD) next.ask(x, delta, at, n, step);
    float s[P][8];
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[p][i] = next.a[p].at(i) + next.b[p].at(i);
    }
    if (AHEAD && row + (int)gridDim.x < rows) next.ask(x, delta, at + (size_t)gridDim.x * n, n, step);
    float sq = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      float part = 0.f;                    // (short sums first: the row's sum keeps its last bits)
#pragma unroll
      for (int i = 0; i < 8; ++i) part = fmaf(s[p][i], s[p][i], part);
      sq += part;
    }
    sq = jk_warp_sum(sq);
    if (lane == 0) red[turn][warp] = sq;   // (the turns' arrays alternate: one barrier a row)
    if (out_sum) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = threadIdx.x * 8 + p * step;
        if (c < n) piece<T>::store(out_sum + at + c, s[p]);
      }
    }
    __syncthreads();
    const float total = jk_warp_sum(lane < warps ? red[turn][lane] : 0.f);
    const float r = 1.f / sqrtf(total / (float)n + eps);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = threadIdx.x * 8 + p * step;
      const bool live = c < n;
      if (!AHEAD && weight && live) w[p].load(weight + c);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[p][i] = s[p][i] * r * w[p].at(i);
      if (out && live) piece<T>::store(out + at + c, s[p]);
      if (codes) mx_store_piece(s[p], live, codes + at + c, scales + mx_scale_at(row, c >> 5, k_tiles));
    }
  }
}

// ------------------------------------------------------------------------------------------ rows to 8 bits
// Pieces of all rows in one line: a thread takes every (grid size)-th.
template <typename T>
__global__ void __launch_bounds__(256) k_quantize_mx8(const T* __restrict__ x, long long x_stride, long long pieces,
                                                      int per_row, uint8_t* __restrict__ codes,
                                                      uint8_t* __restrict__ scales, int k_tiles) {
  jk_pdl_wait();
  jk_pdl_trigger();
  const long long step = (long long)gridDim.x * blockDim.x;
  for (long long i0 = (long long)blockIdx.x * blockDim.x; i0 < pieces; i0 += step) {
    const long long i = i0 + threadIdx.x;
    const bool live = i < pieces;
    const long long row = live ? i / per_row : 0;
    const int c = live ? (int)(i - row * per_row) * 8 : 0;
    piece<T> a;
    float v[8];
    if (live) a.load(x + row * x_stride + c);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = live ? a.at(j) : 0.f;
    mx_store_piece(v, live, codes + row * (long long)per_row * 8 + c, scales + mx_scale_at(row, c >> 5, k_tiles));
  }
}

// ------------------------------------------------------------------------------------------ host side
extern "C" int64_t jk_row_scale_bytes(int64_t rows, int64_t n) {
  if (rows < 1 || rows > (1 << 24) || n < MX_BLOCK || n > (1 << 20) || n % MX_BLOCK) return 0;
  return (rows + 127) / 128 * mx_k_tiles(n) * MX_TILE_BYTES;
}

// Pieces a thread holds: 1 up to n = 2048, 2 up to 8192, 4 beyond; past 16384, where a block has 1024 threads, one
// row at a time (two do not fit the registers).  As many blocks as are resident: the rows are walked.
template <typename T>
static void launch_norm(cudaStream_t st, int sms, int rows, int n, const void* x, const void* delta, const void* weight,
                        float eps, void* out_sum, void* out, void* codes, uint8_t* scales) {
  const int pieces = n / 8, k_tiles = mx_k_tiles(n);
  const int P = pieces <= 256 ? 1 : pieces <= 1024 ? 2 : 4;
  const int threads = (int)jk_align_up((pieces + P - 1) / P, 32);
  const long long most = (long long)sms * (threads > 512 ? 1 : (P == 4 ? 512 : 1024) / threads);
  auto k = P == 1 ? k_add_norm<T, 1, true> : P == 2 ? k_add_norm<T, 2, true>
           : threads <= 512 ? k_add_norm<T, 4, true> : k_add_norm<T, 4, false>;
  jk_launch_pdl(k, dim3((unsigned)(rows < most ? rows : most)), dim3(threads), 0, st, (const T*)x, (const T*)delta,
                (const T*)weight, rows, n, eps, (T*)out_sum, (T*)out, (uint8_t*)codes, scales, k_tiles);
}

extern "C" int jk_add_norm(jk_ctx* ctx, void* stream, int32_t rows, int32_t n, const void* x, const void* delta,
                           const void* weight, void* out_sum, void* out, void* out_mx8, uint8_t* out_scale) {
  if (!ctx || !x || (!out_sum && !out && !out_mx8) || !out_mx8 != !out_scale) return JK_ERR_NULL;
  if (rows < 1 || rows > (1 << 24) || n < 8 || n > 32768 || n % 8 || (out_mx8 && n % MX_BLOCK)) return JK_ERR_SHAPE;
  const size_t es = jk_elem_size(ctx->cfg.dtype), bytes = (size_t)rows * n * es;
  const void* in[] = {x, delta, weight};
  const size_t in_b[] = {bytes, bytes, (size_t)n * es};
  void* o[] = {out_sum, out, out_mx8, out_scale};
  const size_t o_b[] = {bytes, bytes, (size_t)rows * n,
                        out_mx8 ? (size_t)((rows + 127) / 128) * mx_k_tiles(n) * MX_TILE_BYTES : 0};
  for (int i = 0; i < 3; ++i)
    if (!jk_aligned16(in[i])) return JK_ERR_ALIGN;
  for (int i = 0; i < 4; ++i)
    if (!jk_aligned16(o[i])) return JK_ERR_ALIGN;
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 3; ++j)            // (a row is read whole before it is written, so in place is sound)
      if (jk_overlap(o[i], o_b[i], in[j], in_b[j]) && !(i < 2 && j < 2 && o[i] == in[j])) return JK_ERR_SHAPE;
    for (int j = 0; j < i; ++j)
      if (jk_overlap(o[i], o_b[i], o[j], o_b[j])) return JK_ERR_SHAPE;
  }
  int rc = jk_ensure_device_info(ctx);
  if (rc != JK_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  JK_PROF(ctx, st, JK_ST_NORM);
  if (ctx->cfg.dtype == JK_BF16)
    launch_norm<__nv_bfloat16>(st, ctx->sm_count, rows, n, x, delta, weight, ctx->cfg.rms_eps, out_sum, out, out_mx8, out_scale);
  else
    launch_norm<float>(st, ctx->sm_count, rows, n, x, delta, weight, ctx->cfg.rms_eps, out_sum, out, out_mx8, out_scale);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}

extern "C" int jk_quantize_rows(jk_ctx* ctx, void* stream, int64_t rows, int32_t n, const void* x, int64_t x_stride,
                               void* out, uint8_t* out_scale) {
  if (!ctx || !x || !out || !out_scale) return JK_ERR_NULL;
  const int64_t scale_bytes = jk_row_scale_bytes(rows, n);
  if (!scale_bytes) return JK_ERR_SHAPE;
  if (x_stride == 0) x_stride = n;
  if (x_stride < n || x_stride > ((int64_t)1 << 31)) return JK_ERR_SHAPE;
  const size_t es = jk_elem_size(ctx->cfg.dtype);
  if (!jk_aligned16(x) || !jk_aligned16(out) || !jk_aligned16(out_scale) || (x_stride * es) % 16) return JK_ERR_ALIGN;
  const size_t in_b = ((size_t)(rows - 1) * x_stride + n) * es;
  if (jk_overlap(out, (size_t)rows * n, x, in_b) || jk_overlap(out_scale, scale_bytes, x, in_b) ||
      jk_overlap(out, (size_t)rows * n, out_scale, scale_bytes))
    return JK_ERR_SHAPE;
  int rc = jk_ensure_device_info(ctx);
  if (rc != JK_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const long long pieces = (long long)rows * (n / 8);
  const long long want = (pieces + 255) / 256, most = 8ll * ctx->sm_count;
  const dim3 grid((unsigned)(want < most ? want : most));
  JK_PROF(ctx, st, JK_ST_NORM);
  if (ctx->cfg.dtype == JK_BF16)
    jk_launch_pdl(k_quantize_mx8<__nv_bfloat16>, grid, dim3(256), 0, st, (const __nv_bfloat16*)x, (long long)x_stride,
                  pieces, n / 8, (uint8_t*)out, out_scale, mx_k_tiles(n));
  else
    jk_launch_pdl(k_quantize_mx8<float>, grid, dim3(256), 0, st, (const float*)x, (long long)x_stride, pieces, n / 8,
                  (uint8_t*)out, out_scale, mx_k_tiles(n));
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}
