// Rotary positions with one or several axes, and the place of K and V (jk_rope_qkv).
//
// Pair (i, i + d/2) of a q or k head turns by pos[axis of i] * theta^(-2i/d).  All heads of a token
// share its d/2 angles: a block takes a few tokens, forms their sines and cosines once in shared memory
// (the angle as a product in 64 bits, reduced to [-pi, pi] there, so that positions of a million
// keep their last bits; sine and cosine of the remainder in 32) and then streams the heads, 16 bytes
// per thread and access.  Bound by memory: every element is read and written once; 2 x 2047 tokens of 96 heads of 128, 201 MB
// in 35.6 us (5.65 TB/s), 4 x 60 tokens 2.8 us.  Four blocks to an SM: more loads in flight for each thread at fewer
// blocks took 44 us.
#include <math.h>

#include "jk_mx8.cuh"

#define ROPE_THREADS 256
#define ROPE_TOKENS 4                      // tokens of a block, at most

struct rope_axes {
  int axis_end[4];                         // frequencies below axis_end[a] (and not below axis_end[a - 1]) turn with axis a
  int n_axes;
};

template <typename T> struct rope_vec;     // 16 bytes of T
template <> struct rope_vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void open(const uint4& r, float (&o)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __uint_as_float(w[i] << 16);
      o[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
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
template <> struct rope_vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void open(const uint4& r, float (&o)[4]) {
    o[0] = __uint_as_float(r.x); o[1] = __uint_as_float(r.y); o[2] = __uint_as_float(r.z); o[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};

// theta^(-2i/d), formed on the host once for each theta
struct rope_freq { double f[64]; };

// The heads that stand side by side in a row: LH lanes turn a head (VN pairs each), a block 256 / LH heads at a time.
template <typename T, int D>
__global__ void __launch_bounds__(ROPE_THREADS, 4) k_rope_qkv(
    const T* __restrict__ qkv, long long row_stride, const int32_t* __restrict__ pos, const rope_axes ax,
    const __grid_constant__ rope_freq freq, int n_tokens, int per_block, int Hq, int Hkv, T* __restrict__ q_out,
    T* __restrict__ k_out, T* __restrict__ v_out, long long sb, long long sh, int rows,
    const int32_t* __restrict__ first_row, int32_t* status) {
  constexpr int VN = rope_vec<T>::N, HALF = D / 2, LH = HALF / VN, HEADS = ROPE_THREADS / LH, UNROLL = 2;
  __shared__ __align__(16) float s_cos[ROPE_TOKENS][HALF], s_sin[ROPE_TOKENS][HALF];
  __shared__ int s_bad[ROPE_TOKENS];
  if (threadIdx.x < ROPE_TOKENS) s_bad[threadIdx.x] = 0;
  __syncthreads();
  // The successor is released when this kernel ends: the tree attention reads committed rows of a cache
  // ahead of its own wait, and a prompt's rows may be committed by what this call writes.
  jk_pdl_wait();
  const int b = blockIdx.y, t0 = blockIdx.x * per_block, nt = min(per_block, n_tokens - t0);
  const size_t tok0 = (size_t)b * n_tokens + t0;
  for (int i = threadIdx.x; i < nt * HALF; i += ROPE_THREADS) {
    const int t = i / HALF, j = i % HALF;
    int a = 0;
    while (a + 1 < ax.n_axes && j >= ax.axis_end[a]) ++a;
    const int p = pos[(tok0 + t) * ax.n_axes + a];
    if (p < 0) s_bad[t] = 1;
    const double ang = (double)p * freq.f[j];
    const double turns = rint(ang * 0.15915494309189535);            // 1 / (2 pi)
    double red = fma(-turns, 6.283185307179586, ang);                // 2 pi, leading part
    red = fma(-turns, 2.4492935982947064e-16, red);                  // 2 pi, the rest
    sincosf((float)red, &s_sin[t][j], &s_cos[t][j]);
  }
  const int r0 = first_row ? first_row[b] : 0;
  const bool fits = r0 >= 0 && r0 <= rows - n_tokens;
  __syncthreads();
  if (threadIdx.x < nt && (s_bad[threadIdx.x] || !fits)) jk_set_status(status, JK_ERR_BOUNDS);
  // (token, head) pairs in one line, 256 / LH at a time
  const int j = threadIdx.x % LH * VN, heads = fits ? Hq + Hkv : Hq;
  int t = 0, h = threadIdx.x / LH;
  while (h >= heads && t < nt) { h -= heads; ++t; }
  while (t < nt) {
    uint4 lo[UNROLL], hi[UNROLL];
    int ts[UNROLL], hs[UNROLL];
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      ts[i] = t;
      hs[i] = h;
      if (t < nt) {
        const T* src = qkv + (tok0 + t) * row_stride + (size_t)h * D + j;
        lo[i] = *reinterpret_cast<const uint4*>(src);
        hi[i] = *reinterpret_cast<const uint4*>(src + HALF);
        h += HEADS;
        while (h >= heads && t < nt) { h -= heads; ++t; }
      }
    }
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      if (ts[i] >= nt || s_bad[ts[i]]) continue;
      float x1[VN], x2[VN], cs[VN], sn[VN], o1[VN], o2[VN];
#pragma unroll
      for (int e = 0; e < VN; e += 4) {
        *reinterpret_cast<float4*>(&cs[e]) = *reinterpret_cast<const float4*>(&s_cos[ts[i]][j + e]);
        *reinterpret_cast<float4*>(&sn[e]) = *reinterpret_cast<const float4*>(&s_sin[ts[i]][j + e]);
      }
      rope_vec<T>::open(lo[i], x1);
      rope_vec<T>::open(hi[i], x2);
#pragma unroll
      for (int e = 0; e < VN; ++e) {
        o1[e] = x1[e] * cs[e] - x2[e] * sn[e];
        o2[e] = x2[e] * cs[e] + x1[e] * sn[e];
      }
      T* dst = hs[i] < Hq ? q_out + ((tok0 + ts[i]) * Hq + hs[i]) * D + j
                          : k_out + (size_t)b * sb + (size_t)(hs[i] - Hq) * sh + (size_t)(r0 + t0 + ts[i]) * D + j;
      rope_vec<T>::store(dst, o1);
      rope_vec<T>::store(dst + HALF, o2);
    }
  }
  if (!fits) return;
  // V moves as it is
  constexpr int DV = D / VN;
  const int per_tok = Hkv * DV;
  for (t = 0; t < nt; ++t) {
    if (s_bad[t]) continue;
    const T* row = qkv + (tok0 + t) * row_stride + (size_t)(Hq + Hkv) * D;
    T* v = v_out + (size_t)b * sb + (size_t)(r0 + t0 + t) * D;
    for (int i0 = threadIdx.x; i0 < per_tok; i0 += ROPE_THREADS * UNROLL) {
      uint4 x[UNROLL];
#pragma unroll
      for (int i = 0; i < UNROLL; ++i)
        if (i0 + i * ROPE_THREADS < per_tok) x[i] = *reinterpret_cast<const uint4*>(row + (size_t)(i0 + i * ROPE_THREADS) * VN);
#pragma unroll
      for (int i = 0; i < UNROLL; ++i) {
        const int at = i0 + i * ROPE_THREADS;
        if (at < per_tok) *reinterpret_cast<uint4*>(v + (size_t)(at / DV) * sh + at % DV * VN) = x[i];
      }
    }
  }
}

// Pieces of `part` bytes lie at i inner + j outer, 0 <= i < ni, 0 <= j < no, with inner >= part and outer >= (ni - 1) inner + part
// where there is more than one: does one of them share a byte with one of those that lie `off` further?  The distance of
// two pieces is off - i inner - j outer with |i| < ni, |j| < no, and only the two multiples next to what is left can come near.
static bool rope_pieces_meet(int64_t off, int64_t part, int64_t inner, int64_t ni, int64_t outer, int64_t no) {
  for (int64_t j = no > 1 ? off / outer : 0, last = j + 1; j <= last && j < no; ++j) {
    const int64_t r = off > j * outer ? off - j * outer : j * outer - off;
    for (int64_t i = ni > 1 ? r / inner : 0, end = i + 1; i <= end && i < ni; ++i)
      if ((r > i * inner ? r - i * inner : i * inner - r) < part) return true;
  }
  return false;
}

extern "C" int jk_rope_qkv(jk_ctx* ctx, void* stream, int32_t batch, int32_t n_tokens, const void* qkv,
                           int64_t row_stride, const int32_t* pos, int32_t n_axes, const int32_t* sections,
                           float theta, void* q_out, void* k_out, void* v_out, int64_t sb, int64_t sh, int32_t rows,
                           const int32_t* first_row) {
  if (!ctx || !qkv || !pos || !sections || !q_out || !k_out || !v_out) return JK_ERR_NULL;
  const jk_config& c = ctx->cfg;
  const int D = c.head_dim, Hq = c.n_q_heads, Hkv = c.n_kv_heads;
  if (batch < 1 || batch > 65535 || n_tokens < 1 || n_tokens > (1 << 20) || rows < n_tokens || n_axes < 1 ||
      n_axes > 4 || !(theta > 0.f) || theta > 3.4e38f)
    return JK_ERR_SHAPE;
  rope_axes ax;
  ax.n_axes = n_axes;
  int64_t sum = 0;
  for (int a = 0; a < 4; ++a) {
    if (a < n_axes && (sections[a] < 0 || sections[a] > D / 2)) return JK_ERR_SHAPE;
    sum += a < n_axes ? sections[a] : 0;
    ax.axis_end[a] = (int)sum;
  }
  if (sum != D / 2) return JK_ERR_SHAPE;
  const int64_t width = (int64_t)(Hq + 2 * Hkv) * D;
  if (row_stride == 0) row_stride = width;
  if (row_stride < width || row_stride > ((int64_t)1 << 31)) return JK_ERR_SHAPE;
  const int64_t part = (int64_t)rows * D;              // heads within a sequence, or sequences within a head
  if (Hkv == 1) sh = part;                             // (the stride of a dimension of one does not count)
  if (batch == 1) sb = Hkv * part;
  if (sh < part || sh > ((int64_t)1 << 40) || sb < 0 || sb > ((int64_t)1 << 40)) return JK_ERR_SHAPE;
  if (batch > 1 && sb < (Hkv - 1) * sh + part && (sb < part || sh < (batch - 1) * sb + part)) return JK_ERR_SHAPE;
  const int es = jk_elem_size(c.dtype);
  const void* ptrs[] = {qkv, q_out, k_out, v_out};
  for (const void* p : ptrs)
    if (!jk_aligned16(p)) return JK_ERR_ALIGN;
  if ((row_stride * es) % 16 || (sb * es) % 16 || (sh * es) % 16) return JK_ERR_ALIGN;
  if (((uintptr_t)pos & 3) || ((uintptr_t)first_row & 3)) return JK_ERR_ALIGN;
  const size_t tokens = (size_t)batch * n_tokens;
  const size_t in_b = ((tokens - 1) * row_stride + width) * es, q_b = tokens * Hq * D * es;
  const size_t kv_b = ((size_t)(batch - 1) * sb + (size_t)(Hkv - 1) * sh + (size_t)rows * D) * es;
  if (jk_overlap(q_out, q_b, qkv, in_b) || jk_overlap(k_out, kv_b, qkv, in_b) || jk_overlap(v_out, kv_b, qkv, in_b) ||
      jk_overlap(q_out, q_b, k_out, kv_b) || jk_overlap(q_out, q_b, v_out, kv_b))
    return JK_ERR_SHAPE;
  // (K and V may be halves of one buffer: their pieces may lie between one another)
  const int64_t kv_off = (int64_t)((uintptr_t)k_out > (uintptr_t)v_out ? (uintptr_t)k_out - (uintptr_t)v_out : (uintptr_t)v_out - (uintptr_t)k_out);
  const bool by_seq = batch == 1 || sb >= (Hkv - 1) * sh + part;
  if (by_seq ? rope_pieces_meet(kv_off, part * es, sh * es, Hkv, sb * es, batch) : rope_pieces_meet(kv_off, part * es, sb * es, batch, sh * es, Hkv))
    return JK_ERR_SHAPE;
  if (!ctx->ws) return JK_ERR_WORKSPACE;
  int32_t* status = (int32_t*)(ctx->ws + ctx->lay.status);
  cudaStream_t st = (cudaStream_t)stream;
  int rc = jk_ensure_device_info(ctx);
  if (rc != JK_OK) return rc;
  if (ctx->rope_theta != theta) {            // (64 powers take longer than a small call)
    for (int j = 0; j < D / 2; ++j) ctx->rope_freq[j] = pow((double)theta, -2.0 * j / D);
    ctx->rope_theta = theta;
  }
  rope_freq freq;
  memset(&freq, 0, sizeof(freq));
  memcpy(freq.f, ctx->rope_freq, sizeof(double) * (D / 2));
  // tokens of a block: as many as leave four blocks to an SM
  long long per = (long long)tokens / (4ll * ctx->sm_count);
  const int per_block = per < 1 ? 1 : per > ROPE_TOKENS ? ROPE_TOKENS : (int)per;
  const dim3 grid((unsigned)((n_tokens + per_block - 1) / per_block), (unsigned)batch);
  JK_PROF(ctx, st, JK_ST_PRE_ROPE);
  auto go = [&](auto kernel, auto tag) {
    typedef decltype(tag) T;
    jk_launch_pdl(kernel, grid, dim3(ROPE_THREADS), 0, st, (const T*)qkv, (long long)row_stride, pos, ax, freq,
                  n_tokens, per_block, Hq, Hkv, (T*)q_out, (T*)k_out, (T*)v_out, (long long)sb, (long long)sh, rows, first_row,
                  status);
  };
  if (c.dtype == JK_BF16) {
    if (D == 128) go(k_rope_qkv<__nv_bfloat16, 128>, __nv_bfloat16());
    else go(k_rope_qkv<__nv_bfloat16, 64>, __nv_bfloat16());
  } else {
    if (D == 128) go(k_rope_qkv<float, 128>, float());
    else go(k_rope_qkv<float, 64>, float());
  }
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}
