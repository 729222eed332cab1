// jk_tree_verify_attn_paged: tree-masked attention (arXiv 2502.06282, Sec. 2.1 step 2, mask of Fig. 4) over a
// paged 8-bit KV cache.  Columns of sequence b: full pages (e4m3 codes times a scale per page and kv
// head), the open page's tokens in T, the tree tokens in T.
//
// This file holds the entry point and the CUDA-core kernel (fp32 contexts, and bf16 with the tensor
// path off).  One CTA = (sequence, kv head, 64 query rows, slice of the key range); the partials of
// the slices are merged by the kernel of jk_attn.cu.  Bound by its shared-memory reads, not by HBM.
#include <math.h>

#include "jk_paged.cuh"

#define KA_QB 64
#define KA_KEYS 32

template <int D>
struct ka_smem {
  float q[KA_QB][D];                 // pre-scaled queries
  float o[KA_QB][D];                 // running outputs
  float k[KA_KEYS][D + 4];           // padded rows: conflict-free float4 reads
  float v[KA_KEYS][D];
  float m[KA_QB];
  float l[KA_QB];
  unsigned long long anc[JK_MAX_TREE][2];
};

template <typename T, int D>
__global__ void __launch_bounds__(256) k_paged_attn(
    jk_paged c, int layer, const T* __restrict__ q, const T* __restrict__ k_tree,
    const T* __restrict__ v_tree, long long tsb, long long tsh, const int32_t* __restrict__ parent,
    float scale, int M, int Hq, int Hkv, int n_split, int n_qblk, float* __restrict__ part_o,
    float* __restrict__ part_ml, int32_t* status) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  ka_smem<D>& S = *reinterpret_cast<ka_smem<D>*>(smem_raw);
  constexpr int DPL = D / 32;
  jk_pdl_wait();
  const int split = blockIdx.x % n_split, qblk = blockIdx.x / n_split;
  const int kvh = blockIdx.y, b = blockIdx.z;
  const int G = Hq / Hkv;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ps = c.page_size;
  const int P = c.kv_len[b], nf = P / ps * ps;
  if (P < 0 || P > c.max_pages * ps) {
    if (tid == 0) jk_set_status(status, JK_ERR_BOUNDS);
    return;
  }
  const int Ltot = P + M;
  const int n_rows = G * M;
  const int row0 = qblk * KA_QB;
  const int rows_here = min(KA_QB, n_rows - row0);
  if (tid < M) {
    unsigned long long lo = 0ull, hi = 0ull;
    int n = tid;
    for (int guard = 0; n >= 0 && guard <= JK_MAX_TREE; ++guard) {
      if (n < 64) lo |= 1ull << n; else hi |= 1ull << (n - 64);
      const int p = parent[(size_t)b * M + n];
      n = (p < n) ? p : -1;
    }
    S.anc[tid][0] = lo;
    S.anc[tid][1] = hi;
  }
  for (int idx = tid; idx < KA_QB * D; idx += 256) {
    const int r = idx / D, x = idx % D;
    float v = 0.f;
    if (r < rows_here) {
      const int g = (row0 + r) / M, i = (row0 + r) % M;
      v = jk_to_float(q[(((size_t)b * M + i) * Hq + kvh * G + g) * D + x]) * scale;
    }
    S.q[r][x] = v;
    S.o[r][x] = 0.f;
  }
  if (tid < KA_QB) { S.m[tid] = -INFINITY; S.l[tid] = 0.f; }
  const int n_tiles = (Ltot + KA_KEYS - 1) / KA_KEYS;
  const int tiles_per = (n_tiles + n_split - 1) / n_split;
  const int t0 = split * tiles_per, t1 = min(n_tiles, t0 + tiles_per);
  const size_t open_off = (((size_t)layer * c.max_seqs + b) * Hkv + kvh) * 2 * ps * D;
  const size_t tree_off = (size_t)b * tsb + (size_t)kvh * tsh;
  for (int tile = t0; tile < t1; ++tile) {
    __syncthreads();
    const int key0 = tile * KA_KEYS;
    for (int idx = tid; idx < KA_KEYS * (D / 16); idx += 256) {
      const int j = idx / (D / 16), x = (idx % (D / 16)) * 16;
      const int col = key0 + j;
      float kv[16], vv[16];
      if (col < nf) {
        int page = c.page_table[(size_t)b * c.max_pages + col / ps];
        if (page < 0 || page >= c.n_pages) { jk_set_status(status, JK_ERR_BOUNDS); page = 0; }
        const size_t blk = ((size_t)layer * c.n_pages + page) * Hkv + kvh;
        const size_t at = (blk * ps + col % ps) * D + x;
        const float sk = c.k_scale[blk], sv = c.v_scale[blk];
        const uint4 kw = *reinterpret_cast<const uint4*>((const uint8_t*)c.k_pages + at);
        const uint4 vw = *reinterpret_cast<const uint4*>((const uint8_t*)c.v_pages + at);
        const uint32_t ka[4] = {kw.x, kw.y, kw.z, kw.w}, va[4] = {vw.x, vw.y, vw.z, vw.w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float2 k0 = paged_unpack2(ka[t]), k1 = paged_unpack2(ka[t] >> 16);
          const float2 v0 = paged_unpack2(va[t]), v1 = paged_unpack2(va[t] >> 16);
          kv[4 * t] = k0.x * sk; kv[4 * t + 1] = k0.y * sk;
          kv[4 * t + 2] = k1.x * sk; kv[4 * t + 3] = k1.y * sk;
          vv[4 * t] = v0.x * sv; vv[4 * t + 1] = v0.y * sv;
          vv[4 * t + 2] = v1.x * sv; vv[4 * t + 3] = v1.y * sv;
        }
      } else if (col < P) {
        const size_t at = open_off + (size_t)(col & (2 * ps - 1)) * D + x;
        paged_load16((const T*)c.k_open + at, kv);
        paged_load16((const T*)c.v_open + at, vv);
      } else if (col < Ltot) {
        const size_t at = tree_off + (size_t)(col - P) * D + x;
        paged_load16(k_tree + at, kv);
        paged_load16(v_tree + at, vv);
      } else {
#pragma unroll
        for (int t = 0; t < 16; ++t) { kv[t] = 0.f; vv[t] = 0.f; }
      }
#pragma unroll
      for (int t = 0; t < 16; ++t) { S.k[j][x + t] = kv[t]; S.v[j][x + t] = vv[t]; }
    }
    __syncthreads();
    const int key = key0 + lane;
    for (int r = warp; r < rows_here; r += 8) {
      const int i = (row0 + r) % M;
      bool vis = key < P;
      if (!vis && key < Ltot) vis = (S.anc[i][(key - P) >> 6] >> ((key - P) & 63)) & 1ull;
      float s = 0.f;
#pragma unroll 8
      for (int x = 0; x < D; x += 4) {
        const float4 qv = *reinterpret_cast<const float4*>(&S.q[r][x]);
        const float4 kv = *reinterpret_cast<const float4*>(&S.k[lane][x]);
        s = fmaf(qv.x, kv.x, s); s = fmaf(qv.y, kv.y, s);
        s = fmaf(qv.z, kv.z, s); s = fmaf(qv.w, kv.w, s);
      }
      s = vis ? s : -INFINITY;
      const float m_old = S.m[r];
      const float m_new = fmaxf(m_old, jk_warp_max(s));
      if (m_new == -INFINITY) continue;           // nothing visible yet (warp-uniform)
      const float p = vis ? __expf(s - m_new) : 0.f;
      const float corr = __expf(m_old - m_new);   // 0 when m_old = -inf
      const float psum = jk_warp_sum(p);
      float acc[DPL];
#pragma unroll
      for (int t = 0; t < DPL; ++t) acc[t] = S.o[r][lane * DPL + t] * corr;
#pragma unroll 8
      for (int j = 0; j < KA_KEYS; ++j) {
        const float pj = __shfl_sync(0xffffffffu, p, j);
#pragma unroll
        for (int t = 0; t < DPL; ++t) acc[t] = fmaf(pj, S.v[j][lane * DPL + t], acc[t]);
      }
#pragma unroll
      for (int t = 0; t < DPL; ++t) S.o[r][lane * DPL + t] = acc[t];
      if (lane == 0) { S.m[r] = m_new; S.l[r] = S.l[r] * corr + psum; }
      __syncwarp();
    }
  }
  __syncthreads();
  const size_t n_out = (size_t)gridDim.z * M * Hq;
  for (int idx = tid; idx < rows_here * D; idx += 256) {
    const int r = idx / D, x = idx % D;
    const int g = (row0 + r) / M, i = (row0 + r) % M;
    const size_t orow = ((size_t)b * M + i) * Hq + kvh * G + g;
    part_o[((size_t)split * n_out + orow) * D + x] = S.o[r][x];
    if (x == 0) {
      part_ml[((size_t)split * n_out + orow) * 2] = S.m[r];
      part_ml[((size_t)split * n_out + orow) * 2 + 1] = S.l[r];
    }
  }
}

int jk_attn_combine_launch(jk_ctx* ctx, cudaStream_t st, int n_split, size_t n_out, void* out);

template <typename T, int D>
static int ka_launch(jk_ctx* ctx, cudaStream_t st, const jk_paged* c, int layer, int B, int M, const void* q,
                     const void* kt, const void* vt, int64_t sb, int64_t sh, const int32_t* parent,
                     float scale, void* out) {
  const jk_config& g = ctx->cfg;
  const int n_qblk = (g.n_q_heads / g.n_kv_heads * M + KA_QB - 1) / KA_QB;
  const int base = n_qblk * g.n_kv_heads * B;
  // enough slices to cover the SMs twice, each at least 64 keys long
  int n_split = (2 * ctx->sm_count + base - 1) / base;
  const int by_len = (int)(((int64_t)c->max_pages * c->page_size + M + 63) / 64);
  if (n_split > by_len) n_split = by_len;
  if (n_split > ctx->lay.attn_max_split) n_split = ctx->lay.attn_max_split;
  if (n_split < 1) n_split = 1;
  auto kern = k_paged_attn<T, D>;
  const size_t smem = sizeof(ka_smem<D>);
  JK_CUDA_CHECK(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  JK_PROF(ctx, st, JK_ST_PAGED_ATTN);
  jk_launch_pdl(kern, dim3(n_split * n_qblk, g.n_kv_heads, B), dim3(256), smem, st, *c, layer,
                (const T*)q, (const T*)kt, (const T*)vt, (long long)sb, (long long)sh, parent, scale, M,
                g.n_q_heads, g.n_kv_heads, n_split, n_qblk, (float*)(ctx->ws + ctx->lay.attn_o),
                (float*)(ctx->ws + ctx->lay.attn_ml), (int32_t*)(ctx->ws + ctx->lay.status));
  JK_LAUNCH_CHECK(ctx);
  const int booked = ctx->st_combine;
  ctx->st_combine = JK_ST_PAGED_COMBINE;
  const int rc = jk_attn_combine_launch(ctx, st, n_split, (size_t)B * M * g.n_q_heads, out);
  ctx->st_combine = booked;
  return rc;
}

// jk_paged_tc.cu
int jk_paged_attn_tc(jk_ctx* ctx, cudaStream_t st, const jk_paged* c, int layer, int B, int M, const void* q,
                     const void* kt, const void* vt, int64_t sb, int64_t sh, const int32_t* parent, float scale,
                     void* out);

extern "C" int jk_tree_verify_attn_paged(jk_ctx* ctx, void* stream, const jk_paged* c, int32_t layer,
                                       int32_t batch, int32_t tree_size, const void* q,
                                       const void* k_tree, const void* v_tree, int64_t tree_stride_b,
                                       int64_t tree_stride_h, const int32_t* parent,
                                       float softmax_scale, void* out) {
  int rc = jk_paged_check(ctx, c);
  if (rc != JK_OK) return rc;
  if (!q || !k_tree || !v_tree || !parent || !out) return JK_ERR_NULL;
  const jk_config& g = ctx->cfg;
  if (layer < 0 || layer >= c->n_layers || batch < 1 || tree_size < 1 || !(softmax_scale > 0.f))
    return JK_ERR_SHAPE;
  if (batch > g.max_batch || batch > c->max_seqs || tree_size > g.max_tree) return JK_ERR_CAPACITY;
  if (tree_stride_h < (int64_t)tree_size * g.head_dim ||
      (batch > 1 && tree_stride_b < (int64_t)tree_size * g.head_dim))
    return JK_ERR_SHAPE;
  const void* ptrs[] = {q, k_tree, v_tree, out};
  for (const void* p : ptrs)
    if (!jk_aligned16(p)) return JK_ERR_ALIGN;
  const int es = jk_elem_size(g.dtype);
  if ((tree_stride_b * es) % 16 || (tree_stride_h * es) % 16) return JK_ERR_ALIGN;
  if ((rc = jk_ensure_device_info(ctx)) != JK_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (g.dtype == JK_BF16 && ctx->tensor_path)
    return jk_paged_attn_tc(ctx, st, c, layer, batch, tree_size, q, k_tree, v_tree, tree_stride_b, tree_stride_h,
                            parent, softmax_scale, out);
#define KA_CASE(T, D)                                                                              \
  return ka_launch<T, D>(ctx, st, c, layer, batch, tree_size, q, k_tree, v_tree, tree_stride_b,    \
                         tree_stride_h, parent, softmax_scale, out)
  if (g.dtype == JK_BF16) {
    if (g.head_dim == 128) KA_CASE(__nv_bfloat16, 128);
    KA_CASE(__nv_bfloat16, 64);
  }
  if (g.head_dim == 128) KA_CASE(float, 128);
  KA_CASE(float, 64);
#undef KA_CASE
}
