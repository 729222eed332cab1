// jk_tree_verify_attn_paged: tree-masked attention (arXiv 2502.06282, Sec. 2.1 step 2, mask of Fig. 4) over a
// paged 8-bit KV cache.  Columns of sequence b: full pages (e4m3 codes times a scale per page and kv
// head), the open page's tokens in T, the tree tokens in T.
//
// This file holds the entry point and the CUDA-core kernel: one query row per kv head, fp32 contexts, and bf16 with the
// tensor path off.
#include <math.h>

#include "jk_paged.cuh"

// A cluster of C blocks per (sequence, kv head, 1 or 4 query rows); one launch, no partials in memory.  A key's D codes lie
// in D / 16 lanes, 16 bytes each, so a warp reads 512 contiguous bytes per access; each such group of lanes goes
// through its own keys, KU at a time (within a page), with its own running maximum, and holds R rows of its 16
// dims of query and output.  What groups, warps and blocks found is merged at the end, in a fixed order.
// Per key and row this takes about 2 instructions per dim on top of 3 to widen the codes of K and V: with one row the
// bytes bound it, with more the instructions.  More than four rows are more clusters, which read the pages again, from
// L2: fp32, 60 rows, prefix 8192, batch 4, 4 heads 220 us (234 without paired multiply-adds); tiles of 64 rows and 32
// keys in shared memory took 458, and were slower at every size from 16 rows on.
#define KR_THREADS 256
#define KR_WARPS (KR_THREADS / 32)
#define KR_CLUSTER 8

// Two multiply-adds in one instruction.
__device__ __forceinline__ float2 kr_fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
// 16 bytes; where they may be missing, zeros if !live (codes of pages that are not the sequence's may be NaN, and a weight of
// 0 does not undo that).
template <bool MISSING> __device__ __forceinline__ uint4 kr_load(const void* p, bool live) {
  uint4 v;
  if constexpr (MISSING)
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %5, 0;\n\t"
                 "mov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t"
                 "@q ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"((uint32_t)live));
  else
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void kr_widen(const uint4& w, float* o) {
  const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = paged_unpack2(a[i]), y = paged_unpack2(a[i] >> 16);
    o[4 * i] = x.x; o[4 * i + 1] = x.y; o[4 * i + 2] = y.x; o[4 * i + 3] = y.y;
  }
}

template <typename T, int D, int R>
__global__ void __launch_bounds__(KR_THREADS, R == 1 ? 2 : 1) k_paged_attn_rows(
    jk_paged c, int layer, const T* __restrict__ q, const T* __restrict__ k_tree, const T* __restrict__ v_tree,
    long long tsb, long long tsh, const int32_t* __restrict__ parent, float scale, int M, int Hq, int Hkv, int C,
    T* __restrict__ out, int32_t* status) {
  constexpr int LPK = D / 16, GR = 32 / LPK, KU = R == 1 ? 8 : 4, STEP = GR * KU;
  constexpr bool ENDS = STEP > 16;       // a step may reach past the last page: pages hold 16 tokens or a multiple
  __shared__ float s_o[KR_WARPS][R][D];
  __shared__ float s_m[KR_WARPS][R], s_l[KR_WARPS][R];
  __shared__ float c_o[KR_CLUSTER][R][D], c_m[KR_CLUSTER][R], c_l[KR_CLUSTER][R];   // of the blocks, in the first one
  __shared__ uint32_t s_anc[R][4];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t rank = 0;
  if (C > 1) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  // (a block's memory may be written once it runs: waited for before that)
  if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  jk_pdl_wait();
  jk_pdl_trigger();
  const int row0 = blockIdx.x / C * R, h = blockIdx.y, b = blockIdx.z;
  const int G = Hq / Hkv, n_rows = G * M, ps = c.page_size;
  const int grp = lane / LPK, x0 = lane % LPK * 16;
  const int W = C * KR_WARPS, gw = (int)rank * KR_WARPS + warp;
  const int32_t* tab = c.page_table + (size_t)b * c.max_pages;
  // length, queries, parents and the first page's id are asked for together: one after the other these trips took longer
  // than a short prefix
  const int P = c.kv_len[b];
  const int t_first = (gw * STEP + grp * KU) / ps, first = t_first < c.max_pages ? tab[t_first] : -1;
  float qf[R][16];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = min(row0 + r, n_rows - 1), g = row / M, i = row % M;
    paged_load16(q + (((size_t)b * M + i) * Hq + h * G + g) * D + x0, qf[r]);
#pragma unroll
    for (int x = 0; x < 16; ++x) qf[r][x] *= scale * 1.4426950408889634f;
  }
  if (tid < R) {
    uint32_t a[4] = {0u, 0u, 0u, 0u};
    int n = min(row0 + tid, n_rows - 1) % M;
    for (int guard = 0; n >= 0 && guard <= JK_MAX_TREE; ++guard) {
#pragma unroll
      for (int w = 0; w < 4; ++w) a[w] |= w == n >> 5 ? 1u << (n & 31) : 0u;
      const int p = parent[(size_t)b * M + n];
      n = p < n ? p : -1;
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) s_anc[tid][w] = a[w];
  }
  if (P < 0 || P > c.max_pages * ps) {                   // (the same for the whole cluster)
    if (tid == 0) jk_set_status(status, JK_ERR_BOUNDS);
    if (C > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    return;
  }
  const int nf = P / ps * ps, n_open = P - nf, tail = n_open + M;
  __syncthreads();
  float acc[R][16], m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int x = 0; x < 16; ++x) acc[r][x] = 0.f;
  }
  // KU keys: scores s (log2, -inf = not seen), values v(u)[16] times sv
  auto take = [&](float (*s)[R], auto value) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float top = m[r];
#pragma unroll
      for (int u = 0; u < KU; ++u) top = fmaxf(top, s[u][r]);
      const float ref = top == -INFINITY ? 0.f : top;
      const float corr = exp2f(m[r] - ref);
      m[r] = top;
      l[r] *= corr;
#pragma unroll
      for (int x = 0; x < 16; ++x) acc[r][x] *= corr;
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        s[u][r] = exp2f(s[u][r] - ref);
        l[r] += s[u][r];
      }
    }
#pragma unroll
    for (int u = 0; u < KU; ++u) {
      float v[16];
      const float sv = value(u, v);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float w = s[u][r] * sv;
#pragma unroll
        for (int x = 0; x < 16; x += 2) {
          const float2 a = kr_fma2(make_float2(w, w), make_float2(v[x], v[x + 1]), make_float2(acc[r][x], acc[r][x + 1]));
          acc[r][x] = a.x;
          acc[r][x + 1] = a.y;
        }
      }
    }
  };
  auto dot = [&](const float* k, float* s) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float2 a = make_float2(0.f, 0.f);
#pragma unroll
      for (int x = 0; x < 16; x += 2) a = kr_fma2(make_float2(qf[r][x], qf[r][x + 1]), make_float2(k[x], k[x + 1]), a);
      s[r] = a.x + a.y;
#pragma unroll
      for (int o = LPK / 2; o > 0; o >>= 1) s[r] += __shfl_xor_sync(0xffffffffu, s[r], o);
    }
  };
  const int n_it = (nf + STEP - 1) / STEP;
  // ------------------------------------------------ pages
  {
    auto page_of = [&](int key, int id) {                // id: the table's entry, if there is such a key
      if (key >= nf) return 0;
      if (id < 0 || id >= c.n_pages) {
        jk_set_status(status, JK_ERR_BOUNDS);
        id = 0;
      }
      return id;
    };
    int next = page_of(gw * STEP + grp * KU, first);
    for (int it = gw; it < n_it; it += W) {
      const int key = it * STEP + grp * KU, id = next;
      const bool live = !ENDS || key < nf;
      const size_t blk = ((size_t)layer * c.n_pages + id) * Hkv + h;
      const size_t at = (blk * ps + (key & (ps - 1))) * D + x0;
      uint4 kw[KU], vw[KU];
#pragma unroll
      for (int u = 0; u < KU; ++u) kw[u] = kr_load<ENDS>((const uint8_t*)c.k_pages + at + (size_t)u * D, live);
#pragma unroll
      for (int u = 0; u < KU; ++u) vw[u] = kr_load<ENDS>((const uint8_t*)c.v_pages + at + (size_t)u * D, live);
      const float sk = live ? c.k_scale[blk] : 0.f, sv = live ? c.v_scale[blk] : 0.f;
      const int key_next = key + W * STEP;
      next = page_of(key_next, key_next < nf ? tab[key_next / ps] : 0);
      float s[KU][R];
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        float k[16];
        kr_widen(kw[u], k);
        dot(k, s[u]);
#pragma unroll
        for (int r = 0; r < R; ++r) s[u][r] = live ? s[u][r] * sk : -INFINITY;
      }
      take(s, [&](int u, float* v) {
        kr_widen(vw[u], v);
        return sv;
      });
    }
  }
  // ------------------------------------------------ the open page's tokens, the tree
  {
    const size_t open_off = (((size_t)layer * c.max_seqs + b) * Hkv + h) * 2 * ps * D + x0;
    const size_t tree_off = (size_t)b * tsb + (size_t)h * tsh + x0;
    const int turn = (gw + W - n_it % W) % W;            // the turns go on where the pages' end
    for (int it = turn; it * STEP < tail; it += W) {
      const int e0 = it * STEP + grp * KU;
      float s[KU][R];
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        const int e = e0 + u, node = e - n_open;
        float k[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) k[x] = 0.f;
        if (e < n_open) paged_load16((const T*)c.k_open + open_off + (size_t)((nf + e) & (2 * ps - 1)) * D, k);
        else if (e < tail) paged_load16(k_tree + tree_off + (size_t)node * D, k);
        dot(k, s[u]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const bool seen = e < n_open || (e < tail && ((s_anc[r][(node >> 5) & 3] >> (node & 31)) & 1u));
          if (!seen) s[u][r] = -INFINITY;
        }
      }
      take(s, [&](int u, float* o) {
        const int e = e0 + u;
        float v[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) v[x] = 0.f;
        if (e < n_open) paged_load16((const T*)c.v_open + open_off + (size_t)((nf + e) & (2 * ps - 1)) * D, v);
        else if (e < tail) paged_load16(v_tree + tree_off + (size_t)(e - n_open) * D, v);
#pragma unroll
        for (int x = 0; x < 16; ++x) o[x] = v[x];
        return 1.f;
      });
    }
  }
  // ------------------------------------------------ groups of a warp, warps of a block, blocks of the cluster
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float top = m[r];
#pragma unroll
    for (int o = LPK; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float corr = m[r] == -INFINITY ? 0.f : exp2f(m[r] - top);
    l[r] *= corr;
#pragma unroll
    for (int o = LPK; o < 32; o <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      acc[r][x] *= corr;
#pragma unroll
      for (int o = LPK; o < 32; o <<= 1) acc[r][x] += __shfl_xor_sync(0xffffffffu, acc[r][x], o);
    }
    if (grp == 0) {
#pragma unroll
      for (int x = 0; x < 16; x += 4)
        *reinterpret_cast<float4*>(&s_o[warp][r][x0 + x]) = make_float4(acc[r][x], acc[r][x + 1], acc[r][x + 2], acc[r][x + 3]);
    }
    if (lane == 0) { s_m[warp][r] = top; s_l[warp][r] = l[r]; }
  }
  __syncthreads();
  if (C > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // every block runs
  for (int i = tid; i < R * D; i += KR_THREADS) {
    const int r = i / D, x = i % D;
    float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < KR_WARPS; ++w) top = fmaxf(top, s_m[w][r]);
#pragma unroll
    for (int w = 0; w < KR_WARPS; ++w) {
      const float f = s_m[w][r] == -INFINITY ? 0.f : exp2f(s_m[w][r] - top);
      sum = fmaf(f, s_l[w][r], sum);
      o = fmaf(f, s_o[w][r][x], o);
    }
    float *po = &c_o[rank][r][x], *pm = &c_m[rank][r], *pl = &c_l[rank][r];
    if (C > 1) { po = jk_cluster_map(po, 0); pm = jk_cluster_map(pm, 0); pl = jk_cluster_map(pl, 0); }
    *po = o;
    if (x == 0) { *pm = top; *pl = sum; }
  }
  if (C > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank != 0) return;                               // (blocks that left before the others made calls in a row 8 % slower)
  } else {
    __syncthreads();
  }
  for (int i = tid; i < R * D; i += KR_THREADS) {
    const int r = i / D, x = i % D, row = row0 + r;
    float top = -INFINITY, sum = 0.f, o = 0.f;
    for (int k = 0; k < C; ++k) top = fmaxf(top, c_m[k][r]);
#pragma unroll 4
    for (int k = 0; k < C; ++k) {
      const float f = c_m[k][r] == -INFINITY ? 0.f : exp2f(c_m[k][r] - top);
      sum = fmaf(f, c_l[k][r], sum);
      o = fmaf(f, c_o[k][r][x], o);
    }
    if (row < n_rows) {
      const int g = row / M, n = row % M;
      out[(((size_t)b * M + n) * Hq + h * G + g) * D + x] = jk_from_float<T>(o / sum);
    }
  }
}

template <typename T, int D, int R>
static int kr_launch(jk_ctx* ctx, cudaStream_t st, const jk_paged* c, int layer, int B, int M, const void* q,
                     const void* kt, const void* vt, int64_t sb, int64_t sh, const int32_t* parent, float scale,
                     void* out) {
  const jk_config& g = ctx->cfg;
  const int n_rb = (g.n_q_heads / g.n_kv_heads * M + R - 1) / R;
  const int64_t base = (int64_t)n_rb * g.n_kv_heads * B;
  const int64_t keys = (int64_t)c->max_pages * c->page_size;
  // one wave of two blocks per SM, 128 keys a block at least: 4 sequences of 2048 with the 7B heads 17.1 us, with
  // two waves 23, with four 34; 8 blocks for 1024 keys 7.4 us, 4 blocks 8.9
  int C = KR_CLUSTER;
  while (C > 1 && (base * C > 2ll * ctx->sm_count || keys / C < 128)) C >>= 1;
  JK_PROF(ctx, st, JK_ST_PAGED_ATTN);
  jk_launch_pdl_cluster(k_paged_attn_rows<T, D, R>, dim3((unsigned)(n_rb * C), g.n_kv_heads, B), dim3(KR_THREADS),
                        (unsigned)C, 0, st, *c, layer, (const T*)q, (const T*)kt, (const T*)vt, (long long)sb,
                        (long long)sh, parent, scale, M, g.n_q_heads, g.n_kv_heads, C, (T*)out,
                        (int32_t*)(ctx->ws + ctx->lay.status));
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
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
  const int rows = g.n_q_heads / g.n_kv_heads * tree_size;
  // One query row per kv head (single tokens without grouped heads): the CUDA cores keep up with the pages, 7B heads,
  // prefix 1024 7.4 us (tensor cores 16.8), 13B heads, batch 16, prefix 4096 122 (141).  More rows take the tensor cores
  // whatever the lengths, which the host does not know.  Both, 8 kv heads of 128, pages of 64, graph replay, CUDA cores
  // (tensor cores), us, by prefix:
  //                        128           512           1024          2048          4096          8192
  //   2 rows, batch 1      8.4 (10.2)    8.7 (10.3)    8.9 (10.8)    10.7 (11.9)   14.3 (12.7)   21.3 (17.1)
  //           batch 4      8.3 (10.5)    9.1 (11.4)    23.7 (15.7)   29.1 (16.9)   40.5 (19.1)   61.5 (24.4)
  //           batch 16     8.6 (16.5)    21.1 (18.2)   28.6 (20.6)   43.2 (25.6)   72.2 (34.9)   129 (53.4)
  //   8 rows, batch 1      8.4 (10.4)    9.0 (10.5)    16.3 (11.0)   19.8 (12.2)   26.7 (12.9)   41.1 (17.4)
  //           batch 16     16.3 (16.7)   26.8 (18.5)   41.3 (20.8)   68.7 (25.5)   124 (35.2)    230 (53.9)
  // 4 rows are within 3 % of 2.  So the tensor cores lose up to 2 us (8 at batch 16, prefix 128) and win up to a factor of 4.
  if (rows > 1 && g.dtype == JK_BF16 && ctx->tensor_path)
    return jk_paged_attn_tc(ctx, st, c, layer, batch, tree_size, q, k_tree, v_tree, tree_stride_b, tree_stride_h,
                            parent, softmax_scale, out);
#define KR_CASE(T, D)                                                                                              \
  return rows == 1 ? kr_launch<T, D, 1>(ctx, st, c, layer, batch, tree_size, q, k_tree, v_tree, tree_stride_b,     \
                                        tree_stride_h, parent, softmax_scale, out)                                 \
                   : kr_launch<T, D, 4>(ctx, st, c, layer, batch, tree_size, q, k_tree, v_tree, tree_stride_b,     \
                                        tree_stride_h, parent, softmax_scale, out)
  if (g.dtype == JK_BF16) {
    if (g.head_dim == 128) KR_CASE(__nv_bfloat16, 128);
    KR_CASE(__nv_bfloat16, 64);
  }
  if (g.head_dim == 128) KR_CASE(float, 128);
  KR_CASE(float, 64);
#undef KR_CASE
}
