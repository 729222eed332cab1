// Paged 8-bit KV cache: import of prompts, commit of accepted nodes, and the bookkeeping of its pages
// (fork, free, compact, copy).  No counterpart in arXiv 2502.06282, which keeps one 16-bit cache per
// sequence; jk_paged_commit takes the place of the compaction of Sec. 2.1 step 3.
//
// Every call is a plan followed by the data's movement.  The plan is one block: it checks the whole
// request before it changes anything and leaves its verdict in the cache's scratch array, where the
// kernels behind it find it.  One block is enough for what a plan reads (the table rows of the
// sequences named, for free and compact one pass over the reference counts) and lets it number pages
// by prefix sums, so that results do not depend on timing.  The movement is bound by memory: 16-byte
// accesses, a page's block (page_size * d elements, contiguous on both sides) held in registers
// between its maximum and its rounding, so every element is read once.
#include "jk_paged.cuh"

static inline size_t paged_block_elems(const jk_ctx* ctx, const jk_paged* c) {
  return (size_t)c->page_size * ctx->cfg.head_dim;
}

int jk_paged_check(const jk_ctx* ctx, const jk_paged* c) {
  if (!ctx || !c) return JK_ERR_NULL;
  const void* ptrs[] = {c->k_pages, c->v_pages, c->k_scale, c->v_scale, c->k_open, c->v_open,
                        c->kv_len, c->page_table, c->refcount, c->free_list, c->n_free, c->scratch};
  for (const void* p : ptrs)
    if (!p) return JK_ERR_NULL;
  if (c->n_layers < 1 || c->n_layers > 4096 || c->n_pages < 1 || c->n_pages > PAGED_MAX_POOL)
    return JK_ERR_SHAPE;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
    return JK_ERR_SHAPE;
  if (c->max_seqs < 1 || c->max_seqs > PAGED_MAX_SEQS || c->max_pages < 1 ||
      (int64_t)c->max_pages * c->page_size > (1 << 30) ||
      (int64_t)c->n_layers * c->n_pages > (1ll << 31) - 1)
    return JK_ERR_SHAPE;
  for (int i = 0; i < 6; ++i)
    if (!jk_aligned16(ptrs[i])) return JK_ERR_ALIGN;
  for (int i = 6; i < 12; ++i)
    if ((uintptr_t)ptrs[i] & 3) return JK_ERR_ALIGN;
  if (!ctx->ws) return JK_ERR_WORKSPACE;
  return JK_OK;
}

extern "C" int64_t jk_paged_scratch_ints(int32_t n_pages) {
  return n_pages < 1 || n_pages > PAGED_MAX_POOL ? 0 : PAGED_LISTS + 3ll * n_pages;
}

// ---------------------------------------------------------------------------- block-wide helpers
#define PLAN_THREADS 1024
#define PLAN_STEPS 8

// Exclusive prefix sum over the block; *total gets the sum.  red: 33 ints of shared memory.
__device__ __forceinline__ int plan_scan(int v, int* red, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();
  if (lane == 31) red[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    const int w = lane < nw ? red[lane] : 0;
    int wi = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, wi, o);
      if (lane >= o) wi += y;
    }
    if (lane < nw) red[lane] = wi - w;
    if (lane == 31) red[32] = wi;
  }
  __syncthreads();
  *total = red[32];
  return red[warp] + incl - v;
}

// The verdict every later kernel of the call reads.  Called by all threads of the plan's block.
__device__ __forceinline__ void plan_verdict(const jk_paged& c, int32_t* status, int bad, int error) {
  if (threadIdx.x == 0) {
    c.scratch[PAGED_OK] = bad ? 0 : 1;
    if (bad) jk_set_status(status, error);
  }
}

// ---------------------------------------------------------------------------- quantisation
// Largest finite |x| of raw 16-byte pieces.  bf16: as 16-bit integers, two at a time; only where an infinity or a
// NaN shows are the elements looked at one by one.
template <typename T, int N> __device__ __forceinline__ float paged_max(const uint4 (&r)[N]) {
  float amax = 0.f;
  if (sizeof(T) == 2) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      m = __vmaxu2(m, r[i].x & 0x7fff7fffu);
      m = __vmaxu2(m, r[i].y & 0x7fff7fffu);
      m = __vmaxu2(m, r[i].z & 0x7fff7fffu);
      m = __vmaxu2(m, r[i].w & 0x7fff7fffu);
    }
    const uint32_t top = max(m & 0xffffu, m >> 16);
    amax = __uint_as_float(top << 16);
    if (top >= 0x7f80u) {
      amax = 0.f;
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        uint4 q = r[0];
#pragma unroll
        for (int j = 1; j < N; ++j)
          if (i == j) q = r[j];
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          amax = fmaxf(amax, fmaxf(paged_mag(__uint_as_float(w[j] << 16)), paged_mag(__uint_as_float(w[j] & 0xffff0000u))));
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      amax = fmaxf(fmaxf(fmaxf(amax, paged_mag(__uint_as_float(r[i].x))), fmaxf(paged_mag(__uint_as_float(r[i].y)),
                   paged_mag(__uint_as_float(r[i].z)))), paged_mag(__uint_as_float(r[i].w)));
  }
  return amax;
}
// 4 codes of 4 elements from element 4 k of raw pieces on
template <typename T, int N> __device__ __forceinline__ uint32_t paged_codes(const uint4* r, int k, float inv) {
  float v[4];
  if (sizeof(T) == 2) {
    const uint4 q = r[k >> 1];
    const uint32_t a = k & 1 ? q.z : q.x, b = k & 1 ? q.w : q.y;
    v[0] = __uint_as_float(a << 16); v[1] = __uint_as_float(a & 0xffff0000u);
    v[2] = __uint_as_float(b << 16); v[3] = __uint_as_float(b & 0xffff0000u);
  } else {
    const uint4 q = r[k];
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
  }
  return paged_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
}

// `tpu` threads (16 .. 256, a power of two) quantise one block of tpu * 64 elements: each holds four
// runs of 16 elements, as they are in memory, from their load to their rounding: held as floats, bf16 took twice the
// registers, and an SM held two thread blocks instead of four.  Threads of inactive units take part in the
// barriers.  red: 8 floats.
template <typename T>
__device__ __forceinline__ void paged_load_block(const T* src, int t, int tpu, uint4 (&raw)[4 * sizeof(T)]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < (int)sizeof(T); ++j)
      raw[i * sizeof(T) + j] = __ldcs(reinterpret_cast<const uint4*>(src + (size_t)(i * tpu + t) * 16) + j);
}
template <typename T>
__device__ __forceinline__ void paged_quantise(const uint4 (&raw)[4 * sizeof(T)], uint8_t* dst, float* scale, int t, int tpu,
                                               bool active, float* red) {
  constexpr int RUN = sizeof(T);                         // pieces of 16 elements
  float amax = active ? paged_max<T>(raw) : 0.f;
  const int lanes = tpu < 32 ? tpu : 32;
  for (int o = lanes >> 1; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (tpu > 32) {
    const int warp = threadIdx.x >> 5, wpu = tpu >> 5;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[warp] = amax;
    __syncthreads();
    const int w0 = warp / wpu * wpu;
    for (int w = 0; w < wpu; ++w) amax = fmaxf(amax, red[w0 + w]);
  }
  if (!active) return;
  const int e = paged_scale_exp(amax);
  const float inv = paged_pow2(-e);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4* r = raw + i * RUN;
    uint4 o;
    o.x = paged_codes<T, RUN>(r, 0, inv);
    o.y = paged_codes<T, RUN>(r, 1, inv);
    o.z = paged_codes<T, RUN>(r, 2, inv);
    o.w = paged_codes<T, RUN>(r, 3, inv);
    __stcs(reinterpret_cast<uint4*>(dst + (size_t)(i * tpu + t) * 16), o);
  }
  if (t == 0) *scale = paged_pow2(e);
}

// ---------------------------------------------------------------------------- import, commit: plan
// One request per sequence i: row r, pages [from, to) of it have to exist and be its own.
// import: r = seqs[i], [0, n_tokens / ps), nothing may lie behind.  commit: r = i, the pages that
// tokens kv_len - 1 - n_acc .. kv_len - 1 complete.
__global__ void __launch_bounds__(PLAN_THREADS) k_paged_plan(
    jk_paged c, int batch, const int32_t* __restrict__ seqs, const int32_t* __restrict__ n_tokens,
    int src_rows, const int32_t* __restrict__ n_acc, const int32_t* __restrict__ acc_idx,
    int max_depth, int M, int32_t* status) {
  __shared__ int s_row[PAGED_MAX_SEQS], s_from[PAGED_MAX_SEQS], s_to[PAGED_MAX_SEQS], s_miss[PAGED_MAX_SEQS];
  __shared__ int s_seen[PAGED_MAX_SEQS];
  __shared__ int red[33];
  __shared__ int s_bad;
  jk_pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cap = c.max_pages * c.page_size;
  const bool import = n_tokens != nullptr;
  for (int i = tid; i < PAGED_MAX_SEQS; i += PLAN_THREADS) s_seen[i] = 0;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  if (tid < batch) {
    int row = tid, from = 0, to = 0;
    bool bad = false;
    if (import) {
      row = seqs ? seqs[tid] : tid;
      const int n = n_tokens[tid];
      bad = row < 0 || row >= c.max_seqs || n < 0 || n > src_rows || n > cap;
      if (!bad) {
        bad = atomicExch(&s_seen[row], 1) != 0;
        to = n / c.page_size;
      }
    } else {
      const int n = n_acc[tid], len = c.kv_len[tid];
      if (n >= 0) {
        bad = n > max_depth || n >= M || len > cap || len <= n;
        if (!bad) {
          for (int j = 0; j < n; ++j) {
            const int a = acc_idx[(size_t)tid * max_depth + j];
            bad |= a < 0 || a >= M;
          }
          from = (len - 1 - n) / c.page_size;
          to = len / c.page_size;
        }
      }
    }
    if (bad) { s_bad = 1; row = 0; from = to = 0; }
    s_row[tid] = row; s_from[tid] = from; s_to[tid] = to;
  }
  __syncthreads();
  // pages that are there have to be this row's alone; count those that are not
  for (int i = warp; i < batch; i += PLAN_THREADS / 32) {
    const int32_t* tab = c.page_table + (size_t)s_row[i] * c.max_pages;
    const int end = import ? c.max_pages : s_to[i];
    int miss = 0;
    bool bad = false;
    for (int t = s_from[i] + lane; t < end; t += 32) {
      const int e = tab[t];
      if (t >= s_to[i]) bad |= e >= 0;
      else if (e < 0) ++miss;
      else bad |= e >= c.n_pages || c.refcount[e] != 1;
    }
    for (int o = 16; o > 0; o >>= 1) miss += __shfl_xor_sync(0xffffffffu, miss, o);
    if (bad) s_bad = 1;
    if (lane == 0) s_miss[i] = miss;
  }
  __syncthreads();
  int total;
  const int base = plan_scan(tid < batch ? s_miss[tid] : 0, red, &total);
  if (tid < batch) s_miss[tid] = base;
  const int n_free = *c.n_free;
  const int bad = s_bad;
  const bool room = n_free >= total && n_free <= c.n_pages;
  // the ids to be handed out have to be pages
  int wrong = 0;
  if (!bad && room)
    for (int k = tid; k < total; k += PLAN_THREADS) {
      const int e = c.free_list[n_free - 1 - k];
      wrong |= e < 0 || e >= c.n_pages;
    }
  wrong = __syncthreads_or(wrong);
  plan_verdict(c, status, bad || wrong || !room, bad || wrong ? JK_ERR_BOUNDS : JK_ERR_CAPACITY);
  if (bad || wrong || !room) return;
  for (int i = warp; i < batch; i += PLAN_THREADS / 32) {
    int32_t* tab = c.page_table + (size_t)s_row[i] * c.max_pages;
    int at = s_miss[i];
    for (int t0 = s_from[i]; t0 < s_to[i]; t0 += 32) {
      const int t = t0 + lane;
      const bool take = t < s_to[i] && tab[t] < 0;
      const unsigned m = __ballot_sync(0xffffffffu, take);
      if (take) {
        const int e = c.free_list[n_free - 1 - (at + __popc(m & ((1u << lane) - 1u)))];
        tab[t] = e;
        c.refcount[e] = 1;
      }
      at += __popc(m);
    }
    if (import && lane == 0) c.kv_len[s_row[i]] = n_tokens[i];
  }
  if (tid == 0) *c.n_free = n_free - total;
}

// ---------------------------------------------------------------------------- import: movement
// Block (x = (page group, sequence, head), y = (layer, K or V)); the last page group copies the
// tokens behind the last full page to the open rows.
template <typename T>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) k_paged_import(
    jk_paged c, int Hkv, int d, int groups, int first_layer, const int32_t* __restrict__ seqs,
    const int32_t* __restrict__ n_tokens, void* const* __restrict__ k_src,
    void* const* __restrict__ v_src, long long sb, long long sh) {
  __shared__ float red[8];
  jk_pdl_wait();
  jk_pdl_trigger();
  // (what the block needs to know is asked for at once, and the data before the verdict and the page: one after
  // the other these were longer than the movement)
  const int grp = blockIdx.x % groups, bh = blockIdx.x / groups;
  const int i = bh / Hkv, h = bh % Hkv;
  const int layer = first_layer + (blockIdx.y >> 1);
  const bool is_v = blockIdx.y & 1;
  const int ok = c.scratch[PAGED_OK], n = n_tokens[i];
  const int row = seqs ? seqs[i] : i;
  const T* src = (const T*)(is_v ? v_src : k_src)[blockIdx.y >> 1] + (size_t)i * sb + (size_t)h * sh;
  if (!ok) return;
  const int ps = c.page_size, nf = n / ps;
  if (grp == groups - 1) {
    T* dst = (T*)(is_v ? c.v_open : c.k_open) +
             ((((size_t)layer * c.max_seqs + row) * Hkv + h) * 2 * ps + (size_t)(nf & 1) * ps) * d;
    const uint4* s4 = reinterpret_cast<const uint4*>(src + (size_t)nf * ps * d);
    const int n16 = (n - nf * ps) * d * (int)sizeof(T) / 16;
    for (int k = threadIdx.x; k < n16; k += 256) reinterpret_cast<uint4*>(dst)[k] = s4[k];
    return;
  }
  const int be = ps * d, tpu = be / 64, upb = 256 / tpu;
  const int t = grp * upb + (int)threadIdx.x / tpu;
  if (grp * upb >= nf) return;
  const bool active = t < nf;
  uint4 raw[4 * sizeof(T)] = {};
  if (active) paged_load_block<T>(src + (size_t)t * be, threadIdx.x & (tpu - 1), tpu, raw);
  const int page = active ? c.page_table[(size_t)row * c.max_pages + t] : 0;
  const size_t blk = ((size_t)layer * c.n_pages + page) * Hkv + h;
  paged_quantise<T>(raw, (uint8_t*)(is_v ? c.v_pages : c.k_pages) + blk * be, (is_v ? c.v_scale : c.k_scale) + blk,
                    threadIdx.x & (tpu - 1), tpu, active, red);
}

// ---------------------------------------------------------------------------- commit: movement
// Block (x = (sequence, head), y = layer), K and V: the new rows join the open rows, then the pages
// they complete are quantised from there.  At most 17 new rows: at most two pages.  Bound by latency: what a
// block needs to know is asked for at once, the rows behind it, and the grid is a few blocks per SM.
template <typename T>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) k_paged_commit(
    jk_paged c, int Hkv, int d, void* const* __restrict__ k_tree, void* const* __restrict__ v_tree,
    long long sb, long long sh, const int32_t* __restrict__ n_acc, const int32_t* __restrict__ acc_idx,
    int max_depth) {
  __shared__ float red[8];
  __shared__ int s_node[33];
  jk_pdl_wait();
  jk_pdl_trigger();
  const int b = blockIdx.x / Hkv, h = blockIdx.x % Hkv, tid = threadIdx.x;
  const int layer = blockIdx.y;
  const int ok = c.scratch[PAGED_OK], n = n_acc[b], len = c.kv_len[b];
  const T* ksrc = (const T*)k_tree[layer] + (size_t)b * sb + (size_t)h * sh;
  const T* vsrc = (const T*)v_tree[layer] + (size_t)b * sb + (size_t)h * sh;
  if (tid <= max_depth && tid < 33) s_node[tid] = tid == 0 ? 0 : acc_idx[(size_t)b * max_depth + tid - 1];
  if (!ok || n < 0) return;
  __syncthreads();
  const int ps = c.page_size, old = len - 1 - n;
  const size_t at_open = (((size_t)layer * c.max_seqs + b) * Hkv + h) * 2 * ps * d;
  T* kopen = (T*)c.k_open + at_open;
  T* vopen = (T*)c.v_open + at_open;
  const int row16 = d * (int)sizeof(T) / 16, half = (n + 1) * row16;
#pragma unroll 2
  for (int k = tid; k < 2 * half; k += 256) {
    const bool is_v = k >= half;
    const int e = is_v ? k - half : k, j = e / row16, p = e % row16;
    const int at = (old + j) & (2 * ps - 1);
    reinterpret_cast<uint4*>((is_v ? vopen : kopen) + (size_t)at * d)[p] =
        reinterpret_cast<const uint4*>((is_v ? vsrc : ksrc) + (size_t)s_node[j] * d)[p];
  }
  const int t0 = old / ps, units = 2 * (len / ps - t0);     // (page, K or V)
  if (units == 0) return;
  __syncthreads();
  const int be = ps * d, tpu = be / 64, upb = 256 / tpu;
  for (int u0 = 0; u0 < units; u0 += upb) {
    const int u = u0 + tid / tpu, t = t0 + (u >> 1);
    const bool active = u < units, is_v = u & 1;
    uint4 raw[4 * sizeof(T)] = {};
    if (active) paged_load_block<T>((is_v ? vopen : kopen) + (size_t)(t & 1) * be, tid & (tpu - 1), tpu, raw);
    const int page = active ? c.page_table[(size_t)b * c.max_pages + t] : 0;
    const size_t blk = ((size_t)layer * c.n_pages + page) * Hkv + h;
    paged_quantise<T>(raw, (uint8_t*)(is_v ? c.v_pages : c.k_pages) + blk * be, (is_v ? c.v_scale : c.k_scale) + blk,
                      tid & (tpu - 1), tpu, active, red);
  }
}

// ---------------------------------------------------------------------------- fork
__global__ void __launch_bounds__(PLAN_THREADS) k_paged_fork_plan(jk_paged c, int n,
                                                                const int32_t* __restrict__ src,
                                                                const int32_t* __restrict__ dst,
                                                                int32_t* status) {
  __shared__ int s_dst[PAGED_MAX_SEQS];
  jk_pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < PAGED_MAX_SEQS; i += PLAN_THREADS) s_dst[i] = 0;
  __syncthreads();
  int bad = 0, from = -1;
  if (tid < n) {
    from = src[tid];
    const int to = dst[tid];
    bad = from < 0 || from >= c.max_seqs || to < 0 || to >= c.max_seqs;
    if (!bad) bad = atomicExch(&s_dst[to], 1) != 0;
  }
  bad = __syncthreads_or(bad);
  if (!bad && tid < n) {
    const int len = c.kv_len[from];
    bad = s_dst[from] || len < 0 || len > c.max_pages * c.page_size || c.kv_len[dst[tid]] != 0;
  }
  bad = __syncthreads_or(bad);
  if (!bad)
    for (int i = warp; i < n; i += PLAN_THREADS / 32) {
      const int nf = c.kv_len[src[i]] / c.page_size;
      const int32_t* ts = c.page_table + (size_t)src[i] * c.max_pages;
      const int32_t* td = c.page_table + (size_t)dst[i] * c.max_pages;
      for (int t = lane; t < c.max_pages; t += 32) {
        bad |= td[t] >= 0;
        if (t < nf) bad |= ts[t] < 0 || ts[t] >= c.n_pages || c.refcount[ts[t]] < 1;
      }
    }
  bad = __syncthreads_or(bad);
  plan_verdict(c, status, bad, JK_ERR_BOUNDS);
  if (!bad && tid < n) c.kv_len[dst[tid]] = c.kv_len[from];
}

// Block (i, 0): table row and reference counts (integer atomics: any order gives the same).
// Block (i, 1 + (layer, K or V)): the open rows.
__global__ void __launch_bounds__(256) k_paged_fork(jk_paged c, int Hkv, int row_bytes,
                                                  const int32_t* __restrict__ src,
                                                  const int32_t* __restrict__ dst) {
  jk_pdl_wait();
  jk_pdl_trigger();
  if (!c.scratch[PAGED_OK]) return;
  const int from = src[blockIdx.x], to = dst[blockIdx.x];
  const int len = c.kv_len[from], ps = c.page_size, nf = len / ps;
  if (blockIdx.y == 0) {
    for (int t = threadIdx.x; t < nf; t += 256) {
      const int e = c.page_table[(size_t)from * c.max_pages + t];
      c.page_table[(size_t)to * c.max_pages + t] = e;
      atomicAdd(&c.refcount[e], 1);
    }
    return;
  }
  const int y = blockIdx.y - 1, layer = y >> 1;
  char* base = (char*)((y & 1) ? c.v_open : c.k_open);
  const size_t seq_bytes = (size_t)Hkv * 2 * ps * row_bytes;
  const char* s = base + ((size_t)layer * c.max_seqs + from) * seq_bytes;
  char* o = base + ((size_t)layer * c.max_seqs + to) * seq_bytes;
  const int head16 = (len - nf * ps) * row_bytes / 16;            // live 16-byte pieces per head
  const size_t off = (size_t)(nf & 1) * ps * row_bytes;
  const int total = head16 * Hkv;
#pragma unroll 4
  for (int k = threadIdx.x; k < total; k += 256) {
    const int h = k / head16, p = k - h * head16;
    const size_t at = (size_t)h * 2 * ps * row_bytes + off + (size_t)p * 16;
    *reinterpret_cast<uint4*>(o + at) = *reinterpret_cast<const uint4*>(s + at);
  }
}

// ---------------------------------------------------------------------------- free
__global__ void __launch_bounds__(PLAN_THREADS) k_paged_free(jk_paged c, int n,
                                                           const int32_t* __restrict__ seqs,
                                                           int32_t* status) {
  __shared__ int s_seen[PAGED_MAX_SEQS];
  __shared__ int red[33];
  jk_pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int32_t* mark = c.scratch + PAGED_LISTS;
  for (int i = tid; i < PAGED_MAX_SEQS; i += PLAN_THREADS) s_seen[i] = 0;
  for (int i = tid; i < c.n_pages; i += PLAN_THREADS) mark[i] = 0;
  __syncthreads();
  int bad = 0;
  if (tid < n) {
    const int r = seqs[tid];
    bad = r < 0 || r >= c.max_seqs;
    if (!bad) bad = atomicExch(&s_seen[r], 1) != 0;
  }
  const int n_free = *c.n_free;
  bad |= n_free < 0 || n_free > c.n_pages;
  bad = __syncthreads_or(bad);
  if (!bad)
    for (int i = warp; i < n; i += PLAN_THREADS / 32) {
      const int32_t* tab = c.page_table + (size_t)seqs[i] * c.max_pages;
      for (int t = lane; t < c.max_pages; t += 32) {
        const int e = tab[t];
        // marks count how often a page is named, so that a count too low is seen before any change
        if (e >= c.n_pages) bad = 1;
        else if (e >= 0) bad |= atomicAdd(&mark[e], 1) >= c.refcount[e];
      }
    }
  bad = __syncthreads_or(bad);
  plan_verdict(c, status, bad, JK_ERR_BOUNDS);
  if (bad) return;
  for (int i = warp; i < n; i += PLAN_THREADS / 32) {
    const int r = seqs[i];
    int32_t* tab = c.page_table + (size_t)r * c.max_pages;
    for (int t = lane; t < c.max_pages; t += 32) tab[t] = -1;
    if (lane == 0) c.kv_len[r] = 0;
  }
  // pages whose count the marks use up go to the free list, ascending
  // (PLAN_STEPS times the block's pages are looked at together: most of a large pool is not concerned)
  int at = n_free;
  for (int i0 = 0; i0 < c.n_pages; i0 += PLAN_STEPS * PLAN_THREADS) {
    int named[PLAN_STEPS], any = 0;
#pragma unroll
    for (int s = 0; s < PLAN_STEPS; ++s) {
      const int e = i0 + s * PLAN_THREADS + tid;
      named[s] = e < c.n_pages ? mark[e] : 0;
      any |= named[s];
    }
    if (!__syncthreads_or(any)) continue;
#pragma unroll
    for (int s = 0; s < PLAN_STEPS; ++s) {
      const int e = i0 + s * PLAN_THREADS + tid;
      if (e - tid >= c.n_pages) break;
      int empty = 0;
      if (named[s] > 0) {
        const int left = c.refcount[e] - named[s];
        c.refcount[e] = left;
        empty = left == 0;
      }
      if (!__syncthreads_or(empty)) continue;
      int total;
      const int k = plan_scan(empty, red, &total);
      if (empty && at + k < c.n_pages) c.free_list[at + k] = e;
      at += total;
    }
  }
  if (tid == 0) *c.n_free = at < c.n_pages ? at : c.n_pages;
}

// ---------------------------------------------------------------------------- compact, copy
__global__ void __launch_bounds__(PLAN_THREADS) k_paged_compact_plan(jk_paged c, int32_t* n_moved) {
  __shared__ int red[33];
  jk_pdl_wait();
  const int tid = threadIdx.x;
  int32_t* map = c.scratch + PAGED_LISTS;
  int32_t* from = map + c.n_pages;
  int32_t* to = from + c.n_pages;
  int mine = 0, live;
#pragma unroll 8
  for (int e = tid; e < c.n_pages; e += PLAN_THREADS) {
    mine += c.refcount[e] > 0;
    map[e] = e;
  }
  plan_scan(mine, red, &live);
  int holes = 0, movers = 0;
  for (int e0 = 0; e0 < c.n_pages; e0 += PLAN_STEPS * PLAN_THREADS) {
    unsigned kind = 0u;                                  // two bits a step: hole, mover
#pragma unroll
    for (int s = 0; s < PLAN_STEPS; ++s) {
      const int e = e0 + s * PLAN_THREADS + tid;
      const bool used = e < c.n_pages && c.refcount[e] > 0;
      kind |= (unsigned)((e < live && !used) | (e >= live && used) << 1) << (2 * s);
    }
    if (!__syncthreads_or(kind != 0u)) continue;
    for (int s = 0; s < PLAN_STEPS; ++s) {
      if (e0 + s * PLAN_THREADS >= c.n_pages) break;
      const int e = e0 + s * PLAN_THREADS + tid, hole = (kind >> (2 * s)) & 1u, mover = (kind >> (2 * s + 1)) & 1u;
      if (!__syncthreads_or(hole | mover)) continue;
      int th, tm;
      const int kh = plan_scan(hole, red, &th);
      const int km = plan_scan(mover, red, &tm);
      if (hole) to[holes + kh] = e;
      if (mover) from[movers + km] = e;
      holes += th;
      movers += tm;
    }
  }
  __syncthreads();
  for (int i = tid; i < movers; i += PLAN_THREADS) {
    const int s = from[i], d = to[i];
    c.refcount[d] = c.refcount[s];
    c.refcount[s] = 0;
    map[s] = d;
  }
  for (int i = tid; i < c.n_pages - live; i += PLAN_THREADS) c.free_list[i] = c.n_pages - 1 - i;
  if (tid == 0) {
    *c.n_free = c.n_pages - live;
    c.scratch[PAGED_OK] = 1;
    c.scratch[PAGED_N_MOVED] = movers;
    if (n_moved) *n_moved = movers;
  }
}

// A list for jk_paged_copy: ids in range, no destination twice and, within one pool, none that is
// also a source (blocks copy in any order).
__global__ void __launch_bounds__(PLAN_THREADS) k_paged_copy_plan(jk_paged src, jk_paged dst, int same, int n,
                                                                const int32_t* __restrict__ src_ids,
                                                                const int32_t* __restrict__ dst_ids,
                                                                int32_t* status) {
  jk_pdl_wait();
  const int tid = threadIdx.x;
  int32_t* mark = dst.scratch + PAGED_LISTS;
  for (int i = tid; i < n; i += PLAN_THREADS) {
    const int d = dst_ids[i];
    if (d >= 0 && d < dst.n_pages) mark[d] = 0;
    if (same && src_ids[i] >= 0 && src_ids[i] < dst.n_pages) mark[src_ids[i]] = 0;
  }
  __syncthreads();
  int bad = 0;
  for (int i = tid; i < n; i += PLAN_THREADS) {
    const int d = dst_ids[i], s = src_ids[i];
    bad |= s < 0 || s >= src.n_pages || d < 0 || d >= dst.n_pages;
    if (d >= 0 && d < dst.n_pages) bad |= atomicExch(&mark[d], 1) != 0;
  }
  __syncthreads();
  if (same)
    for (int i = tid; i < n; i += PLAN_THREADS) {
      const int s = src_ids[i];
      if (s >= 0 && s < src.n_pages) bad |= mark[s] != 0;
    }
  bad = __syncthreads_or(bad);
  plan_verdict(dst, status, bad, JK_ERR_BOUNDS);
}

// Pages from[i] -> to[i] of all layers, K and V, in pieces of 16 KB dealt over the grid; with `rename`
// (compaction) the table entries too.  Sources and destinations are disjoint.
__global__ void __launch_bounds__(256) k_paged_move(jk_paged src, jk_paged dst, int Hkv, int page_bytes, int n,
                                                  const int32_t* __restrict__ from,
                                                  const int32_t* __restrict__ to, int rename) {
  jk_pdl_wait();
  jk_pdl_trigger();
  if (!dst.scratch[PAGED_OK]) return;
  const int tid = threadIdx.x;
  if (rename) {
    n = dst.scratch[PAGED_N_MOVED];
    const int32_t* map = dst.scratch + PAGED_LISTS;
    if (n > 0)
      for (int64_t i = (int64_t)blockIdx.x * 256 + tid; i < (int64_t)dst.max_seqs * dst.max_pages;
           i += (int64_t)gridDim.x * 256) {
        const int e = dst.page_table[i];
        if (e >= 0 && e < dst.n_pages && map[e] != e) dst.page_table[i] = map[e];
      }
  }
  const int pieces = (page_bytes + 16383) / 16384;
  const int64_t items = (int64_t)n * dst.n_layers * 2 * pieces;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int piece = (int)(it % pieces);
    const int64_t rest = it / pieces;
    const int which = (int)(rest & 1);
    const int layer = (int)((rest >> 1) % dst.n_layers);
    const int i = (int)((rest >> 1) / dst.n_layers);
    const size_t ps = (size_t)layer * src.n_pages + from[i], pd = (size_t)layer * dst.n_pages + to[i];
    const int n16 = min(1024, (page_bytes - piece * 16384) / 16);
    const uint4* s4 = reinterpret_cast<const uint4*>((const char*)(which ? src.v_pages : src.k_pages) +
                                                     ps * page_bytes) + piece * 1024;
    uint4* d4 = reinterpret_cast<uint4*>((char*)(which ? dst.v_pages : dst.k_pages) + pd * page_bytes) +
                piece * 1024;
    uint4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (tid + k * 256 < n16) v[k] = __ldcs(s4 + tid + k * 256);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (tid + k * 256 < n16) __stcs(d4 + tid + k * 256, v[k]);
    if (piece == 0)
      for (int h = tid; h < Hkv; h += 256)
        (which ? dst.v_scale : dst.k_scale)[pd * Hkv + h] = (which ? src.v_scale : src.k_scale)[ps * Hkv + h];
  }
}

__global__ void __launch_bounds__(256) k_paged_init(jk_paged c) {
  jk_pdl_wait();
  jk_pdl_trigger();
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)c.max_seqs * c.max_pages; i += step)
    c.page_table[i] = -1;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < c.n_pages; i += step) {
    c.refcount[i] = 0;
    c.free_list[i] = c.n_pages - 1 - (int)i;
  }
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < c.max_seqs; i += step) c.kv_len[i] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *c.n_free = c.n_pages;
}

// ---------------------------------------------------------------------------- entry points
static int32_t* paged_status(jk_ctx* ctx) { return (int32_t*)(ctx->ws + ctx->lay.status); }

extern "C" int jk_paged_init(jk_ctx* ctx, void* stream, const jk_paged* c) {
  int rc = jk_paged_check(ctx, c);
  if (rc != JK_OK) return rc;
  JK_PROF(ctx, (cudaStream_t)stream, JK_ST_PAGED_PLAN);
  jk_launch_pdl(k_paged_init, dim3(148), dim3(256), 0, (cudaStream_t)stream, *c);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}

static int paged_strides(const jk_ctx* ctx, int64_t sb, int64_t sh) {
  const int es = jk_elem_size(ctx->cfg.dtype);
  if (sb < 0 || sh < 0) return JK_ERR_SHAPE;
  return (sb * es) % 16 || (sh * es) % 16 ? JK_ERR_ALIGN : JK_OK;
}

extern "C" int jk_paged_import(jk_ctx* ctx, void* stream, const jk_paged* c, int32_t batch,
                             const int32_t* seqs, const int32_t* n_tokens, int32_t first_layer,
                             int32_t n_layers, void* const* k_src, void* const* v_src, int64_t sb,
                             int64_t sh, int32_t src_rows) {
  int rc = jk_paged_check(ctx, c);
  if (rc != JK_OK) return rc;
  if (!n_tokens || !k_src || !v_src) return JK_ERR_NULL;
  if (batch < 1 || src_rows < 1 || first_layer < 0 || n_layers < 1 ||
      n_layers > c->n_layers - first_layer)
    return JK_ERR_SHAPE;
  if (batch > c->max_seqs) return JK_ERR_CAPACITY;
  const jk_config& g = ctx->cfg;
  if (sh < (int64_t)src_rows * g.head_dim) return JK_ERR_SHAPE;
  if ((rc = paged_strides(ctx, sb, sh)) != JK_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  JK_PROF(ctx, st, JK_ST_PAGED_PLAN);
  jk_launch_pdl(k_paged_plan, dim3(1), dim3(PLAN_THREADS), 0, st, *c, batch, seqs, n_tokens, src_rows,
                (const int32_t*)nullptr, (const int32_t*)nullptr, 0, 0, paged_status(ctx));
  JK_LAUNCH_CHECK(ctx);
  const int upb = 256 / (int)(paged_block_elems(ctx, c) / 64);
  const int groups = (src_rows / c->page_size + upb - 1) / upb + 1;
  const int64_t gx = (int64_t)groups * batch * g.n_kv_heads;
  if (gx > 0x7fffffff) return JK_ERR_SHAPE;
  JK_PROF(ctx, st, JK_ST_PAGED_MOVE);
  if (g.dtype == JK_BF16)
    jk_launch_pdl(k_paged_import<__nv_bfloat16>, dim3((unsigned)gx, 2 * n_layers), dim3(256), 0, st, *c,
                  g.n_kv_heads, g.head_dim, groups, first_layer, seqs, n_tokens, k_src, v_src,
                  (long long)sb, (long long)sh);
  else
    jk_launch_pdl(k_paged_import<float>, dim3((unsigned)gx, 2 * n_layers), dim3(256), 0, st, *c,
                  g.n_kv_heads, g.head_dim, groups, first_layer, seqs, n_tokens, k_src, v_src,
                  (long long)sb, (long long)sh);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}

extern "C" int jk_paged_commit(jk_ctx* ctx, void* stream, const jk_paged* c, int32_t batch,
                             int32_t tree_size, void* const* k_tree, void* const* v_tree, int64_t sb,
                             int64_t sh, const int32_t* n_acc, const int32_t* acc_idx) {
  int rc = jk_paged_check(ctx, c);
  if (rc != JK_OK) return rc;
  if (!k_tree || !v_tree || !n_acc || !acc_idx) return JK_ERR_NULL;
  const jk_config& g = ctx->cfg;
  if (batch < 1 || tree_size < 1) return JK_ERR_SHAPE;
  if (batch > g.max_batch || batch > c->max_seqs || tree_size > g.max_tree) return JK_ERR_CAPACITY;
  if (sh < (int64_t)tree_size * g.head_dim) return JK_ERR_SHAPE;
  if ((rc = paged_strides(ctx, sb, sh)) != JK_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  JK_PROF(ctx, st, JK_ST_PAGED_PLAN);
  jk_launch_pdl(k_paged_plan, dim3(1), dim3(PLAN_THREADS), 0, st, *c, batch, (const int32_t*)nullptr,
                (const int32_t*)nullptr, 0, n_acc, acc_idx, g.max_depth, tree_size, paged_status(ctx));
  JK_LAUNCH_CHECK(ctx);
  JK_PROF(ctx, st, JK_ST_PAGED_MOVE);
  const dim3 grid(batch * g.n_kv_heads, c->n_layers);
  if (g.dtype == JK_BF16)
    jk_launch_pdl(k_paged_commit<__nv_bfloat16>, grid, dim3(256), 0, st, *c, g.n_kv_heads, g.head_dim,
                  k_tree, v_tree, (long long)sb, (long long)sh, n_acc, acc_idx, g.max_depth);
  else
    jk_launch_pdl(k_paged_commit<float>, grid, dim3(256), 0, st, *c, g.n_kv_heads, g.head_dim, k_tree,
                  v_tree, (long long)sb, (long long)sh, n_acc, acc_idx, g.max_depth);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}

extern "C" int jk_paged_fork(jk_ctx* ctx, void* stream, const jk_paged* c, int32_t n, const int32_t* src,
                           const int32_t* dst) {
  int rc = jk_paged_check(ctx, c);
  if (rc != JK_OK) return rc;
  if (!src || !dst) return JK_ERR_NULL;
  if (n < 1) return JK_ERR_SHAPE;
  if (n > c->max_seqs) return JK_ERR_CAPACITY;
  cudaStream_t st = (cudaStream_t)stream;
  JK_PROF(ctx, st, JK_ST_PAGED_PLAN);
  jk_launch_pdl(k_paged_fork_plan, dim3(1), dim3(PLAN_THREADS), 0, st, *c, n, src, dst, paged_status(ctx));
  JK_LAUNCH_CHECK(ctx);
  JK_PROF(ctx, st, JK_ST_PAGED_MOVE);
  jk_launch_pdl(k_paged_fork, dim3(n, 1 + 2 * c->n_layers), dim3(256), 0, st, *c, ctx->cfg.n_kv_heads,
                ctx->cfg.head_dim * jk_elem_size(ctx->cfg.dtype), src, dst);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}

extern "C" int jk_paged_free(jk_ctx* ctx, void* stream, const jk_paged* c, int32_t n, const int32_t* seqs) {
  int rc = jk_paged_check(ctx, c);
  if (rc != JK_OK) return rc;
  if (!seqs) return JK_ERR_NULL;
  if (n < 1) return JK_ERR_SHAPE;
  if (n > c->max_seqs) return JK_ERR_CAPACITY;
  JK_PROF(ctx, (cudaStream_t)stream, JK_ST_PAGED_PLAN);
  jk_launch_pdl(k_paged_free, dim3(1), dim3(PLAN_THREADS), 0, (cudaStream_t)stream, *c, n, seqs,
                paged_status(ctx));
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}

static int paged_move(jk_ctx* ctx, cudaStream_t st, const jk_paged* src, const jk_paged* dst, int n,
                    const int32_t* from, const int32_t* to, int rename) {
  int rc = jk_ensure_device_info(ctx);
  if (rc != JK_OK) return rc;
  JK_PROF(ctx, st, JK_ST_PAGED_MOVE);
  jk_launch_pdl(k_paged_move, dim3(ctx->sm_count * 8), dim3(256), 0, st, *src, *dst, ctx->cfg.n_kv_heads,
                (int)(paged_block_elems(ctx, dst) * ctx->cfg.n_kv_heads), n, from, to, rename);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}

extern "C" int jk_paged_compact(jk_ctx* ctx, void* stream, const jk_paged* c, int32_t* n_moved) {
  int rc = jk_paged_check(ctx, c);
  if (rc != JK_OK) return rc;
  if ((uintptr_t)n_moved & 3) return JK_ERR_ALIGN;
  cudaStream_t st = (cudaStream_t)stream;
  JK_PROF(ctx, st, JK_ST_PAGED_PLAN);
  jk_launch_pdl(k_paged_compact_plan, dim3(1), dim3(PLAN_THREADS), 0, st, *c, n_moved);
  JK_LAUNCH_CHECK(ctx);
  const int32_t* from = c->scratch + PAGED_LISTS + c->n_pages;
  return paged_move(ctx, st, c, c, 0, from, from + c->n_pages, 1);
}

extern "C" int jk_paged_copy(jk_ctx* ctx, void* stream, const jk_paged* src, const jk_paged* dst,
                                 int32_t n, const int32_t* src_ids, const int32_t* dst_ids) {
  int rc = jk_paged_check(ctx, src);
  if (rc == JK_OK) rc = jk_paged_check(ctx, dst);
  if (rc != JK_OK) return rc;
  if (!src_ids || !dst_ids) return JK_ERR_NULL;
  if (n < 1 || src->n_layers != dst->n_layers || src->page_size != dst->page_size) return JK_ERR_SHAPE;
  if (n > dst->n_pages) return JK_ERR_CAPACITY;
  const int same = src->k_pages == dst->k_pages || src->v_pages == dst->v_pages;
  if (same && (src->k_pages != dst->k_pages || src->v_pages != dst->v_pages ||
               src->k_scale != dst->k_scale || src->v_scale != dst->v_scale ||
               src->n_pages != dst->n_pages))
    return JK_ERR_SHAPE;
  if (!same) {
    // (pools that overlap in part: a page may be read here and written there, in any order)
    const size_t heads = (size_t)src->n_layers * ctx->cfg.n_kv_heads, block = paged_block_elems(ctx, src);
    const void* from[] = {src->k_pages, src->v_pages, src->k_scale, src->v_scale};
    const void* to[] = {dst->k_pages, dst->v_pages, dst->k_scale, dst->v_scale};
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const uintptr_t a = (uintptr_t)from[i], b = (uintptr_t)to[j];
        if (a < b + heads * dst->n_pages * (j < 2 ? block : 4) && b < a + heads * src->n_pages * (i < 2 ? block : 4))
          return JK_ERR_SHAPE;
      }
  }
  cudaStream_t st = (cudaStream_t)stream;
  JK_PROF(ctx, st, JK_ST_PAGED_PLAN);
  jk_launch_pdl(k_paged_copy_plan, dim3(1), dim3(PLAN_THREADS), 0, st, *src, *dst, same, n, src_ids,
                dst_ids, paged_status(ctx));
  JK_LAUNCH_CHECK(ctx);
  return paged_move(ctx, st, src, dst, n, src_ids, dst_ids, 0);
}
