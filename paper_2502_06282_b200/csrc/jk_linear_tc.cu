// jk_linear on the tensor cores: out[r, n] = epilogue(sum_k x[r, k] w[n, k]) for bf16 and for 8-bit
// rows with a scale per 32 elements, gated or not.
//
// Weights stand on the 128-row M side of tcgen05.mma and rows of x on N (16 .. 256), so that a call
// of a few rows streams the weights once and wastes nothing on padding.  Both operand types move as the
// same boxes (rows of 128 bytes, 128-byte swizzle): 64 bf16 or 128 codes along k.  8-bit rows use
// kind::mxf8f6f4 with block scales: the scale tiles (128 rows x 4 blocks, 512 bytes) come with the box
// they belong to and are copied to tensor memory by tcgen05.cp ahead of its products.  A gated block
// multiplies the same x box with a tile of w and a tile of w_up into two accumulators.
//
// The k steps of all tiles form one line, dealt out evenly over one CTA per SM: whatever the shape,
// every SM streams the same share of the weights.  A tile that spans CTAs is finished by the CTA that
// has its last k step; the others hand over f32 partials through the workspace.  A CTA works its share
// from the back, so its only unfinished tile comes first and its partial is long there when the
// CTA behind it asks; it waits only for CTAs of lower index, which were launched before it.  Sums
// are formed in the same order on every run.
//
// Roles: warp 0 loads (TMA), warp 1 issues products, warps 2-5 drain accumulators and do the epilogue.  Every
// wait is bounded: after about 2 s it records JK_ERR_TIMEOUT, the CTA lets its copies land, frees its
// tensor memory and returns.
#include <cuda.h>

#include "jk_linear.cuh"
#include "jk_tcgen05.cuh"

int jk_tma_encode_u8(jk_ctx* ctx, CUtensorMap* out, const void* ptr, int rank, const uint64_t* dims,
                     const uint64_t* strides_bytes, const uint32_t* box);
int jk_tma_available(jk_ctx* ctx);

#define LT_M 128                          // weights of a tile
#define LT_BOX 128                        // bytes of a box row
#define LT_THREADS 192
#define LT_MAX_STAGES 12
#define LT_SMEM (224 * 1024)
#define LT_ACC_COLS 256                   // columns of the accumulators of one tile, at most
#define LT_MAX_CTAS 192
#define LT_SLOT (LT_ACC_COLS * LT_M)      // floats of a partial

size_t jk_linear_part_bytes() { return (size_t)LT_MAX_CTAS * LT_SLOT * sizeof(float); }
size_t jk_linear_flag_bytes() { return LT_MAX_CTAS * sizeof(int32_t); }

struct lt_params {
  int nt;                                 // rows of a tile of x, a multiple of 16
  int r_tiles, w_tiles;
  int boxes;                              // boxes along k
  int subs;                               // products along k (16 bf16 or 32 codes each)
  int kb;                                 // boxes of a stage
  int ks;                                 // stages along k
  int stages, stage_bytes;
  int a_box, b_box;                       // bytes of a box of weights and of x
  int bufs;                               // accumulator buffers: 2, or 1 where two do not fit
  int tmem_cols, sf_col;                  // columns held, first column of the scales
  int sfb;                                // scale tiles of a tile of x (8-bit rows)
  int stream;                             // 1: weights are read once, L2 need not keep them
  long long units;                        // stages of all tiles
};

struct __align__(16) lt_tail {
  uint64_t full[LT_MAX_STAGES], empty[LT_MAX_STAGES];
  uint64_t acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort_flag;
  unsigned done, seen;                    // epilogue warps that handed over their partials / have added up others'
};

// ------------------------------------------------------------------------------------------ PTX
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void l2_prefetch_box(const CUtensorMap* map, int x, int y) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
// D[tmem] (+)= A[smem] B[smem]^T over 32 codes along k, each operand's block scale from tensor memory
__device__ __forceinline__ void tc_mma_mx8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}
// 512 bytes of shared memory, 32 rows of 16, to 4 columns of tensor memory, the same for all four quarters of the lanes
__device__ __forceinline__ void tc_copy_scales(uint32_t dst, uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(128 >> 4) << 32;                       // groups of 8 rows are 128 bytes apart
  d |= (uint64_t)1 << 46;                                // no swizzle
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(dst), "l"(d) : "memory");
}
__host__ __device__ inline uint32_t lt_idesc_bf16(int n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(LT_M >> 4) << 24);
}
// e4m3 x e4m3, scales ue8m0; `k` says which of the four blocks of a scale column
__host__ __device__ inline uint32_t lt_idesc_mx8(int n, int k) {
  return ((uint32_t)k << 4) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(LT_M >> 7) << 27) |
         ((uint32_t)k << 29);
}
__device__ __forceinline__ int ld_acquire(const int32_t* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void st_release(int32_t* p, int v) {
  asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// True in the last of the four epilogue warps to come by (in its lane 0): what the warps before it did is
// ordered before what follows.  Nobody waits, so a warp that gave up holds up no other.
__device__ __forceinline__ bool last_of_four(unsigned* count) {
  __syncwarp();
  if ((threadIdx.x & 31) != 0) return false;
  __threadfence();
  const bool last = (atomicAdd(count, 1u) & 3u) == 3u;
  __threadfence();
  return last;
}

// ------------------------------------------------------------------------------------------ the deal
// CTA i has the units [i U / G, (i + 1) U / G); unit u is stage u % ks of tile u / ks.
__device__ __forceinline__ long long lt_first(const lt_params& p, int i) { return p.units * i / gridDim.x; }

struct lt_walk {                           // a CTA's segments, last tile first
  long long lo, hi;
  __device__ __forceinline__ lt_walk(const lt_params& p) : lo(lt_first(p, blockIdx.x)), hi(lt_first(p, blockIdx.x + 1)) {}
  __device__ __forceinline__ bool next(const lt_params& p, int& tile, int& k0, int& k1) {
    if (hi <= lo) return false;
    tile = (int)((hi - 1) / p.ks);
    const long long t0 = (long long)tile * p.ks;
    k1 = (int)(hi - t0);
    k0 = lo > t0 ? (int)(lo - t0) : 0;
    hi = t0 + k0;
    return true;
  }
};

// ------------------------------------------------------------------------------------------ epilogue
// One thread holds output n of up to 32 rows.
template <bool GATED>
__device__ __forceinline__ void lt_store(const lin_args& a, float (&v)[32], float (&u)[GATED ? 32 : 1], int cols, int r0, int n,
                                         float bias, float bias_up, const uint16_t (&res)[32]) {
  const bool live = n < a.n_out;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    float y = v[j] + bias;
    if (a.act == JK_ACT_SILU) y = __fdividef(y, 1.f + __expf(-y));
    else if (a.act == JK_ACT_GELU) y = 0.5f * y * erfcf(-0.70710678118654752f * y);
    if (GATED) y *= u[j] + bias_up;
    if (a.residual) y += __uint_as_float((uint32_t)res[j] << 16);
    v[j] = y;
  }
  if (a.out_type == JK_ROWS_MX8) {
    if (!live) return;                       // n_out is a multiple of 32: a warp is live as a whole
    int my_e = 0;
    uint8_t* o = (uint8_t*)a.out + (size_t)r0 * a.n_out + n;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(paged_mag(v[j])));
      const int e = paged_scale_exp(__uint_as_float(m));
      if (lane == j) my_e = e;
      const uint32_t c = __nv_cvt_float_to_fp8(v[j] * paged_pow2(-e), __NV_SATFINITE, __NV_E4M3);
      if (j < cols) o[(size_t)j * a.n_out] = (uint8_t)c;
    }
    if (lane < cols) a.out_scale[mx_scale_at(r0 + lane, n >> 5, a.k_tiles_out)] = (uint8_t)(my_e + 127);
  } else if (a.out_type == JK_ROWS_F32) {
    float* o = (float*)a.out + (size_t)r0 * a.o_stride + n;
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (live && j < cols) o[(size_t)j * a.o_stride] = v[j];
  } else {
    __nv_bfloat16* o = (__nv_bfloat16*)a.out + (size_t)r0 * a.o_stride + n;
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (live && j < cols) o[(size_t)j * a.o_stride] = __float2bfloat16_rn(v[j]);
  }
}

// ------------------------------------------------------------------------------------------ the kernel
template <bool MX, bool GATED>
__global__ void __launch_bounds__(LT_THREADS, 1) k_linear_tc(const __grid_constant__ CUtensorMap map_w,
                                                             const __grid_constant__ CUtensorMap map_u,
                                                             const __grid_constant__ CUtensorMap map_x,
                                                             const lt_params p, const lin_args a,
                                                             float* __restrict__ partial, int32_t* flags, int32_t* status) {
  constexpr int G = 1 + GATED;
  constexpr int BOX_EL = MX ? 128 : 64;    // elements of a box row
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  lt_tail& T = *reinterpret_cast<lt_tail*>(smem + (size_t)p.stages * p.stage_bytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &T.abort_flag;
  // a stage: kb boxes of w, kb of w_up, kb of x, then the scale tiles in the same order
  const int off_x = G * p.kb * p.a_box, off_sw = off_x + p.kb * p.b_box, off_sx = off_sw + G * p.kb * MX_TILE_BYTES;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) { mbar_init(&T.full[s], 1); mbar_init(&T.empty[s], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&T.acc_full[i], 1); mbar_init(&T.acc_empty[i], 4); }
    T.abort_flag = 0;
    T.done = T.seen = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc(&T.tmem_base, (uint32_t)p.tmem_cols);
    tmem_relinquish();
  }
  if (warp == 0 && lane == 0) {
    // The first ring of weights is asked into L2 while the kernel before still runs.  (Into L2 only: were
    // the weights that kernel's output, nothing stale would be kept.)
    lt_walk walk(p);
    int tile, k0, k1, left = p.stages;
    while (left > 0 && walk.next(p, tile, k0, k1)) {
      const int row = tile / p.r_tiles * LT_M;
      for (int k = k0; k < k1 && left > 0; ++k, --left)
        for (int b = k * p.kb; b < min(p.boxes, (k + 1) * p.kb); ++b) {
          l2_prefetch_box(&map_w, b * BOX_EL, row);
          if (GATED) l2_prefetch_box(&map_u, b * BOX_EL, row);
        }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = T.tmem_base;
  jk_pdl_wait();
  jk_pdl_trigger();

  if (warp == 0 && lane == 0) {
    // ------------------------------------------------------------------ copies
    const uint64_t once = l2_policy_evict_first();
    bool ok = true;
    int s = 0;
    long long issued = 0;
    uint32_t ph = 0;
    lt_walk walk(p);
    int tile, k0, k1;
    while (ok && walk.next(p, tile, k0, k1)) {
      const int wt = tile / p.r_tiles, rt = tile - wt * p.r_tiles;
      for (int k = k0; k < k1; ++k) {
        if (issued >= p.stages) ok = mbar_wait(&T.empty[s], ph ^ 1u, abort_flag, status);
        if (!ok) break;
        unsigned char* st = smem + (size_t)s * p.stage_bytes;
        const int b0 = k * p.kb, nb = min(p.kb, p.boxes - b0);
        mbar_expect_tx(&T.full[s], (uint32_t)(nb * (G * p.a_box + p.b_box + (MX ? (G + p.sfb) * MX_TILE_BYTES : 0))));
        for (int b = 0; b < nb; ++b) {
          const int x = (b0 + b) * BOX_EL;
          if (p.stream) {
            tma_load_2d_hint(st + b * p.a_box, &map_w, x, wt * LT_M, &T.full[s], once);
            if (GATED) tma_load_2d_hint(st + (p.kb + b) * p.a_box, &map_u, x, wt * LT_M, &T.full[s], once);
          } else {
            tma_load_2d(st + b * p.a_box, &map_w, x, wt * LT_M, &T.full[s]);
            if (GATED) tma_load_2d(st + (p.kb + b) * p.a_box, &map_u, x, wt * LT_M, &T.full[s]);
          }
          tma_load_2d(st + off_x + b * p.b_box, &map_x, x, rt * p.nt, &T.full[s]);
        }
        if (MX) {
          // scale tiles of neighbouring boxes lie side by side
          const size_t at = ((size_t)wt * a.k_tiles_in + b0) * MX_TILE_BYTES;
          bulk_load(st + off_sw, a.w_scale + at, nb * MX_TILE_BYTES, &T.full[s]);
          if (GATED) bulk_load(st + off_sw + p.kb * MX_TILE_BYTES, a.w_up_scale + at, nb * MX_TILE_BYTES, &T.full[s]);
          for (int i = 0; i < p.sfb; ++i) {
            // (a tile of x begins at a multiple of 128 rows wherever there is more than one)
            const size_t ax = ((size_t)(rt * (p.nt >> 7) + i) * a.k_tiles_in + b0) * MX_TILE_BYTES;
            const bool in = rt * p.nt + i * 128 < a.rows;            // the last tile of x may have fewer scale tiles
            bulk_load(st + off_sx + i * p.kb * MX_TILE_BYTES, a.x_scale + (in ? ax : 0), nb * MX_TILE_BYTES, &T.full[s]);
          }
        }
        ++issued;
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok) {
      // gave up: the copies in flight land before the CTA's memory goes away
      for (long long i = issued > p.stages ? issued - p.stages : 0; i < issued; ++i) {
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(&T.full[i % p.stages], (uint32_t)(i / p.stages) & 1u))
          if (global_ns() - t0 > TC_WAIT_NS) break;
      }
    }
  } else if (warp == 1 && lane == 0) {
    // ------------------------------------------------------------------ products
    bool ok = true;
    int s = 0, seg = 0, par = 0;
    uint32_t ph = 0;
    lt_walk walk(p);
    int tile, k0, k1;
    const uint32_t idesc = lt_idesc_bf16(p.nt);
    while (ok && walk.next(p, tile, k0, k1)) {
      const int buf = p.bufs == 2 ? seg & 1 : 0;
      const int use = p.bufs == 2 ? seg >> 1 : seg;
      if (use > 0) ok = mbar_wait(&T.acc_empty[buf], ((uint32_t)use & 1u) ^ 1u, abort_flag, status);
      if (!ok) break;
      tc_fence_after();
      const uint32_t d = tmem_base + (uint32_t)(buf * G * p.nt);
      uint32_t acc = 0;
      for (int k = k0; k < k1; ++k) {
        ok = mbar_wait(&T.full[s], ph, abort_flag, status);
        if (!ok) break;
        tc_fence_after();
        const uint32_t st = smem_u32(smem + (size_t)s * p.stage_bytes);
        const int b0 = k * p.kb, nb = min(p.kb, p.boxes - b0);
        for (int b = 0; b < nb; ++b) {
          const uint64_t dw = smem_desc_sw128(st + b * p.a_box), du = smem_desc_sw128(st + (p.kb + b) * p.a_box);
          const uint64_t dx = smem_desc_sw128(st + off_x + b * p.b_box);
          const int n_sub = min(4, p.subs - (b0 + b) * 4);           // products past the end of k are left out
          uint32_t sf = 0;
          if (MX) {
            // two sets of scale columns take turns: a box's scales do not land on those that the products
            // of the box before may still read
            sf = tmem_base + (uint32_t)(p.sf_col + par * 4 * (G + p.sfb));
            par ^= 1;
            tc_copy_scales(sf, st + off_sw + b * MX_TILE_BYTES);
            if (GATED) tc_copy_scales(sf + 4, st + off_sw + (p.kb + b) * MX_TILE_BYTES);
            for (int i = 0; i < p.sfb; ++i)
              tc_copy_scales(sf + 4 * (G + i), st + off_sx + (i * p.kb + b) * MX_TILE_BYTES);
          }
          for (int k4 = 0; k4 < n_sub; ++k4) {
            const uint64_t step = (uint64_t)(2 * k4);                // 32 bytes along k
            if (MX) {
              const uint32_t id = lt_idesc_mx8(p.nt, k4);
              tc_mma_mx8(d, dw + step, dx + step, id, sf, sf + 4 * G, acc);
              if (GATED) tc_mma_mx8(d + p.nt, du + step, dx + step, id, sf + 4, sf + 4 * G, acc);
            } else {
              tc_mma_bf16(d, dw + step, dx + step, idesc, acc);
              if (GATED) tc_mma_bf16(d + p.nt, du + step, dx + step, idesc, acc);
            }
            acc = 1;
          }
        }
        tc_commit(&T.empty[s]);            // the stage is free once these products have read it
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
      if (ok) tc_commit(&T.acc_full[buf]);
      ++seg;
    }
  } else if (warp >= 2) {
    // ------------------------------------------------------------------ epilogue
    const int quarter = warp & 3;          // the lanes of tensor memory this warp may read
    const int m = quarter * 32 + lane;
    int seg = 0;
    bool ok = true;
    lt_walk walk(p);
    int tile, k0, k1;
    while (ok && walk.next(p, tile, k0, k1)) {
      const int wt = tile / p.r_tiles, rt = tile - wt * p.r_tiles;
      const int n = wt * LT_M + m, r0 = rt * p.nt, rows = min(p.nt, a.rows - r0);
      const int buf = p.bufs == 2 ? seg & 1 : 0;
      const int use = p.bufs == 2 ? seg >> 1 : seg;
      const bool whole = k1 == p.ks;       // this CTA finishes the tile
      const bool live = n < a.n_out;
      float bias = 0.f, bias_up = 0.f;
      if (whole && live && a.bias) bias = __bfloat162float(((const __nv_bfloat16*)a.bias)[n]);
      if (GATED && whole && live && a.bias_up) bias_up = __bfloat162float(((const __nv_bfloat16*)a.bias_up)[n]);
      // the CTAs that have the tile's first k steps: all between the one with its first unit and this one
      int from = blockIdx.x;
      if (whole && k0 > 0) {
        const long long t0 = (long long)tile * p.ks;
        while (from > 0 && lt_first(p, from) > t0) --from;
        for (int j = from; j < (int)blockIdx.x && ok; ++j) {
          const long long c0 = clock64();
          while (ld_acquire(flags + j) == 0) {
            if (*abort_flag) ok = false;
            else if (clock64() - c0 > TC_WAIT_CYCLES) {
              *abort_flag = 1;
              jk_set_status(status, JK_ERR_TIMEOUT);
              ok = false;
            }
            if (!ok) break;
          }
        }
      }
      ok = ok && mbar_wait(&T.acc_full[buf], (uint32_t)use & 1u, abort_flag, status);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * G * p.nt);
      for (int c = 0; c < rows; c += 32) {
        const int cols = min(32, rows - c);
        uint16_t res[32];
        if (whole && a.residual) {
          const uint16_t* rp = (const uint16_t*)a.residual + (size_t)(r0 + c) * a.r_stride + n;
#pragma unroll
          for (int j = 0; j < 32; ++j) res[j] = live && j < cols ? rp[(size_t)j * a.r_stride] : (uint16_t)0;
        }
        // (a tile of 16 more rows than a multiple of 32 reads 16 columns that are not its own and leaves them)
        float v[32], u[GATED ? 32 : 1];
        {
          uint32_t t[32];
          tmem_ld32(t_addr + (uint32_t)c, t);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(t[j]);
          if constexpr (GATED) {
            tmem_ld32(t_addr + (uint32_t)(p.nt + c), t);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] = __uint_as_float(t[j]);
          }
        }
        if (c + 32 >= rows) {              // all of the accumulator has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&T.acc_empty[buf]);
        }
        if (!whole) {
          float* o = partial + (size_t)blockIdx.x * LT_SLOT + m;
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (j < cols) {
              __stcg(o + (size_t)(c + j) * LT_M, v[j]);
              if constexpr (GATED) __stcg(o + (size_t)(p.nt + c + j) * LT_M, u[j]);
            }
          continue;
        }
        for (int i = (int)blockIdx.x - 1; i >= from; --i) {
          const float* o = partial + (size_t)i * LT_SLOT + m;
          float t[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) t[j] = j < cols ? __ldcg(o + (size_t)(c + j) * LT_M) : 0.f;
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] += t[j];
          if constexpr (GATED) {
#pragma unroll
            for (int j = 0; j < 32; ++j) t[j] = j < cols ? __ldcg(o + (size_t)(p.nt + c + j) * LT_M) : 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] += t[j];
          }
        }
        lt_store<GATED>(a, v, u, cols, r0 + c, n, bias, bias_up, res);
      }
      if (!whole) {
        if (last_of_four(&T.done)) st_release(flags + blockIdx.x, 1);
      } else if (from < (int)blockIdx.x) {
        // everyone has seen the flags: they are put back for the next call
        if (last_of_four(&T.seen))
          for (int j = from; j < (int)blockIdx.x; ++j) flags[j] = 0;
      }
      ++seg;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, (uint32_t)p.tmem_cols);
  }
}

// ------------------------------------------------------------------------------------------ host side
int jk_linear_tc(jk_ctx* ctx, cudaStream_t st, const lin_args& a, bool mx) {
  const int G = a.w_up ? 2 : 1, es = mx ? 1 : 2, box_el = LT_BOX / es;
  lt_params p;
  memset(&p, 0, sizeof(p));
  const int most = LT_ACC_COLS / G;
  p.nt = a.rows <= most ? (int)jk_align_up(a.rows, 16) : most;
  p.r_tiles = (a.rows + p.nt - 1) / p.nt;
  p.w_tiles = (a.n_out + LT_M - 1) / LT_M;
  p.boxes = (a.n_in + box_el - 1) / box_el;
  p.subs = (a.n_in * es + 31) / 32;
  p.a_box = LT_M * LT_BOX;
  p.b_box = p.nt * LT_BOX;
  p.sfb = mx ? (p.nt + 127) / 128 : 0;
  const int box_bytes = G * p.a_box + p.b_box + (mx ? (G + p.sfb) * MX_TILE_BYTES : 0);
  const int room = LT_SMEM - (int)sizeof(lt_tail) - 1024;
  p.kb = room / (2 * box_bytes) >= 4 && p.boxes > 1 ? 2 : 1;
  p.ks = (p.boxes + p.kb - 1) / p.kb;
  p.stage_bytes = (int)jk_align_up((size_t)p.kb * box_bytes, 1024);
  p.stages = room / p.stage_bytes < LT_MAX_STAGES ? room / p.stage_bytes : LT_MAX_STAGES;
  const int sf_cols = mx ? 2 * 4 * (G + p.sfb) : 0;
  p.bufs = 2 * G * p.nt + sf_cols <= 512 ? 2 : 1;
  p.sf_col = p.bufs * G * p.nt;
  p.tmem_cols = 32;
  // (the epilogue reads 32 columns at a time: up to 16 past the accumulators' end)
  while (p.tmem_cols < p.sf_col + sf_cols || p.tmem_cols < jk_align_up(p.sf_col, 32)) p.tmem_cols <<= 1;
  p.stream = p.r_tiles == 1;
  p.units = (long long)p.w_tiles * p.r_tiles * p.ks;
  int grid = ctx->sm_count < LT_MAX_CTAS ? ctx->sm_count : LT_MAX_CTAS;
  if (p.units < grid) grid = (int)p.units;
  CUtensorMap mw, mu, mx_;
  auto map = [&](CUtensorMap* m, const void* ptr, uint64_t rows, uint64_t stride, uint32_t box_rows) {
    const uint64_t dims[2] = {(uint64_t)a.n_in, rows}, str[1] = {stride * es};
    const uint32_t box[2] = {(uint32_t)box_el, box_rows};
    return mx ? jk_tma_encode_u8(ctx, m, ptr, 2, dims, str, box) : jk_tma_encode_bf16(ctx, m, ptr, 2, dims, str, box);
  };
  int rc = map(&mw, a.w, a.n_out, a.n_in, LT_M);
  if (rc == JK_OK) rc = map(&mu, a.w_up ? a.w_up : a.w, a.n_out, a.n_in, LT_M);
  if (rc == JK_OK) rc = map(&mx_, a.x, a.rows, a.x_stride, p.nt);
  if (rc != JK_OK) return rc;
  auto kernel = mx ? (G == 2 ? k_linear_tc<true, true> : k_linear_tc<true, false>)
                   : (G == 2 ? k_linear_tc<false, true> : k_linear_tc<false, false>);
  const int bit = 1 << (2 * mx + G - 1);
  if (!(ctx->lin_smem_set & bit)) {
    JK_CUDA_CHECK(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LT_SMEM));
    ctx->lin_smem_set |= bit;
  }
  const size_t smem = (size_t)p.stages * p.stage_bytes + sizeof(lt_tail) + 1024;
  JK_PROF(ctx, st, JK_ST_LINEAR);
  jk_launch_pdl(kernel, dim3(grid), dim3(LT_THREADS), smem, st, mw, mu, mx_, p, a,
                (float*)(ctx->ws + ctx->lay.lin_part), (int32_t*)(ctx->ws + ctx->lay.lin_flag),
                (int32_t*)(ctx->ws + ctx->lay.status));
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}
