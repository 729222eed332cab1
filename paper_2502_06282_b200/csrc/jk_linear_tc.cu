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
// Three deals, by their cost (jk_linear_tc_plan).  Whole tiles, one after the other for each CTA.  Or the k steps of
// all tiles as one line, dealt out evenly: a tile that spans CTAs is finished by the CTA that
// has its last k step; the others hand over f32 partials through the workspace, which the copy engine brings into the
// ring.  A CTA works its share from the back, so its only unfinished tile comes first and its partial is long there when
// the CTA behind it asks; it waits only for CTAs of lower index, which were launched before it.  Or, for few tiles, a
// cluster of 2, 4 or 8 CTAs for each, whose sums pass through the cluster's shared memory.  Sums are formed in
// the same order on every run.
//
// Bound by the weights' way from memory: 60 rows, 11008 x 4096 gated in bf16 32 to 37 us (5.6 to 4.9 TB/s), 1 row 14336 x 4096
// gated in 8 bits 19.4 to 21.3 us (6.25 to 5.7); short calls by the gap between launches (1.2 us), the first boxes (1.3) and
// the hand-over: 60 rows 4096 x 4096 9.7 to 10.7 us (3.5 to 3.2 TB/s).
//
// Roles: warp 0 loads (TMA), warp 1 issues products, warps 2-17 drain accumulators and do the epilogue.  Every
// wait is bounded: after about 2 s it records JK_ERR_TIMEOUT, the CTA lets its copies land, frees its
// tensor memory and returns.
#include "jk_linear_tc.cuh"

int jk_tma_encode_u8(jk_ctx* ctx, CUtensorMap* out, const void* ptr, int rank, const uint64_t* dims,
                     const uint64_t* strides_bytes, const uint32_t* box);
struct lp_params;
double jk_linear_pair_plan(const lin_args& a, bool mx, int sms, lp_params* out);

#define LT_EPI_WARPS 16                   // four for each quarter of the lanes of tensor memory
#define LT_THREADS (64 + 32 * LT_EPI_WARPS)   // and two warps that load and multiply
#define LT_MAX_SPLIT 8                    // CTAs that share a tile, at most
#define LT_MAX_STAGES 12

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
  int by_tile;                            // 1: whole tiles, the shares end with them
  int grid;
  int cluster;                            // CTAs of a cluster that share a tile; 1: none
  int slots, exchange;                    // clusters: runs of 8 rows that a CTA finishes, and bytes of what it is handed
                                          // (0: it is handed into the ring, once all CTAs' products are done)
};

struct __align__(16) lt_tail {
  uint64_t full[LT_MAX_STAGES], empty[LT_MAX_STAGES];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t part_full, part_empty;         // others' partials in the ring, and read
  uint32_t tmem_base;
  int abort_flag;
};

__host__ __device__ inline uint32_t lt_idesc_bf16(int n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(LT_M >> 4) << 24);
}
// e4m3 x e4m3, scales ue8m0; `k` says which of the four blocks of a scale column
__host__ __device__ inline uint32_t lt_idesc_mx8(int n, int k) {
  return ((uint32_t)k << 4) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(LT_M >> 7) << 27) |
         ((uint32_t)k << 29);
}
// ------------------------------------------------------------------------------------------ the deal
// CTA i has the units [i U / G, (i + 1) U / G), or as many tiles; unit u is stage u % ks of tile u / ks.
__device__ __forceinline__ long long lt_first(const lt_params& p, int i) {
  return p.by_tile ? p.units / p.ks * i / gridDim.x * p.ks : p.units * i / gridDim.x;
}

struct lt_walk {                           // a CTA's segments, last tile first
  long long lo, hi;
  __device__ __forceinline__ lt_walk(const lt_params& p) {
    if (p.cluster > 1) {                   // one tile for each cluster, cut evenly
      const int rank = blockIdx.x % p.cluster;
      const long long t0 = (long long)(blockIdx.x / p.cluster) * p.ks;
      lo = t0 + p.ks * rank / p.cluster;
      hi = t0 + p.ks * (rank + 1) / p.cluster;
    } else {
      lo = lt_first(p, blockIdx.x);
      hi = lt_first(p, blockIdx.x + 1);
    }
  }
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

// The first of the CTAs that have the first k steps of a tile this CTA finishes from step k0 on (itself at k0 = 0).
__device__ __forceinline__ int lt_from(const lt_params& p, int tile, int k0) {
  int from = blockIdx.x;
  const long long t0 = (long long)tile * p.ks;
  while (k0 > 0 && from > 0 && lt_first(p, from) > t0) --from;
  return from;
}
// Their partials come through the ring, as many columns at a time as it holds.
__device__ __forceinline__ int lt_round_cols(const lt_params& p, int parts, int G) {
  return max(16, min(p.nt, p.stages * p.stage_bytes / (parts * G * LT_M * 4) / 16 * 16));
}

// ------------------------------------------------------------------------------------------ epilogue
// One thread holds output n of up to 8 rows.
#define LT_COLS 8
template <bool GATED>
__device__ __forceinline__ void lt_store(const lin_args& a, float (&v)[LT_COLS], float (&u)[GATED ? LT_COLS : 1], int cols,
                                         int r0, int n, float bias, float bias_up, const uint16_t (&res)[LT_COLS]) {
  const bool live = n < a.n_out;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < LT_COLS; ++j) v[j] += bias;
  lin_act_all(v, a.act, a.out_type == JK_ROWS_F32);
  if constexpr (GATED) {
#pragma unroll
    for (int j = 0; j < LT_COLS; ++j) v[j] *= u[j] + bias_up;
  }
  if (a.residual) {
#pragma unroll
    for (int j = 0; j < LT_COLS; ++j) v[j] += __uint_as_float((uint32_t)res[j] << 16);
  }
  if (a.out_type == JK_ROWS_MX8) {
    if (!live) return;                       // n_out is a multiple of 32: a warp is live as a whole
    int my_e = 0;
    uint8_t* o = (uint8_t*)a.out + (size_t)r0 * a.n_out + n;
#pragma unroll
    for (int j = 0; j < LT_COLS; ++j) {
      const uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(paged_mag(v[j])));
      const int e = paged_scale_exp(__uint_as_float(m));
      if (lane == j) my_e = e;
      if (j < cols) *o = (uint8_t)__nv_cvt_float_to_fp8(v[j] * paged_pow2(-e), __NV_SATFINITE, __NV_E4M3);
      o += a.n_out;
    }
    if (lane < cols) a.out_scale[mx_scale_at(r0 + lane, n >> 5, a.k_tiles_out)] = (uint8_t)(my_e + 127);
  } else if (a.out_type == JK_ROWS_F32) {
    float* o = (float*)a.out + (size_t)r0 * a.o_stride + n;
#pragma unroll
    for (int j = 0; j < LT_COLS; ++j, o += a.o_stride)
      if (live && j < cols) *o = v[j];
  } else {
    __nv_bfloat16* o = (__nv_bfloat16*)a.out + (size_t)r0 * a.o_stride + n;
#pragma unroll
    for (int j = 0; j < LT_COLS; ++j, o += a.o_stride)
      if (live && j < cols) *o = __float2bfloat16_rn(v[j]);
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
  unsigned char* handed = p.exchange ? smem + (size_t)p.stages * p.stage_bytes : smem;
  lt_tail& T = *reinterpret_cast<lt_tail*>(smem + (size_t)p.stages * p.stage_bytes + p.exchange);
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  volatile int* abort_flag = &T.abort_flag;
  // a stage: kb boxes of w, kb of w_up, kb of x, then the scale tiles in the same order
  const int off_x = G * p.kb * p.a_box, off_sw = off_x + p.kb * p.b_box, off_sx = off_sw + G * p.kb * MX_TILE_BYTES;

  if (warp == 0) {
    // This warp needs nothing of the others: it does not wait for them (nor for tensor memory) before it
    // asks for the first boxes.
    if (lane == 0) {
      for (int s = 0; s < p.stages; ++s) { mbar_init(&T.full[s], 1); mbar_init(&T.empty[s], 1); }
      for (int i = 0; i < 2; ++i) { mbar_init(&T.acc_full[i], 1); mbar_init(&T.acc_empty[i], LT_EPI_WARPS); }
      mbar_init(&T.part_full, 1);
      mbar_init(&T.part_empty, LT_EPI_WARPS);
      T.abort_flag = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("bar.arrive 1, %0;" ::"n"(LT_THREADS) : "memory");
  } else {
    if (warp == 1) {
      tmem_alloc(&T.tmem_base, (uint32_t)p.tmem_cols);
      tmem_relinquish();
    }
    tc_fence_before();
    asm volatile("bar.sync 1, %0;" ::"n"(LT_THREADS) : "memory");
    tc_fence_after();
  }
  lt_walk walk(p);
  int tile, k0, k1;
  bool more = walk.next(p, tile, k0, k1);
  if (warp == 2) {
    // The boxes of the first ring are asked into L2 while the kernel before still runs.  (Into L2 only: what
    // that kernel writes meanwhile, it writes there.)
    const int k = k0 + lane / p.kb, b = k * p.kb + lane % p.kb;
    if (lane < p.stages * p.kb && k < k1 && b < p.boxes) {
      const int row = tile / p.r_tiles;
      l2_prefetch_box(&map_w, b * BOX_EL, row * LT_M);
      if (GATED) l2_prefetch_box(&map_u, b * BOX_EL, row * LT_M);
      l2_prefetch_box(&map_x, b * BOX_EL, (tile - row * p.r_tiles) * p.nt);
    }
    __syncwarp();
  }
  const uint32_t tmem_base = warp ? T.tmem_base : 0;       // (warp 0 may be ahead of the allocation; it needs no address)
  if (p.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  jk_pdl_wait();
  jk_pdl_trigger();
  // (a CTA's memory is written from outside only once it runs)
  if (p.cluster > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");

  if (warp == 0) {
    // ------------------------------------------------------------------ copies
    const uint64_t once = l2_policy_evict_first();
    const uint32_t lead = lt_elect(), base = smem_u32(smem), full0 = smem_u32(T.full);
    bool ok = true;
    int s = 0;
    long long issued = 0;
    uint32_t ph = 0;
    for (; ok && more; more = walk.next(p, tile, k0, k1)) {
      const int wt = tile / p.r_tiles, rt = tile - wt * p.r_tiles;
      // (a tile of x begins at a multiple of 128 rows wherever there is more than one; the last may have fewer
      // scale tiles, and reads the first in place of those)
      const uint8_t* sw = MX ? a.w_scale + (size_t)wt * a.k_tiles_in * MX_TILE_BYTES : nullptr;
      const uint8_t* su = MX && GATED ? a.w_up_scale + (size_t)wt * a.k_tiles_in * MX_TILE_BYTES : nullptr;
      const uint8_t* sx0 = MX ? a.x_scale + (size_t)(rt * (p.nt >> 7)) * a.k_tiles_in * MX_TILE_BYTES : nullptr;
      const uint8_t* sx1 = MX && rt * p.nt + 128 < a.rows ? sx0 + (size_t)a.k_tiles_in * MX_TILE_BYTES : sx0;
      for (int k = k0; k < k1; ++k) {
        if (issued >= p.stages) ok = mbar_wait(&T.empty[s], ph ^ 1u, abort_flag, status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t st = base + (uint32_t)s * (uint32_t)p.stage_bytes, bar = full0 + 8u * (uint32_t)s;
        const int b0 = k * p.kb, nb = min(p.kb, p.boxes - b0);
        lt_expect(bar, (uint32_t)(nb * (G * p.a_box + p.b_box + (MX ? (G + p.sfb) * MX_TILE_BYTES : 0))), lead);
        for (int b = 0; b < nb; ++b) {
          const int x = (b0 + b) * BOX_EL;
          if (p.stream) {
            lt_box_once(st + b * p.a_box, &map_w, x, wt * LT_M, bar, once, lead);
            if (GATED) lt_box_once(st + (p.kb + b) * p.a_box, &map_u, x, wt * LT_M, bar, once, lead);
          } else {
            lt_box(st + b * p.a_box, &map_w, x, wt * LT_M, bar, lead);
            if (GATED) lt_box(st + (p.kb + b) * p.a_box, &map_u, x, wt * LT_M, bar, lead);
          }
          lt_box(st + off_x + b * p.b_box, &map_x, x, rt * p.nt, bar, lead);
        }
        if (MX) {
          // scale tiles of neighbouring boxes lie side by side
          const int at = b0 * MX_TILE_BYTES, bytes = nb * MX_TILE_BYTES, step = p.kb * MX_TILE_BYTES;
          lt_bulk(st + off_sw, sw + at, bytes, bar, lead);
          if (GATED) lt_bulk(st + off_sw + step, su + at, bytes, bar, lead);
          lt_bulk(st + off_sx, sx0 + at, bytes, bar, lead);
          if (p.sfb > 1) lt_bulk(st + off_sx + step, sx1 + at, bytes, bar, lead);
        }
        ++issued;
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
    }
    // The tile this CTA finishes last may have begun in others: once its products are done and the ring is free,
    // their partials come through it, one lane looking after each.
    const long long lo = lt_first(p, blockIdx.x);
    tile = (int)(lo / p.ks);
    k0 = (int)(lo - (long long)tile * p.ks);
    if (ok && p.cluster == 1 && k0 > 0 && lt_first(p, blockIdx.x + 1) - lo >= p.ks - k0) {
      const int parts = (int)blockIdx.x - lt_from(p, tile, k0), cols = lt_round_cols(p, parts, G);
      const int rows = min(p.nt, a.rows - tile % p.r_tiles * p.nt);
      const int other = (int)blockIdx.x - 1 - lane;
      // (products end in order: when the last stage has been read, all have)
      ok = mbar_wait(&T.empty[(issued - 1) % p.stages], (uint32_t)((issued - 1) / p.stages) & 1u, abort_flag, status);
      ok = __all_sync(0xffffffffu, ok);
      uint32_t round = 0;
      for (int c = 0; c < rows && ok; c += cols, ++round) {
        if (round > 0) ok = mbar_wait(&T.part_empty, (round & 1u) ^ 1u, abort_flag, status);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        if (lane < parts) {
          if (round == 0) {
            const long long c0 = clock64();
            while (ok && ld_acquire(flags + other) != LT_EPI_WARPS) {
              if (*abort_flag) ok = false;
              else if (clock64() - c0 > TC_WAIT_CYCLES) {
                *abort_flag = 1;
                jk_set_status(status, JK_ERR_TIMEOUT);
                ok = false;
              }
            }
            asm volatile("fence.proxy.async.global;" ::: "memory");     // the partials were written by ordinary stores
          }
          if (ok) {
            const uint32_t bytes = (uint32_t)min(cols, p.nt - c) * LT_M * 4;
            mbar_add_tx(&T.part_full, bytes * G);
            for (int g = 0; g < G; ++g)
              lt_bulk(base + (uint32_t)((lane * G + g) * cols * LT_M * 4),
                      partial + (size_t)other * LT_SLOT + (size_t)(g * p.nt + c) * LT_M, bytes, smem_u32(&T.part_full), 1u);
            if (round == 0) flags[other] = 0;    // for the next call; nobody else looks at it in this one
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&T.part_full);            // every piece has been announced
        ok = __all_sync(0xffffffffu, ok);
      }
      if (!ok && round > 0 && lane == 0) {
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(&T.part_full, (round - 1) & 1u))
          if (global_ns() - t0 > TC_WAIT_NS) break;
      }
    }
    if (!ok && lane == 0) {
      // gave up: the copies in flight land before the CTA's memory goes away
      for (long long i = issued > p.stages ? issued - p.stages : 0; i < issued; ++i) {
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(&T.full[i % p.stages], (uint32_t)(i / p.stages) & 1u))
          if (global_ns() - t0 > TC_WAIT_NS) break;
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products
    const uint32_t lead = lt_elect(), tm = __shfl_sync(0xffffffffu, tmem_base, 0);
    const uint32_t empty0 = smem_u32(T.empty);
    const uint64_t d0 = smem_desc_sw128(smem_u32(smem));   // further descriptors: sixteenths of bytes are added
    const uint64_t s0 = LT_SCALE_DESC | (uint64_t)((smem_u32(smem) & 0x3FFFFu) >> 4);
    const uint32_t idesc = lt_idesc_bf16(p.nt);
    bool ok = true;
    int s = 0, seg = 0, par = 0;
    uint32_t ph = 0;
    for (; ok && more; more = walk.next(p, tile, k0, k1)) {
      const int buf = p.bufs == 2 ? seg & 1 : 0;
      const int use = p.bufs == 2 ? seg >> 1 : seg;
      if (use > 0) ok = mbar_wait(&T.acc_empty[buf], ((uint32_t)use & 1u) ^ 1u, abort_flag, status);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const uint32_t d = tm + (uint32_t)(buf * G * p.nt);
      uint32_t acc = 0;
      for (int k = k0; k < k1; ++k) {
        ok = mbar_wait(&T.full[s], ph, abort_flag, status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t st = (uint32_t)s * (uint32_t)(p.stage_bytes >> 4);
        const int b0 = k * p.kb, nb = min(p.kb, p.boxes - b0);
        for (int b = 0; b < nb; ++b) {
          const uint64_t dw = d0 + (st + (uint32_t)(b * p.a_box >> 4)), du = dw + (uint32_t)(p.kb * p.a_box >> 4);
          const uint64_t dx = d0 + (st + (uint32_t)((off_x + b * p.b_box) >> 4));
          const int n_sub = p.subs - (b0 + b) * 4;                   // products past the end of k are left out
          uint32_t sf = 0;
          if (MX) {
            // two sets of scale columns take turns: a box's scales do not land on those that the products
            // of the box before may still read
            sf = tm + (uint32_t)(p.sf_col + par * 4 * (G + p.sfb));
            par ^= 1;
            const uint64_t ds = s0 + (st + (uint32_t)((off_sw + b * MX_TILE_BYTES) >> 4));
            const uint32_t step = (uint32_t)(p.kb * MX_TILE_BYTES) >> 4;
            lt_copy_scales(sf, ds, lead);
            lt_copy_scales(sf + 4, ds + step, lead);                 // gated: of w_up; else the first of x
            if (GATED || p.sfb > 1) lt_copy_scales(sf + 8, ds + 2 * step, lead);
            if (GATED && p.sfb > 1) lt_copy_scales(sf + 12, ds + 3 * step, lead);
          }
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4) {
            if (k4 >= n_sub) break;
            const uint64_t step = (uint64_t)(2 * k4);                // 32 bytes along k
            if (MX) {
              const uint32_t id = lt_idesc_mx8(p.nt, k4);
              lt_mma_mx8(d, dw + step, dx + step, id, sf, sf + 4 * G, acc, lead);
              if (GATED) lt_mma_mx8(d + p.nt, du + step, dx + step, id, sf + 4, sf + 4 * G, acc, lead);
            } else {
              lt_mma_bf16(d, dw + step, dx + step, idesc, acc, lead);
              if (GATED) lt_mma_bf16(d + p.nt, du + step, dx + step, idesc, acc, lead);
            }
            acc = 1;
          }
        }
        lt_commit(empty0 + 8u * (uint32_t)s, lead);        // the stage is free once these products have read it
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
      if (ok) lt_commit(smem_u32(&T.acc_full[buf]), lead);
      ++seg;
    }
  } else if (p.cluster > 1) {
    // ------------------------------------------------------------------ epilogue of a shared tile
    // Each CTA of the cluster finishes every cluster-th run of 8 rows: it is handed the others' sums of
    // those in its shared memory, and its own.  While the products run the warps go through it once without effect, so
    // that its instructions are there when it counts.
    const int quarter = warp & 3, sub = (warp - 2) >> 2, m = quarter * 32 + lane, rank = blockIdx.x % p.cluster;
    const int wt = tile / p.r_tiles, rt = tile - wt * p.r_tiles;
    const int n = wt * LT_M + m, r0 = rt * p.nt, rows = min(p.nt, a.rows - r0);
    const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const bool live = n < a.n_out;
    uint16_t res[LT_COLS];
    float bias = 0.f, bias_up = 0.f;
    auto ask_residual = [&](int c) {
      const uint16_t* rp = (const uint16_t*)a.residual + (size_t)(r0 + c) * a.r_stride + n;
#pragma unroll
      for (int j = 0; j < LT_COLS; ++j, rp += a.r_stride) res[j] = live && c + j < rows ? *rp : (uint16_t)0;
    };
    if (live && a.bias) bias = __bfloat162float(((const __nv_bfloat16*)a.bias)[n]);
    if (GATED && live && a.bias_up) bias_up = __bfloat162float(((const __nv_bfloat16*)a.bias_up)[n]);
    if (a.residual) ask_residual((sub * p.cluster + rank) * 8);
#pragma unroll 1
    for (int real = 0; real < 2; ++real) {
      bool ok = true;
      if (real) {
        ok = mbar_wait(&T.acc_full[0], 0, abort_flag, status);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        if (!p.exchange) lt_cluster_sync();
      }
      const int end = !real ? 8 : ok ? rows : 0;
#pragma unroll 1
      for (int j = real ? sub : 0; j * 8 < end; j += LT_EPI_WARPS / 4) {
        uint32_t v[8], u[8];
        lt_ld8(t_addr + (uint32_t)(j * 8), v);
        if constexpr (GATED) lt_ld8(t_addr + (uint32_t)(p.nt + j * 8), u);
        tmem_ld_wait();
        const uint32_t to = lt_map(smem_u32(handed) + (uint32_t)(((rank * p.slots + j / p.cluster) * G * 8 * LT_M + m) * 4),
                                   (uint32_t)(j % p.cluster));
        if (real) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(to + i * LT_M * 4), "r"(v[i]) : "memory");
            if constexpr (GATED) asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(to + (8 + i) * LT_M * 4), "r"(u[i]) : "memory");
          }
        }
      }
      __syncwarp();
      if (real) lt_cluster_sync();
#pragma unroll 1
      for (int slot = real ? sub : 0; slot < (real ? p.slots : 1); slot += LT_EPI_WARPS / 4) {
        const int c = (slot * p.cluster + rank) * 8, cols = real ? min(LT_COLS, rows - c) : 0;
        if (real && cols <= 0) break;
        if (a.residual && real && slot != sub) ask_residual(c);
        float v[LT_COLS], u[GATED ? LT_COLS : 1];
#pragma unroll
        for (int j = 0; j < LT_COLS; ++j) {
          v[j] = 0.f;
          if constexpr (GATED) u[j] = 0.f;
        }
        for (int i = 0; i < p.cluster; ++i) {              // in the order of k
          const float* o = reinterpret_cast<const float*>(handed) + (size_t)((i * p.slots + slot) * G * 8) * LT_M + m;
#pragma unroll
          for (int j = 0; j < LT_COLS; ++j) {
            v[j] += o[j * LT_M];
            if constexpr (GATED) u[j] += o[(8 + j) * LT_M];
          }
        }
        lt_store<GATED>(a, v, u, cols, r0 + c, n, bias, bias_up, res);
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue
    const int quarter = warp & 3;          // the lanes of tensor memory this warp may read
    const int sub = (warp - 2) >> 2;       // its warps take 8 columns in turn
    const int m = quarter * 32 + lane;
    int seg = 0;
    bool ok = true;
    for (; ok && more; more = walk.next(p, tile, k0, k1)) {
      const int wt = tile / p.r_tiles, rt = tile - wt * p.r_tiles;
      const int n = wt * LT_M + m, r0 = rt * p.nt, rows = min(p.nt, a.rows - r0);
      const int buf = p.bufs == 2 ? seg & 1 : 0;
      const int use = p.bufs == 2 ? seg >> 1 : seg;
      const bool whole = k1 == p.ks;       // this CTA finishes the tile
      const bool live = n < a.n_out;
      float bias = 0.f, bias_up = 0.f;
      if (whole && live && a.bias) bias = __bfloat162float(((const __nv_bfloat16*)a.bias)[n]);
      if (GATED && whole && live && a.bias_up) bias_up = __bfloat162float(((const __nv_bfloat16*)a.bias_up)[n]);
      const int parts = whole ? (int)blockIdx.x - lt_from(p, tile, k0) : 0;
      const int round_cols = parts ? lt_round_cols(p, parts, G) : p.nt;
      uint16_t res[LT_COLS];
      auto ask_residual = [&](int c) {
        const uint16_t* rp = (const uint16_t*)a.residual + (size_t)(r0 + c) * a.r_stride + n;
#pragma unroll
        for (int j = 0; j < LT_COLS; ++j, rp += a.r_stride) res[j] = live && c + j < rows ? *rp : (uint16_t)0;
      };
      if (whole && a.residual) ask_residual(sub * LT_COLS);      // the first of them ahead of the wait
      ok = mbar_wait(&T.acc_full[buf], (uint32_t)use & 1u, abort_flag, status);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * G * p.nt);
      uint32_t round = 0;
      for (int c0 = 0; c0 < rows; c0 += round_cols, ++round) {
        if (parts) {
          ok = mbar_wait(&T.part_full, round & 1u, abort_flag, status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
        }
        const int c1 = min(rows, c0 + round_cols);
        for (int c = c0 + sub * LT_COLS; c < c1; c += LT_EPI_WARPS / 4 * LT_COLS) {
          const int cols = min(LT_COLS, rows - c);
          if (whole && a.residual && c != sub * LT_COLS) ask_residual(c);
          float v[LT_COLS], u[GATED ? LT_COLS : 1];
          {
            uint32_t t[LT_COLS], t2[LT_COLS];
            lt_ld8(t_addr + (uint32_t)c, t);
            if constexpr (GATED) lt_ld8(t_addr + (uint32_t)(p.nt + c), t2);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < LT_COLS; ++j) {
              v[j] = __uint_as_float(t[j]);
              if constexpr (GATED) u[j] = __uint_as_float(t2[j]);
            }
          }
          if (!whole) {
            float* o = partial + (size_t)blockIdx.x * LT_SLOT + (size_t)c * LT_M + m;
#pragma unroll
            for (int j = 0; j < LT_COLS; ++j) {
              __stcg(o + (size_t)j * LT_M, v[j]);
              if constexpr (GATED) __stcg(o + (size_t)(p.nt + j) * LT_M, u[j]);
            }
            continue;
          }
          const float* o = reinterpret_cast<const float*>(smem) + (size_t)(c - c0) * LT_M + m;
          for (int i = 0; i < parts; ++i, o += (size_t)G * round_cols * LT_M) {
#pragma unroll
            for (int j = 0; j < LT_COLS; ++j) {
              v[j] += o[j * LT_M];
              if constexpr (GATED) u[j] += o[(round_cols + j) * LT_M];
            }
          }
          lt_store<GATED>(a, v, u, cols, r0 + c, n, bias, bias_up, res);
        }
        if (parts) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&T.part_empty);
        }
      }
      if (!ok) break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&T.acc_empty[buf]);       // all of the accumulator has been read
      if (!whole && lane == 0) add_release(flags + blockIdx.x, 1);      // (behind the warp's stores: the barrier above)
      ++seg;
    }
  }
  if (p.cluster > 1 && warp < 2) {         // (the meetings of the epilogue's warps are all warps')
    __syncwarp();
    if (!p.exchange) lt_cluster_sync();
    lt_cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, (uint32_t)p.tmem_cols);
  }
}

// ------------------------------------------------------------------------------------------ host side
// Into how many shares the tiles are cut.  One SM takes in about 118 bytes a nanosecond and one box in 0.19 us at best
// (gated: two); all together 6400.  What is cut has to be handed over: 1.5 us and 0.02 for each column of the
// accumulators, a quarter more for each further share.  Measured with 4096 outputs, 64 boxes (bf16, 4096 inputs), us:
// 60 rows 18.3 whole, 15.1, 13.5, 12.5 with 2, 3, 4 shares, 12.5 with 4.6; 8 boxes: 7.3 whole, 8.4, 8.3, 8.8.  The costs,
// in us and with a launch, also choose between this kernel and that for many rows.
double jk_linear_tc_plan(const lin_args& a, bool mx, int sms, const int* clusters, lt_params* out) {
  const int G = a.w_up ? 2 : 1, es = mx ? 1 : 2, box_el = LT_BOX / es;
  lt_params p;
  memset(&p, 0, sizeof(p));
  const int most = LT_ACC_COLS / G;
  p.r_tiles = (a.rows + most - 1) / most;
  p.nt = p.r_tiles > 1 && mx ? most : (int)jk_align_up((a.rows + p.r_tiles - 1) / p.r_tiles, 16);     // (scale tiles: 128 rows)
  p.w_tiles = (a.n_out + LT_M - 1) / LT_M;
  p.boxes = (a.n_in + box_el - 1) / box_el;
  p.subs = (a.n_in * es + 31) / 32;
  p.a_box = LT_M * LT_BOX;
  p.b_box = p.nt * LT_BOX;
  p.sfb = mx ? (p.nt + 127) / 128 : 0;
  const int box_bytes = G * p.a_box + p.b_box + (mx ? (G + p.sfb) * MX_TILE_BYTES : 0);
  // The ring: stages of two boxes while four of them fit (8-bit rows, which bring scales with every stage: three).
  auto ring = [&](int room) {
    p.kb = room / (2 * box_bytes) >= (mx ? 3 : 4) && p.boxes > 1 ? 2 : 1;
    p.ks = (p.boxes + p.kb - 1) / p.kb;
    p.stage_bytes = (int)jk_align_up((size_t)p.kb * box_bytes, 1024);
    p.stages = room / p.stage_bytes < LT_MAX_STAGES ? room / p.stage_bytes : LT_MAX_STAGES;
  };
  const int room = LT_SMEM - (int)sizeof(lt_tail) - 1024;
  ring(room);
  const int sf_cols = mx ? 2 * 4 * (G + p.sfb) : 0;
  p.bufs = 2 * G * p.nt + sf_cols <= 512 ? 2 : 1;
  p.sf_col = p.bufs * G * p.nt;
  p.tmem_cols = 32;
  while (p.tmem_cols < p.sf_col + sf_cols) p.tmem_cols <<= 1;
  p.stream = p.r_tiles == 1;
  const long long tiles = (long long)p.w_tiles * p.r_tiles;
  p.units = tiles * p.ks;
  const double box_us = box_bytes / 118e3 > 0.185 * G ? box_bytes / 118e3 : 0.185 * G;
  const double tile_us = box_us * p.boxes, hbm_us = (double)a.n_out * a.n_in * es * G / 6.4e6, per_tile_hbm = hbm_us / p.w_tiles;
  const long long full = tiles / sms, left = tiles - full * sms;
  const auto larger = [](double x, double y) { return x > y ? x : y; };
  double best = full * larger(tile_us, sms * per_tile_hbm) + (left ? larger(tile_us, left * per_tile_hbm) : 0.);
  p.by_tile = 1;
  p.cluster = 1;
  p.grid = tiles < sms ? (int)tiles : sms;
  for (int s = 2; s <= LT_MAX_SPLIT && s <= p.ks; s = s < 4 ? s + 1 : 2 * s) {
    if (s > 4 && G * p.nt > 64) break;                     // (their partials do not fit the ring at once)
    const int grid = tiles * s < sms ? (int)(tiles * s) : sms;
    const double shares = (double)grid / tiles, over = 1.5 + 0.02 * G * p.nt * (shares > 2. ? 0.5 + 0.25 * shares : 1.);
    const double cost = larger(tile_us / shares, hbm_us * p.r_tiles) + over;
    if (cost < best) { best = cost; p.by_tile = 0; p.grid = grid; }
    if (grid == sms) break;
  }
  // Few tiles: a cluster for each, whose CTAs hand their sums over through shared memory: 0.011 us for each column, less what
  // sharing the epilogue saves.  (4096 x 4096 in bf16, us: 60 rows 10.7, dealt evenly 12.5; 256 rows 16.2, dealt evenly 25.0.)
  for (int i = 0; i < 3 && clusters; ++i) {
    const int c = 2 << i;
    if (2 * c > p.boxes || tiles > clusters[i]) continue;  // (a stage for every CTA)
    const int slots = (p.nt / 8 + c - 1) / c, bytes = c * slots * G * 8 * LT_M * 4;
    const bool apart = bytes <= 64 * 1024;                 // (the ring needs the rest)
    if (!apart && bytes > p.stages * p.stage_bytes) continue;
    const double cost = larger(tile_us / c, larger(hbm_us, hbm_us * 60 / (tiles * c))) + 0.011 * G * p.nt - 0.4;
    if (cost < best) {
      best = cost;
      p.cluster = c;
      p.slots = slots;
      p.exchange = apart ? bytes : 0;
      p.by_tile = 0;
      p.grid = (int)tiles * c;
    }
  }
  if (p.cluster > 1) ring(room - p.exchange);
  if (out) *out = p;
  return best + 4.9 + 0.01 * G * p.nt;
}

typedef void (*lt_kernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const lt_params, const lin_args, float*,
                          int32_t*, int32_t*);
static lt_kernel lt_pick(bool mx, bool gated) {
  return mx ? (gated ? k_linear_tc<true, true> : k_linear_tc<true, false>)
            : (gated ? k_linear_tc<false, true> : k_linear_tc<false, false>);
}
// How many clusters of 2, 4 and 8 CTAs (one to an SM) run at a time; asked once for each context.
static int lt_clusters(jk_ctx* ctx) {
  if (ctx->lin_clusters[0]) return JK_OK;
  const lt_kernel kernel = lt_pick(false, false);
  JK_CUDA_CHECK(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LT_SMEM));
  for (int i = 2; i >= 0; --i) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(8 * (LT_MAX_CTAS / 8));
    cfg.blockDim = dim3(LT_THREADS);
    cfg.dynamicSmemBytes = LT_SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2 << i;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    JK_CUDA_CHECK(ctx, cudaOccupancyMaxActiveClusters(&n, kernel, &cfg));
    ctx->lin_clusters[i] = n > 0 ? n : 1;
  }
  return JK_OK;
}
// The costs of the two kernels (us): is this one's the lower?
int jk_linear_tc_pays(jk_ctx* ctx, const lin_args& a, bool mx, bool* pays) {
  const int rc = lt_clusters(ctx);
  if (rc != JK_OK) return rc;
  const int sms = ctx->sm_count < LT_MAX_CTAS ? ctx->sm_count : LT_MAX_CTAS;
  *pays = jk_linear_tc_plan(a, mx, sms, ctx->lin_clusters, nullptr) <= jk_linear_pair_plan(a, mx, sms, nullptr);
  return JK_OK;
}

int jk_linear_tc(jk_ctx* ctx, cudaStream_t st, const lin_args& a, bool mx) {
  const int G = a.w_up ? 2 : 1, es = mx ? 1 : 2, box_el = LT_BOX / es;
  lt_params p;
  jk_linear_tc_plan(a, mx, ctx->sm_count < LT_MAX_CTAS ? ctx->sm_count : LT_MAX_CTAS, ctx->lin_clusters, &p);
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
  const lt_kernel kernel = lt_pick(mx, G == 2);
  const int bit = 1 << (2 * mx + G - 1);
  if (!(ctx->lin_smem_set & bit)) {
    JK_CUDA_CHECK(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LT_SMEM));
    ctx->lin_smem_set |= bit;
  }
  const size_t smem = (size_t)p.stages * p.stage_bytes + p.exchange + sizeof(lt_tail) + 1024;
  JK_PROF(ctx, st, JK_ST_LINEAR);
  float* part = (float*)(ctx->ws + ctx->lay.lin_part);
  int32_t* flags = (int32_t*)(ctx->ws + ctx->lay.lin_flag);
  int32_t* status = (int32_t*)(ctx->ws + ctx->lay.status);
  if (p.cluster > 1)
    jk_launch_pdl_cluster(kernel, dim3(p.grid), dim3(LT_THREADS), p.cluster, smem, st, mw, mu, mx_, p, a, part, flags, status);
  else
    jk_launch_pdl(kernel, dim3(p.grid), dim3(LT_THREADS), smem, st, mw, mu, mx_, p, a, part, flags, status);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}
