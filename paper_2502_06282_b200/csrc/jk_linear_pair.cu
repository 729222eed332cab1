// jk_linear for many rows: the kernel whose time is the tensor cores'.
//
// A pair of CTAs (a cluster of two SMs) makes a tile of 256 rows of x times 256 weight rows with tcgen05.mma
// cta_group::2: each CTA brings 128 rows of x and 128 weight rows and holds the sums of its 128 rows,
// so a byte that arrives in shared memory serves twice the products of a single CTA's tile (64 bytes a
// clock and SM at the full rate, where 128 x 256 tiles of single CTAs ask for 96).  A gated block takes 128
// rows of w and 128 of w_up as the 256: one CTA brings the one, the other the other, and the two sums of an
// output stand in the same lane.  Rows of x stand on the lanes here: a thread of the epilogue holds 32
// consecutive outputs of a row, which are a scale block of 8-bit rows, without any exchange.
//
// Tiles are dealt to the pairs in turn, in bands of 8 tiles of x, so that what runs at one time shares
// its operands in L2.  The tiles left over for a last, incomplete turn come first and are cut along k
// into even shares: the pair that has a tile's end finishes it from the others' f32 partials, as in the
// kernel for few rows.
//
// Accumulators: two of 256 columns for bf16.  8-bit rows need 24 columns for scales; there the second
// accumulator begins at column 232, and of the 24 columns that both use the epilogue reads first.
//
// Roles: warp 0 loads, warp 1 (of the pair's first CTA) multiplies, warps 2-9 are the epilogue.  Waits are bounded as
// in the kernel for few rows.
#include "jk_linear_tc.cuh"

int jk_tma_encode_u8(jk_ctx* ctx, CUtensorMap* out, const void* ptr, int rank, const uint64_t* dims,
                     const uint64_t* strides_bytes, const uint32_t* box);
int jk_tma_encode_scales(jk_ctx* ctx, CUtensorMap* out, const void* ptr, uint64_t tiles);
int jk_tma_encode_piece(jk_ctx* ctx, CUtensorMap* out, const void* ptr, int es, uint64_t cols, uint64_t rows, uint64_t stride,
                        uint32_t box_cols);

#define LP_ROWS 256                       // rows of x of a pair's tile
#define LP_N 256                          // weight rows of a pair's tile
#define LP_BAND 8                         // tiles of x of a band
#define LP_MAX_SPLIT 4                    // pairs that share a tile, at most
#define LP_EPI_WARPS 8
#define LP_THREADS (64 + 32 * LP_EPI_WARPS)
#define LP_A_BYTES (LT_M * LT_BOX)        // of each operand in a box
#define LP_SF_COL 488                     // 8-bit rows: first column of the scales, two sets of 12
#define LP_ACC2_MX 232                    // 8-bit rows: first column of the second accumulator
#define LP_MAX_STAGES 6
#define LP_OUT_BYTES 2048                 // an epilogue warp's piece of the output: 32 rows of at most 64 bytes; two of them
#define LP_X_PITCH 34                     // the same memory as a 32 x 32 exchange: elements of a row

struct lp_params {
  int r_tiles, w_tiles;
  int boxes, subs;                        // boxes and products along k
  int n_tile;                             // outputs of a tile: 256, gated 128
  int full;                               // tiles dealt whole
  int left, sk_pairs;                     // tiles cut along k, and the pairs that share them
  int pairs;
};

struct __align__(16) lp_tail {
  uint64_t full[LP_MAX_STAGES], empty[LP_MAX_STAGES];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t shared_free;                   // the columns both accumulators use have been read
  uint64_t res_full[LP_EPI_WARPS][2];     // a warp's piece of the residual
  uint32_t tmem_base;
  int abort_flag;
  unsigned seen;                          // epilogue warps that have seen all flags
};

template <bool MX> struct lp_ring { static constexpr int BYTES = 2 * LP_A_BYTES + (MX ? 2048 : 0), STAGES = MX ? 5 : 6; };

// ------------------------------------------------------------------------------------------ PTX
// Loads of a pair: the barrier is the first CTA's, whichever CTA the data is for.
__device__ __forceinline__ void lp_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar, uint32_t lead) {
  asm volatile(LT_IF("%5")
               "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], "
               "[%4];\n\t}"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "r"(lead)
               : "memory");
}
__device__ __forceinline__ void lp_mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void lp_mma_mx8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                           uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(acc), "r"(lead)
      : "memory");
}
// (each CTA's scales from its own shared memory to its own tensor memory)
__device__ __forceinline__ void lp_copy_scales(uint32_t dst, uint64_t desc, uint32_t lead) {
  asm volatile(LT_IF("%2") "tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(dst), "l"(desc), "r"(lead) : "memory");
}
// An arrival on the barrier at this place in both CTAs, when the products issued so far have completed.
__device__ __forceinline__ void lp_commit(uint32_t bar, uint32_t lead) {
  asm volatile(LT_IF("%1")
               "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %2;\n\t}"
               ::"r"(bar), "r"(lead), "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ uint32_t lp_map(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void lp_arrive(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void lp_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__host__ __device__ inline uint32_t lp_idesc_bf16() {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(LP_N >> 3) << 17) | ((uint32_t)(LP_ROWS >> 4) << 24);
}
__host__ __device__ inline uint32_t lp_idesc_mx8(int k) {
  return ((uint32_t)k << 4) | ((uint32_t)(LP_N >> 3) << 17) | (1u << 23) | ((uint32_t)(LP_ROWS >> 7) << 27) | ((uint32_t)k << 29);
}
// A warp's piece of the output, 32 rows, from shared memory; columns and rows past the array's end are left out.
__device__ __forceinline__ void lp_put(const CUtensorMap* map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
template <int LEFT> __device__ __forceinline__ void lp_put_read() {        // all but the last LEFT pieces have been read
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory");
}

// ------------------------------------------------------------------------------------------ the deal
// Of pair i: its share of the tiles cut along k (unit u = box u % boxes of tile full + u / boxes), last tile first;
// then the whole tiles i, i + pairs, ...
struct lp_walk {
  long long lo, hi;
  int next_full;
  static __device__ __forceinline__ long long first(const lp_params& p, int i) {
    return i >= p.sk_pairs ? (long long)p.left * p.boxes : (long long)p.left * p.boxes * i / p.sk_pairs;
  }
  __device__ __forceinline__ lp_walk(const lp_params& p, int pair)
      : lo(p.left ? first(p, pair) : 0), hi(p.left ? first(p, pair + 1) : 0), next_full(pair) {}
  __device__ __forceinline__ bool next(const lp_params& p, int pairs, int& tile, int& k0, int& k1) {
    if (hi > lo) {
      const int t = (int)((hi - 1) / p.boxes);
      const long long t0 = (long long)t * p.boxes;
      k1 = (int)(hi - t0);
      k0 = lo > t0 ? (int)(lo - t0) : 0;
      hi = t0 + k0;
      tile = p.full + t;
      return true;
    }
    if (next_full >= p.full) return false;
    tile = next_full;
    next_full += pairs;
    k0 = 0;
    k1 = p.boxes;
    return true;
  }
};
// Tile of x and tile of weights.
__device__ __forceinline__ void lp_place(const lp_params& p, int tile, int& rt, int& wt) {
  const int band = tile / (LP_BAND * p.w_tiles), in = tile - band * LP_BAND * p.w_tiles;
  const int rows = min(LP_BAND, p.r_tiles - band * LP_BAND);
  wt = in / rows;
  rt = band * LP_BAND + in - wt * rows;
}

// ------------------------------------------------------------------------------------------ epilogue
__device__ __forceinline__ uint32_t lp_pack(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// 32 elements of T from p as f32, the same for all lanes; those from `most` on are 0.
__device__ __forceinline__ void lp_add32(float (&v)[32], const uint16_t* p, int most) {
  if (most >= 32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 r = __ldg(reinterpret_cast<const uint4*>(p) + i);
      const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[8 * i + 2 * j] += __uint_as_float(w[j] << 16);
        v[8 * i + 2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] += j < most ? __uint_as_float((uint32_t)p[j] << 16) : 0.f;
  }
}
// Where the copy engine has 16-byte chunk c of row r: pieces with rows of 64 bytes, and of 32.
__device__ __forceinline__ uint32_t lp_at64(int r, int c) { return (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4)); }
__device__ __forceinline__ uint32_t lp_at32(int r, int c) { return (uint32_t)(r * 32 + ((c ^ ((r >> 2) & 1)) << 4)); }

// ------------------------------------------------------------------------------------------ the kernel
template <bool MX, bool GATED>
__global__ void __launch_bounds__(LP_THREADS, 1) k_linear_pair(
    const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_u,
    const __grid_constant__ CUtensorMap map_sx, const __grid_constant__ CUtensorMap map_sw,
    const __grid_constant__ CUtensorMap map_su, const __grid_constant__ CUtensorMap map_out,
    const __grid_constant__ CUtensorMap map_res, const lp_params p, const lin_args a, int wide_out, int wide_res,
    float* __restrict__ partial, int32_t* flags, int32_t* status) {
  constexpr int BOX_EL = MX ? 128 : 64, STAGE = lp_ring<MX>::BYTES, LP_STAGES = lp_ring<MX>::STAGES;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* pieces = smem + LP_STAGES * STAGE;
  lp_tail& T = *reinterpret_cast<lp_tail*>(pieces + LP_EPI_WARPS * 2 * LP_OUT_BYTES);
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  volatile int* abort_flag = &T.abort_flag;

  if (threadIdx.x == 0) {
    for (int s = 0; s < LP_STAGES; ++s) { mbar_init(&T.full[s], 1); mbar_init(&T.empty[s], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&T.acc_full[i], 1); mbar_init(&T.acc_empty[i], 2 * LP_EPI_WARPS); }
    mbar_init(&T.shared_free, LP_EPI_WARPS);           // four warps of each CTA
    for (int i = 0; i < LP_EPI_WARPS; ++i) { mbar_init(&T.res_full[i][0], 1); mbar_init(&T.res_full[i][1], 1); }
    T.abort_flag = 0;
    T.seen = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&T.tmem_base)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  lp_cluster_sync();                       // the barriers of both CTAs exist
  tc_fence_after();
  const uint32_t tmem_base = T.tmem_base;
  lp_walk walk(p, pair);
  int tile, k0, k1;
  bool more = walk.next(p, pairs, tile, k0, k1);
  jk_pdl_wait();
  jk_pdl_trigger();

  if (warp == 0) {
    // ------------------------------------------------------------------ copies
    const uint32_t lead = lt_elect(), base = smem_u32(smem);
    const uint32_t full0 = lp_map(smem_u32(T.full), 0), own_full0 = smem_u32(T.full);
    bool ok = true;
    int s = 0;
    long long issued = 0;
    uint32_t ph = 0;
    for (; ok && more; more = walk.next(p, pairs, tile, k0, k1)) {
      int rt, wt;
      lp_place(p, tile, rt, wt);
      const int xr = rt * LP_ROWS + rank * LT_M;
      const int wr = GATED ? wt * LT_M : wt * LP_N + rank * LT_M;
      const CUtensorMap* mw = GATED && rank ? &map_u : &map_w;
      for (int k = k0; k < k1; ++k) {
        if (issued >= LP_STAGES) ok = mbar_wait(&T.empty[s], ph ^ 1u, abort_flag, status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t st = base + (uint32_t)s * STAGE, bar = full0 + 8u * (uint32_t)s;
        // (both CTAs' bytes; what the other's copies bring may arrive before it is expected)
        if (rank == 0) lt_expect(own_full0 + 8u * (uint32_t)s, 2u * (2 * LP_A_BYTES + (MX ? 3 * MX_TILE_BYTES : 0)), lead);
        lp_box(st, &map_x, k * BOX_EL, xr, bar, lead);
        lp_box(st + LP_A_BYTES, mw, k * BOX_EL, wr, bar, lead);
        if (MX) {
          // scales: of this CTA's rows of x, and of all 256 weight rows
          lp_box(st + 2 * LP_A_BYTES, &map_sx, 0, (rt * 2 + rank) * a.k_tiles_in + k, bar, lead);
          lp_box(st + 2 * LP_A_BYTES + MX_TILE_BYTES, &map_sw, 0, (GATED ? wt : 2 * wt) * a.k_tiles_in + k, bar, lead);
          lp_box(st + 2 * LP_A_BYTES + 2 * MX_TILE_BYTES, GATED ? &map_su : &map_sw, 0,
                 (GATED ? wt : 2 * wt + 1) * a.k_tiles_in + k, bar, lead);
        }
        ++issued;
        if (++s == LP_STAGES) { s = 0; ph ^= 1u; }
      }
    }
    // (the last stages' releases come from the other CTA: they have to be there before this one's memory goes)
    for (long long i = issued > LP_STAGES ? issued - LP_STAGES : 0; i < issued && ok; ++i)
      ok = mbar_wait(&T.empty[i % LP_STAGES], (uint32_t)(i / LP_STAGES) & 1u, abort_flag, status);
    if (!ok && rank == 0) {
      // gave up: the copies in flight land before the CTA's memory goes away (the second CTA's are waited for
      // here too: the barriers count both)
      for (long long i = issued > LP_STAGES ? issued - LP_STAGES : 0; i < issued; ++i) {
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(&T.full[i % LP_STAGES], (uint32_t)(i / LP_STAGES) & 1u))
          if (global_ns() - t0 > TC_WAIT_NS) break;
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products
    if (rank == 0) {
      const uint32_t lead = lt_elect(), tm = __shfl_sync(0xffffffffu, tmem_base, 0);
      const uint32_t empty0 = smem_u32(T.empty);
      const uint64_t d0 = smem_desc_sw128(smem_u32(smem));
      const uint64_t s0 = LT_SCALE_DESC | (uint64_t)(((smem_u32(smem) + 2 * LP_A_BYTES) & 0x3FFFFu) >> 4);
      bool ok = true;
      int s = 0, seg = 0, par = 0;
      uint32_t ph = 0;
      for (; ok && more; more = walk.next(p, pairs, tile, k0, k1)) {
        const int buf = seg & 1, use = seg >> 1;
        if (use > 0) ok = mbar_wait(&T.acc_empty[buf], ((uint32_t)use & 1u) ^ 1u, abort_flag, status);
        if (MX && seg > 0) ok = ok && mbar_wait(&T.shared_free, ((uint32_t)seg & 1u) ^ 1u, abort_flag, status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tm + (uint32_t)(buf * (MX ? LP_ACC2_MX : LP_N));
        uint32_t acc = 0;
        for (int k = k0; k < k1; ++k) {
          ok = mbar_wait(&T.full[s], ph, abort_flag, status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          const uint32_t st = (uint32_t)s * (uint32_t)(STAGE >> 4);
          const uint64_t dx = d0 + st, dw = dx + (LP_A_BYTES >> 4);
          const int n_sub = p.subs - k * 4;                          // products past the end of k are left out
          uint32_t sf = 0;
          if (MX) {
            sf = tm + (uint32_t)(LP_SF_COL + par * 12);              // two sets take turns
            par ^= 1;
            const uint64_t ds = s0 + st;
            lp_copy_scales(sf, ds, lead);
            lp_copy_scales(sf + 4, ds + (MX_TILE_BYTES >> 4), lead);
            lp_copy_scales(sf + 8, ds + (2 * MX_TILE_BYTES >> 4), lead);
          }
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4) {
            if (k4 >= n_sub) break;
            if (MX) lp_mma_mx8(d, dx + 2 * k4, dw + 2 * k4, lp_idesc_mx8(k4), sf, sf + 4, acc, lead);
            else lp_mma_bf16(d, dx + 2 * k4, dw + 2 * k4, lp_idesc_bf16(), acc, lead);
            acc = 1;
          }
          lp_commit(empty0 + 8u * (uint32_t)s, lead);
          if (++s == LP_STAGES) { s = 0; ph ^= 1u; }
        }
        if (ok) lp_commit(smem_u32(&T.acc_full[buf]), lead);
        ++seg;
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue
    const int quarter = warp & 3;          // the lanes of tensor memory this warp may read
    const int half = (warp - 2) >> 2;      // the columns 0 .. 127 upwards, or 255 .. 128 downwards
    unsigned char* mine = pieces + (warp - 2) * 2 * LP_OUT_BYTES;    // 1024-byte aligned: two pieces
    const uint32_t mine_u32 = smem_u32(mine);
    uint64_t* res_full = T.res_full[warp - 2];
    uint32_t res_ph = 0;                   // phases of the two, a bit each
    const uint32_t acc_empty0 = lp_map(smem_u32(T.acc_empty), 0), shared0 = lp_map(smem_u32(&T.shared_free), 0);
    constexpr int CHUNKS = GATED ? 2 : 4;  // of 32 outputs, for this warp
    int seg = 0;
    bool ok = true;
    for (; ok && more; more = walk.next(p, pairs, tile, k0, k1)) {
      int rt, wt;
      lp_place(p, tile, rt, wt);
      const int row0 = rt * LP_ROWS + rank * LT_M + quarter * 32, n0 = wt * p.n_tile;
      const int buf = seg & 1, use = seg >> 1;
      const bool whole = k1 == p.boxes;    // this pair finishes the tile
      // the pairs that have the tile's first k steps
      int from = pair;
      if (whole && k0 > 0) {
        const long long t0 = (long long)(tile - p.full) * p.boxes;
        while (from > 0 && lp_walk::first(p, from) > t0) --from;
        for (int j = from; j < pair && ok; ++j) {
          const long long c0 = clock64();
          while (ok && ld_acquire(flags + 2 * j + rank) != LP_EPI_WARPS) {
            if (*abort_flag) ok = false;
            else if (clock64() - c0 > TC_WAIT_CYCLES) {
              *abort_flag = 1;
              jk_set_status(status, JK_ERR_TIMEOUT);
              ok = false;
            }
          }
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        // the last warp to have seen them puts the flags back for the next call
        if (lane == 0 && atomicAdd(&T.seen, 1u) == LP_EPI_WARPS - 1)
          for (int j = from; j < pair; ++j) flags[2 * j + rank] = 0;
        __syncwarp();
      }
      auto chunk = [&](int c) { return half ? (GATED ? 3 : 7) - c : c; };
      const bool rows_live = row0 < a.rows;
      // The residual of a chunk is brought to the piece that the chunk's outputs will take.
      auto ask_residual = [&](int c) {
        const int n = n0 + chunk(c) * 32;
        if (lane == 0 && n < a.n_out && rows_live) {
          lp_put_read<0>();                // (the piece's last outputs have been read)
          lt_expect(smem_u32(&res_full[c & 1]), LP_OUT_BYTES, 1u);
          lt_box(mine_u32 + (c & 1) * LP_OUT_BYTES, &map_res, n, row0, smem_u32(&res_full[c & 1]), 1u);
        }
      };
      const bool res_tma = whole && a.residual && wide_res;
      if (res_tma) ask_residual(0);
      // (a partial: 16 bytes of a lane next to the next lane's, 8 times for a chunk of 32 columns)
      const size_t my_part = (size_t)quarter * LP_N * 32 + lane * 4;
      float4 t[8], tu[GATED ? 8 : 1];
      auto ask_part = [&](int i, int q) {
        const float* o = partial + (size_t)(2 * i + rank) * LT_SLOT + my_part + (size_t)q * 32 * 32;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          t[j] = __ldcg(reinterpret_cast<const float4*>(o + j * 128));
          if constexpr (GATED) tu[j] = __ldcg(reinterpret_cast<const float4*>(o + LT_M * 32 + j * 128));
        }
      };
      // (one other pair's partials are asked for a chunk ahead; not in a gated block, whose chunk fills the registers)
      constexpr bool AHEAD = !GATED;
      if (AHEAD && from < pair) ask_part(pair - 1, chunk(0));
      ok = mbar_wait(&T.acc_full[buf], (uint32_t)use & 1u, abort_flag, status);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * (MX ? LP_ACC2_MX : LP_N));
#pragma unroll 1
      for (int c = 0; c < CHUNKS; ++c) {
        __syncwarp();
        const int q = chunk(c);            // chunk of 32 outputs
        float v[32], u[GATED ? 32 : 1];
        {
          uint32_t w[32];
          tmem_ld32(t_addr + (uint32_t)(q * 32), w);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(w[j]);
          if constexpr (GATED) {
            tmem_ld32(t_addr + (uint32_t)(LT_M + q * 32), w);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] = __uint_as_float(w[j]);
          }
        }
        if ((MX && c == 0) || c == CHUNKS - 1) {
          tc_fence_before();
          __syncwarp();
          // the columns that both accumulators use: the last 24 of the first, the first 24 of the second
          if (MX && c == 0 && half != buf && lane == 0) lp_arrive(shared0);
          if (c == CHUNKS - 1 && lane == 0) lp_arrive(acc_empty0 + 8u * (uint32_t)buf);
        }
        if (!whole) {
          float* o = partial + (size_t)blockIdx.x * LT_SLOT + my_part + (size_t)q * 32 * 32;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            __stcg(reinterpret_cast<float4*>(o + j * 128), make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
            if constexpr (GATED)
              __stcg(reinterpret_cast<float4*>(o + LT_M * 32 + j * 128),
                     make_float4(u[4 * j], u[4 * j + 1], u[4 * j + 2], u[4 * j + 3]));
          }
          continue;
        }
        for (int i = pair - 1; i >= from; --i) {
          if (!AHEAD || i < pair - 1) ask_part(i, q);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            v[4 * j] += t[j].x; v[4 * j + 1] += t[j].y; v[4 * j + 2] += t[j].z; v[4 * j + 3] += t[j].w;
            if constexpr (GATED) {
              u[4 * j] += tu[j].x; u[4 * j + 1] += tu[j].y; u[4 * j + 2] += tu[j].z; u[4 * j + 3] += tu[j].w;
            }
          }
        }
        if (AHEAD && from < pair && c + 1 < CHUNKS) ask_part(pair - 1, chunk(c + 1));
        if (res_tma && c + 1 < CHUNKS) ask_residual(c + 1);
        const int n = n0 + q * 32, most = a.n_out - n;
        if (most <= 0 || !rows_live) continue;
        unsigned char* piece = mine + (c & 1) * LP_OUT_BYTES;
        // ---- the epilogue proper: the lane's row, outputs n .. n + 31
        if (a.bias) lp_add32(v, (const uint16_t*)a.bias + n, most);
        lin_act_all(v, a.act, a.out_type == JK_ROWS_F32);
        if constexpr (GATED) {
          if (a.bias_up) lp_add32(u, (const uint16_t*)a.bias_up + n, most);
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] *= u[j];
        }
        if (res_tma) {
          ok = mbar_wait(&res_full[c & 1], (res_ph >> (c & 1)) & 1u, abort_flag, status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          res_ph ^= 1u << (c & 1);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 r = *reinterpret_cast<const uint4*>(piece + lp_at64(lane, i));
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              v[8 * i + 2 * j] += __uint_as_float(w[j] << 16);
              v[8 * i + 2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u);
            }
          }
        } else {
          if (lane == 0) {                 // the piece's last outputs have been read
            if (wide_out && a.out_type != JK_ROWS_F32 && !a.residual) lp_put_read<1>();
            else lp_put_read<0>();
          }
          __syncwarp();
          if (a.residual) {
            // rows that begin anywhere: read along the rows, handed out through shared memory
            uint16_t* X = reinterpret_cast<uint16_t*>(mine);
            const uint16_t* rp = (const uint16_t*)a.residual + (size_t)row0 * a.r_stride + n + lane;
#pragma unroll 8
            for (int j = 0; j < 32; ++j, rp += a.r_stride)
              X[j * LP_X_PITCH + lane] = row0 + j < a.rows && lane < most ? *rp : (uint16_t)0;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += __uint_as_float((uint32_t)X[lane * LP_X_PITCH + j] << 16);
            __syncwarp();
          }
        }
        if (a.out_type == JK_ROWS_MX8) {   // n_out is a multiple of 32: all of the block or nothing
          float m = 0.f;
#pragma unroll
          for (int j = 0; j < 32; ++j) m = fmaxf(m, paged_mag(v[j]));
          const int e = paged_scale_exp(m);
          const float inv = paged_pow2(-e);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
              o[j] = paged_pack4(v[16 * i + 4 * j] * inv, v[16 * i + 4 * j + 1] * inv, v[16 * i + 4 * j + 2] * inv, v[16 * i + 4 * j + 3] * inv);
            *reinterpret_cast<uint4*>(piece + lp_at32(lane, i)) = make_uint4(o[0], o[1], o[2], o[3]);
          }
          if (row0 + lane < a.rows) a.out_scale[mx_scale_at(row0 + lane, n >> 5, a.k_tiles_out)] = (uint8_t)(e + 127);
        } else if (a.out_type == JK_ROWS_T) {
          if (wide_out) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<uint4*>(piece + lp_at64(lane, i)) =
                  make_uint4(lp_pack(v[8 * i], v[8 * i + 1]), lp_pack(v[8 * i + 2], v[8 * i + 3]),
                             lp_pack(v[8 * i + 4], v[8 * i + 5]), lp_pack(v[8 * i + 6], v[8 * i + 7]));
          } else {
            uint16_t* X = reinterpret_cast<uint16_t*>(mine);
            uint32_t* x32 = reinterpret_cast<uint32_t*>(&X[lane * LP_X_PITCH]);
#pragma unroll
            for (int j = 0; j < 16; ++j) x32[j] = lp_pack(v[2 * j], v[2 * j + 1]);
            __syncwarp();
            uint16_t* o = (uint16_t*)a.out + (size_t)row0 * a.o_stride + n + lane;
#pragma unroll 8
            for (int j = 0; j < 32; ++j, o += a.o_stride)
              if (row0 + j < a.rows && lane < most) *o = X[j * LP_X_PITCH + lane];
          }
        } else if (wide_out) {             // f32: 16 outputs to a piece
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<uint4*>(mine + h * LP_OUT_BYTES + lp_at64(lane, i)) =
                  make_uint4(__float_as_uint(v[16 * h + 4 * i]), __float_as_uint(v[16 * h + 4 * i + 1]),
                             __float_as_uint(v[16 * h + 4 * i + 2]), __float_as_uint(v[16 * h + 4 * i + 3]));
        } else if (row0 + lane < a.rows) {
          float* o = (float*)a.out + (size_t)(row0 + lane) * a.o_stride + n;
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (j < most) o[j] = v[j];
        }
        if (wide_out) {
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (a.out_type == JK_ROWS_F32) {
              lp_put(&map_out, n, row0, mine_u32);
              if (most > 16) lp_put(&map_out, n + 16, row0, mine_u32 + LP_OUT_BYTES);
            } else {
              lp_put(&map_out, n, row0, mine_u32 + (c & 1) * LP_OUT_BYTES);
            }
          }
        }
      }
      if (!ok) break;
      if (!whole) {
        __syncwarp();
        if (lane == 0) add_release(flags + blockIdx.x, 1);
      }
      ++seg;
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  lp_cluster_sync();                       // nobody's memory is used any more
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem_base) : "memory");
  }
}

// ------------------------------------------------------------------------------------------ host side
// The deal.  The tiles of the last, incomplete turn: whole (a turn more), or cut among 2, 3 or 4 pairs each, which costs
// the hand-over: 18, 24, 31 boxes' time (5.6, 7.5 and 9.6 us measured at 16 tiles, a box 0.31).  Cut at K = 8192 in bf16,
// 16 tiles: 43.7 us whole, 31.9, 28.1, 27.2 among 2, 3, 4; at K = 2048: 16.4 whole, 17.5, 18.0, 19.4.  Returns the cost
// in us, with a launch.
double jk_linear_pair_plan(const lin_args& a, bool mx, int sms, lp_params* out) {
  const bool gated = a.w_up != nullptr;
  const int es = mx ? 1 : 2, box_el = LT_BOX / es;
  lp_params p;
  memset(&p, 0, sizeof(p));
  p.n_tile = gated ? LT_M : LP_N;
  p.r_tiles = (a.rows + LP_ROWS - 1) / LP_ROWS;
  p.w_tiles = (a.n_out + p.n_tile - 1) / p.n_tile;
  p.boxes = (a.n_in + box_el - 1) / box_el;
  p.subs = (a.n_in * es + 31) / 32;
  const long long tiles = (long long)p.r_tiles * p.w_tiles;
  const int pairs = sms / 2, left = (int)(tiles % pairs);
  static const int hand_over[LP_MAX_SPLIT] = {0, 18, 24, 31};
  int split = 1;
  double best = left ? p.boxes : 0;
  for (int s = 2; left && s <= LP_MAX_SPLIT && s <= p.boxes && left * (s - 1) < pairs; ++s) {
    const int on = left * s < pairs ? left * s : pairs;
    const double cost = (double)left * p.boxes / on + hand_over[s - 1];
    if (cost < best) { best = cost; split = s; }
  }
  p.left = split > 1 ? left : 0;
  p.full = (int)(tiles - p.left);
  p.sk_pairs = p.left * split < pairs ? p.left * split : pairs;
  p.pairs = tiles >= pairs ? pairs : p.left ? p.sk_pairs : p.full;
  if (out) *out = p;
  const double us = 0.31 * (best + (double)(tiles / pairs) * p.boxes), hbm_us = (double)a.n_out * a.n_in * es * (1 + gated) / 6.4e6;
  return 6.9 + (us > hbm_us ? us : hbm_us);
}

int jk_linear_pair(jk_ctx* ctx, cudaStream_t st, const lin_args& a, bool mx) {
  const bool gated = a.w_up != nullptr;
  const int es = mx ? 1 : 2, box_el = LT_BOX / es;
  lp_params p;
  jk_linear_pair_plan(a, mx, ctx->sm_count < LT_MAX_CTAS ? ctx->sm_count : LT_MAX_CTAS, &p);
  CUtensorMap mx_map, mw, mu, msx, msw, msu;
  auto map = [&](CUtensorMap* m, const void* ptr, uint64_t rows, uint64_t stride) {
    const uint64_t dims[2] = {(uint64_t)a.n_in, rows}, str[1] = {stride * es};
    const uint32_t box[2] = {(uint32_t)box_el, LT_M};
    return mx ? jk_tma_encode_u8(ctx, m, ptr, 2, dims, str, box) : jk_tma_encode_bf16(ctx, m, ptr, 2, dims, str, box);
  };
  int rc = map(&mx_map, a.x, a.rows, a.x_stride);
  if (rc == JK_OK) rc = map(&mw, a.w, a.n_out, a.n_in);
  mu = mw;
  if (rc == JK_OK && gated) rc = map(&mu, a.w_up, a.n_out, a.n_in);
  msx = msw = msu = mw;
  if (mx) {
    const uint64_t xt = (uint64_t)((a.rows + 127) / 128) * a.k_tiles_in, wt = (uint64_t)((a.n_out + 127) / 128) * a.k_tiles_in;
    if (rc == JK_OK) rc = jk_tma_encode_scales(ctx, &msx, a.x_scale, xt);
    if (rc == JK_OK) rc = jk_tma_encode_scales(ctx, &msw, a.w_scale, wt);
    if (rc == JK_OK && gated) rc = jk_tma_encode_scales(ctx, &msu, a.w_up_scale, wt);
  }
  if (rc != JK_OK) return rc;
  // Outputs and residuals whose rows begin at multiples of 16 bytes go through the copy engine, in pieces of 32 rows.
  const bool f32 = a.out_type == JK_ROWS_F32, q8 = a.out_type == JK_ROWS_MX8;
  const int os = q8 ? 1 : f32 ? 4 : 2;
  const int wide_out = (a.o_stride * os) % 16 == 0, wide_res = a.residual && wide_out && !f32 && (a.r_stride * 2) % 16 == 0;
  CUtensorMap mo = mw, mr = mw;
  if (wide_out) rc = jk_tma_encode_piece(ctx, &mo, a.out, q8 ? 1 : f32 ? 4 : 2, a.n_out, a.rows, a.o_stride, f32 ? 16 : 32);
  if (rc == JK_OK && wide_res) rc = jk_tma_encode_piece(ctx, &mr, a.residual, 2, a.n_out, a.rows, a.r_stride, 32);
  if (rc != JK_OK) return rc;
  auto kernel = mx ? (gated ? k_linear_pair<true, true> : k_linear_pair<true, false>)
                   : (gated ? k_linear_pair<false, true> : k_linear_pair<false, false>);
  const size_t smem = (size_t)(mx ? lp_ring<true>::STAGES * lp_ring<true>::BYTES : lp_ring<false>::STAGES * lp_ring<false>::BYTES) +
                      LP_EPI_WARPS * 2 * LP_OUT_BYTES + sizeof(lp_tail) + 1024;
  const int bit = 16 << (2 * mx + gated);
  if (!(ctx->lin_smem_set & bit)) {
    JK_CUDA_CHECK(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    ctx->lin_smem_set |= bit;
  }
  JK_PROF(ctx, st, JK_ST_LINEAR);
  jk_launch_pdl_cluster(kernel, dim3(2 * p.pairs), dim3(LP_THREADS), 2, smem, st, mx_map, mw, mu, msx, msw, msu, mo, mr, p, a,
                        wide_out, wide_res,                        (float*)(ctx->ws + ctx->lay.lin_part), (int32_t*)(ctx->ws + ctx->lay.lin_flag),
                        (int32_t*)(ctx->ws + ctx->lay.status));
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}
