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
// its operands in L2.  The tiles left over for a last, incomplete turn may come first, cut along k
// into even shares (jk_linear_pair_plan): the pair that has a tile's end finishes it from the others' f32 partials, as in
// the kernel for few rows.
//
// Accumulators: two of 256 columns for bf16.  8-bit rows need 24 columns for scales; there the second
// accumulator begins at column 232, and of the 24 columns that both use the epilogue reads first.
//
// Roles: warp 0 loads, warp 1 (of the pair's first CTA) multiplies, the others (8, or 16 where nothing hides them) are the
// epilogue.  It works on 16 columns at a time: its instructions come through a loop that stays in the cache (32 columns
// at a time waited for instructions, 8 for latency).  Outputs and the residual go through the copy engine
// where their rows begin and end at multiples of 16 bytes.  Waits are bounded as in the kernel for few rows.
//
// Bound by the tensor cores and the power they take: 2047 rows, 5120 x 5120 in bf16 79 us on a cool card (1360 TFLOP/s), 87 to
// 92 back to back, where the clock falls to 1.5 GHz; 4099 rows, 14336 x 4096 gated in 8 bits 365 us (2640), 430 back to
// back.  480 rows, 5120 x 13824 in 8 bits 40 us (1690), 42 to 48 back to back: 40 tiles among 74 pairs, of which the hand-over
// takes 13.
#include <type_traits>

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
#define LP_W 16                           // columns that an epilogue warp works on at a time
#define LP_A_BYTES (LT_M * LT_BOX)        // of each operand in a box
#define LP_SF_COL 488                     // 8-bit rows: first column of the scales, two sets of 12
#define LP_ACC2_MX 232                    // 8-bit rows: first column of the second accumulator
#define LP_MAX_STAGES 7
#define LP_MAX_EPI 16
#define LP_PIECE 2048                     // an epilogue warp's piece of the output: 32 rows of 64 bytes; two of them
#define LP_PIECE8 1024                    // ... of 8-bit outputs: 32 rows of 32; behind 32 x 32 f32
#define LP_PART 2048                      // an epilogue warp's piece of a partial: 32 rows of LP_W columns, f32
#define LP_MAX_PARTS 5
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
  uint64_t res_full[LP_MAX_EPI][2];       // a warp's piece of the residual
  uint64_t part_full[LP_MAX_EPI][LP_MAX_PARTS];      // ... its pieces of the partials
  uint32_t tmem_base;
  int abort_flag;
  unsigned seen;                          // epilogue warps that have seen all flags
};

// LAST: a pair finishes at most one tile, and does so last.  The ring is free by then and holds the epilogue's pieces
// and what it is handed; it has a stage more for that, and 16 warps, not 8, get the epilogue done, which nothing hides.
template <bool MX, bool OUT8, bool LAST> struct lp_smem {
  static constexpr int EPI = LAST ? 16 : 8, THREADS = 64 + 32 * EPI;
  static constexpr int STAGE = 2 * LP_A_BYTES + (MX ? 2048 : 0), STAGES = (MX || (OUT8 && !LAST) ? 5 : 6) + LAST;
  static constexpr int WARP = 2 * LP_PIECE + (OUT8 ? 2 * LP_PIECE8 : 0);           // of an epilogue warp
  static constexpr int PARTS = (STAGES * STAGE / EPI - WARP) / LP_PART < LP_MAX_PARTS ? (STAGES * STAGE / EPI - WARP) / LP_PART : LP_MAX_PARTS;
  static constexpr size_t BYTES = (size_t)STAGES * STAGE + (LAST ? 0 : EPI * WARP) + sizeof(lp_tail) + 1024;
  static_assert(BYTES <= LT_SMEM && STAGES <= LP_MAX_STAGES && PARTS >= 1, "shared memory");
};

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
__device__ __forceinline__ void lp_arrive(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
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

// Elements of T added to f32: 8 of a 16-byte piece; LP_W from p, where those from `most` on do not exist.
template <int AT> __device__ __forceinline__ void lp_add8(float (&v)[LP_W], const uint4& r) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[AT + 2 * j] += __uint_as_float(w[j] << 16);
    v[AT + 2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u);
  }
}
__device__ __forceinline__ void lp_add(float (&v)[LP_W], const uint16_t* p, int most) {
  if (most >= LP_W && ((uintptr_t)p & 15) == 0) {
    const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
    lp_add8<0>(v, a);
    lp_add8<8>(v, b);
  } else {
#pragma unroll
    for (int j = 0; j < LP_W; ++j) v[j] += j < most ? __uint_as_float((uint32_t)p[j] << 16) : 0.f;
  }
}
// Where the copy engine has 16-byte chunk c of row r: pieces with rows of 64 bytes, and of 32.
__device__ __forceinline__ uint32_t lp_at64(int r, int c) { return (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4)); }
__device__ __forceinline__ uint32_t lp_at32(int r, int c) { return (uint32_t)(r * 32 + ((c ^ ((r >> 2) & 1)) << 4)); }
// (and where an f32 row of 128 bytes is kept, so that neighbouring rows meet in different banks)
__device__ __forceinline__ uint32_t lp_at128(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }

// ------------------------------------------------------------------------------------------ the kernel
template <bool MX, bool GATED, bool OUT8, bool LAST>
__global__ void __launch_bounds__((lp_smem<MX, OUT8, LAST>::THREADS), 1) k_linear_pair(
    const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_u,
    const __grid_constant__ CUtensorMap map_sx, const __grid_constant__ CUtensorMap map_sw,
    const __grid_constant__ CUtensorMap map_su, const __grid_constant__ CUtensorMap map_out,
    const __grid_constant__ CUtensorMap map_res, const lp_params p, const lin_args a, int wide_out, int wide_res,
    float* __restrict__ partial, int32_t* flags, int32_t* status) {
  typedef lp_smem<MX, OUT8, LAST> L;
  constexpr int BOX_EL = MX ? 128 : 64, STAGE = L::STAGE, LP_STAGES = L::STAGES, WARP = L::WARP, EPI = L::EPI, PARTS = L::PARTS;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* pieces = LAST ? smem : smem + LP_STAGES * STAGE;
  lp_tail& T = *reinterpret_cast<lp_tail*>(smem + LP_STAGES * STAGE + (LAST ? 0 : EPI * WARP));
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  volatile int* abort_flag = &T.abort_flag;

  if (threadIdx.x == 0) {
    for (int s = 0; s < LP_STAGES; ++s) { mbar_init(&T.full[s], 1); mbar_init(&T.empty[s], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&T.acc_full[i], 1); mbar_init(&T.acc_empty[i], 2 * EPI); }
    mbar_init(&T.shared_free, 8);          // four warps of each CTA
    for (int i = 0; i < EPI; ++i) { mbar_init(&T.res_full[i][0], 1); mbar_init(&T.res_full[i][1], 1); }
    for (int i = 0; LAST && i < EPI * LP_MAX_PARTS; ++i) mbar_init(&T.part_full[0][0] + i, 1);
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
  lt_cluster_sync();                       // the barriers of both CTAs exist
  tc_fence_after();
  const uint32_t tmem_base = T.tmem_base;
  lp_walk walk(p, pair);
  int tile, k0, k1;
  bool more = walk.next(p, pairs, tile, k0, k1);
  if (warp == 2 && more && lane < LP_STAGES && k0 + lane < k1) {
    // The boxes of the first ring are asked into L2 while the kernel before still runs.
    int rt, wt;
    lp_place(p, tile, rt, wt);
    l2_prefetch_box(&map_x, (k0 + lane) * BOX_EL, rt * LP_ROWS + rank * LT_M);
    l2_prefetch_box(GATED && rank ? &map_u : &map_w, (k0 + lane) * BOX_EL, GATED ? wt * LT_M : wt * LP_N + rank * LT_M);
  }
  __syncwarp();
  jk_pdl_wait();
  jk_pdl_trigger();

  if (warp == 0) {
    // ------------------------------------------------------------------ copies
    const uint32_t lead = lt_elect(), base = smem_u32(smem);
    const uint32_t full0 = lt_map(smem_u32(T.full), 0), own_full0 = smem_u32(T.full);
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
    const int share = (warp - 2) >> 2;     // of the columns: the first half's are taken upwards, the others downwards
    unsigned char* mine = pieces + (warp - 2) * WARP;                // 1024-byte aligned
    const uint32_t mine_u32 = smem_u32(mine);
    uint64_t* res_full = T.res_full[warp - 2];
    uint32_t res_ph = 0;                   // phases of the two, a bit each
    const uint32_t acc_empty0 = lt_map(smem_u32(T.acc_empty), 0), shared0 = lt_map(smem_u32(&T.shared_free), 0);
    constexpr int G = 1 + GATED, CHUNKS = 32 / EPI / G;      // of 32 outputs, for this warp
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
          while (ok && ld_acquire(flags + 2 * j + rank) != EPI) {
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
        if (lane == 0 && atomicAdd(&T.seen, 1u) == EPI - 1)
          for (int j = from; j < pair; ++j) flags[2 * j + rank] = 0;
        __syncwarp();
      }
      auto chunk = [&](int c) { return share < EPI / 8 ? share * CHUNKS + c : (share + 1) * CHUNKS - 1 - c; };
      const bool rows_live = row0 < a.rows, live = row0 + lane < a.rows;
      // The residual of a chunk is brought to the piece that the chunk's outputs will take.
      auto ask_residual = [&](int c) {
        const int n = n0 + chunk(c) * 32;
        if (lane == 0 && n < a.n_out && rows_live) {
          lp_put_read<0>();                // (the piece's last outputs have been read)
          lt_expect(smem_u32(&res_full[c & 1]), LP_PIECE, 1u);
          lt_box(mine_u32 + (c & 1) * LP_PIECE, &map_res, n, row0, smem_u32(&res_full[c & 1]), 1u);
        }
      };
      // (where neither the residual's nor the outputs' rows begin at multiples of 16 bytes, both pass through an exchange;
      // where only one does, and for f32 and 8-bit outputs, a lane reads its row)
      const bool res_tma = !OUT8 && whole && a.residual && wide_res;
      const bool res_x = !OUT8 && a.residual && a.out_type == JK_ROWS_T && !wide_out;
      if (res_tma && !LAST) ask_residual(0);
      if (res_tma && LAST && lane < CHUNKS && rows_live && n0 + chunk(lane) * 32 < a.n_out)
        l2_prefetch_box(&map_res, n0 + chunk(lane) * 32, row0);
      // (a partial: 16 bytes of a lane next to the next lane's; one other pair's are asked for LP_W columns ahead)
      const size_t my_part = (size_t)quarter * LP_N * 32 + lane * 4;
      float4 t[LP_W / 4], tu[GATED ? LP_W / 4 : 1];
      auto ask_part = [&](int i, int col) {
        const float* o = partial + (size_t)(2 * i + rank) * LT_SLOT + my_part + (size_t)col * 32;
#pragma unroll
        for (int j = 0; j < LP_W / 4; ++j) {
          t[j] = __ldcg(reinterpret_cast<const float4*>(o + j * 128));
          if constexpr (GATED) tu[j] = __ldcg(reinterpret_cast<const float4*>(o + LT_M * 32 + j * 128));
        }
      };
      const int parts = pair - from, asks = parts * (CHUNKS * 32 / LP_W) * G;
      unsigned char* part_smem = smem + EPI * WARP + (warp - 2) * (PARTS * LP_PART);
      int asked = 0, taken = 0;            // (LAST: pieces come in the order in which they are added)
      auto ask_parts = [&] {
        for (; asked < asks && asked < taken + PARTS; ++asked) {
          if (lane) continue;
          const int g = asked % G, k = pair - 1 - asked / G % parts, step = asked / G / parts;
          const uint32_t bar = smem_u32(&T.part_full[warp - 2][asked % PARTS]);
          const int col = chunk(step * LP_W / 32) * 32 + step * LP_W % 32 + g * LT_M;
          lt_expect(bar, LP_PART, 1u);
          lt_bulk(smem_u32(part_smem) + (uint32_t)(asked % PARTS) * LP_PART,
                  partial + (size_t)(2 * k + rank) * LT_SLOT + (size_t)(quarter * LP_N + col) * 32, LP_PART, bar, 1u);
        }
      };
      if (!LAST && parts) ask_part(pair - 1, chunk(0) * 32);
      ok = mbar_wait(&T.acc_full[buf], (uint32_t)use & 1u, abort_flag, status);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      if (LAST && whole) {                 // (the products of all boxes are done)
        if (res_tma) ask_residual(0);
        if (parts) {
          asm volatile("fence.proxy.async;" ::: "memory");       // the partials were written by ordinary stores
          ask_parts();
        }
      }
      const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * (MX ? LP_ACC2_MX : LP_N));
      bool first = true;                   // no output of this tile has been stored yet
#pragma unroll 1
      for (int c = 0; c < CHUNKS; ++c) {
        const int q = chunk(c), n = n0 + q * 32, most = a.n_out - n;
        const bool out_live = whole && most > 0 && rows_live;
        unsigned char* piece = mine + (OUT8 ? 2 * LP_PIECE + (c & 1) * LP_PIECE8 : (c & 1) * LP_PIECE);
        uint16_t* X = reinterpret_cast<uint16_t*>(mine);
        // ---- the piece's memory: its last outputs have been read, or the residual has come
        if (res_tma) {
          if (c + 1 < CHUNKS) ask_residual(c + 1);
          if (out_live) {
            ok = mbar_wait(&res_full[c & 1], (res_ph >> (c & 1)) & 1u, abort_flag, status);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            res_ph ^= 1u << (c & 1);
          }
        } else if (out_live) {
          // (within a tile the latest store has the other piece; chunks past the outputs store nothing, so that of the tile
          // before may have this one)
          if (lane == 0) {
            if (wide_out && (OUT8 || a.out_type == JK_ROWS_T) && !first) lp_put_read<1>();
            else lp_put_read<0>();
          }
          first = false;
          __syncwarp();
          if (res_x) {
            // rows that begin anywhere: read along the rows, handed out through shared memory
            const uint16_t* rp = (const uint16_t*)a.residual + (size_t)row0 * a.r_stride + n + lane;
#pragma unroll 4
            for (int j = 0; j < 32; ++j, rp += a.r_stride)
              X[j * LP_X_PITCH + lane] = row0 + j < a.rows && lane < most ? *rp : (uint16_t)0;
            __syncwarp();
          }
        }
        float top = 0.f;                   // 8-bit outputs: the block's largest magnitude
#pragma unroll 1
        for (int i = 0; i < 32; i += LP_W) {
          const int col = q * 32 + i, nw = n + i, most_w = most - i;
          float v[LP_W], u[LP_W];
          // (the biases are asked for ahead of the sums; n is a multiple of 16, so they are aligned)
          uint4 b[2], bu[2];
          const bool bias_full = out_live && most_w >= LP_W;
          if (bias_full && a.bias) {
            const uint4* bp = reinterpret_cast<const uint4*>((const uint16_t*)a.bias + nw);
            b[0] = bp[0];
            b[1] = bp[1];
          }
          if (GATED && bias_full && a.bias_up) {
            const uint4* bp = reinterpret_cast<const uint4*>((const uint16_t*)a.bias_up + nw);
            bu[0] = bp[0];
            bu[1] = bp[1];
          }
          {
            uint32_t w[LP_W], w2[LP_W];
            tmem_ld16(t_addr + (uint32_t)col, w);
            if constexpr (GATED) tmem_ld16(t_addr + (uint32_t)(LT_M + col), w2);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < LP_W; ++j) {
              v[j] = __uint_as_float(w[j]);
              u[j] = GATED ? __uint_as_float(w2[j]) : 0.f;
            }
          }
          if (i + LP_W == 32 && ((MX && c == 0) || c == CHUNKS - 1)) {
            tc_fence_before();
            __syncwarp();
            // the columns that both accumulators use: the last 24 of the first, the first 24 of the second
            if (MX && c == 0 && share == (buf ? 0 : EPI / 4 - 1) && lane == 0) lp_arrive(shared0);
            if (c == CHUNKS - 1 && lane == 0) lp_arrive(acc_empty0 + 8u * (uint32_t)buf);
          }
          if (!whole) {
            float* o = partial + (size_t)blockIdx.x * LT_SLOT + my_part + (size_t)col * 32;
#pragma unroll
            for (int j = 0; j < LP_W / 4; ++j) {
              __stcg(reinterpret_cast<float4*>(o + j * 128), make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
              if constexpr (GATED)
                __stcg(reinterpret_cast<float4*>(o + LT_M * 32 + j * 128),
                       make_float4(u[4 * j], u[4 * j + 1], u[4 * j + 2], u[4 * j + 3]));
            }
            continue;
          }
          if constexpr (LAST) {
            for (int k = 0; k < parts; ++k) {
#pragma unroll
              for (int g = 0; g < G; ++g, ++taken) {
                ok = ok && mbar_wait(&T.part_full[warp - 2][taken % PARTS], (uint32_t)(taken / PARTS) & 1u, abort_flag, status);
                const float4* o = reinterpret_cast<const float4*>(part_smem + taken % PARTS * LP_PART) + lane;
                float(&to)[LP_W] = g ? u : v;
#pragma unroll
                for (int j = 0; j < LP_W / 4; ++j) {
                  const float4 y = o[j * 32];
                  to[4 * j] += y.x; to[4 * j + 1] += y.y; to[4 * j + 2] += y.z; to[4 * j + 3] += y.w;
                }
              }
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
              __syncwarp();
              ask_parts();
            }
            if (!ok) break;
          } else for (int k = pair - 1; k >= from; --k) {
            if (k < pair - 1) ask_part(k, col);
#pragma unroll
            for (int j = 0; j < LP_W / 4; ++j) {
              v[4 * j] += t[j].x; v[4 * j + 1] += t[j].y; v[4 * j + 2] += t[j].z; v[4 * j + 3] += t[j].w;
              if constexpr (GATED) {
                u[4 * j] += tu[j].x; u[4 * j + 1] += tu[j].y; u[4 * j + 2] += tu[j].z; u[4 * j + 3] += tu[j].w;
              }
            }
          }
          const bool last = i + LP_W == 32;
          if (!LAST && parts && (!last || c + 1 < CHUNKS)) ask_part(pair - 1, last ? chunk(c + 1) * 32 : col + LP_W);
          if (!out_live) continue;
          if (a.bias) {
            if (bias_full) { lp_add8<0>(v, b[0]); lp_add8<8>(v, b[1]); }
            else lp_add(v, (const uint16_t*)a.bias + nw, most_w);
          }
          lin_act_all(v, a.act, !OUT8 && a.out_type == JK_ROWS_F32);
          if constexpr (GATED) {
            if (a.bias_up) {
              if (bias_full) { lp_add8<0>(u, bu[0]); lp_add8<8>(u, bu[1]); }
              else lp_add(u, (const uint16_t*)a.bias_up + nw, most_w);
            }
#pragma unroll
            for (int j = 0; j < LP_W; ++j) v[j] *= u[j];
          }
          if (a.residual && !res_tma && !res_x && live)
            lp_add(v, (const uint16_t*)a.residual + (size_t)(row0 + lane) * a.r_stride + nw, most_w);
          if constexpr (OUT8) {
#pragma unroll
            for (int j = 0; j < LP_W; ++j) top = fmaxf(top, fabsf(v[j]));          // (leaves NaN out)
#pragma unroll
            for (int j = 0; j < LP_W / 4; ++j)
              *reinterpret_cast<float4*>(mine + lp_at128(lane, i / 4 + j)) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          } else {
            if (res_tma) {
              lp_add8<0>(v, *reinterpret_cast<const uint4*>(piece + lp_at64(lane, i / 8)));
              lp_add8<8>(v, *reinterpret_cast<const uint4*>(piece + lp_at64(lane, i / 8 + 1)));
            } else if (res_x) {
#pragma unroll
              for (int j = 0; j < LP_W; ++j) v[j] += __uint_as_float((uint32_t)X[lane * LP_X_PITCH + i + j] << 16);
            }
            if (a.out_type == JK_ROWS_T) {
              uint32_t o[LP_W / 2];
#pragma unroll
              for (int j = 0; j < LP_W / 2; ++j) o[j] = lp_pack(v[2 * j], v[2 * j + 1]);
              if (wide_out) {
                *reinterpret_cast<uint4*>(piece + lp_at64(lane, i / 8)) = make_uint4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<uint4*>(piece + lp_at64(lane, i / 8 + 1)) = make_uint4(o[4], o[5], o[6], o[7]);
              } else {
                uint32_t* x32 = reinterpret_cast<uint32_t*>(&X[lane * LP_X_PITCH + i]);
#pragma unroll
                for (int j = 0; j < LP_W / 2; ++j) x32[j] = o[j];
              }
            } else if (wide_out) {         // f32: 16 outputs to a piece
#pragma unroll
              for (int j = 0; j < 4; ++j)
                *reinterpret_cast<float4*>(mine + i / 16 * LP_PIECE + lp_at64(lane, j)) =
                    make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            } else if (live) {
              float* p32 = (float*)a.out + (size_t)(row0 + lane) * a.o_stride + nw;
#pragma unroll
              for (int j = 0; j < LP_W; ++j)
                if (j < most_w) p32[j] = v[j];
            }
          }
        }
        if (!ok) break;
        __syncwarp();
        if (!out_live) continue;
        if constexpr (OUT8) {              // n_out is a multiple of 32: all of the block or nothing
          if (top > 3.402823466e38f) {     // an infinity does not count for the scale
            top = 0.f;
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
              const float4 y = *reinterpret_cast<const float4*>(mine + lp_at128(lane, j));
              top = fmaxf(fmaxf(fmaxf(top, paged_mag(y.x)), fmaxf(paged_mag(y.y), paged_mag(y.z))), paged_mag(y.w));
            }
          }
          const int e = paged_scale_exp(top);
          const float inv = paged_pow2(-e);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float4 y = *reinterpret_cast<const float4*>(mine + lp_at128(lane, 4 * i + j));
              o[j] = paged_pack4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
            }
            *reinterpret_cast<uint4*>(piece + lp_at32(lane, i)) = make_uint4(o[0], o[1], o[2], o[3]);
          }
          if (live) a.out_scale[mx_scale_at(row0 + lane, n >> 5, a.k_tiles_out)] = (uint8_t)(e + 127);
        } else if (a.out_type == JK_ROWS_T && !wide_out) {
          uint16_t* o = (uint16_t*)a.out + (size_t)row0 * a.o_stride + n + lane;
#pragma unroll 4
          for (int j = 0; j < 32; ++j, o += a.o_stride)
            if (row0 + j < a.rows && lane < most) *o = X[j * LP_X_PITCH + lane];
        }
        if (wide_out) {
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (!OUT8 && a.out_type == JK_ROWS_F32) {
              lp_put(&map_out, n, row0, mine_u32);
              if (most > 16) lp_put(&map_out, n + 16, row0, mine_u32 + LP_PIECE);
            } else {
              lp_put(&map_out, n, row0, smem_u32(piece));
            }
          }
        }
      }
      if (!ok) {                           // gave up: what was asked for lands before the memory goes away
        for (int i = taken; i < asked && lane == 0; ++i) {
          const unsigned long long t0 = global_ns();
          while (!mbar_try_wait(&T.part_full[warp - 2][i % PARTS], (uint32_t)(i / PARTS) & 1u))
            if (global_ns() - t0 > TC_WAIT_NS) break;
        }
        break;
      }
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
  lt_cluster_sync();                       // nobody's memory is used any more
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem_base) : "memory");
  }
}

// ------------------------------------------------------------------------------------------ host side
// The deal.  The tiles of the last, incomplete turn: whole (a turn more), or cut among 2, 3 or 4 pairs each, which costs
// the hand-over in boxes' time (a box 0.31 us): 18, 24, 31 where whole tiles follow and hide a part, 28, 34, 42 where none do
// or, in 8 bits, the two accumulators wait for one another.  Measured, us, whole and cut among 2, 3, 4 pairs: 16 tiles in
// bf16, K = 2048 16.4, 18.9, 19.3, 20.9, K = 4096 25.3, 24.2, 24.1, 25.2; in 8 bits, K = 4096 16.5, 19.9, 20.6, 21.6; 160
// tiles (12 left over), K = 5120 in bf16 88.3, 81.4, 79.7, 77.4, in 8 bits 49.1, 50.6, 50.0, 50.0.  Returns the cost in us,
// with a launch.
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
  static const int next_turn[LP_MAX_SPLIT] = {0, 18, 24, 31}, exposed[LP_MAX_SPLIT] = {0, 28, 34, 42};
  const int* hand_over = mx || tiles < pairs ? exposed : next_turn;
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

template <typename K>
static int launch_pair(jk_ctx* ctx, cudaStream_t st, K kernel, int threads, size_t smem, int bit, const CUtensorMap& x, const CUtensorMap& w,
                       const CUtensorMap& u, const CUtensorMap& sx, const CUtensorMap& sw, const CUtensorMap& su,
                       const CUtensorMap& o, const CUtensorMap& r, const lp_params& p, const lin_args& a, int wide_out,
                       int wide_res) {
  if (!(ctx->lin_smem_set & bit)) {
    JK_CUDA_CHECK(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    ctx->lin_smem_set |= bit;
  }
  JK_PROF(ctx, st, JK_ST_LINEAR);
  jk_launch_pdl_cluster(kernel, dim3(2 * p.pairs), dim3(threads), 2, smem, st, x, w, u, sx, sw, su, o, r, p, a, wide_out, wide_res,
                        (float*)(ctx->ws + ctx->lay.lin_part), (int32_t*)(ctx->ws + ctx->lay.lin_flag),
                        (int32_t*)(ctx->ws + ctx->lay.status));
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
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
  // Outputs and residuals whose rows begin and end at multiples of 16 bytes go through the copy engine, in pieces of 32
  // rows.  (It stores 16 bytes at least: the last of a row that ends elsewhere would reach into what lies between the rows.)
  const bool f32 = a.out_type == JK_ROWS_F32, q8 = a.out_type == JK_ROWS_MX8;
  const int os = q8 ? 1 : f32 ? 4 : 2;
  const int wide_out = (a.o_stride * os) % 16 == 0 && ((long long)a.n_out * os) % 16 == 0, wide_res = a.residual && wide_out && !f32 && (a.r_stride * 2) % 16 == 0;
  CUtensorMap mo = mw, mr = mw;
  if (wide_out) rc = jk_tma_encode_piece(ctx, &mo, a.out, q8 ? 1 : f32 ? 4 : 2, a.n_out, a.rows, a.o_stride, f32 ? 16 : 32);
  if (rc == JK_OK && wide_res) rc = jk_tma_encode_piece(ctx, &mr, a.residual, 2, a.n_out, a.rows, a.r_stride, 32);
  if (rc != JK_OK) return rc;
  // (8-bit outputs are always wide: n_out is a multiple of 32)
  auto pick = [&](auto m, auto g, auto o, auto l) {
    constexpr bool M = decltype(m)::value, G = decltype(g)::value, O = decltype(o)::value, LAST = decltype(l)::value;
    typedef lp_smem<M, O, LAST> S;
    return launch_pair(ctx, st, k_linear_pair<M, G, O, LAST>, S::THREADS, S::BYTES, 16 << (8 * LAST + 4 * M + 2 * G + O), mx_map, mw,
                       mu, msx, msw, msu, mo, mr, p, a, wide_out, wide_res);
  };
  const bool last = (long long)p.r_tiles * p.w_tiles <= p.pairs;
  auto pick_l = [&](auto m, auto g, auto o) { return last ? pick(m, g, o, std::true_type()) : pick(m, g, o, std::false_type()); };
  auto pick_g = [&](auto m, auto g) { return q8 ? pick_l(m, g, std::true_type()) : pick_l(m, g, std::false_type()); };
  auto pick_m = [&](auto m) { return gated ? pick_g(m, std::true_type()) : pick_g(m, std::false_type()); };
  return mx ? pick_m(std::true_type()) : pick_m(std::false_type());
}
