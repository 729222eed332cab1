// Tensor-core (tcgen05) kernel of jk_tree_verify_attn_paged for bf16 contexts.
//
// For a block of query rows (pairs of a q head of the group and a tree node) and tiles of 128 keys:
//   S^T = K Q^T   (keys on the 128 lanes, query rows on the columns), then
//   O^T = V^T P^T (head dims on the lanes, query rows on the columns).
// Keys on the lanes because a call has few query rows (1 .. 128 per kv head): with rows on the lanes a
// block of 60 would leave half of the SM's sub-partitions idle in the softmax, and a single token
// 127 of 128 lanes.  A thread owns one key: its page's scales are two constants of the thread.
//
// Full pages stay 8-bit up to the tensor core.  A bf16 query has 8 significant bits, an e4m3 number 4, so
// q 2^a = hi + lo with hi = e4m3(q 2^a) and lo = e4m3(q 2^a - hi) is exact down to 2^-17 of the block's
// largest q, and S is two e4m3 products into one fp32 accumulator.  The softmax weights go the same
// way: p = hi + lo keeps 8 significant bits, as bf16 would.  Two e4m3 products cost what one bf16
// product costs, and no code is ever widened.  V's scale (a power of two) is added to the logit, so
// that p already carries it: x = s scale_k + log2(scale_v), p = 2^(x - ref), and the row sum takes
// 2^(x - ref) / scale_v.
//
// ref is the (rounded up) maximum of this row in this tile, not the running one: e4m3 reaches down to
// 2^-18 of the tile's largest weight, so what is lost of a tile is below 2^-11 of its own weight,
// however small that is against another tile (with a running reference a long prefix behind one
// dominant key would vanish).  So every tile has its own product O_t, and the running output is
// kept in registers: acc = alpha acc + beta O_t with powers of two alpha, beta.
//
// The open page and the tree tokens are bf16 tiles at the end of the sequence (16-row boxes of either
// array, dead rows cleared in V): the same pipeline with kind::f16 products.
//
// One CTA per SM; all tiles of the call are dealt out evenly in order (sequence, kv head, row block,
// tile), so a unit (sequence, kv head, row block) spans CTAs where it has to; such a CTA leaves an
// unnormalised partial, which k_paged_merge adds up, and a unit inside one CTA is written directly.
// Warps: four softmax groups of four, TMA producers for K and for V, an MMA issuer.  A group takes 32 rows (16 where the block
// has no more) of every NP-th tile: 128 rows 4 x 32, 64 rows 2 x 32 with two tiles at a time, fewer rows
// with four.  Two groups of 64 rows each had 168 registers and spilled, two warps per scheduler to hide
// every wait, and took twice as long.
#include <math.h>

#include "jk_paged.cuh"
#include "jk_tcgen05.cuh"

#define PT_KEYS 128
#define PT_SOFTMAX 512              // threads of the softmax groups
#define PT_THREADS (PT_SOFTMAX + 96)
#define PT_MAX_CTAS 160
#define PT_INFO 8                    // ring of stage descriptions
#define PT_PSHIFT 8.f                // weights are scaled by 2^8: the largest lie in (2^7, 2^8]

// ------------------------------------------------------------------------------------------ PTX
__device__ __forceinline__ void pt_mma_f8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
// Maxima (sums) over the warp's lanes of N = 16 or 32 rows held one value per lane: lane l ends up with
// row l mod N.  Half of the rows changes sides at every step, so 31 exchanges serve 32 rows.
template <int N, bool SUM> __device__ __forceinline__ float pt_rows_reduce(const float* x, int lane) {
  float v[N];
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = x[j];
  if (N == 16) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float y = __shfl_xor_sync(0xffffffffu, v[j], 16);
      v[j] = SUM ? v[j] + y : fmaxf(v[j], y);
    }
  }
#pragma unroll
  for (int h = N / 2; h >= 1; h >>= 1) {
    const bool up = lane & h;
#pragma unroll
    for (int j = 0; j < h; ++j) {
      const float keep = up ? v[j + h] : v[j], send = up ? v[j] : v[j + h];
      const float y = __shfl_xor_sync(0xffffffffu, send, h);
      v[j] = SUM ? keep + y : fmaxf(keep, y);
    }
  }
  return v[0];
}
template <int ID, int N> __device__ __forceinline__ void pt_bar() {
  asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(N) : "memory");
}
// Shared-memory matrix descriptor; layout 2 / 4 / 6 / 0 = 128 / 64 / 32-byte swizzle / none.
__device__ __forceinline__ uint64_t pt_desc(uint32_t addr, uint32_t lbo, uint32_t sbo, uint32_t layout) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(lbo >> 4) << 16;
  d |= (uint64_t)(sbo >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)layout << 61;
  return d;
}
// Layout code of rows of `bytes` bytes (one row = one swizzle span).
__host__ __device__ constexpr uint32_t pt_layout(int bytes) {
  return bytes == 128 ? 2u : bytes == 64 ? 4u : bytes == 32 ? 6u : 0u;
}
// Byte offset of 16-byte piece c of row r in such an array.
template <int BYTES> __device__ __forceinline__ uint32_t pt_piece(int r, int c) {
  const int x = BYTES == 128 ? (r & 7) : BYTES == 64 ? ((r >> 1) & 3) : BYTES == 32 ? ((r >> 2) & 1) : 0;
  return (uint32_t)(r * BYTES + ((c ^ x) << 4));
}
// Instruction descriptor, fp32 accumulate, M = 128; fmt 1 = bf16 (kind::f16), 0 = e4m3 (kind::f8f6f4).
__device__ __forceinline__ uint32_t pt_idesc(uint32_t fmt, int n, int a_mn, int b_mn) {
  return (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

// ------------------------------------------------------------------------------------------ layout
template <int D, int NR> struct pt_cfg {
  static constexpr int RW = NR < 32 ? NR : 32;         // rows of a softmax group
  static constexpr int NRG = NR / RW;                  // groups that share a tile
  static constexpr int NP = 4 / NRG;                   // tiles in the groups' hands at a time
  static constexpr int TPS = NP == 1 ? 1 : 2;          // 8-bit tiles of a stage
  static constexpr int WK = NP == 1 ? 64 : 128;        // keys of a bf16 tile
  static constexpr int SLOT = WK * D * 2;              // a bf16 tile, or TPS 8-bit tiles
  static constexpr int KST = NR == 128 ? 3 : 2;
  static constexpr int VST = NR == 128 || NR == 16 ? 3 : 2;
  static constexpr int Q8 = NR * D;                    // one of the two e4m3 parts of the queries
  static constexpr int Q16 = NR * D * 2;
  static constexpr int PG = PT_KEYS * RW * 2;          // a group's weights: two e4m3 parts, or bf16
  static constexpr int PT = NRG * PG;                  // the weights of a tile
  static constexpr int MB = (NP - 1) * NR * 512;       // sums handed over at a unit's end, over the weights
  static constexpr int PBYTES = 4 * PG > MB ? 4 * PG : MB;
  static constexpr int OFF_Q16 = 2 * Q8;
  static constexpr int OFF_P = OFF_Q16 + Q16;
  static constexpr int OFF_K = OFF_P + PBYTES;
  static constexpr int OFF_V = OFF_K + KST * SLOT;
  static constexpr int OFF_X = OFF_V + VST * SLOT + 1024;   // (a head size of 64 reads one row group further)
  static constexpr uint32_t COLS = 16 * RW;            // S and O, two buffers each, of four groups
};

struct pt_info {                     // one stage, written by the producer
  int live[2];                       // live keys of the tile(s), may pass the tile's
  int open_rows, open16;             // bf16 tile: first row past the open page's tokens, and past their padding
  float sk[16], lsv[16], isv[16];    // per page: K scale, log2 and inverse of the V scale
};

template <int D, int NR> struct alignas(16) pt_tail {
  uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4];
  uint64_t info_full[PT_INFO], s_full[4][2], p_full[4], o_full[4], q_full;
  uint32_t tmem_base;
  int abort_flag;
  long long cum[JK_MAX_ROWS + 1];    // tiles before each sequence
  int n8[JK_MAX_ROWS], n16[JK_MAX_ROWS];
  pt_info info[PT_INFO];
  float q_max[16];
  int rowoff[NR];                    // output row of each query row, -1 = none
  int parent[JK_MAX_TREE];
  alignas(16) uint32_t anc[4][NR];   // tree nodes each query row sees
  // per warp and row, so that a step has one barrier: the four warps of a group form the same values
  alignas(16) float ref[16][32], alpha[16][2][32], beta[16][2][32];
  float wmax[4][2][4][32], m_run[4][32], lsum[16][32];
};

// The stages of a segment [t0, t1) of a unit with n8 8-bit tiles in front: every role walks them.
template <int TPS, int NP> struct pt_iter {
  int tile, t1, n8, turn;
  __device__ __forceinline__ void start(int t0, int end, int n8_) { tile = t0; t1 = end; n8 = n8_; turn = 0; }
  // n tiles from `first` on; tile j is worked on by the groups of turn (w + j) mod NP
  __device__ __forceinline__ bool next(int& first, int& n, int& w, bool& wide) {
    if (tile >= t1) return false;
    first = tile;
    wide = tile >= n8;
    n = (TPS == 2 && !wide && tile + 1 < t1 && tile + 1 < n8) ? 2 : 1;
    w = turn;
    turn = (turn + n) & (NP - 1);
    tile += n;
    return true;
  }
};

// Tiles of every sequence, and their prefix sums, by one warp.  wk: keys of a bf16 tile.
__device__ __forceinline__ void pt_count(const jk_paged& c, int B, int M, int wk, int units, int lane, long long* cum,
                                         int* n8, int* n16, int32_t* status) {
  long long run = 0;
  for (int b0 = 0; b0 < B; b0 += 32) {
    const int b = b0 + lane;
    int a = 0, w = 0;
    if (b < B) {
      const int P = c.kv_len[b];
      if (P < 0 || P > c.max_pages * c.page_size) {
        if (status) jk_set_status(status, JK_ERR_BOUNDS);
      } else {
        const int nf = P / c.page_size * c.page_size;
        a = (nf + PT_KEYS - 1) / PT_KEYS;
        w = (((P - nf + 15) & ~15) + M + wk - 1) / wk;
      }
    }
    long long incl = (long long)(a + w) * units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (b < B) {
      cum[b + 1] = run + incl;
      n8[b] = a;
      if (n16) n16[b] = w;
    }
    run += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (lane == 0) cum[0] = 0;
}

// ------------------------------------------------------------------------------------------ kernel
template <int D, int NR>
__global__ void __launch_bounds__(PT_THREADS, 1) k_paged_attn_tc(
    const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
    const __grid_constant__ CUtensorMap map_ko, const __grid_constant__ CUtensorMap map_vo,
    const __grid_constant__ CUtensorMap map_kt, const __grid_constant__ CUtensorMap map_vt, const jk_paged c,
    int layer, const __nv_bfloat16* __restrict__ q, const int32_t* __restrict__ parent, float scale, int B, int M,
    int Hq, int Hkv, int n_qblk, __nv_bfloat16* __restrict__ out, float* __restrict__ part_o,
    float* __restrict__ part_ml, int32_t* status) {
  typedef pt_cfg<D, NR> F;
  constexpr int RW = F::RW, NRG = F::NRG, NP = F::NP, KST = F::KST, VST = F::VST, WK = F::WK;
  constexpr int KB = D / 64;
  constexpr uint32_t O_COL = 8 * RW;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* sk = smem + F::OFF_K;
  unsigned char* sv = smem + F::OFF_V;
  typedef pt_tail<D, NR> tail_t;
  tail_t& X = *reinterpret_cast<tail_t*>(smem + F::OFF_X);
  volatile int* abort_flag = &X.abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = Hq / Hkv, units = Hkv * n_qblk, ps = c.page_size;

  if (tid == 0) {
    for (int i = 0; i < 4; ++i) {
      mbar_init(&X.k_full[i], 1); mbar_init(&X.k_empty[i], 1);
      mbar_init(&X.v_full[i], 1); mbar_init(&X.v_empty[i], 1);
    }
    for (int i = 0; i < PT_INFO; ++i) mbar_init(&X.info_full[i], 1);
    for (int i = 0; i < 4; ++i) {
      mbar_init(&X.s_full[i][0], 1); mbar_init(&X.s_full[i][1], 1);
      mbar_init(&X.p_full[i], 4 * NRG); mbar_init(&X.o_full[i], 1);
    }
    mbar_init(&X.q_full, PT_SOFTMAX / 32);
    X.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 17) {
    tmem_alloc(&X.tmem_base, F::COLS);
    tmem_relinquish();
  }
  jk_pdl_wait();
  if (warp == 16) pt_count(c, B, M, F::WK, units, lane, X.cum, X.n8, X.n16, blockIdx.x == 0 ? status : nullptr);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = X.tmem_base;
  const long long total = X.cum[B];
  // with fewer tiles than CTAs the first `total` CTAs take one each (an empty share would leave a gap)
  const long long ctas = total < gridDim.x ? total : gridDim.x;
  const bool idle = blockIdx.x >= ctas;
  const long long w0 = idle ? 0 : total * blockIdx.x / ctas, w1 = idle ? 0 : total * (blockIdx.x + 1) / ctas;
  bool ok = true;

  // a segment of the CTA's range: unit (b, u), tiles [t0, t1)
  auto segment = [&](long long t, int& b, int& u, int& t0, int& t1, int& nt) {
    b = 0;
    while (X.cum[b + 1] <= t) ++b;
    nt = X.n8[b] + X.n16[b];
    const long long off = t - X.cum[b];
    u = (int)(off / nt);
    t0 = (int)(off - (long long)u * nt);
    const long long left = w1 - t;
    t1 = left < nt - t0 ? t0 + (int)left : nt;
  };

  if (warp == 16 || warp == 18) {
    // ==================================================================== TMA producers: K (16), V (18)
    const bool is_k = warp == 16;
    const int NST = is_k ? KST : VST;
    uint64_t* full = is_k ? X.k_full : X.v_full;
    uint64_t* empty = is_k ? X.k_empty : X.v_empty;
    unsigned char* ring = is_k ? sk : sv;
    const CUtensorMap* map = is_k ? &map_k : &map_v;
    int sc = 0, s_slot = 0, s_par = 1;                  // stages so far, their slot and its parity
    // pages are read once, unless several row blocks of a kv head come by
    const uint64_t pol = l2_policy_evict_first();
    const bool once = n_qblk == 1;
    const int per = PT_KEYS / ps;                       // pages of a tile
    for (long long t = w0; t < w1 && ok;) {
      int b, u, t0, t1, nt;
      segment(t, b, u, t0, t1, nt);
      t += t1 - t0;
      const int h = u / n_qblk, n8 = X.n8[b];
      const int P = c.kv_len[b], nf = P / ps * ps, n_pg = P / ps;
      const int open_rows = P - nf, open16 = (open_rows + 15) & ~15;
      const int32_t* tab = c.page_table + (size_t)b * c.max_pages;
      pt_iter<F::TPS, NP> it;
      it.start(t0, t1, n8);
      int first, n, w;
      bool wide;
      // Page ids and scales in batches of 32 pages, lane l the batch's page l, the ids of the next batch
      // asked for a batch ahead: two dependent loads per stage would be the stage's time.
      int at = t0 * per, id = 0, id_next = 0;
      float ksc = 1.f, vsc = 1.f;
      auto ask = [&](int p0) { return p0 + lane < n_pg ? tab[p0 + lane] : 0; };
      auto take = [&](int raw) {                        // the batch from `at` on
        id = raw;
        if (id < 0 || id >= c.n_pages) {
          jk_set_status(status, JK_ERR_BOUNDS);
          id = 0;
        }
        if (is_k) {
          const size_t blk = ((size_t)layer * c.n_pages + id) * Hkv + h;
          ksc = c.k_scale[blk];
          vsc = c.v_scale[blk];
        }
        id_next = ask(at + 32);
      };
      if (t0 < n8) take(ask(at));
      while (ok && it.next(first, n, w, wide)) {
        ok = __all_sync(0xffffffffu, mbar_wait(&empty[s_slot], s_par, abort_flag, status));
        unsigned char* dst = ring + s_slot * F::SLOT;
        pt_info& I = X.info[sc % PT_INFO];
        if (!wide) {
          const int p0 = first * per, np = min(n * per, n_pg - p0);
          // a stage has at most 16 pages and starts at a multiple of its tile: it may span two batches
          if (p0 >= at + 32) { at += 32; take(id_next); }
          int page = __shfl_sync(0xffffffffu, id, (p0 - at + lane) & 31);
          float k1 = __shfl_sync(0xffffffffu, ksc, (p0 - at + lane) & 31);
          float v1 = __shfl_sync(0xffffffffu, vsc, (p0 - at + lane) & 31);
          if (p0 + np > at + 32) {
            const int split = at + 32 - p0;             // lanes from here on belong to the next batch
            at += 32;
            take(id_next);
            const int pg2 = __shfl_sync(0xffffffffu, id, (p0 - at + lane) & 31);
            const float k2 = __shfl_sync(0xffffffffu, ksc, (p0 - at + lane) & 31);
            const float v2 = __shfl_sync(0xffffffffu, vsc, (p0 - at + lane) & 31);
            if (lane >= split) { page = pg2; k1 = k2; v1 = v2; }
          }
          if (ok && lane == 0) mbar_expect_tx(&full[s_slot], (uint32_t)np * ps * D);
          __syncwarp();
          if (ok && lane < np) {
            const int row = layer * c.n_pages + page;
            if (once) tma_load_4d_hint(dst + lane * ps * D, map, 0, 0, h, row, &full[s_slot], pol);
            else tma_load_4d(dst + lane * ps * D, map, 0, 0, h, row, &full[s_slot]);
          }
          if (is_k) {
            if (lane < 16) {
              const int e = (int)(__float_as_uint(v1) >> 23) - 127;
              I.sk[lane] = k1;
              I.lsv[lane] = (float)e;
              I.isv[lane] = paged_pow2(-e);
            }
            if (lane < 2) I.live[lane] = min(PT_KEYS, nf - (first + lane) * PT_KEYS);
          }
        } else {
          // bf16 tile: rows g of (open rows, padded to 16, then tree rows) in boxes of 16
          const int base = (first - n8) * WK;
          const int g = base + (lane / KB) * 16, kb = lane % KB;
          const bool in_open = g < open16;
          const bool mine = lane < WK / 16 * KB && (in_open || g - open16 < M);
          const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * 16 * 64 * 2;
          const int row = in_open ? (nf & (2 * ps - 1)) + g : g - open16;
          const int outer = in_open ? layer * c.max_seqs + b : b;
          if (ok && lane == 0) mbar_expect_tx(&full[s_slot], bytes);
          __syncwarp();
          if (ok && mine)
            tma_load_4d(dst + kb * (WK * 128) + (lane / KB) * 16 * 128,
                        is_k ? (in_open ? &map_ko : &map_kt) : (in_open ? &map_vo : &map_vt), kb * 64, row, h, outer,
                        &full[s_slot]);
          if (is_k && lane == 0) {
            I.live[0] = open16 + M - base;
            I.open_rows = open_rows - base;
            I.open16 = open16 - base;
          }
        }
        __syncwarp();
        if (is_k && lane == 0) mbar_arrive(&X.info_full[sc % PT_INFO]);
        ++sc;
        if (++s_slot == NST) { s_slot = 0; s_par ^= 1; }
      }
    }
    if (!ok) {
      // gave up, possibly with copies still in flight: give them a bounded time to land
      const unsigned long long ts = global_ns();
      while (global_ns() - ts < 2000000ull) { /* 2 ms: far longer than any TMA copy */ }
    }
  } else if (warp == 17) {
    if (lane == 0) {
      // ================================================================== MMA issuer
      const uint32_t q8 = smem_u32(smem), q16 = smem_u32(smem + F::OFF_Q16), pb = smem_u32(smem + F::OFF_P);
      const uint32_t ka0 = smem_u32(sk), va0 = smem_u32(sv);
      const uint32_t id_s8 = pt_idesc(0, NR, 0, 0), id_s16 = pt_idesc(1, NR, 0, 0);
      const uint32_t id_p8 = pt_idesc(0, NR, 1, 1), id_p16 = pt_idesc(1, NR, 1, 1);
      int ks_n = 0, vs_n = 0, segs = 0;
      uint32_t cs = 0, cp = 0;                          // tiles per turn so far, a byte each (mod 256)
      auto issue_s = [&](int n, int w, bool wide) {
        const int slot = ks_n % KST;
        if (!mbar_wait(&X.k_full[slot], (ks_n / KST) & 1, abort_flag, status)) { ok = false; return; }
        tc_fence_after();
        const uint32_t ka = ka0 + slot * F::SLOT;
        for (int j = 0; j < n; ++j) {
          const int tp = (w + j) & (NP - 1);
          const uint32_t buf = (cs >> (8 * tp)) & 1;
          const uint32_t d = tmem + (buf * NP + tp) * NR;
          if (!wide) {
            const uint32_t kt = ka + j * (PT_KEYS * D);
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
              for (int k = 0; k < D / 32; ++k)
                pt_mma_f8(d, pt_desc(kt + k * 32, 16, 8 * D, pt_layout(D)),
                          pt_desc(q8 + part * F::Q8 + k * 32, 16, 8 * D, pt_layout(D)), id_s8, (part | k) ? 1u : 0u);
          } else {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                tc_mma_bf16(d, pt_desc(ka + kb * (WK * 128) + k * 32, 16, 1024, 2),
                            pt_desc(q16 + kb * (NR * 128) + k * 32, 16, 1024, 2), id_s16, (kb | k) ? 1u : 0u);
          }
          tc_commit(&X.s_full[tp][buf]);
          cs = (cs & ~(0xffu << (8 * tp))) | ((((cs >> (8 * tp)) + 1) & 0xffu) << (8 * tp));
        }
        tc_commit(&X.k_empty[slot]);
        ++ks_n;
      };
      auto issue_pv = [&](int n, int w, bool wide) {
        const int slot = vs_n % VST;
        if (!mbar_wait(&X.v_full[slot], (vs_n / VST) & 1, abort_flag, status)) { ok = false; return; }
        const uint32_t va = va0 + slot * F::SLOT;
        for (int j = 0; j < n; ++j) {
          const int tp = (w + j) & (NP - 1);
          const uint32_t buf = (cp >> (8 * tp)) & 1;
          if (!mbar_wait(&X.p_full[tp], buf, abort_flag, status)) { ok = false; return; }
          tc_fence_after();
          const uint32_t d = tmem + O_COL + (buf * NP + tp) * NR;
          const uint32_t p = pb + tp * F::PT;
          if (!wide) {
            const uint32_t vt = va + j * (PT_KEYS * D);
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
              for (int k = 0; k < PT_KEYS / 32; ++k)
                pt_mma_f8(d, pt_desc(vt + k * 32 * D, 8 * D, 8 * D, pt_layout(D)),
                          pt_desc(p + part * (PT_KEYS * RW) + k * 32 * RW, NRG > 1 ? F::PG : 8 * RW, 8 * RW, pt_layout(RW)),
                          id_p8, (part | k) ? 1u : 0u);
          } else {
#pragma unroll
            for (int k = 0; k < WK / 16; ++k)
              tc_mma_bf16(d, pt_desc(va + k * 2048, KB == 2 ? WK * 128 : 1024, 1024, 2),
                          pt_desc(p + k * 32 * RW, NRG > 1 ? F::PG : 16 * RW, 16 * RW, pt_layout(2 * RW)), id_p16, k ? 1u : 0u);
          }
          tc_commit(&X.o_full[tp]);
          cp = (cp & ~(0xffu << (8 * tp))) | ((((cp >> (8 * tp)) + 1) & 0xffu) << (8 * tp));
        }
        tc_commit(&X.v_empty[slot]);
        ++vs_n;
      };
      for (long long t = w0; t < w1 && ok;) {
        int b, u, t0, t1, nt;
        segment(t, b, u, t0, t1, nt);
        t += t1 - t0;
        ok = mbar_wait(&X.q_full, segs & 1, abort_flag, status);
        ++segs;
        if (!ok) break;
        tc_fence_after();
        pt_iter<F::TPS, NP> is, ip;
        is.start(t0, t1, X.n8[b]);
        ip.start(t0, t1, X.n8[b]);
        int first, n, w, ahead = 0;
        bool wide, more = true;
        // S runs two stages ahead of the second product: S of stage i + 2 reuses the columns of stage i,
        // which are free once the weights of stage i have been written
        while (ok) {
          if (more && (more = is.next(first, n, w, wide))) {
            issue_s(n, w, wide);
            ++ahead;
          }
          if (!ok) break;
          if (ahead == 2 || (!more && ahead > 0)) {
            ip.next(first, n, w, wide);
            issue_pv(n, w, wide);
            --ahead;
          }
          if (!more && ahead == 0) break;
        }
      }
      if (!ok) {                                        // products still in flight get a bounded time to end
        const unsigned long long ts = global_ns();
        while (global_ns() - ts < 2000000ull) { }
      }
    }
  } else if (warp < 16) {
    // ==================================================================== softmax groups
    const int grp = warp >> 2, wq = warp & 3;           // group, tensor-memory lane quarter
    const int rg = grp % NRG, tp = grp / NRG;           // its rows of the block, its turn among the tiles
    const int kl = wq * 32 + lane;                      // this thread's key of a tile / head dim of O
    const uint32_t lane_base = (uint32_t)(wq * 32) << 16;
    unsigned char* pbuf = smem + F::OFF_P + tp * F::PT + rg * F::PG;
    const int grow = rg * RW;                           // first row of this group in the block
    auto group_bar = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(grp + 1) : "memory"); };
    int cnt = 0, sc = 0;                                // tiles of this group, stages of the CTA
    for (long long t = w0; t < w1;) {
      int b, u, t0, t1, nt;
      segment(t, b, u, t0, t1, nt);
      const bool whole = t0 == 0 && t1 == nt;
      // a partial that does not start its unit is this CTA's first, else its last
      const int slot = (int)(blockIdx.x * 2 + (t0 == 0 ? 1 : 0));
      t += t1 - t0;
      const int h = u / n_qblk, row0 = (u % n_qblk) * NR, n_rows = G * M, n8 = X.n8[b];
      // ------------------------------------------------ queries of the unit
      constexpr int QV = (NR * (D / 8) + PT_SOFTMAX - 1) / PT_SOFTMAX;
      uint4 qv[QV];
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const int idx = tid + i * PT_SOFTMAX, r = idx / (D / 8), ch = idx % (D / 8);
        qv[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < NR && row0 + r < n_rows) {
          const int gg = (row0 + r) / M, ii = (row0 + r) % M;
          qv[i] = *reinterpret_cast<const uint4*>(q + (((size_t)b * M + ii) * Hq + h * G + gg) * D + ch * 8);
        }
      }
      if (t1 > n8 && tid < M) X.parent[tid] = parent[(size_t)b * M + tid];
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const uint32_t qw[4] = {qv[i].x, qv[i].y, qv[i].z, qv[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          amax = fmaxf(amax, fmaxf(paged_mag(__uint_as_float(qw[j] << 16)),
                                   paged_mag(__uint_as_float(qw[j] & 0xffff0000u))));
      }
      amax = jk_warp_max(amax);
      if (lane == 0) X.q_max[warp] = amax;
      // (also: all groups are done with the previous unit's queries, sums and row tables)
      pt_bar<5, PT_SOFTMAX>();
      amax = jk_warp_max(X.q_max[lane & 15]);
      int qe = (int)(__float_as_uint(amax) >> 23) - 127 - 8 + ((__float_as_uint(amax) & 0x7fffffu) > 0x600000u ? 1 : 0);
      qe = max(-100, min(100, qe));
      const float qinv = paged_pow2(-qe);
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const int idx = tid + i * PT_SOFTMAX, r = idx / (D / 8), ch = idx % (D / 8);
        if (r < NR) {
          *reinterpret_cast<uint4*>(smem + F::OFF_Q16 + (ch >> 3) * (NR * 128) + pt_piece<128>(r, ch & 7)) = qv[i];
          const uint32_t qw[4] = {qv[i].x, qv[i].y, qv[i].z, qv[i].w};
          uint32_t hi[2], lo[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float v0 = __uint_as_float(qw[2 * j] << 16) * qinv, v1 = __uint_as_float(qw[2 * j] & 0xffff0000u) * qinv;
            const float v2 = __uint_as_float(qw[2 * j + 1] << 16) * qinv;
            const float v3 = __uint_as_float(qw[2 * j + 1] & 0xffff0000u) * qinv;
            hi[j] = paged_pack4(v0, v1, v2, v3);
            const float2 b0 = paged_unpack2(hi[j]), b1 = paged_unpack2(hi[j] >> 16);
            lo[j] = paged_pack4(v0 - b0.x, v1 - b0.y, v2 - b1.x, v3 - b1.y);
          }
          const uint32_t at = pt_piece<D>(r, ch >> 1) + (ch & 1) * 8;
          *reinterpret_cast<uint2*>(smem + at) = make_uint2(hi[0], hi[1]);
          *reinterpret_cast<uint2*>(smem + F::Q8 + at) = make_uint2(lo[0], lo[1]);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&X.q_full);
      if (tid < NR) {
        const bool live = row0 + tid < n_rows;
        const int gg = live ? (row0 + tid) / M : 0, ii = live ? (row0 + tid) % M : 0;
        X.rowoff[tid] = live ? ii * Hq + h * G + gg : -1;
        uint32_t a[4] = {0u, 0u, 0u, 0u};
        if (live && t1 > n8) {                          // (only the last tiles look at it)
          int node = ii;
          for (int guard = 0; node >= 0 && guard <= JK_MAX_TREE; ++guard) {
            const uint32_t bit = 1u << (node & 31);
            const int wd = node >> 5;
            a[0] |= wd == 0 ? bit : 0u; a[1] |= wd == 1 ? bit : 0u;
            a[2] |= wd == 2 ? bit : 0u; a[3] |= wd == 3 ? bit : 0u;
            const int pp = X.parent[node];
            node = pp < node ? pp : -1;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) X.anc[i][tid] = a[i];
      }
      pt_bar<5, PT_SOFTMAX>();                          // row tables are visible
      const float c16 = scale * 1.4426950408889634f, c8 = c16 * paged_pow2(qe);

      float acc[RW], lacc[RW];
#pragma unroll
      for (int i = 0; i < RW; ++i) acc[i] = lacc[i] = 0.f;
      float run = -INFINITY;                            // running reference of row lane (mod RW)
      bool pending = false, moved_before = false;       // the last tile's product is still to be added
      // acc = alpha acc + beta O of tile `count`.  Its completion has been waited for by every thread of
      // the group: a wait here, after the arrival for the next tile, could find the barrier two phases on.
      auto take_o = [&](int count, bool moved) {
        const int sb = count & 1;
        __syncwarp();
        tc_fence_after();
        const uint32_t oa = tmem + lane_base + O_COL + (sb * NP + tp) * NR + grow;
        uint32_t r[RW];
        if constexpr (RW == 32) tmem_ld32(oa, r); else tmem_ld16(oa, r);
        tmem_ld_wait();
        if (moved) {
#pragma unroll
          for (int j = 0; j < RW; j += 4) {
            const float4 al = *reinterpret_cast<const float4*>(&X.alpha[warp][sb][j]);
            acc[j] *= al.x; acc[j + 1] *= al.y; acc[j + 2] *= al.z; acc[j + 3] *= al.w;
          }
        }
#pragma unroll
        for (int j = 0; j < RW; j += 4) {
          const float4 be = *reinterpret_cast<const float4*>(&X.beta[warp][sb][j]);
          acc[j] = fmaf(__uint_as_float(r[j]), be.x, acc[j]);
          acc[j + 1] = fmaf(__uint_as_float(r[j + 1]), be.y, acc[j + 1]);
          acc[j + 2] = fmaf(__uint_as_float(r[j + 2]), be.z, acc[j + 2]);
          acc[j + 3] = fmaf(__uint_as_float(r[j + 3]), be.w, acc[j + 3]);
        }
      };

      pt_iter<F::TPS, NP> it;
      it.start(t0, t1, n8);
      int first, n, w;
      bool wide;
      for (; it.next(first, n, w, wide); ++sc) {
        const int part = (tp - w) & (NP - 1);           // tile of the stage
        if (part >= n) continue;
        const pt_info& I = X.info[sc % PT_INFO];
        const int sb = cnt & 1;
        if (ok) ok = mbar_wait(&X.info_full[sc % PT_INFO], (sc / PT_INFO) & 1, abort_flag, status);
        float ck = c16, lsv = 0.f, isv = 1.f;
        bool dead;
        int tree_row = -1;
        if (!wide) {
          const int pg = (part * PT_KEYS + kl) / ps;
          dead = kl >= I.live[part];
          ck = c8 * I.sk[pg];
          lsv = I.lsv[pg];
          isv = I.isv[pg];
        } else {
          dead = kl >= min(WK, I.live[0]) || (kl >= I.open_rows && kl < I.open16);
          if (kl >= I.open16) tree_row = kl - I.open16;
        }
        if (ok) ok = mbar_wait(&X.s_full[tp][sb], (cnt >> 1) & 1, abort_flag, status);
        __syncwarp();
        tc_fence_after();
        const uint32_t sa = tmem + lane_base + (sb * NP + tp) * NR + grow;
        const bool masked = __any_sync(0xffffffffu, dead || tree_row >= 0);
        // rows of V that no live key owns may hold anything, NaN included, and 0 * NaN would reach every row
        if (dead && (!wide || kl < WK)) {
          if (ok) ok = mbar_wait(&X.v_full[sc % VST], (sc / VST) & 1, abort_flag, status);
          unsigned char* row = sv + (sc % VST) * F::SLOT + (wide ? kl * 128 : part * (PT_KEYS * D) + kl * D);
          if (ok) {
#pragma unroll 1
            for (int j = 0; j < (wide ? D / 8 : D / 16); ++j)
              *reinterpret_cast<uint4*>(row + (wide ? (j >> 3) * (WK * 128) + (j & 7) * 16 : j * 16)) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        __syncwarp();
        // rows of the block this key is visible to
        uint32_t vis = 0xffffffffu;
        if (masked) {
          if (dead) vis = 0u;
          else if (tree_row >= 0) {
            const uint32_t* aw = &X.anc[(tree_row >> 5) & 3][grow];
            vis = 0u;
#pragma unroll
            for (int j = 0; j < RW; ++j) vis |= ((aw[j] >> (tree_row & 31)) & 1u) << j;
          }
        }
        // ---- maxima over the tile of the logits of each row (base 2, with log2 of the V scale)
        {
          float x[RW];
          uint32_t r[RW];
          if constexpr (RW == 32) tmem_ld32(sa, r); else tmem_ld16(sa, r);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < RW; ++j) x[j] = fmaf(__uint_as_float(r[j]), ck, lsv);
          if (masked) {
#pragma unroll
            for (int j = 0; j < RW; ++j)
              if (!((vis >> j) & 1u)) x[j] = -INFINITY;
          }
          const float m = pt_rows_reduce<RW, false>(x, lane);
          if (lane < RW) X.wmax[grp][sb][wq][lane] = m;
        }
        group_bar();
        bool moved = false;
        {
          const float* wm = &X.wmax[grp][sb][0][lane & (RW - 1)];
          const float m = fmaxf(fmaxf(wm[0], wm[32]), fmaxf(wm[64], wm[96]));
          float ref = 0.f, be = 0.f, al = 1.f;
          if (m != -INFINITY) {
            ref = ceilf(m);
            const float now = fmaxf(run, ref);
            al = run == -INFINITY ? 0.f : fast_exp2(run - now);
            be = fast_exp2(ref - now);
            moved = run != now;
            run = now;
          }
          if (lane < RW) {
            X.ref[warp][lane] = ref - PT_PSHIFT;
            X.alpha[warp][sb][lane] = al;
            X.beta[warp][sb][lane] = be;
          }
        }
        moved = __any_sync(0xffffffffu, moved);         // (orders the writes above within the warp)
        __syncwarp();
        // ---- the previous product is complete: its weights may be overwritten
        if (pending && ok) ok = mbar_wait(&X.o_full[tp], (cnt - 1) & 1, abort_flag, status);
        __syncwarp();
        if (moved) {
#pragma unroll
          for (int j = 0; j < RW; j += 4) {
            const float4 al = *reinterpret_cast<const float4*>(&X.alpha[warp][sb][j]);
            lacc[j] *= al.x; lacc[j + 1] *= al.y; lacc[j + 2] *= al.z; lacc[j + 3] *= al.w;
          }
        }
#pragma unroll
        for (int j0 = 0; j0 < RW; j0 += 16) {
          uint32_t r[16];
          float e[16];
          tmem_ld16(sa + j0, r);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            const float4 rf = *reinterpret_cast<const float4*>(&X.ref[warp][j0 + j]);
            e[j] = fast_exp2(fmaf(__uint_as_float(r[j]), ck, lsv - rf.x));
            e[j + 1] = fast_exp2(fmaf(__uint_as_float(r[j + 1]), ck, lsv - rf.y));
            e[j + 2] = fast_exp2(fmaf(__uint_as_float(r[j + 2]), ck, lsv - rf.z));
            e[j + 3] = fast_exp2(fmaf(__uint_as_float(r[j + 3]), ck, lsv - rf.w));
          }
          if (masked) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (!((vis >> (j0 + j)) & 1u)) e[j] = 0.f;
          }
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            const float4 be = *reinterpret_cast<const float4*>(&X.beta[warp][sb][j0 + j]);
            lacc[j0 + j] = fmaf(e[j], isv * be.x, lacc[j0 + j]);
            lacc[j0 + j + 1] = fmaf(e[j + 1], isv * be.y, lacc[j0 + j + 1]);
            lacc[j0 + j + 2] = fmaf(e[j + 2], isv * be.z, lacc[j0 + j + 2]);
            lacc[j0 + j + 3] = fmaf(e[j + 3], isv * be.w, lacc[j0 + j + 3]);
          }
          if (!wide) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              // the remainder is formed in fp16 (11 significant bits where 8 are kept)
              const __half2 h0 = __floats2half2_rn(e[4 * j], e[4 * j + 1]);
              const __half2 h1 = __floats2half2_rn(e[4 * j + 2], e[4 * j + 3]);
              const uint32_t p0 = __nv_cvt_halfraw2_to_fp8x2(*reinterpret_cast<const __half2_raw*>(&h0), __NV_SATFINITE, __NV_E4M3);
              const uint32_t p1 = __nv_cvt_halfraw2_to_fp8x2(*reinterpret_cast<const __half2_raw*>(&h1), __NV_SATFINITE, __NV_E4M3);
              const __half2_raw r0 = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)p0, __NV_E4M3);
              const __half2_raw r1 = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)p1, __NV_E4M3);
              const __half2 d0 = __hsub2(h0, *reinterpret_cast<const __half2*>(&r0));
              const __half2 d1 = __hsub2(h1, *reinterpret_cast<const __half2*>(&r1));
              const uint32_t l0 = __nv_cvt_halfraw2_to_fp8x2(*reinterpret_cast<const __half2_raw*>(&d0), __NV_SATFINITE, __NV_E4M3);
              const uint32_t l1 = __nv_cvt_halfraw2_to_fp8x2(*reinterpret_cast<const __half2_raw*>(&d1), __NV_SATFINITE, __NV_E4M3);
              hi[j] = p0 | (p1 << 16);
              lo[j] = l0 | (l1 << 16);
            }
            const uint32_t at = pt_piece<RW>(kl, j0 >> 4);
            *reinterpret_cast<uint4*>(pbuf + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4*>(pbuf + PT_KEYS * RW + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          } else {
            uint32_t pk[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const __nv_bfloat162 v = __floats2bfloat162_rn(e[2 * j], e[2 * j + 1]);
              pk[j] = *reinterpret_cast<const uint32_t*>(&v);
            }
            *reinterpret_cast<uint4*>(pbuf + pt_piece<2 * RW>(kl, j0 >> 3)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            *reinterpret_cast<uint4*>(pbuf + pt_piece<2 * RW>(kl, (j0 >> 3) + 1)) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
          }
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&X.p_full[tp]);
        if (pending) take_o(cnt - 1, moved_before);
        pending = true;
        moved_before = moved;
        ++cnt;
      }
      if (pending) {
        if (ok) ok = mbar_wait(&X.o_full[tp], (cnt - 1) & 1, abort_flag, status);
        take_o(cnt - 1, moved_before);
      }
      tc_fence_before();

      // ------------------------------------------------ the segment's result
      {
        const float l = pt_rows_reduce<RW, true>(lacc, lane);
        if (lane < RW) {
          X.lsum[warp][lane] = l;
          if (wq == 0) X.m_run[grp][lane] = run;
        }
      }
      float* po = part_o + (size_t)slot * NR * D;
      float* pml = part_ml + (size_t)slot * NR * 2;
      float* mb = reinterpret_cast<float*>(smem + F::OFF_P);     // [NP - 1][NR][128] over the weights
      pt_bar<5, PT_SOFTMAX>();                          // every product has been read: the weights are free
      if (NP > 1 && tp > 0) {
#pragma unroll
        for (int j = 0; j < RW; ++j) mb[((tp - 1) * NR + grow + j) * 128 + kl] = acc[j];
      }
      if (tp == 0 && kl < RW) {
        // row kl of this group: what each turn's sum weighs
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < NP; ++i) m = fmaxf(m, X.m_run[i * NRG + rg][kl]);
        float wt[NP], l = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int g = i * NRG + rg;
          const float mi = X.m_run[g][kl];
          wt[i] = mi == -INFINITY ? 0.f : fast_exp2(mi - m);
          l = fmaf(wt[i], (X.lsum[g * 4][kl] + X.lsum[g * 4 + 1][kl]) + (X.lsum[g * 4 + 2][kl] + X.lsum[g * 4 + 3][kl]), l);
        }
        const float inv = whole ? 1.f / l : 1.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) X.beta[grp * 4 + i][0][kl] = wt[i] * inv;
        if (!whole) {
          pml[(grow + kl) * 2] = m;
          pml[(grow + kl) * 2 + 1] = l;
        }
      }
      pt_bar<5, PT_SOFTMAX>();
      if (tp == 0 && kl < D) {
#pragma unroll
        for (int j = 0; j < RW; ++j) {
          float v = acc[j] * X.beta[grp * 4][0][j];
#pragma unroll
          for (int i = 1; i < NP; ++i) v = fmaf(mb[((i - 1) * NR + grow + j) * 128 + kl], X.beta[grp * 4 + i][0][j], v);
          if (whole) {
            const int off = X.rowoff[grow + j];
            if (off >= 0) out[((size_t)b * M * Hq + off) * D + kl] = __float2bfloat16_rn(v);
          } else {
            po[(size_t)(grow + j) * D + kl] = v;
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 17) {
    tc_fence_after();
    tmem_dealloc(tmem, F::COLS);
  }
  jk_pdl_trigger();
}

// ------------------------------------------------------------------------------------------ merge
// out = sum_s 2^(m_s - m) acc_s / sum_s 2^(m_s - m) l_s over the partials of a unit that spans CTAs; one warp
// per query row.  CTA s holds tiles [total s / G, total (s + 1) / G), so which CTAs hold a unit's tiles, and
// under which of its two slots, follows from the tile counts alone.
template <int D, int NR>
__global__ void __launch_bounds__(256) k_paged_merge(const jk_paged c, int B, int M, int Hq, int Hkv, int n_qblk,
                                                     int grid, const float* __restrict__ part_o,
                                                     const float* __restrict__ part_ml, __nv_bfloat16* __restrict__ out) {
  __shared__ long long cum[JK_MAX_ROWS + 1];
  __shared__ int n8[JK_MAX_ROWS];
  constexpr int DPL = D / 32, NB = 8;
  jk_pdl_wait();
  jk_pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int units = Hkv * n_qblk, G = Hq / Hkv;
  if (warp == 0) pt_count(c, B, M, pt_cfg<D, NR>::WK, units, lane, cum, n8, nullptr, nullptr);
  __syncthreads();
  const int64_t row = (int64_t)blockIdx.x * 8 + warp;
  const int64_t unit = row / NR;
  const int r = (int)(row % NR);
  const int b = (int)(unit / units), u = (int)(unit % units);
  if (b >= B) return;
  const int nr = (u % n_qblk) * NR + r;
  if (nr >= G * M) return;
  const long long total = cum[B], per = (cum[b + 1] - cum[b]) / units;
  if (per == 0) return;
  const long long a = cum[b] + (long long)u * per;
  const long long ctas = total < grid ? total : grid;
  const int c0 = (int)(((a + 1) * ctas - 1) / total), c1 = (int)(((a + per) * ctas - 1) / total);
  if (c0 == c1) return;                                 // one CTA held it all and has written it
  // slot of CTA s: its last segment where the unit begins, its first everywhere else
  float m = -INFINITY;
  for (int s0 = c0; s0 <= c1; s0 += 32) {
    const int s = s0 + lane;
    if (s <= c1) m = fmaxf(m, part_ml[((size_t)(s * 2 + (s == c0 ? 1 : 0)) * NR + r) * 2]);
  }
  m = jk_warp_max(m);
  float acc[DPL], l = 0.f;
#pragma unroll
  for (int t = 0; t < DPL; ++t) acc[t] = 0.f;
  for (int s0 = c0; s0 <= c1; s0 += NB) {
    float v[NB][DPL];
    float2 ml[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int s = s0 + j;
      ml[j] = make_float2(-INFINITY, 0.f);
      if (s > c1) continue;
      const size_t at = (size_t)(s * 2 + (s == c0 ? 1 : 0)) * NR + r;
      ml[j] = *reinterpret_cast<const float2*>(part_ml + at * 2);
      if (DPL == 4) {
        const float4 x = *reinterpret_cast<const float4*>(part_o + at * D + lane * DPL);
        v[j][0] = x.x; v[j][1] = x.y; v[j][DPL - 2] = x.z; v[j][DPL - 1] = x.w;
      } else {
        const float2 x = *reinterpret_cast<const float2*>(part_o + at * D + lane * DPL);
        v[j][0] = x.x; v[j][DPL - 1] = x.y;
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      if (s0 + j > c1 || ml[j].x == -INFINITY) continue;
      const float w = fast_exp2(ml[j].x - m);
      l = fmaf(w, ml[j].y, l);
#pragma unroll
      for (int t = 0; t < DPL; ++t) acc[t] = fmaf(w, v[j][t], acc[t]);
    }
  }
  const float inv = 1.f / l;
  const int gg = nr / M, ii = nr % M;
  __nv_bfloat16* o = out + (((size_t)b * M + ii) * Hq + (u / n_qblk) * G + gg) * D + lane * DPL;
#pragma unroll
  for (int t = 0; t < DPL; ++t) o[t] = __float2bfloat16_rn(acc[t] * inv);
}

// ------------------------------------------------------------------------------------------ host
int jk_tma_encode_bf16(jk_ctx* ctx, CUtensorMap* out, const void* ptr, int rank, const uint64_t* dims,
                       const uint64_t* strides_bytes, const uint32_t* box);
int jk_tma_encode_u8(jk_ctx* ctx, CUtensorMap* out, const void* ptr, int rank, const uint64_t* dims,
                     const uint64_t* strides_bytes, const uint32_t* box);

// Query rows of a block: the smallest of 16, 32, 64, 128 that holds the rows of a kv head, 128 past that.
static int pt_rows(const jk_config& g, int M) {
  const int rows = g.n_q_heads / g.n_kv_heads * M;
  return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
}

// Workspace of the partials: two slots per CTA.
size_t jk_paged_part_floats(const jk_config& g, int with_ml) {
  if (g.dtype != JK_BF16) return 0;
  return (size_t)PT_MAX_CTAS * 2 * pt_rows(g, g.max_tree) * (with_ml ? 2 : g.head_dim);
}

template <int D, int NR>
static int pt_launch(jk_ctx* ctx, cudaStream_t st, const CUtensorMap* maps, const jk_paged* c, int layer, int B, int M,
                     const void* q, const int32_t* parent, float scale, void* out) {
  typedef pt_cfg<D, NR> F;
  const jk_config& g = ctx->cfg;
  const int rows = g.n_q_heads / g.n_kv_heads * M;
  const int n_qblk = (rows + NR - 1) / NR, units = g.n_kv_heads * n_qblk;
  const int64_t most = (int64_t)B * units * (((int64_t)c->max_pages * c->page_size + PT_KEYS - 1) / PT_KEYS +
                                             (c->page_size + M + F::WK - 1) / F::WK);
  int ctas = ctx->sm_count < PT_MAX_CTAS ? ctx->sm_count : PT_MAX_CTAS;
  if (most < ctas) ctas = (int)most;
  const size_t smem = F::OFF_X + sizeof(pt_tail<D, NR>) + 1024;
  static_assert(F::OFF_X + sizeof(pt_tail<D, NR>) + 1024 <= 232448, "shared memory of one CTA");
  auto kern = k_paged_attn_tc<D, NR>;
  JK_CUDA_CHECK(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  float* part_o = (float*)(ctx->ws + ctx->lay.paged_o);
  float* part_ml = (float*)(ctx->ws + ctx->lay.paged_ml);
  JK_PROF(ctx, st, JK_ST_PAGED_ATTN);
  jk_launch_pdl(kern, dim3(ctas), dim3(PT_THREADS), smem, st, maps[0], maps[1], maps[2], maps[3], maps[4], maps[5], *c,
                layer, (const __nv_bfloat16*)q, parent, scale, B, M, g.n_q_heads, g.n_kv_heads, n_qblk,
                (__nv_bfloat16*)out, part_o, part_ml, (int32_t*)(ctx->ws + ctx->lay.status));
  JK_LAUNCH_CHECK(ctx);
  if (ctas == 1) return JK_OK;
  JK_PROF(ctx, st, JK_ST_PAGED_COMBINE);
  jk_launch_pdl(k_paged_merge<D, NR>, dim3((unsigned)((int64_t)B * units * NR / 8)), dim3(256), 0, st, *c, B, M,
                g.n_q_heads, g.n_kv_heads, n_qblk, ctas, (const float*)part_o, (const float*)part_ml,
                (__nv_bfloat16*)out);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}

// Arguments are checked.  Tensor maps are made per call (they are host arithmetic on the arguments).
int jk_paged_attn_tc(jk_ctx* ctx, cudaStream_t st, const jk_paged* c, int layer, int B, int M, const void* q,
                     const void* kt, const void* vt, int64_t sb, int64_t sh, const int32_t* parent, float scale,
                     void* out) {
  const jk_config& g = ctx->cfg;
  const uint64_t D = g.head_dim, ps = c->page_size, H = g.n_kv_heads;
  CUtensorMap maps[6];
  {
    const uint64_t dims[4] = {D, ps, H, (uint64_t)c->n_layers * c->n_pages};
    const uint64_t strides[3] = {D, ps * D, H * ps * D};
    const uint32_t box[4] = {(uint32_t)D, (uint32_t)ps, 1, 1};
    int rc = jk_tma_encode_u8(ctx, &maps[0], c->k_pages, 4, dims, strides, box);
    if (rc == JK_OK) rc = jk_tma_encode_u8(ctx, &maps[1], c->v_pages, 4, dims, strides, box);
    if (rc != JK_OK) return rc;
  }
  const uint32_t box[4] = {64, 16, 1, 1};
  {
    const uint64_t dims[4] = {D, 2 * ps, H, (uint64_t)c->n_layers * c->max_seqs};
    const uint64_t strides[3] = {D * 2, 2 * ps * D * 2, H * 2 * ps * D * 2};
    int rc = jk_tma_encode_bf16(ctx, &maps[2], c->k_open, 4, dims, strides, box);
    if (rc == JK_OK) rc = jk_tma_encode_bf16(ctx, &maps[3], c->v_open, 4, dims, strides, box);
    if (rc != JK_OK) return rc;
  }
  {
    // (rows behind the tree read as zero; with one sequence its stride is never used)
    const uint64_t dims[4] = {D, (uint64_t)M, H, (uint64_t)B};
    const uint64_t strides[3] = {D * 2, (uint64_t)sh * 2, B > 1 ? (uint64_t)sb * 2 : H * (uint64_t)sh * 2};
    int rc = jk_tma_encode_bf16(ctx, &maps[4], kt, 4, dims, strides, box);
    if (rc == JK_OK) rc = jk_tma_encode_bf16(ctx, &maps[5], vt, 4, dims, strides, box);
    if (rc != JK_OK) return rc;
  }
#define PT_CASE(DD, NN) \
  if (g.head_dim == DD && nr == NN) return pt_launch<DD, NN>(ctx, st, maps, c, layer, B, M, q, parent, scale, out)
  const int nr = pt_rows(g, M);
  PT_CASE(128, 16); PT_CASE(128, 32); PT_CASE(128, 64); PT_CASE(128, 128);
  PT_CASE(64, 16); PT_CASE(64, 32); PT_CASE(64, 64); PT_CASE(64, 128);
#undef PT_CASE
  return JK_ERR_SHAPE;
}
