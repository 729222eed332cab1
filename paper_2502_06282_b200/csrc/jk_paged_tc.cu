// Tensor-core (tcgen05) kernel of jk_tree_verify_attn_paged for bf16 contexts.
//
// For a block of query rows (pairs of a q head of the group and a tree node) and tiles of 128 keys:
//   S^T = K Q^T   (keys on the 128 lanes, query rows on the columns), then
//   O^T += V^T P^T (head dims on the lanes, query rows on the columns).
// Keys on the lanes because a call has few query rows (1 .. 64 per block): with rows on the lanes a block of 60
// would leave half of the SM's sub-partitions idle in the softmax, and a single token 127 of 128 lanes.
// A thread owns one key: its page's scales are constants of the thread.
//
// K stays 8-bit up to the tensor core.  A bf16 query has 8 significant bits, an e4m3 number 4, so q becomes two of them,
// q 2^a = hi + lo with hi = e4m3(q 2^a) and lo = e4m3(q 2^a - hi), and S is two e4m3 products into one fp32
// accumulator, the price of one bf16 product.  The block's largest q is put between 224 and 448, where the low part's
// steps of 2^-9 end: values down to 2^-2 there are exact (2^-10 of the largest), smaller ones off by 2^-10 at most.
// Rows whose largest values lie within 2^4 of each other share the power of two, so that a value is off by at most
// 2^-13 of its row's largest; rows further apart take one each (2^-17), and S is multiplied by the difference.
// V is widened to fp16 (exact) by a warpgroup of its own, 32 KB per tile, because the softmax weights need more
// than 8 bits: two 8-bit parts per weight cost the softmax three times as many instructions as one
// conversion to fp16, and their range (2^-17) made every few stages form new maxima.
//   x = s scale_k + log2(scale_v),  p = 2^(x - ref + 6) in fp16 (11 significant bits),
// so p carries V's scale (a power of two); the row sum takes p / scale_v in fp32.  ref is the rounded-up
// maximum of the row's first tile in this CTA and only rises: when a weight passes fp16's range (2^10 above the
// reference) the references follow, sums and products so far are scaled, and the tile's weights are formed
// again.  Weights down to 2^-20 of 2^ref keep 11 bits, below 2^-31 they become 0: the tail behind one
// dominant key survives to lengths of 2^20.
//
// The open page and the tree tokens are bf16 tiles of 64 keys at the end of the sequence (16-row boxes of
// either array, dead rows cleared in V): the same pipeline with bf16 products.  V is bf16 there, so the weights are too, as
// in the attention over a 16-bit cache.  Where these keys carry the result (short prefixes) its error against 64 bits is 0.0024
// instead of the 0.0017 of its own rounding; a second bf16 part of the weights gives 0.0017, and was measured at 3.5 % of
// the 7B tree's time at prefix 1024, 5 % of the ragged batch's with G = 4, 1.7 % of 13B's: not taken.
//
// One CTA per SM; all tiles of the call are dealt out evenly in order (sequence, kv head, row block,
// tile), so a unit (sequence, kv head, row block) spans CTAs where it has to; such a CTA leaves an
// unnormalised partial, which k_paged_merge adds up, and a unit inside one CTA is written directly.
// Warps: four softmax groups of four (32 rows of every second tile, with up to 16 rows every fourth tile), four that
// widen V, TMA producers for K and for V, an issuer of either product.  Registers are moved to the softmax
// warps, each role setting its own: with the shared memory this kernel takes a spill is a trip to L2.
//
// Measured (B200, graph replay on the same inputs; in brackets calls one after the other on inputs that leave L2 in
// between, by machine): 13B heads, batch 8, prefix 8192, trees of 60 (690 MB): 169 us = 4.1 TB/s, 0.63 of the measured copy
// bandwidth (190 to 200 us, 0.54 to 0.56); 70B heads, 32 ragged sequences up to 16384, single tokens: 134 us, 0.84 of it (137
// to 147).  A 64-row tile takes about 1700 cycles in the steady state: its share of HBM bandwidth 1424, its
// shared-memory traffic of 190 KB (K read twice, V copied, widened and read, weights written and read) 1490, its 4700
// warp instructions 1180 issue slots per sub-partition; no stage alone is the limit (leaving the widening of V out, as a
// probe, saved 8 %).  At 13B those tiles are 124 us (143 per CTA), the start and the merge 14; the other 30 are the ends of
// units, 3.2 per CTA: both products drain, the softmax groups meet twice, and the next unit's queries and parents are
// loaded, converted and walked before its first weight is formed.
#include <math.h>
#include <stdio.h>

#include "jk_paged.cuh"
#include "jk_tcgen05.cuh"

#define PT_KEYS 128
#define PT_WKEYS 64                  // keys of a bf16 tile
#define PT_SOFTMAX 512               // threads of the softmax groups
#define PT_THREADS 768
#define PT_MAX_CTAS 160
#define PT_INFO 16                   // tile descriptions: at least K slots + 3 tiles per turn (S is two ahead of the weights)
#define PT_SHIFT 6.f                 // a weight at its reference is 2^6

// ------------------------------------------------------------------------------------------ PTX
// The whole warp runs the issuing code and one lane issues: with values the compiler knows to be the same in
// all lanes, descriptors live in uniform registers.  (Issued from inside `if (lane == 0)`, every product
// cost its thread about 90 cycles of register moves, and the tensor core waited.)
__device__ __forceinline__ uint32_t pt_elect() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r));
  return r;
}
__device__ __forceinline__ void pt_mma_f8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void pt_mma_16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void pt_commit(uint64_t* bar, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
      ::"r"(smem_u32(bar)), "r"(lead)
      : "memory");
}
// Bounded wait, kept short (the 32-bit cycle counter, about a second): the loops of this kernel are long, and what
// does not fit the instruction caches is fetched again for every tile.
__device__ __forceinline__ bool pt_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  if (mbar_try_wait(bar, parity)) return true;
  uint32_t t0, t;
  asm volatile("mov.u32 %0, %%clock;" : "=r"(t0));
  do {
    if (mbar_try_wait(bar, parity)) return true;
    asm volatile("mov.u32 %0, %%clock;" : "=r"(t));
  } while (t - t0 < 2000000000u && !*abort_flag);
  *abort_flag = 1;
  jk_set_status(status, JK_ERR_TIMEOUT);
  return false;
}
// Maxima (sums) over lanes of rows held one value per lane and row.  Half of the rows changes sides at every
// step, so each step costs what is left of the rows: pt_fold sends rows j and j + N/2 to the two halves of
// the lanes that differ in bit h, pt_rows_reduce goes on from N rows to one.
template <bool SUM> __device__ __forceinline__ float pt_fold(float a, float b, int h, bool up) {
  const float keep = up ? b : a, send = up ? a : b;
  const float y = __shfl_xor_sync(0xffffffffu, send, h);
  return SUM ? keep + y : fmaxf(keep, y);
}
template <int N, bool SUM> __device__ __forceinline__ float pt_rows_reduce(float (&v)[N], int lane) {
#pragma unroll
  for (int h = N / 2; h >= 1; h >>= 1)
#pragma unroll
    for (int j = 0; j < h; ++j) v[j] = pt_fold<SUM>(v[j], v[j + h], h, lane & h);
  return v[0];
}
// Two fp32 values at a time.
__device__ __forceinline__ uint64_t pt_pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 pt_unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t pt_fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t pt_mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t pt_add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
template <int N> __device__ __forceinline__ void pt_ld(uint32_t addr, uint32_t (&r)[N]) {
  if constexpr (N == 16) tmem_ld16(addr, r);
  else tmem_ld32(addr, r);
}
__device__ __forceinline__ void pt_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15, %16};"
      ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
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
// Four e4m3 codes as fp16.
__device__ __forceinline__ void pt_widen(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(codes));
}
// Instruction descriptor, fp32 accumulate, M = 128; formats: kind::f16 1 = bf16, kind::f8f6f4 0 = e4m3, 1 = e5m2.
__device__ __forceinline__ uint32_t pt_idesc(uint32_t fmt_a, uint32_t fmt_b, int n, int a_mn, int b_mn) {
  return (1u << 4) | (fmt_a << 7) | (fmt_b << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

// ------------------------------------------------------------------------------------------ layout
template <int D, int NR> struct pt_cfg {
  static constexpr int RW = NR == 64 ? 32 : 16;        // rows of a softmax group
  static constexpr int NRG = NR / RW;                  // groups that share a tile
  static constexpr int NP = 4 / NRG;                   // tiles in the groups' hands: their turns
  static constexpr int SLOT = PT_KEYS * D;             // an 8-bit tile of 128 keys or a bf16 tile of 64
  static constexpr int KST = NR == 64 ? 3 : 4;
  static constexpr int VST = NR == 64 ? 2 : 3;
  static constexpr int Q8 = NR * D;                    // one of the two e4m3 parts of the queries
  static constexpr int PROW = 2 * NR;                  // bytes of a key's weights
  static constexpr int PB = PT_KEYS * PROW;            // the weights of a tile, a buffer per turn
  static constexpr int MB = (NP - 1) * NR * 512;       // sums that the other turns hand to the first, in the same place
  static constexpr int PBYTES = NP * PB > MB ? NP * PB : MB;
  static constexpr int VB = PT_KEYS * D * 2;           // a tile of V in fp16
  static constexpr int OFF_Q16 = 2 * Q8;
  static constexpr int OFF_P = OFF_Q16 + NR * D * 2;
  static constexpr int OFF_W = OFF_P + PBYTES;
  static constexpr int OFF_K = OFF_W + 2 * VB;
  static constexpr int OFF_V = OFF_K + KST * SLOT;
  // (behind the rings: a bf16 K tile is read as 128 rows, a head size of 64 one row group further in V)
  static constexpr int OFF_X = OFF_V + VST * SLOT + 1024;
  static constexpr uint32_t O_COL = NP * 2 * NR;       // S: two buffers per turn
  static constexpr uint32_t COLS = NR == 64 ? 512 : 256;
  static_assert(3 * NP * NR <= COLS, "tensor memory");
  static_assert(KST + 3 * NP <= PT_INFO, "tile descriptions");
};

struct pt_info {                     // one tile, written by the producer; bf16 tiles: rows of the tile
  int live;                          // live keys (may pass the tile's)
  int open_rows, open16;             // first row past the open page's tokens, and past their padding
  int pad;
  float sk[8], sv[8], lsv[8];        // per page: K scale, V scale and its log2
};

template <int D, int NR> struct alignas(16) pt_tail {
  uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4];
  uint64_t info_full[PT_INFO], s_full[4][2], s_empty[4][2], p_full[4], p_empty[4], w_full[8], w_empty[2], q_full;
  uint32_t tmem_base;
  int abort_flag;
  long long cum[JK_MAX_ROWS + 1];    // tiles before each sequence
  int n8[JK_MAX_ROWS], n16[JK_MAX_ROWS];
  pt_info info[PT_INFO];
  uint2 q_max[16];                     // per warp, as bits: the largest of the rows' largest magnitudes; the least but 0, less 1
  // of the unit at work, for what comes after its tiles
  int seg_b, seg_slot, seg_whole;
  float c8;                          // logits per product of codes, in units of log2
  uint32_t vis[PT_SOFTMAX];          // masked tiles: rows of the group that see the thread's key
  int rowoff[NR];                    // output row of each query row, -1 = none
  int parent[JK_MAX_TREE];
  alignas(16) uint32_t anc[4][NR];   // tree nodes each query row sees
  // per warp and row (the four warps of a group form the same values); at the end of a unit alpha holds the sums
  alignas(16) float nref[16][32], alpha[16][32];
  alignas(16) float rowf[NR];          // a row's own power of two over the block's, where they are far apart
  float wmax[4][4][32], m_run[4][32], wt[4][NR];
};

// Tiles of every sequence, and their prefix sums, by one warp.
__device__ __forceinline__ void pt_count(const jk_paged& c, int B, int M, int units, int lane, long long* cum,
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
        w = (((P - nf + 15) & ~15) + M + PT_WKEYS - 1) / PT_WKEYS;
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
  constexpr int KST = F::KST, VST = F::VST, RW = F::RW, NRG = F::NRG, NP = F::NP;
  constexpr int KB = D / 64;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* sk = smem + F::OFF_K;
  unsigned char* sv = smem + F::OFF_V;
  typedef pt_tail<D, NR> tail_t;
  tail_t& X = *reinterpret_cast<tail_t*>(smem + F::OFF_X);
  volatile int* abort_flag = &X.abort_flag;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int G = Hq / Hkv, units = Hkv * n_qblk, ps = c.page_size;

  if (warp == 0) {
    // all barriers stand in a row from k_full on; a lane takes two or three
    uint64_t* bars = X.k_full;
    const int n_bars = (int)(&X.q_full - bars) + 1;
    for (int i = lane; i < n_bars; i += 32) {
      uint64_t* bar = bars + i;
      const bool groups = (bar >= &X.s_empty[0][0] && bar <= &X.s_empty[3][1]) || (bar >= X.p_full && bar < X.p_full + 4);
      mbar_init(bar, bar == &X.q_full ? PT_SOFTMAX / 32 : groups ? 4 * NRG : 1);
    }
    if (lane == 0) X.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 21) {
    tmem_alloc(&X.tmem_base, F::COLS);
    tmem_relinquish();
  }
  jk_pdl_wait();
  if (warp == 20) pt_count(c, B, M, units, lane, X.cum, X.n8, X.n16, blockIdx.x == 0 ? status : nullptr);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = X.tmem_base;
  const long long total = X.cum[B];
  // with fewer tiles than CTAs the first `total` CTAs take one each (an empty share would leave a gap)
  const long long ctas = total < gridDim.x ? total : gridDim.x;
  const bool idle = blockIdx.x >= ctas;
  const long long w0 = idle ? 0 : total * blockIdx.x / ctas;
  const int share = idle ? 0 : (int)(total * (blockIdx.x + 1) / ctas - w0);
  bool ok = true;

  // a segment of the CTA's share: unit (b, u), tiles [t0, t1) of its nt; n8 of them 8-bit
  auto segment = [&](int done, int& b, int& u, int& t0, int& t1, int& nt) {
    const long long t = w0 + done;
    b = 0;
    while (X.cum[b + 1] <= t) ++b;
    nt = X.n8[b] + X.n16[b];
    const uint32_t off = (uint32_t)(t - X.cum[b]);      // tiles of one sequence: below 2^32
    u = (int)(off / (uint32_t)nt);
    t0 = (int)(off - (uint32_t)u * (uint32_t)nt);
    t1 = share - done < nt - t0 ? t0 + share - done : nt;
  };

  // registers: 768 x 80 at launch = 512 x 96 + 256 x 48 (each warpgroup sets its own at the top of its roles)
  if (warp >= 20) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
  if (warp == 20 || warp == 22) {
    // ==================================================================== TMA producers: K (20), V (22)
    const bool is_k = warp == 20;
    const int NST = is_k ? KST : VST;
    uint64_t* full = is_k ? X.k_full : X.v_full;
    uint64_t* empty = is_k ? X.k_empty : X.v_empty;
    unsigned char* ring = is_k ? sk : sv;
    const CUtensorMap* map = is_k ? &map_k : &map_v;
    int tc = 0, s_slot = 0, s_par = 1;                  // tiles so far, the slot and its parity
    // pages are read once, unless several row blocks of a kv head come by
    const uint64_t pol = l2_policy_evict_first();
    const bool once = n_qblk == 1;
    const int per = PT_KEYS / ps;                       // pages of a tile
    for (int done = 0; done < share && ok;) {
      int b, u, t0, t1, nt;
      segment(done, b, u, t0, t1, nt);
      done += t1 - t0;
      const int h = u / n_qblk, n8 = X.n8[b];
      const int P = c.kv_len[b], nf = P / ps * ps, n_pg = P / ps;
      const int open_rows = P - nf, open16 = (open_rows + 15) & ~15;
      const int32_t* tab = c.page_table + (size_t)b * c.max_pages;
      // Page ids and scales in batches of 32 pages, lane l the batch's page l, the ids of the next batch
      // asked for a batch ahead: two dependent loads per tile would be the tile's time.
      int at = t0 * per / 32 * 32, id = 0, id_next = 0;
      float ksc = 1.f, vsc = 1.f;
      auto ask = [&](int p0) { return p0 + lane < n_pg ? tab[p0 + lane] : 0; };
      auto take = [&](int raw) {                        // the batch from `at` on
        id = raw;
        if (id < 0 || id >= c.n_pages) {
          jk_set_status(status, JK_ERR_BOUNDS);
          id = 0;
        }
        if (is_k) {
          // (1 behind the last page: no scale of another's page, which may hold anything, reaches a weight of 0)
          const size_t blk = ((size_t)layer * c.n_pages + id) * Hkv + h;
          const bool live = at + lane < n_pg;
          ksc = live ? c.k_scale[blk] : 1.f;
          vsc = live ? c.v_scale[blk] : 1.f;
        }
        id_next = ask(at + 32);
      };
      if (t0 < n8) take(ask(at));
      for (int tile = t0; tile < t1 && ok; ++tile, ++tc) {
        pt_info& I = X.info[tc % PT_INFO];
        ok = __all_sync(0xffffffffu, pt_wait(&empty[s_slot], s_par, abort_flag, status));
        unsigned char* dst = ring + s_slot * F::SLOT;
        if (tile < n8) {
          // (a tile's pages never span two batches: both start at multiples of the tile's page count)
          const int p0 = tile * per, np = min(per, n_pg - p0);
          if (p0 >= at + 32) { at += 32; take(id_next); }
          const int page = __shfl_sync(0xffffffffu, id, (p0 - at + lane) & 31);
          if (ok && lane == 0) mbar_expect_tx(&full[s_slot], (uint32_t)np * ps * D);
          __syncwarp();
          if (ok && lane < np) {
            const int row = layer * c.n_pages + page;
            if (once) tma_load_4d_hint(dst + lane * ps * D, map, 0, 0, h, row, &full[s_slot], pol);
            else tma_load_4d(dst + lane * ps * D, map, 0, 0, h, row, &full[s_slot]);
          }
          if (is_k) {
            const float k1 = __shfl_sync(0xffffffffu, ksc, (p0 - at + lane) & 31);
            const float v1 = __shfl_sync(0xffffffffu, vsc, (p0 - at + lane) & 31);
            if (lane < per) {
              I.sk[lane] = k1;
              I.sv[lane] = v1;
              I.lsv[lane] = (float)((int)(__float_as_uint(v1) >> 23) - 127);
            }
            if (lane == 0) I.live = nf - tile * PT_KEYS;
          }
        } else {
          // bf16 tile: rows g of (open rows, padded to 16, then tree rows) in boxes of 16
          const int base = (tile - n8) * PT_WKEYS;
          const int g = base + (lane / KB) * 16, kb = lane % KB;
          const bool in_open = g < open16;
          const bool mine = lane < PT_WKEYS / 16 * KB && (in_open || g - open16 < M);
          const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * 16 * 64 * 2;
          const int row = in_open ? (nf & (2 * ps - 1)) + g : g - open16;
          const int outer = in_open ? layer * c.max_seqs + b : b;
          if (ok && lane == 0) mbar_expect_tx(&full[s_slot], bytes);
          __syncwarp();
          if (ok && mine)
            tma_load_4d(dst + kb * (PT_WKEYS * 128) + (lane / KB) * 16 * 128,
                        is_k ? (in_open ? &map_ko : &map_kt) : (in_open ? &map_vo : &map_vt), kb * 64, row, h, outer,
                        &full[s_slot]);
          if (is_k && lane == 0) {
            I.live = open16 + M - base;
            I.open_rows = open_rows - base;
            I.open16 = open16 - base;
          }
        }
        __syncwarp();
        if (is_k && lane == 0) mbar_arrive(&X.info_full[tc % PT_INFO]);
        if (++s_slot == NST) { s_slot = 0; s_par ^= 1; }
      }
    }
    if (!ok) {
      // gave up, possibly with copies still in flight: give them a bounded time to land
      const unsigned long long ts = global_ns();
      while (global_ns() - ts < 2000000ull) { /* 2 ms: far longer than any TMA copy */ }
    }
  } else if (warp == 21) {
    // ==================================================================== S issuer
    const uint32_t lead = pt_elect();
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t k8 = pt_desc(smem_u32(sk), 16, 8 * D, pt_layout(D)), q8 = pt_desc(smem_u32(smem), 16, 8 * D, pt_layout(D));
    const uint64_t k16 = pt_desc(smem_u32(sk), 16, 1024, 2), q16 = pt_desc(smem_u32(smem + F::OFF_Q16), 16, 1024, 2);
    const uint32_t id_8 = pt_idesc(0, 0, NR, 0, 0), id_16 = pt_idesc(1, 1, NR, 0, 0);
    int k_slot = 0, k_par = 0, segs = 0;
    uint32_t n = 0;                                     // tiles per turn so far, a byte each
    for (int done = 0; done < share && ok;) {
      int b, u, t0, t1, nt;
      segment(done, b, u, t0, t1, nt);
      done += t1 - t0;
      ok = pt_wait(&X.q_full, segs & 1, abort_flag, status);
      ++segs;
      const int n8 = X.n8[b];
      for (int tile = t0; tile < t1 && ok; ++tile) {
        const int tp = (tile - t0) & (NP - 1);
        const int cg = (n >> (8 * tp)) & 0xff, buf = cg & 1;
        // the columns are free when the weights of the group's tile before last have been written
        ok = pt_wait(&X.s_empty[tp][buf], ((cg >> 1) & 1) ^ 1, abort_flag, status) &&
             pt_wait(&X.k_full[k_slot], k_par, abort_flag, status);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        const uint32_t d = tm + (tp * 2 + buf) * NR;
        const uint32_t at = k_slot * (F::SLOT >> 4);
        if (ok && tile < n8) {
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
              pt_mma_f8(d, k8 + at + k * 2, q8 + part * (F::Q8 >> 4) + k * 2, id_8, (part | k) ? 1u : 0u, lead);
        } else if (ok) {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              pt_mma_16(d, k16 + at + kb * (PT_WKEYS * 8) + k * 2, q16 + kb * (NR * 8) + k * 2, id_16, (kb | k) ? 1u : 0u, lead);
        }
        pt_commit(&X.k_empty[k_slot], lead);
        pt_commit(&X.s_full[tp][buf], lead);
        if (++k_slot == KST) { k_slot = 0; k_par ^= 1; }
        n = (n & ~(0xffu << (8 * tp))) | (((cg + 1u) & 0xffu) << (8 * tp));
      }
    }
    if (!ok) {                                          // products still in flight get a bounded time to end
      const unsigned long long ts = global_ns();
      while (global_ns() - ts < 2000000ull) { }
    }
  } else {
    // ==================================================================== O issuer (warp 23)
    const uint32_t lead = pt_elect();
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t p0 = pt_desc(smem_u32(smem + F::OFF_P), 8 * F::PROW, 8 * F::PROW, pt_layout(F::PROW));
    const uint64_t v16 = pt_desc(smem_u32(smem + F::OFF_W), KB == 2 ? PT_KEYS * 128 : 1024, 1024, 2);
    const uint64_t vw = pt_desc(smem_u32(sv), KB == 2 ? PT_WKEYS * 128 : 1024, 1024, 2);
    const uint32_t id_h = pt_idesc(0, 0, NR, 1, 1), id_b = pt_idesc(1, 1, NR, 1, 1);
    int v_slot = 0, v_tile = 0, w_buf = 0;
    uint32_t n = 0;                                     // tiles per turn so far, a byte each
    for (int done = 0; done < share && ok;) {
      int b, u, t0, t1, nt;
      segment(done, b, u, t0, t1, nt);
      done += t1 - t0;
      const int n8 = X.n8[b];
      for (int tile = t0; tile < t1 && ok; ++tile) {
        const int tp = (tile - t0) & (NP - 1);
        const int cg = (n >> (8 * tp)) & 0xff;
        ok = pt_wait(&X.w_full[v_tile & 7], (v_tile >> 3) & 1, abort_flag, status) &&
             pt_wait(&X.p_full[tp], cg & 1, abort_flag, status);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        const uint32_t d = tm + F::O_COL + tp * NR;
        const uint64_t p = p0 + tp * (F::PB >> 4);
        const bool add = tile - t0 >= NP;
        if (ok && tile < n8) {
          const uint64_t v = v16 + w_buf * (F::VB >> 4);
#pragma unroll
          for (int k = 0; k < PT_KEYS / 16; ++k)
            pt_mma_16(d, v + k * 128, p + k * F::PROW, id_h, (add || k) ? 1u : 0u, lead);
        } else if (ok) {
          const uint64_t v = vw + v_slot * (F::SLOT >> 4);
#pragma unroll
          for (int k = 0; k < PT_WKEYS / 16; ++k)
            pt_mma_16(d, v + k * 128, p + k * F::PROW, id_b, (add || k) ? 1u : 0u, lead);
        }
        pt_commit(&X.p_empty[tp], lead);
        if (tile < n8) {
          pt_commit(&X.w_empty[w_buf], lead);
          w_buf ^= 1;
        } else {
          pt_commit(&X.v_empty[v_slot], lead);
        }
        if (++v_slot == VST) v_slot = 0;
        ++v_tile;
        n = (n & ~(0xffu << (8 * tp))) | (((cg + 1u) & 0xffu) << (8 * tp));
      }
    }
    if (!ok) {
      const unsigned long long ts = global_ns();
      while (global_ns() - ts < 2000000ull) { }
    }
  }
  } else if (warp >= 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    // ==================================================================== V to fp16
    const int ct = tid - PT_SOFTMAX;                    // 0 .. 127
    // Four pieces of 16 codes of rows r and r ^ 5 go through eight lanes: both the 16-byte loads (8 pieces of a
    // swizzled row of codes) and the 16-byte stores (every other piece of a swizzled row of fp16) of such a
    // group fall into different banks.
    const int cw = ct >> 5, qw = lane >> 3, rr = (lane & 4) ? qw ^ 5 : qw;
    // row, piece and so the swizzles' terms of a thread's first step; further steps are whole groups of 8 rows on
    const int half = KB == 2 ? cw & 1 : 0, row0 = (KB == 2 ? cw >> 1 : cw) * 8 + rr;
    const uint32_t at_s = pt_piece<D>(row0, half * 4 + (lane & 3));
    const uint32_t at_d = half * (PT_KEYS * 128) + pt_piece<128>(row0, (lane & 3) * 2);
    int tc = 0, v_slot = 0, v_par = 0, w_n = 0;
    for (int done = 0; done < share;) {
      int b, u, t0, t1, nt;
      segment(done, b, u, t0, t1, nt);
      done += t1 - t0;
      const int n8 = X.n8[b];
      for (int tile = t0; tile < t1; ++tile, ++tc) {
        const pt_info& I = X.info[tc % PT_INFO];
        if (ok) ok = pt_wait(&X.info_full[tc % PT_INFO], (tc / PT_INFO) & 1, abort_flag, status);
        if (ok) ok = pt_wait(&X.v_full[v_slot], v_par, abort_flag, status);
        unsigned char* src = sv + v_slot * F::SLOT;
        if (tile < n8) {
          const int buf = w_n & 1, live = I.live;
          if (ok && w_n >= 2) ok = pt_wait(&X.w_empty[buf], ((w_n >> 1) & 1) ^ 1, abort_flag, status);
          unsigned char* dst = smem + F::OFF_W + buf * F::VB;
          // a warp's step: 8 rows, four pieces (64 dims), then the next 16 (d = 64: 32) rows; four loads are asked for
          // before the first conversion
#pragma unroll 1
          for (int i0 = 0; i0 < 4 * KB; i0 += 4) {
            uint4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint4*>(src + at_s + (i0 + i) * 2048);
            if (live < PT_KEYS) {                       // rows behind the last page may hold anything
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if ((i0 + i) * (32 / KB) + row0 >= live) v[i] = make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t o[8];
              pt_widen(v[i].x, o[0], o[1]);
              pt_widen(v[i].y, o[2], o[3]);
              pt_widen(v[i].z, o[4], o[5]);
              pt_widen(v[i].w, o[6], o[7]);
              *reinterpret_cast<uint4*>(dst + at_d + (i0 + i) * (32 / KB * 128)) = make_uint4(o[0], o[1], o[2], o[3]);
              *reinterpret_cast<uint4*>(dst + (at_d ^ 16u) + (i0 + i) * (32 / KB * 128)) = make_uint4(o[4], o[5], o[6], o[7]);
            }
          }
          ++w_n;
        } else if (ct < PT_WKEYS) {
          // rows that no live key owns may hold anything, NaN included, and 0 * NaN would reach every row
          if (ct >= I.live || (ct >= I.open_rows && ct < I.open16)) {
#pragma unroll 1
            for (int i = 0; i < D / 8; ++i)
              *reinterpret_cast<uint4*>(src + (i >> 3) * (PT_WKEYS * 128) + ct * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        fence_proxy_async_smem();
        pt_bar<6, 128>();
        if (ct == 0) {
          mbar_arrive(&X.w_full[tc & 7]);
          if (tile < n8) mbar_arrive(&X.v_empty[v_slot]);   // (a bf16 tile is read where it is)
        }
        if (++v_slot == VST) { v_slot = 0; v_par ^= 1; }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
    // ==================================================================== softmax groups
    const int grp = warp >> 2, wq = warp & 3;           // group, tensor-memory lane quarter
    const int rg = grp & (NRG - 1), tp = grp / NRG;     // its rows of the block, its turn among the tiles
    const int grow = rg * RW;                           // first row of the group in the block
    const int kl = wq * 32 + lane;                      // this thread's key of a tile / head dim of O
    const uint32_t lane_base = (uint32_t)(wq * 32) << 16;
    unsigned char* pbuf = smem + F::OFF_P + tp * F::PB;
    const uint32_t oa = tmem + lane_base + F::O_COL + tp * NR + grow;
    const int pg = kl / ps;                             // page of the key within a tile
    const float c16 = scale * 1.4426950408889634f;
    auto group_or = [&](bool mine) {                    // a barrier that tells whether any thread said yes
      uint32_t r;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 128, p;\n\t"
          "selp.u32 %0, 1, 0, q;\n\t}"
          : "=r"(r)
          : "r"((uint32_t)mine), "r"(grp + 1)
          : "memory");
      return r != 0;
    };
    auto group_bar = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(grp + 1) : "memory"); };
    auto scale_pow2 = [](float from, float to) { return from == -INFINITY ? 0.f : fast_exp2(from - to); };
    int cnt = 0, tc = 0;                                // tiles of this group, tiles of the CTA
    for (int done = 0; done < share;) {
      int b, u, t0, t1, nt;
      segment(done, b, u, t0, t1, nt);
      done += t1 - t0;
      const int n8 = X.n8[b];
      const int h = u / n_qblk, row0 = (u % n_qblk) * NR, n_rows = G * M;
      // ------------------------------------------------ queries of the unit
      constexpr int QV = (NR * (D / 8) + PT_SOFTMAX - 1) / PT_SOFTMAX;
      uint4 qv[QV];
      static_assert(QV <= 2, "row maxima of all pieces share a word");
      auto q_exp = [](uint32_t a) {                     // the least e with a <= 448 2^e
        return max(-100, min(100, (int)(a >> 23) - 127 - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0)));
      };
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
      // largest magnitude of each piece's row, 16 bits each; infinities and NaN are above all numbers
      uint32_t rmax = 0u;
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const uint32_t m = __vmaxu2(__vmaxu2(qv[i].x & 0x7fff7fffu, qv[i].y & 0x7fff7fffu),
                                    __vmaxu2(qv[i].z & 0x7fff7fffu, qv[i].w & 0x7fff7fffu));
        rmax |= max(m & 0xffffu, m >> 16) << (16 * i);
      }
#pragma unroll
      for (int o = D / 16; o > 0; o >>= 1) rmax = __vmaxu2(rmax, __shfl_xor_sync(0xffffffffu, rmax, o));
      auto row_max = [&](int i) { return rmax >> (16 * i) << 16; };      // as the bits of a float
      uint32_t most = 0u, least = ~0u;
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const uint32_t a = row_max(i);
        if (a < 0x7f800000u) {
          most = max(most, a);
          least = min(least, a - 1u);
        }
      }
      most = __reduce_max_sync(0xffffffffu, most);
      least = __reduce_min_sync(0xffffffffu, least);
      if (lane == 0) X.q_max[warp] = make_uint2(most, least);
      // (also: all groups are done with the previous unit's queries, sums and row tables)
      pt_bar<5, PT_SOFTMAX>();
      {
        const uint2 w = X.q_max[lane & 15];
        most = __reduce_max_sync(0xffffffffu, w.x);
        least = __reduce_min_sync(0xffffffffu, w.y);
      }
      const int qe = q_exp(most);
      // Rows within 2^4 of each other share a power of two.  Else each takes its own, and S is brought to the block's where
      // weights are formed: one row's size must not cost another one its bits.
      const bool apart = least != ~0u && q_exp(least + 1u) < qe - 4;
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const int idx = tid + i * PT_SOFTMAX, r = idx / (D / 8), ch = idx % (D / 8);
        if (r < NR) {
          *reinterpret_cast<uint4*>(smem + F::OFF_Q16 + (ch >> 3) * (NR * 128) + pt_piece<128>(r, ch & 7)) = qv[i];
          const uint32_t a = row_max(i);
          const bool number = a < 0x7f800000u;          // (else all of the row's logits are infinite or NaN: NaN)
          const int re = apart && number && a ? q_exp(a) : qe;
          if (apart && ch == 0) X.rowf[r] = re - qe < -126 ? 0.f : paged_pow2(re - qe);
          const float qinv = number ? paged_pow2(-re) : __int_as_float(0x7fffffff);
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
      if (tid == 0) {
        X.seg_b = b;
        // a partial that does not start its unit is this CTA's first, else its last
        X.seg_slot = (int)(blockIdx.x * 2 + (t0 == 0 ? 1 : 0));
        X.seg_whole = t0 == 0 && t1 == nt;
        X.c8 = scale * 1.4426950408889634f * paged_pow2(qe);
      }
      pt_bar<5, PT_SOFTMAX>();                          // row tables are visible

      float2 lacc[RW / 2];                              // sums of the weights of this thread's keys, unit 2^ref
#pragma unroll
      for (int i = 0; i < RW / 2; ++i) lacc[i] = make_float2(0.f, 0.f);
      float ref = -INFINITY;                            // of row lane (mod RW)
      bool unseen = true;                               // some row has no reference yet
      const int cnt0 = cnt;                             // tiles before this unit

      for (int tile = t0; tile < t1; ++tile, ++tc) {
        if (((tile - t0) & (NP - 1)) != tp) continue;
        const bool wide = tile >= n8;
        const pt_info& I = X.info[tc % PT_INFO];
        if (ok) ok = pt_wait(&X.info_full[tc % PT_INFO], (tc / PT_INFO) & 1, abort_flag, status);
        // A tile with keys that not every row sees (dead ones behind the last, tree nodes) leaves the rows that
        // see this thread's key in vis.
        const bool masked = wide || I.live < PT_KEYS;
        if (masked) {
          bool dead = kl >= I.live;
          int node = -1;
          if (wide) {
            dead = dead || kl >= PT_WKEYS || (kl >= I.open_rows && kl < I.open16);
            if (!dead && kl >= I.open16) node = kl - I.open16;
          }
          uint32_t v = 0xffffffffu;
          if (node >= 0) {
            const uint4* aw = reinterpret_cast<const uint4*>(&X.anc[(node >> 5) & 3][grow]);
            const int sh = node & 31;
            v = 0u;
#pragma unroll 1
            for (int e = 0; e < RW; e += 4) {
              const uint4 a = aw[e >> 2];
              v |= (((a.x >> sh) & 1u) | ((a.y >> sh) & 1u) << 1 | ((a.z >> sh) & 1u) << 2 | ((a.w >> sh) & 1u) << 3) << e;
            }
          }
          X.vis[tid] = dead ? 0u : v;
        }
        const float k1 = wide ? c16 : X.c8 * I.sk[pg], l1 = wide ? 0.f : I.lsv[pg], f1 = wide ? 1.f : I.sv[pg];
        if (ok) ok = pt_wait(&X.s_full[tp][cnt & 1], (cnt >> 1) & 1, abort_flag, status);
        __syncwarp();
        tc_fence_after();
        const uint32_t sa = tmem + lane_base + (tp * 2 + (cnt & 1)) * NR + grow;
        if (__builtin_expect(apart && !wide, 0)) {
          // S from the rows' own powers of two to the block's, where it stands: the loops below do not know of it
#pragma unroll 1
          for (int j0 = 0; j0 < RW; j0 += 16) {
            uint32_t r[16];
            tmem_ld16(sa + j0, r);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * X.rowf[grow + j0 + j]);
            pt_st16(sa + j0, r);
          }
          tmem_st_wait();
        }

        // the weights of the group's last tile have been read, and its product is complete
        auto last_product = [&]() {
          if (cnt > 0) {
            if (ok) ok = pt_wait(&X.p_empty[tp], (cnt - 1) & 1, abort_flag, status);
            __syncwarp();
            tc_fence_after();
          }
        };
        // References, raised to the rounded-up maximum of the tile where that is higher; sums follow.
        auto references = [&]() {
          {
            uint32_t r[RW];
            float m[RW];
            pt_ld<RW>(sa, r);
            tmem_ld_wait();
            const uint32_t v1 = masked ? X.vis[tid] : 0xffffffffu;
#pragma unroll
            for (int j = 0; j < RW; ++j) m[j] = (v1 >> j) & 1u ? fmaf(__uint_as_float(r[j]), k1, l1) : -INFINITY;
            float top = pt_rows_reduce<RW, false>(m, lane);
            if (RW == 16) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            if (lane < RW) X.wmax[grp][wq][lane] = top;
          }
          group_bar();
          const float* wm = &X.wmax[grp][0][lane & (RW - 1)];
          const float now = fmaxf(ref, ceilf(fmaxf(fmaxf(wm[0], wm[32]), fmaxf(wm[64], wm[96]))));
          if (lane < RW) {
            // (a row that sees nothing here has a reference of 0 meanwhile: its weights are all 0)
            X.nref[warp][lane] = PT_SHIFT - (now == -INFINITY ? 0.f : now);
            X.alpha[warp][lane] = scale_pow2(ref, now);
          }
          const bool moved = __any_sync(0xffffffffu, ref != now);
          unseen = __any_sync(0xffffffffu, now == -INFINITY);
          ref = now;
          __syncwarp();
          if (moved && cnt > cnt0) {
#pragma unroll
            for (int j = 0; j < RW / 2; ++j) {
              const float2 al = *reinterpret_cast<const float2*>(&X.alpha[warp][2 * j]);
              lacc[j].x *= al.x;
              lacc[j].y *= al.y;
            }
            last_product();
#pragma unroll 1
            for (int j0 = 0; j0 < RW; j0 += 16) {
              uint32_t r[16];
              tmem_ld16(oa + j0, r);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * X.alpha[warp][j0 + j]);
              pt_st16(oa + j0, r);
            }
            tmem_st_wait();
          }
          group_bar();                                  // wmax may be written again
        };
        // ---- weights; a second time, with higher references, if one passed the range.  The row sums are fp32 and
        // right the first time unless a weight was infinite; such a sum (`lost`) starts again, what it held
        // is below 2^-80 of what comes in.
        uint32_t lost = 0u;
        bool anew = unseen;
        for (int attempt = 0; attempt < 2; ++attempt) {
          if (anew) references();
          uint32_t most = 0u;                           // two maxima of 16-bit patterns: no weight is negative
          const uint64_t kk = pt_pack2(k1, k1), ff = pt_pack2(f1, f1);
#pragma unroll
          for (int j0 = 0; j0 < RW; j0 += 16) {
            uint32_t x[16], pk[8];
            float2 e[8];
            tmem_ld16(sa + j0, x);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
              const ulonglong2 rf = *reinterpret_cast<const ulonglong2*>(&X.nref[warp][j0 + 2 * j]);
              e[j] = pt_unpack2(pt_fma2(pt_pack2(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1])), kk, rf.x));
              e[j + 1] = pt_unpack2(pt_fma2(pt_pack2(__uint_as_float(x[2 * j + 2]), __uint_as_float(x[2 * j + 3])), kk, rf.y));
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = make_float2(fast_exp2(e[j].x), fast_exp2(e[j].y));
            if (masked) {
              const uint32_t v1 = X.vis[tid] >> j0;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                if (!((v1 >> (2 * j)) & 1u)) e[j].x = 0.f;
                if (!((v1 >> (2 * j + 1)) & 1u)) e[j].y = 0.f;
              }
            }
            if (attempt == 0) {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                lacc[j0 / 2 + j] = pt_unpack2(pt_add2(pt_pack2(lacc[j0 / 2 + j].x, lacc[j0 / 2 + j].y), pt_pack2(e[j].x, e[j].y)));
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                if ((lost >> (j0 + 2 * j)) & 1u) lacc[j0 / 2 + j].x += e[j].x;
                if ((lost >> (j0 + 2 * j + 1)) & 1u) lacc[j0 / 2 + j].y += e[j].y;
              }
            }
            if (!wide) {
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const __half2 v = __float22half2_rn(pt_unpack2(pt_mul2(pt_pack2(e[j].x, e[j].y), ff)));
                pk[j] = *reinterpret_cast<const uint32_t*>(&v);
              }
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const __nv_bfloat162 v = __float22bfloat162_rn(e[j]);
                pk[j] = *reinterpret_cast<const uint32_t*>(&v);
              }
            }
#pragma unroll
            for (int j = 0; j < 8; j += 2) most = __vimax3_u16x2(most, pk[j], pk[j + 1]);
            if (j0 == 0) last_product();
            *reinterpret_cast<uint4*>(pbuf + pt_piece<F::PROW>(kl, (grow + j0) >> 3)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            *reinterpret_cast<uint4*>(pbuf + pt_piece<F::PROW>(kl, ((grow + j0) >> 3) + 1)) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
          }
          if (attempt == 1) break;
          // fp16 infinity; 65536 in bf16
          const uint32_t limit = wide ? 0x4780u : 0x7c00u;
          const bool over = (most & 0xffffu) >= limit || (most >> 16) >= limit;
          if (!group_or(over)) break;
#pragma unroll
          for (int j = 0; j < RW / 2; ++j) {
            if (lacc[j].x == INFINITY) { lacc[j].x = 0.f; lost |= 1u << (2 * j); }
            if (lacc[j].y == INFINITY) { lacc[j].y = 0.f; lost |= 2u << (2 * j); }
          }
          anew = true;
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&X.s_empty[tp][cnt & 1]);
          mbar_arrive(&X.p_full[tp]);
        }
        ++cnt;
      }
      if (cnt > cnt0) {
        if (ok) ok = pt_wait(&X.p_empty[tp], (cnt - 1) & 1, abort_flag, status);
        __syncwarp();
        tc_fence_after();
      }

      // ------------------------------------------------ the segment's result
      {
        float l[RW];
#pragma unroll
        for (int j = 0; j < RW / 2; ++j) { l[2 * j] = lacc[j].x; l[2 * j + 1] = lacc[j].y; }
        float sum = pt_rows_reduce<RW, true>(l, lane);
        if (RW == 16) sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        if (lane < RW) {
          X.alpha[warp][lane] = sum;
          if (wq == 0) X.m_run[grp][lane] = ref;
        }
      }
      const int seg_b = X.seg_b;
      const bool whole = X.seg_whole != 0;
      float* po = part_o + (size_t)X.seg_slot * NR * D;
      float* pml = part_ml + (size_t)X.seg_slot * NR * 2;
      float* mb = reinterpret_cast<float*>(smem + F::OFF_P);     // [NP - 1][NR][128] over the weights
      pt_bar<5, PT_SOFTMAX>();                          // every product has been read: the weights are free
      if (tp > 0 && cnt > cnt0) {
#pragma unroll 1
        for (int j0 = 0; j0 < RW; j0 += 16) {
          uint32_t v[16];
          tmem_ld16(oa + j0, v);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) mb[((tp - 1) * NR + grow + j0 + j) * 128 + kl] = __uint_as_float(v[j]);
        }
      }
      if (tid < NR) {
        // row tid: what each turn's sum weighs
        const int g0 = tid / RW, r = tid & (RW - 1);
        float m = -INFINITY, l = 0.f, a[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) m = fmaxf(m, X.m_run[i * NRG + g0][r]);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int w = (i * NRG + g0) * 4;
          a[i] = scale_pow2(X.m_run[i * NRG + g0][r], m);
          l = fmaf(a[i], (X.alpha[w][r] + X.alpha[w + 1][r]) + (X.alpha[w + 2][r] + X.alpha[w + 3][r]), l);
        }
        const float inv = whole ? 1.f / l : 1.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) X.wt[i][tid] = a[i] * inv;
        if (!whole) {
          pml[tid * 2] = m;
          pml[tid * 2 + 1] = l;
        }
      }
      tc_fence_before();
      pt_bar<5, PT_SOFTMAX>();
      if (tp == 0) {                                    // (the first tile was this turn's: there is a sum)
#pragma unroll 1
        for (int j0 = 0; j0 < RW; j0 += 16) {
          uint32_t x[16];
          tmem_ld16(oa + j0, x);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int row = grow + j0 + j;
            float v = __uint_as_float(x[j]) * X.wt[0][row];
#pragma unroll
            for (int i = 1; i < NP; ++i) {
              const float w1 = X.wt[i][row];
              if (w1 != 0.f) v = fmaf(mb[((i - 1) * NR + row) * 128 + kl], w1, v);
            }
            if (kl < D) {
              if (whole) {
                const int off = X.rowoff[row];
                if (off >= 0) out[((size_t)seg_b * M * Hq + off) * D + kl] = __float2bfloat16_rn(v);
              } else {
                po[(size_t)row * D + kl] = v;
              }
            }
          }
        }
        tc_fence_before();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 21) {
    tc_fence_after();
    tmem_dealloc(tmem, F::COLS);
  }
  jk_pdl_trigger();
}

// ------------------------------------------------------------------------------------------ merge
// out = sum_s 2^(m_s - m) acc_s / sum_s 2^(m_s - m) l_s over the partials of a unit that spans CTAs.  CTA s holds
// tiles [total s / G, total (s + 1) / G), so which CTAs hold a unit's tiles, and under which of its two
// slots, follows from the tile counts alone.  A warp takes RPW rows with all their loads under way together: one
// where the rows are few (7B heads, prefix 1024: 5 us against 7 with four), four where each block's search for
// the unit's CTAs would be for few rows (13B heads, batch 8: 10 us against 13 with one).
template <int D, int NR, int RPW>
__global__ void __launch_bounds__(256) k_paged_merge(const jk_paged c, int B, int M, int Hq, int Hkv, int n_qblk,
                                                     int grid, const float* __restrict__ part_o,
                                                     const float* __restrict__ part_ml, __nv_bfloat16* __restrict__ out) {
  __shared__ long long cum[JK_MAX_ROWS + 1];
  __shared__ int n8[JK_MAX_ROWS];
  __shared__ int s_c[2];
  constexpr int DPL = D / 32, RB = 8 * RPW, NB = RPW == 1 ? 8 : 4;
  static_assert(NR % RB == 0, "a block's rows are of one unit");
  jk_pdl_wait();
  jk_pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int units = Hkv * n_qblk, G = Hq / Hkv;
  const int unit = blockIdx.x / (NR / RB), r0 = (blockIdx.x % (NR / RB)) * RB + warp * RPW;
  const int b = unit / units, u = unit % units;
  if (warp == 0) {
    pt_count(c, B, M, units, lane, cum, n8, nullptr, nullptr);
    __syncwarp();
    if (lane < 2) {
      const long long total = cum[B], per = (cum[b + 1] - cum[b]) / units;
      const long long a = cum[b] + (long long)u * per;
      const long long ctas = total < grid ? total : grid;
      s_c[lane] = per == 0 ? 0 : (int)(((lane == 0 ? a + 1 : a + per) * ctas - 1) / total);
    }
  }
  __syncthreads();
  const int c0 = s_c[0], c1 = s_c[1];
  if (c0 == c1) return;                                 // one CTA held it all and has written it (or there is nothing)
  const int live = min(RPW, G * M - ((u % n_qblk) * NR + r0));   // rows of this warp
  if (live <= 0) return;
  // slot of CTA s: its last segment where the unit begins, its first everywhere else
  auto slot = [&](int s, int r) { return (size_t)(s * 2 + (s == c0 ? 1 : 0)) * NR + r; };
  float m[RPW], l[RPW], acc[RPW][DPL];
#pragma unroll
  for (int q = 0; q < RPW; ++q) {
    m[q] = -INFINITY;
    l[q] = 0.f;
#pragma unroll
    for (int t = 0; t < DPL; ++t) acc[q][t] = 0.f;
  }
  for (int s0 = c0; s0 <= c1; s0 += 32) {
#pragma unroll
    for (int q = 0; q < RPW; ++q)
      if (s0 + lane <= c1 && q < live) m[q] = fmaxf(m[q], part_ml[slot(s0 + lane, r0 + q) * 2]);
  }
#pragma unroll
  for (int q = 0; q < RPW; ++q) m[q] = jk_warp_max(m[q]);
  for (int s0 = c0; s0 <= c1; s0 += 32) {
    float w[RPW];                                       // of slot s0 + lane
#pragma unroll
    for (int q = 0; q < RPW; ++q) {
      float2 ml = make_float2(-INFINITY, 0.f);
      if (s0 + lane <= c1 && q < live) ml = *reinterpret_cast<const float2*>(part_ml + slot(s0 + lane, r0 + q) * 2);
      // (a maximum of -inf: nothing seen, the sum is 0; or nothing but NaN, and so is the sum)
      w[q] = ml.x == -INFINITY ? ml.y * 0.f : fast_exp2(ml.x - m[q]);
      l[q] += w[q] == 0.f ? 0.f : w[q] * ml.y;
    }
    const int n = min(32, c1 - s0 + 1);
    for (int j0 = 0; j0 < n; j0 += NB) {
      float4 v[NB][RPW];
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int q = 0; q < RPW; ++q)
          if (j0 + j < n && q < live) {
            const float* p = part_o + slot(s0 + j0 + j, r0 + q) * D + lane * DPL;
            if (DPL == 4) {
              v[j][q] = *reinterpret_cast<const float4*>(p);
            } else {
              const float2 x = *reinterpret_cast<const float2*>(p);
              v[j][q] = make_float4(x.x, x.y, 0.f, 0.f);
            }
          }
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int q = 0; q < RPW; ++q) {
          const float wj = __shfl_sync(0xffffffffu, w[q], (j0 + j) & 31);
          if (j0 + j >= n || q >= live || wj == 0.f) continue;
          const float x[4] = {v[j][q].x, v[j][q].y, v[j][q].z, v[j][q].w};
#pragma unroll
          for (int t = 0; t < DPL; ++t) acc[q][t] = fmaf(wj, x[t], acc[q][t]);
        }
    }
  }
#pragma unroll
  for (int q = 0; q < RPW; ++q) {
    const float inv = 1.f / jk_warp_sum(l[q]);
    if (q >= live) continue;
    const int nr = (u % n_qblk) * NR + r0 + q, gg = nr / M, ii = nr % M;
    __nv_bfloat162* o = reinterpret_cast<__nv_bfloat162*>(
        out + (((size_t)b * M + ii) * Hq + (u / n_qblk) * G + gg) * D + lane * DPL);
#pragma unroll
    for (int t = 0; t < DPL / 2; ++t) o[t] = __floats2bfloat162_rn(acc[q][2 * t] * inv, acc[q][2 * t + 1] * inv);
  }
}

// ------------------------------------------------------------------------------------------ host
int jk_tma_encode_bf16(jk_ctx* ctx, CUtensorMap* out, const void* ptr, int rank, const uint64_t* dims,
                       const uint64_t* strides_bytes, const uint32_t* box);
int jk_tma_encode_u8(jk_ctx* ctx, CUtensorMap* out, const void* ptr, int rank, const uint64_t* dims,
                     const uint64_t* strides_bytes, const uint32_t* box);

// Query rows of a block: the smallest of 16, 32, 64 that holds the rows of a kv head, 64 past that.
static int pt_rows(const jk_config& g, int M) {
  const int rows = g.n_q_heads / g.n_kv_heads * M;
  return rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
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
                                             (c->page_size + M + PT_WKEYS - 1) / PT_WKEYS);
  int ctas = ctx->sm_count < PT_MAX_CTAS ? ctx->sm_count : PT_MAX_CTAS;
  if (most < ctas) ctas = (int)most;
  const size_t smem = F::OFF_X + sizeof(pt_tail<D, NR>) + 1024;
  static_assert(F::OFF_X + sizeof(pt_tail<D, NR>) + 1024 <= 232448, "shared memory of one CTA");
  auto kern = k_paged_attn_tc<D, NR>;
  JK_CUDA_CHECK(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  // what the roles take (512 x 96 + 256 x 48) has to be there at launch, or the kernel would wait for it
  cudaFuncAttributes attr;
  JK_CUDA_CHECK(ctx, cudaFuncGetAttributes(&attr, kern));
  if (attr.numRegs * PT_THREADS < 512 * 96 + 256 * 48) {
    snprintf(ctx->cuda_err, sizeof(ctx->cuda_err), "k_paged_attn_tc was built with %d registers", attr.numRegs);
    return JK_ERR_CUDA;
  }
  float* part_o = (float*)(ctx->ws + ctx->lay.paged_o);
  float* part_ml = (float*)(ctx->ws + ctx->lay.paged_ml);
  JK_PROF(ctx, st, JK_ST_PAGED_ATTN);
  jk_launch_pdl(kern, dim3(ctas), dim3(PT_THREADS), smem, st, maps[0], maps[1], maps[2], maps[3], maps[4], maps[5], *c,
                layer, (const __nv_bfloat16*)q, parent, scale, B, M, g.n_q_heads, g.n_kv_heads, n_qblk,
                (__nv_bfloat16*)out, part_o, part_ml, (int32_t*)(ctx->ws + ctx->lay.status));
  JK_LAUNCH_CHECK(ctx);
  if (ctas == 1) return JK_OK;
  JK_PROF(ctx, st, JK_ST_PAGED_COMBINE);
  const int64_t m_rows = (int64_t)B * units * NR;
  constexpr int WIDE = NR == 16 ? 2 : 4;
  const bool few = m_rows / 8 <= 4ll * ctx->sm_count;
  auto merge = few ? k_paged_merge<D, NR, 1> : k_paged_merge<D, NR, WIDE>;
  jk_launch_pdl(merge, dim3((unsigned)(m_rows / (few ? 8 : 8 * WIDE))), dim3(256), 0, st, *c, B, M, g.n_q_heads,
                g.n_kv_heads, n_qblk, ctas, (const float*)part_o, (const float*)part_ml, (__nv_bfloat16*)out);
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
  PT_CASE(128, 16); PT_CASE(128, 32); PT_CASE(128, 64);
  PT_CASE(64, 16); PT_CASE(64, 32); PT_CASE(64, 64);
#undef PT_CASE
  return JK_ERR_SHAPE;
}
