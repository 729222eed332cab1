// jk_linear's tensor-core kernels: what they share of PTX.
#pragma once

#include <cuda.h>

#include "jk_linear.cuh"
#include "jk_tcgen05.cuh"

#define LT_M 128                          // lanes of tensor memory: rows of an operand on the M side, per CTA
#define LT_BOX 128                        // bytes of a box row
#define LT_SMEM (227 * 1024)
#define LT_ACC_COLS 256                   // columns of the accumulators of one tile, at most
#define LT_MAX_CTAS 192
#define LT_SLOT (LT_ACC_COLS * LT_M)      // floats of a partial

// The warps that load and multiply run their loops with all lanes and one lane issues (`lead`): with values
// that the compiler knows to be the same in all lanes, addresses and descriptors live in uniform registers.
// (Issued from inside `if (lane == 0)`, every product cost about 126 cycles, whatever its size, and every
// box of a copy as much; a product of 128 x 64 x 16 takes 32.)
__device__ __forceinline__ uint32_t lt_elect() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r));
  return r;
}
#define LT_IF(arg) "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, " arg ", 0;\n\t@q "
__device__ __forceinline__ void lt_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar, uint32_t lead) {
  asm volatile(LT_IF("%4")
               "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "r"(lead)
               : "memory");
}
__device__ __forceinline__ void lt_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar, uint32_t lead) {
  asm volatile(LT_IF("%5")
               "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "r"(lead)
               : "memory");
}
__device__ __forceinline__ void lt_box_once(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar, uint64_t policy,
                                            uint32_t lead) {
  asm volatile(LT_IF("%6")
               "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, "
               "%3}], [%4], %5;\n\t}"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "l"(policy), "r"(lead)
               : "memory");
}
__device__ __forceinline__ void lt_expect(uint32_t bar, uint32_t bytes, uint32_t lead) {
  asm volatile(LT_IF("%2") "mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes), "r"(lead)
               : "memory");
}
__device__ __forceinline__ void lt_commit(uint32_t bar, uint32_t lead) {
  asm volatile(LT_IF("%1") "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(lead)
               : "memory");
}
__device__ __forceinline__ void l2_prefetch_box(const CUtensorMap* map, int x, int y) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
// D[tmem] (+)= A[smem] B[smem]^T over 16 bf16 along k
__device__ __forceinline__ void lt_mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(lead)
      : "memory");
}
// ... over 32 codes along k, each operand's block scale from tensor memory
__device__ __forceinline__ void lt_mma_mx8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                           uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(acc), "r"(lead)
      : "memory");
}
// 512 bytes of shared memory, 32 rows of 16, to 4 columns of tensor memory, the same for all four quarters of the
// lanes; the descriptor: no swizzle, groups of 8 rows 128 bytes apart
#define LT_SCALE_DESC (((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46))
__device__ __forceinline__ void lt_copy_scales(uint32_t dst, uint64_t desc, uint32_t lead) {
  asm volatile(LT_IF("%2") "tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(dst), "l"(desc), "r"(lead) : "memory");
}
// More bytes for the running phase, without an arrival.
__device__ __forceinline__ void mbar_add_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ int ld_acquire(const int32_t* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void add_release(int32_t* p, int v) {
  asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// 8 columns of tensor memory, the warp's 32 lanes.
__device__ __forceinline__ void lt_ld8(uint32_t addr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(addr));
}
// The address, in the cluster's window, of this place in another CTA's shared memory.
__device__ __forceinline__ uint32_t lt_map(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void lt_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
