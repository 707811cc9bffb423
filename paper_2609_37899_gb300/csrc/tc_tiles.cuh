// tc_tiles.cuh -- what the 16-bit matrix products of the first-order operators
// need beyond tc_primitives.cuh: tensor maps and tiled bulk copies, and the
// descriptors of 128-byte-swizzled operand tiles, K-major and MN-major.
//
// A stage of an operand is made of boxes of 64 columns (128 bytes) by some
// rows of the matrix in memory, each row 128 bytes further, the 16-byte pieces
// of a row permuted by the row's index modulo 8 (the 128-byte swizzle).
//  - K-major (the columns are the product's depth): one box of 128 rows; eight
//    rows lie 1024 bytes apart from the next eight.
//  - MN-major (the columns are the operand's rows): one box of 64 rows per 64
//    columns; the depth runs over the box's rows.
#pragma once

#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "tc_primitives.cuh"

namespace soma {
namespace tc {

constexpr int kDepth = 64;                  // depth of one stage
constexpr uint32_t kBoxBytes = 64 * 128;    // an MN-major box

// ---- CTA pairs ------------------------------------------------------------
// Two CTAs of a cluster multiply one 256-row tile: each stages 128 rows of A
// and half of B's rows, the even one issues the products for both, and each
// accumulates its own 128 rows.
__device__ __forceinline__ uint32_t pair_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

// Cluster address of the even CTA's shared variable at the same place as *p.
__device__ __forceinline__ uint32_t leader_addr(const void* p) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(p)));
  return r;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
}

// Arrives on a barrier given by its cluster address.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar)
               : "memory");
}

// 2-D tiled copy of one box at (x, y) = (column, row) into this CTA's shared
// memory; the bytes are counted on the barrier at the cluster address `bar`.
__device__ __forceinline__ void tile_g2s_pair(void* smem_dst, const CUtensorMap* map, int x, int y,
                                              uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile"
      ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(smem_dst)),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

__device__ __forceinline__ void tmem_alloc_pair(uint32_t* slot, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                   smem_u32(slot)),
               "r"(ncols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
               : "memory");
}

// D[tmem of both] (+)= A * B^T with operands in both CTAs' shared memory.
__device__ __forceinline__ void mma_f16_ss_pair(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo,
                                                uint32_t desc_hi, uint32_t idesc,
                                                uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 da, db;\n setp.ne.b32 p, %5, 0;\n"
      " mov.b64 da, {%1, %3};\n mov.b64 db, {%2, %3};\n"
      " tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, p;\n}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(desc_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Arrive on *bar of both CTAs once every tcgen05.mma of this thread so far
// has completed.
__device__ __forceinline__ void mma_commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64"
      " [%0], %1;" ::"r"(smem_u32(bar)),
      "h"((uint16_t)3)
      : "memory");
}

// ---- tiled stores ---------------------------------------------------------
__device__ __forceinline__ void tile_s2g(const CUtensorMap* map, int x, int y, const void* src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::
                   "l"(map),
               "r"(x), "r"(y), "r"(smem_u32(src))
               : "memory");
}

// Adds the fp32 box to memory.
__device__ __forceinline__ void tile_add_s2g(const CUtensorMap* map, int x, int y,
                                             const void* src) {
  asm volatile(
      "cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], "
      "[%3];" ::"l"(map),
      "r"(x), "r"(y), "r"(smem_u32(src))
      : "memory");
}

__device__ __forceinline__ void bulk_commit() {
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// This thread's committed stores have read their shared memory.
__device__ __forceinline__ void bulk_wait_read() {
  asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}
// ... and have been made.
__device__ __forceinline__ void bulk_wait() {
  asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// High word of a swizzled operand descriptor: 1024 bytes between groups of
// eight rows, descriptor version 1, 128-byte swizzle.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);

// Low word: start address, and between 64-column blocks of an MN-major
// operand the size of a box (K-major operands have a single block: unused).
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, bool mn_major) {
  return ((saddr & 0x3FFFFu) >> 4) | ((mn_major ? kBoxBytes >> 4 : 1u) << 16);
}

// What 16 steps of depth add to the low word: 32 bytes of a row, or 16 rows.
__host__ __device__ constexpr uint32_t desc_step(bool mn_major) {
  return mn_major ? (16u * 128u) >> 4 : 32u >> 4;
}

// Instruction descriptor of kind::f16 with fp32 accumulation.
__host__ __device__ constexpr uint32_t idesc_16(int M, int N, bool bf16, bool a_mn, bool b_mn) {
  return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) |
         ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(M >> 4) << 24);
}

// 32 consecutive fp32 columns of this thread's TMEM lane; the values are
// there after tmem_wait_ld32() of the same array.
__device__ __forceinline__ void tmem_ld32_nowait(uint32_t taddr, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr));
}

// Waits for this thread's tensor-memory loads; the array goes through the
// statement so that no use of it is moved ahead of the wait.
__device__ __forceinline__ void tmem_wait_ld32(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31]));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

}  // namespace tc

// Tensor map of a row-major matrix [rows][cols] of a soma_dtype, `stride`
// elements between rows, in boxes of 128 bytes of columns by box_rows rows.
// The address must be 16-byte aligned and the stride a multiple of 16 bytes.
// What lies outside the matrix reads as zero and is not written.
bool make_tile_map(CUtensorMap* map, const void* base, int dtype, int64_t rows, int64_t cols,
                   int64_t stride, int box_rows);

// Tensor map of a 3-D tensor, the first dimension adjacent and `stride`
// elements between neighbours of the other two, in plain boxes (no swizzle).
// The address must be 16-byte aligned, the strides multiples of 16 bytes, the
// second a multiple of the first and neither shorter than what it steps over.
bool make_box_map(CUtensorMap* map, const void* base, int dtype, const int64_t (&size)[3],
                  const int64_t (&stride)[2], const int (&box_size)[3]);

// Tensor map of a 4-D tensor of a 16-bit type, the first dimension adjacent and
// `stride` elements between neighbours of the others, in boxes of 64 columns
// (128 bytes, swizzled).  As make_box_map, each stride a multiple of the last.
bool make_swizzled_map(CUtensorMap* map, const void* base, int dtype, const int64_t (&size)[4],
                       const int64_t (&stride)[3], const int (&box_size)[4]);

}  // namespace soma
