// Swizzled operand tiles for tcgen05: tiled bulk copies (TMA) of [rows x 64] bf16 blocks, their descriptors, products whose left
// operand lives in tensor memory, and registers -> tensor memory.
//
// A tile of R rows and D channels is D / 64 blocks of R rows x 128 bytes, each in the 128-byte swizzle: the 16-byte piece p of row r
// lies at piece p ^ (r % 8) of the row.  Blocks start on 1024 bytes.  The same tile serves both roles of a product:
//   K-major   rows are M or N, channels are K:   a K-step of 16 channels is 32 bytes further, 8 rows are 1024 bytes
//   MN-major  rows are K, channels are M or N:   a K-step of 16 rows is 2048 bytes further, 64 channels are one block
#pragma once
#include "ln_umma.cuh"
#include <cuda.h>

namespace ln {
namespace umma {

__device__ __forceinline__ uint64_t tile_desc(uint32_t saddr, uint32_t lbo_bytes) {
  uint64_t d = (uint64_t)((saddr & 0x3FFFF) >> 4);
  d |= (uint64_t)((lbo_bytes >> 4) & 0x3FFF) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;   // descriptor version of sm_100
  d |= (uint64_t)2 << 61;   // 128-byte swizzle
  return d;
}
// Descriptors of a tile as a K-major operand (rows are M or N) and as an MN-major one (rows are K, blocks of `rows` rows), and how
// far K-step ks of it is: a constant once the loop over ks is unrolled, so that a step costs one addition.  (With the descriptor
// formed step by step in a loop that was not unrolled an MMA was issued every 100 clocks, whatever its size.)
__device__ __forceinline__ uint64_t rows_desc(uint32_t tile) { return tile_desc(tile, 16); }
__device__ __forceinline__ uint64_t cols_desc(uint32_t tile, int rows) { return tile_desc(tile, (uint32_t)rows * 128u); }
__device__ __forceinline__ constexpr uint64_t rows_step(int rows, int ks) { return (uint64_t)(((ks >> 2) * rows * 128 + (ks & 3) * 32) >> 4); }
__device__ __forceinline__ constexpr uint64_t cols_step(int ks) { return (uint64_t)(ks * 2048 >> 4); }

// D[tmem] (+)= A[tmem] * B for one K-step: A holds two bf16 of K per 32-bit column, 8 columns a step.  ONE thread.
__device__ __forceinline__ void mma_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, bool accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate ? 1u : 0u) : "memory");
}

// 32 consecutive columns of this thread's TMEM lane without the wait: several loads may be in flight.  The registers may be read
// after tmem_ld_wait() and tie32() of each load (they pass through it, so that no use is moved in front of the wait).
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
        "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]),
        "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]),
        "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld16_async(uint32_t taddr, float* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
        "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tie32(float* r) {
#pragma unroll
  for (int q = 0; q < 32; ++q) asm volatile("" : "+f"(r[q]));
}
__device__ __forceinline__ void tie16(float* r) {
#pragma unroll
  for (int q = 0; q < 16; ++q) asm volatile("" : "+f"(r[q]));
}
// 16 columns of this thread's lane <- registers
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void mbar_arrive(unsigned long long* mbar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(s32(mbar)) : "memory");
}

// One block (64 channels from c) of the rows from r of (head, batch): rows and channels out of range arrive as zeros.  ONE thread.
__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap* map, int c, int r, int h, int b, unsigned long long* mbar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(c), "r"(r), "r"(h), "r"(b), "r"(s32(mbar)) : "memory");
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

}  // namespace umma

// A [B, H, n, d] view as the kernels load it: the tensor map, and whether head and batch are axes of it (a broadcast axis has
// extent one in the map).
struct TileMap { CUtensorMap map; int head, batch; };

}  // namespace ln
