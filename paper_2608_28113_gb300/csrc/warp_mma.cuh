// warp_mma.cuh -- warp-level MMA (m16n8k16, bf16 operands, fp32 sums) for the thin products beside the
// tcgen05 kernels.  Lane = 4 g + q.  A: rows g and g + 8, K slots 2 q, 2 q + 1 and 2 q + 8, 2 q + 9; B: column
// g, the same slots; D: rows g and g + 8, columns 2 q, 2 q + 1.
#pragma once
#include <cstdint>

namespace hscale {

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
               "{%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 8 x 8 bf16 blocks (rows of 16 bytes) from shared memory, transposed: lane 8 u + r gives the address of row r of block u;
// lane (g, q) gets rows 2 q, 2 q + 1 of column g of each of the four.
__device__ __forceinline__ uint4 load_transposed_x4(uint32_t saddr) {
  uint4 r;
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "r"(saddr)
               : "memory");
  return r;
}

}  // namespace hscale
