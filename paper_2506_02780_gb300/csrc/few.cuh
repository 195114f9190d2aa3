// Weight products for a few tokens (up to 8 an MMA, 16 in ee_fp8_linear): a warp takes 16 weight rows
// and some of their 128-byte blocks, straight from global memory into the fragments of an m16n8 MMA (weights the
// 16 side, tokens the 8 side).  So few tokens leave nothing to share between warps but the
// sums, and without rings, tensor memory and barriers a call costs little more than its one wait for memory.
//
// A lane holds, of a 128-byte block of rows g and g + 8 (g = lane / 4) and of token g, the 16 bytes
// at 16 (lane % 4) and those at 64 + 16 (lane % 4).  Which column of the block stands at which place of an
// MMA's inner dimension is free as long as weights and tokens agree, so the four 32-bit words of such a piece
// serve as the k-pairs of two MMAs.  Internal header.
#pragma once
#include "block_mma.cuh"

namespace ee {

constexpr int kFewWarps = 8;           // warps that share the blocks of 16 rows

struct FewFrag {
  uint4 lo, hi;
};
// the lane's pieces of a block of `left` bytes from here; zeros where `in` is false or the row has ended
__device__ __forceinline__ FewFrag few_load(const uint8_t* block, int left, int tq, bool in) {
  FewFrag f;
  f.lo = f.hi = make_uint4(0, 0, 0, 0);
  if (in && tq * 16 < left) f.lo = *reinterpret_cast<const uint4*>(block + tq * 16);
  if (in && tq * 16 + 64 < left) f.hi = *reinterpret_cast<const uint4*>(block + tq * 16 + 64);
  return f;
}
template <bool kFp8>
__device__ __forceinline__ void few_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  if constexpr (kFp8)
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, "
        "%2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, "
        "%2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// c += the block's product: c[0], c[1] of row g and tokens 2 tq, 2 tq + 1, c[2], c[3] of row g + 8
template <bool kFp8>
__device__ __forceinline__ void few_block(float (&c)[4], const FewFrag& r0, const FewFrag& r1, const FewFrag& x) {
  few_mma<kFp8>(c, r0.lo.x, r1.lo.x, r0.lo.y, r1.lo.y, x.lo.x, x.lo.y);
  few_mma<kFp8>(c, r0.lo.z, r1.lo.z, r0.lo.w, r1.lo.w, x.lo.z, x.lo.w);
  few_mma<kFp8>(c, r0.hi.x, r1.hi.x, r0.hi.y, r1.hi.y, x.hi.x, x.hi.y);
  few_mma<kFp8>(c, r0.hi.z, r1.hi.z, r0.hi.w, r1.hi.w, x.hi.z, x.hi.w);
}

}  // namespace ee
