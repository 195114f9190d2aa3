// What the weight products of a pass share (ee_fp8_linear, ee_moe_layer):
// 8-bit MMAs, the promotion of one block's product into fp32 registers, and the
// quantisation of a block.  Internal header.
//
// A product with a scale for each block of 128 along K cannot stay in the
// tensor cores' accumulator: y = sum_b s_b (x_b . w_b).  Each block's product
// goes to tensor memory by itself (two to eight accumulators in turn) and the epilogue
// warps add it, scaled, to sums of their own in registers.  With tokens as the MMA's
// M side (one tensor-memory lane, one thread) a block's scale is one number a
// thread and 128 columns; tiles of few tokens have it the other way round (moe_experts.cu).
#pragma once
#include "ee_common.cuh"
#include "ee_ptx.cuh"

namespace ee {

constexpr int kBlk = 128;              // columns (and weight rows) that share a scale
constexpr float kE4m3Max = 448.f;
constexpr float kLeastMax = 0x1p-100f;   // a block's maximum counts as at least this

// dims[0] bytes are contiguous; 128-byte swizzle, zero fill out of bounds
bool encode_u8_tmap_2d(CUtensorMap* map, const void* base, uint64_t cols, uint64_t rows, uint64_t stride_bytes,
                       uint32_t box_cols, uint32_t box_rows);
// the same in 4-byte elements without a swizzle: rows of a box lie behind one another
bool encode_u32_tmap_2d(CUtensorMap* map, const void* base, uint64_t cols, uint64_t rows, uint64_t stride_bytes,
                        uint32_t box_cols, uint32_t box_rows);

// Instruction descriptor of kind::f8f6f4: e4m3 A and B, fp32 D, both K-major.
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void tc_mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                          uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// acc[16 g .. 16 g + 15] (pairs) += s * 32 columns that a load left in r
template <int G, int N>
__device__ __forceinline__ void add_scaled32(uint64_t (&acc)[N], uint32_t (&r)[32], uint64_t s) {
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[G * 16 + i] = f2_fma(f2_pack(r[2 * i], r[2 * i + 1]), s, acc[G * 16 + i]);
}

// acc += f * the 64 or 128 columns (G groups of 32) from c on of this warp's lanes; the loads of the
// second 64 run behind the sums of the first
template <int G>
__device__ __forceinline__ void promote(uint64_t (&acc)[16 * G], uint32_t c, float f) {
  uint32_t a[32], b[32];
  tc_ld32_nowait(c, a);
  tc_ld32_nowait(c + 32, b);
  const uint64_t p = f2_pack(__float_as_uint(f), __float_as_uint(f));
  tc_wait_ld32(a);
  tc_pin32(b);
  add_scaled32<0>(acc, a, p);
  if constexpr (G == 4) tc_ld32_nowait(c + 64, a);
  add_scaled32<1>(acc, b, p);
  if constexpr (G == 4) {
    tc_ld32_nowait(c + 96, b);
    tc_wait_ld32(a);
    tc_pin32(b);
    add_scaled32<2>(acc, a, p);
    add_scaled32<3>(acc, b, p);
  }
}

// acc += f0 * the 64 columns at c0 and f1 * the 64 at c1
__device__ __forceinline__ void promote_2x64(uint64_t (&acc)[64], uint32_t c0, uint32_t c1, float f0, float f1) {
  uint32_t a[32], b[32];
  tc_ld32_nowait(c0, a);
  tc_ld32_nowait(c0 + 32, b);
  const uint64_t p0 = f2_pack(__float_as_uint(f0), __float_as_uint(f0)), p1 = f2_pack(__float_as_uint(f1), __float_as_uint(f1));
  tc_wait_ld32(a);
  tc_pin32(b);
  add_scaled32<0>(acc, a, p0);
  tc_ld32_nowait(c1, a);
  add_scaled32<1>(acc, b, p0);
  tc_ld32_nowait(c1 + 32, b);
  tc_wait_ld32(a);
  tc_pin32(b);
  add_scaled32<2>(acc, a, p1);
  add_scaled32<3>(acc, b, p1);
}

// The code of x in a block whose largest magnitude is a: the e4m3 number nearest to 448 x / a.
// The quotient is x (hi + lo) with hi + lo = 448 / a to about 48 bits, rounded once to fp32: for a
// bf16 x it is then never on the wrong side of a border between two codes (448 x / a is either a
// border itself, which fp32 holds, or at least 2^-13 of it away), so codes do not depend on how a
// program divides.  A block with an infinity or a NaN has NaN codes throughout.
struct BlockScale {
  float hi, lo, scale;
};
__device__ __forceinline__ BlockScale block_scale(float a) {
  BlockScale b;
  a = a < kLeastMax ? kLeastMax : a;   // (a NaN stays)
  b.hi = __fdiv_rn(kE4m3Max, a);
  b.lo = __fdiv_rn(__fmaf_rn(-b.hi, a, kE4m3Max), a);
  b.scale = __fdiv_rn(a, kE4m3Max);
  return b;
}
__device__ __forceinline__ float to_code(float x, const BlockScale& b) {
  return __fmaf_rn(x, b.hi, __fmul_rn(x, b.lo));
}
__device__ __forceinline__ uint32_t pack_e4m3(float x0, float x1, float x2, float x3) {
  uint32_t d;
  asm("{\n .reg .b16 l, h;\n cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n"
      " mov.b32 %0, {l, h};\n}\n"
      : "=r"(d)
      : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
  return d;
}
// silu(g) u = g u / (1 + e^-g) for two pairs.  An exponent y = x / ln 2 is rounded, which puts 2^y off by more the larger x is; what it
// is off by is put back: e^x = 2^y (1 + c), c = x - y ln 2 with ln 2 in two parts (Cody and Waite).  Errors are counted in 2^-24; ex2.approx's is 4 (2
// units in the last place), rcp.approx's 2.
__device__ __forceinline__ uint64_t f2_both(float f) { return f2_pack(__float_as_uint(f), __float_as_uint(f)); }
__device__ __forceinline__ uint64_t f2_rcp(uint64_t v) {
  uint32_t a, b;
  f2_unpack(v, a, b);
  asm("rcp.approx.ftz.f32 %0, %0;" : "+r"(a));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+r"(b));
  return f2_pack(a, b);
}
// e^x where y is x / ln 2, rounded
__device__ __forceinline__ uint64_t f2_exp(uint64_t x, uint64_t y) {
  uint32_t a, b;
  f2_unpack(y, a, b);
  asm("ex2.approx.ftz.f32 %0, %0;" : "+r"(a));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+r"(b));
  const uint64_t e = f2_pack(a, b), c = f2_fma(y, f2_both(1.90465421e-9f), f2_fma(y, f2_both(-0.693147182f), x));
  return f2_fma(e, c, e);
}
// For |g| <= 80, from -g and -u: errors e^-g 5, 1 + e^-g at most 6, its reciprocal 2, products 2; together 10.
constexpr float kSiluNear = 80.f;
__device__ __forceinline__ uint64_t silu_near2(uint64_t ng, uint64_t nu) {
  const uint64_t e = f2_exp(ng, f2_mul(ng, f2_both(1.44269502f)));
  return f2_mul(f2_mul(ng, f2_rcp(f2_add(e, f2_both(1.f)))), nu);
}
// For every g, with m = e^(-|g| / 2):   g < 0:  (g m) (u m) / (1 + m^2),   else  g u / (1 + m^2),   in which neither e^-g nor a divisor
// above 2 occurs, so that a far gate of a large u keeps its digits.  Errors: m 5, twice in the result, 1 + m^2 at most 6, its reciprocal 2,
// products 4; together 22.  Below g = -174 m is 0, off by less than 1e-35.
__device__ __forceinline__ uint64_t silu_times2(uint64_t g, uint64_t u) {
  uint32_t g0, g1, m0, m1;
  f2_unpack(g, g0, g1);
  // (no further than 2^8: an infinite g would make c a NaN)
  const uint64_t a = f2_pack(__float_as_uint(fminf(fabsf(__uint_as_float(g0)), 256.f)),
                             __float_as_uint(fminf(fabsf(__uint_as_float(g1)), 256.f)));
  uint64_t m = f2_exp(f2_mul(a, f2_both(-0.5f)), f2_mul(a, f2_both(-0.72134751f)));
  const uint64_t r = f2_rcp(f2_fma(m, m, f2_both(1.f)));
  f2_unpack(m, m0, m1);
  m = f2_pack((int)g0 < 0 ? m0 : 0x3f800000u, (int)g1 < 0 ? m1 : 0x3f800000u);
  return f2_mul(f2_mul(f2_mul(g, m), r), f2_mul(u, m));
}
__device__ __forceinline__ float silu_times(float g, float u) {
  uint32_t lo, hi;
  f2_unpack(silu_times2(f2_pack(__float_as_uint(g), __float_as_uint(g)), f2_pack(__float_as_uint(u), __float_as_uint(u))), lo, hi);
  return __uint_as_float(lo);
}

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

__device__ __forceinline__ void st_shared_u4(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared_u4(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}

}  // namespace ee
