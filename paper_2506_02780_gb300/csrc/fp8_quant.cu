// ee_fp8_quantize, ee_fp8_quantize_weights: bf16 arrays as e4m3 codes with an fp32 scale
// for each block, 128 columns of a row (activations) or 128 x 128 (weights).
//   a = max(max |x|, 2^-100),  scale = a / 448,  code = the e4m3 number nearest to 448 x / a
// Gated: x = silu(gate) * up of the row's two halves, in fp32, so that a gated unit's
// output goes from bf16 to codes in one pass.
// Bound by HBM: 3 bytes an element (5 gated).  8,191 gated rows of 14,336: 587 MB in 94 us, 6.2 TB/s; 28,672 x 3,584
// weights: 308 MB in 46 us, 6.7 TB/s.
#include "block_mma.cuh"

namespace {

using namespace ee;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ uint32_t abs_max8(uint4 v) {   // bits of the largest of 8 bf16 magnitudes
  const uint32_t m = 0x7fff7fffu;
  const uint32_t a = __vmaxu2(__vmaxu2(v.x & m, v.y & m), __vmaxu2(v.z & m, v.w & m));
  return max(a & 0xffffu, a >> 16) << 16;   // integer order: a NaN is larger than an infinity
}
__device__ __forceinline__ void unpack8(uint4 v, float (&x)[8]) {
  x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
  x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint2 codes8(const float (&x)[8], const BlockScale& b) {
  const uint64_t hi = f2_both(b.hi), lo = f2_both(b.lo);
  float c[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint64_t v = f2_pack(__float_as_uint(x[i]), __float_as_uint(x[i + 1]));
    uint32_t c0, c1;
    f2_unpack(f2_fma(v, hi, f2_mul(v, lo)), c0, c1);
    c[i] = __uint_as_float(c0);
    c[i + 1] = __uint_as_float(c1);
  }
  return make_uint2(pack_e4m3(c[0], c[1], c[2], c[3]), pack_e4m3(c[4], c[5], c[6], c[7]));
}

// silu(g) u of 8 columns; returns the bits of the largest magnitude
template <bool kNear>
__device__ __forceinline__ uint32_t gated8(uint4 g, uint4 u, float (&h)[8]) {
  if constexpr (kNear) {
    const uint32_t sign = 0x80008000u;
    g = make_uint4(g.x ^ sign, g.y ^ sign, g.z ^ sign, g.w ^ sign);
    u = make_uint4(u.x ^ sign, u.y ^ sign, u.z ^ sign, u.w ^ sign);
  }
  float f[8], up[8];
  unpack8(g, f);
  unpack8(u, up);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint64_t g2 = f2_pack(__float_as_uint(f[i]), __float_as_uint(f[i + 1]));
    const uint64_t u2 = f2_pack(__float_as_uint(up[i]), __float_as_uint(up[i + 1]));
    uint32_t h0, h1;
    f2_unpack(kNear ? silu_near2(g2, u2) : silu_times2(g2, u2), h0, h1);
    h[i] = __uint_as_float(h0);
    h[i + 1] = __uint_as_float(h1);
    top = max(top, max(h0 & 0x7fffffffu, h1 & 0x7fffffffu));
  }
  return top;
}

struct RowParams {
  const __nv_bfloat16* x;
  int64_t x_stride;
  uint8_t* q;
  float* scale;
  int rows, cols, chunks;   // chunks of kUnroll * 256 columns a row
};

// A warp takes kUnroll steps of 256 columns (two blocks, 16 lanes each) of one row; the
// CTA's warps take the same columns of eight rows, whose scales are neighbours.  A lane works out one block's
// scale, for three divisions cost as much as eight values' codes.
template <bool kGated, int kUnroll>
__global__ void __launch_bounds__(kThreads, 4) quant_rows_kernel(const RowParams p) {
  pdl_allow_next();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunk = blockIdx.x % p.chunks;
  const int64_t row = (int64_t)(blockIdx.x / p.chunks) * kWarps + warp;
  if (row >= p.rows) return;
  pdl_wait();
  const __nv_bfloat16* x = p.x + row * p.x_stride;
  uint4 v[kUnroll], w[kGated ? kUnroll : 1];
  const int c0 = chunk * (kUnroll * 256) + lane * 8;
  float h[kGated ? kUnroll : 1][8];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int c = c0 + u * 256;
    v[u] = make_uint4(0, 0, 0, 0);
    if constexpr (kGated) w[u] = v[u];
    if (c < p.cols) {
      v[u] = *reinterpret_cast<const uint4*>(x + c);
      if constexpr (kGated) w[u] = *reinterpret_cast<const uint4*>(x + p.cols + c);
    }
  }
  uint32_t top[kUnroll], my_top = 0;               // lane u of 16: of their u-th block
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) top[u] = abs_max8(v[u]);
  if constexpr (kGated) {
    // gates are near almost always (8,191 rows of 14,336: 94 us; by silu_times2 alone 104, by expf and an ordinary division 128)
    uint32_t far = top[0];
#pragma unroll
    for (int u = 1; u < kUnroll; ++u) far = max(far, top[u]);
    if (far <= __float_as_uint(kSiluNear)) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) top[u] = gated8<true>(v[u], w[u], h[u]);
    } else {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) top[u] = gated8<false>(v[u], w[u], h[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) top[u] = max(top[u], __shfl_xor_sync(0xffffffffu, top[u], d));
    if ((lane & 15) == u) my_top = top[u];
  }
  const BlockScale mine = block_scale(__uint_as_float(my_top));
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int c = c0 + u * 256;
    BlockScale b;
    b.hi = __shfl_sync(0xffffffffu, mine.hi, (lane & 16) + u);
    b.lo = __shfl_sync(0xffffffffu, mine.lo, (lane & 16) + u);
    if constexpr (!kGated) unpack8(v[u], h[0]);
    if (c < p.cols) *reinterpret_cast<uint2*>(p.q + row * p.cols + c) = codes8(h[kGated ? u : 0], b);
  }
  const int cs = c0 + (lane & 15) * (256 - 8);     // a column of the lane's block
  if ((lane & 15) < kUnroll && cs < p.cols) p.scale[(int64_t)(cs / kBlk) * p.rows + row] = mine.scale;
}

struct BlockParams {
  const __nv_bfloat16* w;
  uint8_t* q;
  float* scale;
  int rows, cols, rb, cb;
};

// A CTA takes one block of 128 x 128, held in registers between its maximum and its codes:
// 16 lanes a row, 16 rows at once, eight times.
__global__ void __launch_bounds__(kThreads) quant_blocks_kernel(const BlockParams p) {
  __shared__ uint32_t s_top[kWarps];
  pdl_allow_next();
  pdl_wait();
  const int cbi = blockIdx.x % p.cb;
  const int64_t strip = blockIdx.x / p.cb;            // batch * row blocks
  const int64_t batch = strip / p.rb;
  const int r0 = (int)(strip % p.rb) * kBlk + (threadIdx.x >> 4);
  const int c = cbi * kBlk + (threadIdx.x & 15) * 8;
  const int64_t base = batch * (int64_t)p.rows * p.cols + c;
  uint4 v[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    v[i] = make_uint4(0, 0, 0, 0);
    if (r < p.rows && c < p.cols) v[i] = *reinterpret_cast<const uint4*>(p.w + base + (int64_t)r * p.cols);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, abs_max8(v[i]));
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
  if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWarps; ++i) top = max(top, s_top[i]);
  const BlockScale b = block_scale(__uint_as_float(top));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    float f[8];
    unpack8(v[i], f);
    if (r < p.rows && c < p.cols) *reinterpret_cast<uint2*>(p.q + base + (int64_t)r * p.cols) = codes8(f, b);
  }
  if (threadIdx.x == 0) p.scale[strip * p.cb + cbi] = b.scale;
}

}  // namespace

extern "C" ee_status ee_fp8_quantize(const ee_bf16* x, int64_t x_stride, int32_t rows, int32_t cols, int32_t gated,
                                     uint8_t* q, float* scale, ee_stream_t stream) {
  if (rows < 0 || cols < 1) return EE_ERR_INVALID_ARG;
  if (cols % 16 != 0 || cols > (1 << 24) || rows > (1 << 30)) return EE_ERR_UNSUPPORTED;
  if (rows == 0) return EE_OK;
  if (!x || !q || !scale || !ee::aligned(x, 16) || !ee::aligned(q, 16) || !ee::aligned(scale, 4))
    return EE_ERR_INVALID_ARG;
  if (x_stride % 8 != 0 || x_stride < (int64_t)cols * (gated ? 2 : 1)) return EE_ERR_INVALID_ARG;
  RowParams p;
  p.x = reinterpret_cast<const __nv_bfloat16*>(x);
  p.x_stride = x_stride;
  p.q = q;
  p.scale = scale;
  p.rows = rows;
  p.cols = cols;
  // four steps a warp where that leaves work for every SM, two where it does not (8,191 gated rows of 14,336 94 us, by
  // two steps 116; 16,384 rows of 7,168 56 and 66; 64 rows of 3,584 2.1 and 1.7)
  const int64_t row_ctas = ((int64_t)rows + kWarps - 1) / kWarps;
  const bool many = row_ctas * ((cols + 1023) / 1024) >= 2 * ee::kNumSMs;
  p.chunks = many ? (cols + 1023) / 1024 : (cols + 511) / 512;
  if (row_ctas * p.chunks > 0x7fffffff) return EE_ERR_UNSUPPORTED;
  const auto kernel = gated ? (many ? quant_rows_kernel<true, 4> : quant_rows_kernel<true, 2>)
                            : (many ? quant_rows_kernel<false, 4> : quant_rows_kernel<false, 2>);
  EE_CUDA_OK(ee::launch_pdl(kernel, dim3((unsigned)(row_ctas * p.chunks)), dim3(kThreads), 0, (cudaStream_t)stream, 1, p));
  return EE_OK;
}

extern "C" ee_status ee_fp8_quantize_weights(const ee_bf16* w, int32_t batch, int32_t rows, int32_t cols, uint8_t* q,
                                             float* scale, ee_stream_t stream) {
  if (batch < 0 || rows < 1 || cols < 1) return EE_ERR_INVALID_ARG;
  if (cols % 16 != 0 || cols > (1 << 24) || rows > (1 << 30)) return EE_ERR_UNSUPPORTED;
  if (batch == 0) return EE_OK;
  if (!w || !q || !scale || !ee::aligned(w, 16) || !ee::aligned(q, 16) || !ee::aligned(scale, 4))
    return EE_ERR_INVALID_ARG;
  BlockParams p;
  p.w = reinterpret_cast<const __nv_bfloat16*>(w);
  p.q = q;
  p.scale = scale;
  p.rows = rows;
  p.cols = cols;
  p.rb = (rows + kBlk - 1) / kBlk;
  p.cb = (cols + kBlk - 1) / kBlk;
  const int64_t per = (int64_t)p.rb * p.cb;
  if (per > 0x7fffffff || per * batch > 0x7fffffff) return EE_ERR_UNSUPPORTED;
  EE_CUDA_OK(ee::launch_pdl(quant_blocks_kernel, dim3((unsigned)(per * batch)), dim3(kThreads), 0,
                            (cudaStream_t)stream, 1, p));
  return EE_OK;
}
