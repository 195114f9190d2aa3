// ee_moe_layer for up to 8 tokens, after the router (moe_route.cu): one persistent kernel of which two CTAs
// share an SM.  A CTA draws units from a queue:
//   gate unit    8 columns of h of one expert: a warp's MMAs take its 8 gate rows and its 8 up rows, so that a
//                lane holds both halves of silu(g) u
//   down unit    16 columns of out, over all chosen experts: their sums are weighted on the way, and no y is stored
// and its warps share the unit's 128-byte blocks (few.cuh).  Between the two lies one wait for the gate
// units of the other CTAs, all of which are running; then every CTA brings h into its own shared
// memory, as e4m3 codes for 8-bit weights.
#include <mutex>

#include "moe.cuh"

namespace {

using namespace ee;

constexpr int kThreads = kFewWarps * 32;
constexpr int kFlight = 4;             // blocks of a warp whose loads are under way together
constexpr int kMaxActive = 128;        // experts: 8 tokens of 16 at most
constexpr size_t kMostSmem = 100 * 1024;

__host__ __device__ constexpr int h_stride(int KB2) { return KB2 * 128 + 64; }   // rows two by two on different banks

template <bool kFp8>
__global__ void __launch_bounds__(kThreads, 2) moe_few_kernel(const MoeParams p) {
  constexpr int es = kFp8 ? 1 : 2;
  extern __shared__ __align__(16) uint8_t s_h[];               // [entries] rows of h, then their blocks' scales
  __shared__ float s_part[2][kFewWarps][16][kFewTokens];
  __shared__ float s_p[kMaxActive][kFewTokens];                // an active expert's weight for a token
  __shared__ int16_t s_map[kMaxActive][kFewTokens];            // ... and the entry, or -1
  __shared__ int16_t s_exp[kMaxActive];
  __shared__ int s_unit[2];
  __shared__ int s_ok;
  pdl_allow_next();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, tq = lane & 3;
  pdl_wait();
  const int live = p.live ? max(0, min(p.T, ld_pinned(p.live))) : p.T;
  const int na = (int)p.ctl->tiles;                            // an active expert has one tile
  if (threadIdx.x == 0) s_unit[0] = (int)atomicAdd(&p.ctl->queue, 1u);
  for (int i = threadIdx.x; i < na * kFewTokens; i += kThreads) s_map[i / kFewTokens][i % kFewTokens] = -1;
  __syncthreads();
  if ((int)threadIdx.x < na) {
    const MoeTile e = p.tile[threadIdx.x];
    s_exp[threadIdx.x] = (int16_t)e.expert;
    for (int i = 0; i < e.count; ++i) {
      const int t = p.list[e.entry0 + i];
      s_map[threadIdx.x][t] = (int16_t)(e.entry0 + i);
      s_p[threadIdx.x][t] = p.pe[e.entry0 + i];
    }
  }
  __syncthreads();
  const int per = p.I / 8, gates = na * per, downs = na ? (p.H + 15) / 16 : 0;
  const uint8_t* const w1 = static_cast<const uint8_t*>(p.w1);
  const uint8_t* const w2 = static_cast<const uint8_t*>(p.w2);
  const uint8_t* const x = static_cast<const uint8_t*>(p.x) + (size_t)g * p.x_stride * es;
  const int h_bytes = p.H * es, i_bytes = p.I * es;
  const int t0 = min(2 * tq, p.T - 1), t1 = min(2 * tq + 1, p.T - 1);

  int u = s_unit[0], turn = 0;
  for (; u < gates; turn ^= 1) {
    int next = 0;
    if (threadIdx.x == 0) next = (int)atomicAdd(&p.ctl->queue, 1u);
    const int a = u / per, i8 = u % per, e = s_exp[a];
    const uint8_t* const r0 = w1 + ((size_t)e * 2 * p.I + i8 * 8 + g) * h_bytes;
    const uint8_t* const r1 = r0 + (size_t)p.I * h_bytes;
    const float* const ws0 = kFp8 ? p.s1 + ((size_t)e * 2 * p.IB + i8 * 8 / kBlk) * p.KB1 : nullptr;
    const float* const ws1 = kFp8 ? ws0 + (size_t)p.IB * p.KB1 : nullptr;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = warp; k0 < p.KB1; k0 += kFewWarps * kFlight) {
      FewFrag fa[kFlight], fb[kFlight], fx[kFlight];
      float s[kFlight][4];
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int kb = k0 + j * kFewWarps, left = h_bytes - kb * 128;
        const bool in = kb < p.KB1;
        fa[j] = few_load(r0 + (size_t)kb * 128, left, tq, in);
        fb[j] = few_load(r1 + (size_t)kb * 128, left, tq, in);
        fx[j] = few_load(x + (size_t)kb * 128, left, tq, in && g < live);
        if constexpr (kFp8) {
          s[j][0] = in ? p.xs[(size_t)kb * p.T + t0] : 0.f;
          s[j][1] = in ? p.xs[(size_t)kb * p.T + t1] : 0.f;
          s[j][2] = in ? ws0[kb] : 0.f;
          s[j][3] = in ? ws1[kb] : 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < kFlight; ++j)
        if (k0 + j * kFewWarps < p.KB1) {
          if constexpr (kFp8) {
            float c[4] = {0.f, 0.f, 0.f, 0.f};
            few_block<true>(c, fa[j], fb[j], fx[j]);
            acc[0] = __fmaf_rn(c[0], s[j][0] * s[j][2], acc[0]);
            acc[1] = __fmaf_rn(c[1], s[j][1] * s[j][2], acc[1]);
            acc[2] = __fmaf_rn(c[2], s[j][0] * s[j][3], acc[2]);
            acc[3] = __fmaf_rn(c[3], s[j][1] * s[j][3], acc[3]);
          } else {
            few_block<false>(acc, fa[j], fb[j], fx[j]);
          }
        }
    }
    *reinterpret_cast<float2*>(&s_part[turn][warp][g][2 * tq]) = make_float2(acc[0], acc[1]);
    *reinterpret_cast<float2*>(&s_part[turn][warp][g + 8][2 * tq]) = make_float2(acc[2], acc[3]);
    if (threadIdx.x == 0) s_unit[turn ^ 1] = next;
    __syncthreads();
    u = s_unit[turn ^ 1];
    if (warp < 2) {                                            // token t, column o; the others go on
      const int t = threadIdx.x >> 3, o = threadIdx.x & 7;
      const int entry = s_map[a][t];
      if (entry >= 0) {
        float gs = s_part[turn][0][o][t], us = s_part[turn][0][o + 8][t];
#pragma unroll
        for (int i = 1; i < kFewWarps; ++i) {
          gs += s_part[turn][i][o][t];
          us += s_part[turn][i][o + 8][t];
        }
        const float h = silu_times(gs, us);
        const size_t at = (size_t)entry * p.I + i8 * 8 + o;
        if constexpr (kFp8) __stcg(p.hf + at, h);
        else static_cast<__nv_bfloat16*>(p.h)[at] = __float2bfloat16_rn(h);
      }
      asm volatile("bar.sync 1, 64;" ::: "memory");
      if (threadIdx.x == 0) red_inc_release(&p.ctl->down_done, 0xffffffffu);
    }
  }
  if (u - gates >= downs) return;

  // ---- h, once it is there ------------------------------------------------------------
  if (threadIdx.x == 0) s_ok = wait_count_geq(&p.ctl->down_done, (uint32_t)gates);
  __syncthreads();
  if (!s_ok) {
    if (threadIdx.x == 0) flag_error(p.err, EE_DEVERR_TIMEOUT);
    return;
  }
  const int n = live * p.k, hs = h_stride(p.KB2);
  float* const s_hs = reinterpret_cast<float*>(s_h + (size_t)p.n * hs);   // [entries][IB]
  if constexpr (kFp8) {
    for (int i0 = warp; i0 < n * p.IB; i0 += kFewWarps * 8) {  // a block a warp, eight loads in flight
      float4 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = i0 + j * kFewWarps, m = i / p.IB, col = i % p.IB * kBlk + 4 * lane;
        v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < n * p.IB && col < p.I) v[j] = __ldcg(reinterpret_cast<const float4*>(p.hf + (size_t)m * p.I + col));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = i0 + j * kFewWarps, m = i / p.IB, b = i % p.IB;
        if (i >= n * p.IB) continue;
        const uint32_t k = 0x7fffffffu;
        const uint32_t top = __reduce_max_sync(0xffffffffu, max(max(__float_as_uint(v[j].x) & k, __float_as_uint(v[j].y) & k),
                                                                max(__float_as_uint(v[j].z) & k, __float_as_uint(v[j].w) & k)));
        const BlockScale s = block_scale(__uint_as_float(top));
        *reinterpret_cast<uint32_t*>(s_h + (size_t)m * hs + b * kBlk + 4 * lane) =
            pack_e4m3(to_code(v[j].x, s), to_code(v[j].y, s), to_code(v[j].z, s), to_code(v[j].w, s));
        if (lane == 0) s_hs[m * p.IB + b] = s.scale;
      }
    }
  } else {
    const int chunks = p.KB2 * 8;                              // 16 bytes
    for (int i0 = threadIdx.x; i0 < n * chunks; i0 += kThreads * 4) {
      uint4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = i0 + j * kThreads, m = i / chunks, c = i % chunks * 16;
        v[j] = make_uint4(0, 0, 0, 0);
        if (i < n * chunks && c < i_bytes)
          v[j] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.h) + (size_t)m * i_bytes + c));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = i0 + j * kThreads;
        if (i < n * chunks) *reinterpret_cast<uint4*>(s_h + (size_t)(i / chunks) * hs + i % chunks * 16) = v[j];
      }
    }
  }
  __syncthreads();

  for (int d = u - gates; d < downs; turn ^= 1) {
    int next = 0;
    if (threadIdx.x == 0) next = (int)atomicAdd(&p.ctl->queue, 1u);
    const int o0 = d * 16, items = na * p.KB2;
    const bool in0 = o0 + g < p.H, in1 = o0 + g + 8 < p.H;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = warp; k0 < items; k0 += kFewWarps * kFlight) {
      FewFrag fa[kFlight], fb[kFlight];
      float s[kFlight];
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int i = k0 + j * kFewWarps, a = i < items ? i / p.KB2 : 0, kb = i - a * p.KB2, left = i_bytes - kb * 128;
        const int e = s_exp[a];
        const uint8_t* const r0 = w2 + ((size_t)e * p.H + o0 + g) * i_bytes + (size_t)kb * 128;
        fa[j] = few_load(r0, left, tq, i < items && in0);
        fb[j] = few_load(r0 + (size_t)8 * i_bytes, left, tq, i < items && in1);
        if constexpr (kFp8) s[j] = i < items ? p.s2[((size_t)e * p.HB + o0 / kBlk) * p.KB2 + kb] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int i = k0 + j * kFewWarps;
        if (i >= items) break;
        const int a = i / p.KB2, kb = i - a * p.KB2;
        const int m = s_map[a][g], m0 = s_map[a][2 * tq], m1 = s_map[a][2 * tq + 1];
        FewFrag fx;
        fx.lo = fx.hi = make_uint4(0, 0, 0, 0);
        if (m >= 0) {
          const uint8_t* const r = s_h + (size_t)m * hs + kb * 128 + tq * 16;
          fx.lo = *reinterpret_cast<const uint4*>(r);
          fx.hi = *reinterpret_cast<const uint4*>(r + 64);
        }
        float c[4] = {0.f, 0.f, 0.f, 0.f};
        few_block<kFp8>(c, fa[j], fb[j], fx);
        if (m0 >= 0) {                                         // (a token at other experts takes nothing, not even a NaN)
          const float f = kFp8 ? s_p[a][2 * tq] * (s_hs[m0 * p.IB + kb] * s[j]) : s_p[a][2 * tq];
          acc[0] = __fmaf_rn(c[0], f, acc[0]);
          acc[2] = __fmaf_rn(c[2], f, acc[2]);
        }
        if (m1 >= 0) {
          const float f = kFp8 ? s_p[a][2 * tq + 1] * (s_hs[m1 * p.IB + kb] * s[j]) : s_p[a][2 * tq + 1];
          acc[1] = __fmaf_rn(c[1], f, acc[1]);
          acc[3] = __fmaf_rn(c[3], f, acc[3]);
        }
      }
    }
    *reinterpret_cast<float2*>(&s_part[turn][warp][g][2 * tq]) = make_float2(acc[0], acc[1]);
    *reinterpret_cast<float2*>(&s_part[turn][warp][g + 8][2 * tq]) = make_float2(acc[2], acc[3]);
    if (threadIdx.x == 0) s_unit[turn ^ 1] = next;
    __syncthreads();
    const int t = threadIdx.x >> 4, o = threadIdx.x & 15;
    if (t < live && o0 + o < p.H) {                            // (live is at most 8)
      float f = s_part[turn][0][o][t];
#pragma unroll
      for (int i = 1; i < kFewWarps; ++i) f += s_part[turn][i][o][t];
      p.out[(int64_t)t * p.out_stride + o0 + o] = __float2bfloat16_rn(f);
    }
    d = s_unit[turn ^ 1] - gates;
  }
}

template <bool kFp8>
ee_status launch(const MoeParams& p, size_t smem, cudaStream_t stream) {
  {
    int dev = 0;
    const ee_status ds = current_device(&dev);
    if (ds != EE_OK) return ds;
    static std::mutex mu;
    static bool set[kMaxDevices] = {};
    std::lock_guard<std::mutex> lock(mu);
    if (!set[dev]) {
      EE_CUDA_OK(cudaFuncSetAttribute(moe_few_kernel<kFp8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem));
      set[dev] = true;
    }
  }
  EE_CUDA_OK(launch_pdl(moe_few_kernel<kFp8>, dim3(2 * kNumSMs), dim3(kThreads), smem, stream, 1, p));
  return EE_OK;
}

}  // namespace

namespace ee {

size_t moe_few_smem(int T, int I, int k, bool fp8) {
  if (T > kFewTokens) return 0;
  const int IB = (I + kBlk - 1) / kBlk, KB2 = (I * (fp8 ? 1 : 2) + 127) / 128;
  const size_t bytes = (size_t)T * k * ((size_t)h_stride(KB2) + 4 * (size_t)IB);
  return bytes <= kMostSmem ? bytes : 0;
}

ee_status launch_moe_few(const MoeParams& p, bool fp8, cudaStream_t stream) {
  const size_t smem = moe_few_smem(p.T, p.I, p.k, fp8);
  return fp8 ? launch<true>(p, smem, stream) : launch<false>(p, smem, stream);
}

}  // namespace ee
