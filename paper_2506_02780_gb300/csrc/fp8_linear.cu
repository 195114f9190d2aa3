// ee_fp8_linear: y = x W^T (+ bias) with x and W in e4m3, a scale for each token and 128
// columns of x and for each 128 x 128 block of W, bf16 out.
//
// Warp 0 streams 128-byte-wide tiles of x (up to 128 tokens) and W (BN rows) with TMA into a
// ring, warp 1 multiplies each k-block (128 columns, 4 MMAs of 128 x BN x 32) into one of the
// tensor memory's 512 / BN accumulators, and warps 4..11 add it, scaled, to fp32 sums in their
// registers (block_mma.cuh).  A CTA walks its tiles without a stop between them: the ring and
// the next tile's first MMAs run behind the stores, which go through shared memory (as 16-byte pieces
// of 32 rows straight from the registers they hold the next tile up for 2 us; TMA would take them behind the loads it
// has queued).
// Few tokens: the stream of W bounds the call, so it has to come from every SM.  Where there
// are fewer tiles than SMs, a cluster of up to 8 CTAs shares a tile's k-blocks and adds its
// partial sums through distributed shared memory, always in the same order.
// Many tokens: a k-block is 48 KB a CTA and 0.33 us of MMAs; loads alone run at 0.41 us (L2 to an SM about 118 GB/s),
// the whole at 0.48: 8,191 tokens x 3,584 x 28,672 646 to 690 us in a graph, 694 to 780 one call after another at the power cap
// (2.2 to 2.4 PFLOP/s).  (CTA pairs that share their MMAs load 32 KB, but hand every k-block's accumulator over between two CTAs and
// back: twice the time.)
// Rows of out that are not 16-byte aligned (N or the stride no multiple of 8) are stored by 2 bytes, which the epilogue warps pay for: 4,000
// tokens x 3,584 x 3,584 44 us, with a row of out one element longer 97.  K no multiple of 128 costs loads, for a box's rows then begin inside
// of 128-byte lines: K = 3,600 58 us.
#include <mutex>

#include "few.cuh"

namespace {

using namespace ee;

constexpr int kThreads = 384;          // warp 0 TMA, 1 MMA, 2 TMEM, 3 none; 4..11 epilogue
constexpr int kEpiWarps = 8;           // two per TMEM lane quarter, half of the columns each
constexpr int kRegsAll = 168;          // a warp's at launch; the epilogue's take some of the others', kRegsEpi
constexpr int BM = 128;

struct LinParams {
  int n, N, KB, MT, NT, ks, a_rows, stages;
  const float* xs;     // [KB][n]
  const float* ws;     // [ceil(N / 128)][KB]
  const __nv_bfloat16* bias;
  __nv_bfloat16* out;
  int64_t out_stride;
  int vec;             // rows of out are 16-byte aligned
  int32_t* err;
};

__device__ __forceinline__ void st_shared_f4(uint32_t a, float4 v) {
  asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(a)
               : "memory");
  return v;
}

constexpr uint32_t kOutBytes = 32 * 32 * 2;   // of an epilogue warp: 32 rows of 32 columns on their way out

template <int BN, bool kSplit>
__global__ void __launch_bounds__(kThreads, 1)
fp8_linear_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, const LinParams p) {
  // what spills least
  constexpr int kRegsEpi = BN < 256 ? 208 : kSplit ? 232 : 224, kRegsOther = 3 * kRegsAll - 2 * kRegsEpi;
  constexpr bool kAllPromote = BN == 256;   // (also warps that have nothing to keep)
  constexpr int kBufs = 512 / BN;               // accumulators
  constexpr int kGroups = BN / 64;              // groups of 32 columns of an epilogue warp
  constexpr int kCols = BN / 2;                 // columns of an epilogue warp
  constexpr uint32_t kWBytes = BN * kBlk;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  __shared__ __align__(8) uint64_t s_bars[2 * 16 + 2 * 4 + 1];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ int s_issued, s_consumed;

  pdl_allow_next();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int S = p.stages;
  const uint32_t aBytes = (uint32_t)p.a_rows * kBlk;
  const uint32_t aStage = (aBytes + 1023) & ~1023u;        // x rows, then W rows: an MMA's rows past a_rows are
  const uint32_t stBytes = aStage + kWBytes;               // whatever follows, and so are lanes that nobody reads
  const uint32_t ring = smem_u32(smem), out0 = ring + (uint32_t)S * stBytes;
  const uint32_t full0 = smem_u32(s_bars), empty0 = full0 + 8 * 16, tfull0 = empty0 + 8 * 16, tempty0 = tfull0 + 8 * 4,
                 drain = tempty0 + 8 * 4;
  if (threadIdx.x == 0) {
    s_abort = 0;
    s_issued = 0;
    s_consumed = 0;
    for (int s = 0; s < S; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int a = 0; a < kBufs; ++a) {
      mbar_init(tfull0 + 8 * a, 1);
      mbar_init(tempty0 + 8 * a, kEpiWarps);
    }
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmW)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmX)) : "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const int num_tiles = p.MT * p.NT;
  const int ks = kSplit ? p.ks : 1;
  const int rank = kSplit ? (int)blockIdx.x % ks : 0;
  const int first = (int)blockIdx.x / ks, step = (int)gridDim.x / ks;
  const int kb0 = p.KB * rank / ks, kb1 = p.KB * (rank + 1) / ks;   // (KB is at most 2^17)
  if (warp == 3) {                              // the first weights on their way while the kernel in front still runs
    const int n0 = first / p.MT * BN;
    if (lane < kb1 - kb0 && lane < 2 * S) prefetch_l2_box(&tmW, (kb0 + lane) * kBlk, n0);
    for (int i = 32 * lane; i < kb1 - kb0; i += 32 * 32) {
      prefetch_l2_line(p.ws + (int64_t)(n0 / kBlk) * p.KB + kb0 + i);
      if (n0 + kBlk < p.N) prefetch_l2_line(p.ws + (int64_t)(n0 / kBlk + 1) * p.KB + kb0 + i);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_wait();

  if (warp >= 4) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpi));
    const int q = warp & 3, half = (warp - 4) >> 2;
    const int r = 32 * q + lane;                              // row of the tile
    const uint32_t taddr = tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)(half * kCols);
    uint32_t it = 0;
    bool ok = true;
    for (int t = first; t < num_tiles && ok; t += step) {
      const int nt = t / p.MT, row = (t % p.MT) * BM + r;
      const int c0 = nt * BN + half * kCols;                  // this thread's first column
      const bool mine = (t % p.MT) * BM + 32 * q < p.n && c0 < p.N;     // the warp has something to keep
      const float* xs = p.xs + min(row, p.n - 1);
      const float* ws = p.ws + (int64_t)min(c0 / kBlk, (p.N - 1) / kBlk) * p.KB;   // (a warp's columns have one block)
      uint64_t acc[BN / 4];
#pragma unroll
      for (int i = 0; i < BN / 4; ++i) acc[i] = 0;
      // scales load kAhead blocks ahead (two, where there are registers: those of W come from HBM); turns of kAhead
      // blocks, for a load under way cannot move to another register
      constexpr int kAhead = BN == 256 ? 1 : 2;
      float sx[kAhead], sw[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        sx[j] = sw[j] = 0.f;
        if (kb0 + j < kb1) {
          sx[j] = xs[(int64_t)(kb0 + j) * p.n];
          sw[j] = ws[kb0 + j];
        }
      }
      for (int kb1st = kb0; kb1st < kb1 && ok; kb1st += kAhead) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int kb = kb1st + j;
          if (kb >= kb1) break;
          const float f = sx[j] * sw[j];
          if (kb + kAhead < kb1) {
            sx[j] = xs[(int64_t)(kb + kAhead) * p.n];
            sw[j] = ws[kb + kAhead];
          }
          const uint32_t buf = it % kBufs, ph = (it / kBufs) & 1;
          ++it;
          if (!__all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * buf, ph, &s_abort))) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (kAllPromote || mine) promote<kGroups>(acc, taddr + buf * BN, f);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(tempty0 + 8 * buf);
        }
      }
      if (!ok || !mine) continue;
      if constexpr (kSplit) {
        // to shared memory, 16-byte chunks permuted within a row so that a warp's 32 rows
        // spread over the banks; the ring is idle (every stage was read by an MMA that ended)
        const uint32_t base = ring + (uint32_t)r * (BN * 4);
        if (row < p.n)
#pragma unroll
          for (int i = 0; i < kCols / 4; ++i) {
            uint32_t x, y, z, w;
            f2_unpack(acc[2 * i], x, y);
            f2_unpack(acc[2 * i + 1], z, w);
            const uint32_t ch = (uint32_t)(half * (kCols / 4) + i) ^ (uint32_t)(r & 31);
            st_shared_f4(base + ch * 16, make_float4(__uint_as_float(x), __uint_as_float(y), __uint_as_float(z),
                                                     __uint_as_float(w)));
          }
        continue;
      }
      // 32 columns at a time through shared memory, so that a store is eight rows' 64 bytes
      // (addresses from values that the compiler cannot follow: it would keep them through the k-blocks, and spill)
      uint32_t ln = (uint32_t)lane, tile = (uint32_t)t;
      asm volatile("" : "+r"(ln), "+r"(tile));
      const int o0 = (int)(tile / (uint32_t)p.MT) * BN + half * kCols;
      const uint32_t buf = out0 + (uint32_t)(warp - 4) * kOutBytes;
#pragma unroll
      for (int h = 0; h < kGroups; ++h) {
        if (o0 + 32 * h >= p.N) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t lo, hi;
            f2_unpack(acc[16 * h + 4 * i + j], lo, hi);
            f[2 * j] = __uint_as_float(lo);
            f[2 * j + 1] = __uint_as_float(hi);
          }
          if (p.bias)
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] += __bfloat162float(p.bias[min(o0 + 32 * h + 8 * i + j, p.N - 1)]);
          // pieces permuted within two rows: eight rows' pieces on different banks
          st_shared_u4(buf + ln * 64 + (uint32_t)((i ^ (ln >> 1 & 3)) << 4),
                       make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])));
        }
        __syncwarp();
        const int c = o0 + 32 * h + 8 * (int)(ln & 3), left = p.N - c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int rr = 8 * i + (int)(ln >> 2), orow = (int)(tile % (uint32_t)p.MT) * BM + 32 * q + rr;
          const uint4 v = ld_shared_u4(buf + (uint32_t)rr * 64 + (uint32_t)(((int)(ln & 3) ^ (rr >> 1 & 3)) << 4));
          if (orow >= p.n) continue;
          __nv_bfloat16* o = p.out + (int64_t)orow * p.out_stride + c;
          if (p.vec && left >= 8) {
            *reinterpret_cast<uint4*>(o) = v;
          } else {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (j < left) reinterpret_cast<uint16_t*>(o)[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
          }
        }
        __syncwarp();
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 0) {
      // (the whole warp and an elected lane: the copies' operands stay in uniform registers)
      const uint32_t u_ring = __shfl_sync(0xffffffffu, ring, 0), u_full = __shfl_sync(0xffffffffu, full0, 0);
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = first; t < num_tiles && ok; t += step) {
        const int nt = t / p.MT, mt = t % p.MT;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!__all_sync(0xffffffffu, mbar_wait(empty0 + 8 * stage, phase ^ 1, &s_abort))) {
            ok = false;
            break;
          }
          if (elect_one()) {
            const uint32_t fb = u_full + 8 * stage, at = u_ring + (uint32_t)stage * stBytes;
            mbar_expect_tx(fb, aBytes + kWBytes);
            tma_load_2d(at + aStage, &tmW, fb, kb * kBlk, nt * BN);
            tma_load_2d(at, &tmX, fb, kb * kBlk, mt * BM);
          }
          __syncwarp();
          ++issued;
          if (++stage == S) {
            stage = 0;
            phase ^= 1;
          }
        }
      }
      if (lane == 0) s_issued = issued;
    } else if (warp == 1) {
      const uint32_t idesc = idesc_e4m3(BM, BN);
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      const uint64_t ad0 = smem_desc_sw128(__shfl_sync(0xffffffffu, ring, 0));
      int stage = 0, consumed = 0;
      uint32_t phase = 0, it = 0;
      bool ok = true;
      for (int t = first; t < num_tiles && ok; t += step) {
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          const uint32_t buf = it % kBufs, ph = (it / kBufs) & 1;
          if (!__all_sync(0xffffffffu, mbar_wait(tempty0 + 8 * buf, ph ^ 1, &s_abort)) ||
              !__all_sync(0xffffffffu, mbar_wait(full0 + 8 * stage, phase, &s_abort))) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (elect_one()) {
            const uint64_t ad = ad0 + (uint64_t)(stage * (stBytes >> 4));
            const uint64_t bd = ad + (uint64_t)(aStage >> 4);
#pragma unroll
            for (int k = 0; k < kBlk / 32; ++k)
              tc_mma_f8(tm + buf * BN, ad + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, k != 0 ? 1u : 0u);
            tc_commit(empty0 + 8 * stage);
            tc_commit(tfull0 + 8 * buf);
          }
          __syncwarp();
          ++consumed;
          if (++stage == S) {
            stage = 0;
            phase ^= 1;
          }
        }
      }
      if (lane == 0) s_consumed = consumed;
    }
  }

  // one code for all warps from here: as many registers as it was compiled for (a warpgroup has to
  // meet between two changes of its registers)
  __syncthreads();
  if (warp >= 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsAll));
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsAll));
  tc_fence_before();
  if constexpr (kSplit) {
    cluster_sync();
    const int nt = first / p.MT, m0 = (first % p.MT) * BM;
    const int rows = min(BM, p.n - m0), chunks = rows * (BN / 4);
    for (int i = rank * kThreads + (int)threadIdx.x; i < chunks; i += ks * kThreads) {
      const int r = i / (BN / 4), c4 = i % (BN / 4);
      const int c = nt * BN + 4 * c4;
      if (c >= p.N) continue;
      const uint32_t at = ring + (uint32_t)r * (BN * 4) + (((uint32_t)c4 ^ (uint32_t)(r & 31)) << 4);
      float4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < ks) v[k] = ld_cluster_f4(map_cluster(at, k));
      float f[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
      for (int k = 1; k < 8; ++k)
        if (k < ks) {
          f[0] += v[k].x;
          f[1] += v[k].y;
          f[2] += v[k].z;
          f[3] += v[k].w;
        }
      __nv_bfloat16* o = p.out + (int64_t)(m0 + r) * p.out_stride + c;
      if (p.bias)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c + j < p.N) f[j] += __bfloat162float(p.bias[c + j]);
      if (p.vec && c + 4 <= p.N) {
        *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c + j < p.N) o[j] = __float2bfloat16_rn(f[j]);
      }
    }
    cluster_sync();                    // nobody leaves while a peer still reads its sums
  } else {
    __syncthreads();
  }

  // ---- teardown: drain on abort, free TMEM -----------------------------------------
  if (s_abort) {
    if (threadIdx.x == 0) {
      flag_error(p.err, EE_DEVERR_TIMEOUT);
      for (int k = s_consumed; k < s_issued; ++k)
        if (!mbar_wait_plain(full0 + 8 * (k % S), (uint32_t)((k / S) & 1))) break;
    }
    if (warp == 1) {
      if (elect_one()) {   // the lane that issued the MMAs
        tc_commit(drain);
        mbar_wait_plain(drain, 0);
      }
      __syncwarp();
    }
    __syncthreads();
  }
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// Up to 8 NG tokens: a CTA takes 16 weight rows, its warps every eighth block of them.
template <int NG>
__global__ void __launch_bounds__(kFewWarps * 32, 2) fp8_linear_few_kernel(const uint8_t* x, const uint8_t* w, int K, const LinParams p) {
  constexpr int kFlight = NG == 1 ? 4 : 2;        // blocks of a warp whose loads are under way together
  constexpr int NT = 8 * NG;
  __shared__ float s_part[kFewWarps][16][NT];
  pdl_allow_next();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, tq = lane & 3;
  const int o0 = (int)blockIdx.x * 16;
  const int64_t r0 = o0 + g, r1 = r0 + 8;
  const float* ws = p.ws + (int64_t)(o0 / kBlk) * p.KB;
  float acc[NG][4];
#pragma unroll
  for (int i = 0; i < NG; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
  if (threadIdx.x == 0) prefetch_l2(w + (int64_t)o0 * K, (uint32_t)(min(16, p.N - o0) * K));   // (K is at most 2^24)
  if (threadIdx.x >= 32 && (int)threadIdx.x - 32 < (p.KB + 31) / 32) prefetch_l2_line(ws + ((int)threadIdx.x - 32) * 32);
  pdl_wait();
  for (int k0 = warp; k0 < p.KB; k0 += kFewWarps * kFlight) {
    FewFrag a[kFlight], b[kFlight], v[kFlight][NG];
    float sw[kFlight], sx[kFlight][NG][2];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const int kb = k0 + j * kFewWarps, left = K - kb * kBlk;
      const bool in = kb < p.KB;
      a[j] = few_load(w + r0 * K + (int64_t)kb * kBlk, left, tq, in && r0 < p.N);
      b[j] = few_load(w + r1 * K + (int64_t)kb * kBlk, left, tq, in && r1 < p.N);
      sw[j] = in ? ws[kb] : 0.f;
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        const int t = 8 * i + g;
        v[j][i] = few_load(x + (int64_t)t * K + (int64_t)kb * kBlk, left, tq, in && t < p.n);
#pragma unroll
        for (int d = 0; d < 2; ++d) sx[j][i][d] = in ? p.xs[(int64_t)kb * p.n + min(8 * i + 2 * tq + d, p.n - 1)] : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < kFlight; ++j)
      if (k0 + j * kFewWarps < p.KB)
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          float c[4] = {0.f, 0.f, 0.f, 0.f};
          few_block<true>(c, a[j], b[j], v[j][i]);
          const float f0 = sx[j][i][0] * sw[j], f1 = sx[j][i][1] * sw[j];
          acc[i][0] = __fmaf_rn(c[0], f0, acc[i][0]);
          acc[i][1] = __fmaf_rn(c[1], f1, acc[i][1]);
          acc[i][2] = __fmaf_rn(c[2], f0, acc[i][2]);
          acc[i][3] = __fmaf_rn(c[3], f1, acc[i][3]);
        }
  }
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    *reinterpret_cast<float2*>(&s_part[warp][g][8 * i + 2 * tq]) = make_float2(acc[i][0], acc[i][1]);
    *reinterpret_cast<float2*>(&s_part[warp][g + 8][8 * i + 2 * tq]) = make_float2(acc[i][2], acc[i][3]);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 16 * NT; e += kFewWarps * 32) {
    const int t = e >> 4, o = e & 15;
    if (t >= p.n || o0 + o >= p.N) continue;
    float f = s_part[0][o][t];
#pragma unroll
    for (int i = 1; i < kFewWarps; ++i) f += s_part[i][o][t];
    if (p.bias) f += __bfloat162float(p.bias[o0 + o]);
    p.out[(int64_t)t * p.out_stride + o0 + o] = __float2bfloat16_rn(f);
  }
}

template <int BN, bool kSplit>
ee_status launch(const uint8_t* x, const uint8_t* w, int32_t K, LinParams& p, cudaStream_t stream) {
  p.NT = (p.N + BN - 1) / BN;
  const int tiles = p.MT * p.NT;
  const size_t stage = (((size_t)p.a_rows * kBlk + 1023) & ~(size_t)1023) + (size_t)BN * kBlk;
  const size_t outs = kSplit ? 0 : kEpiWarps * kOutBytes;
  p.stages = (int)std::min<size_t>(16, ((size_t)(224 * 1024) - outs) / stage);
  const size_t smem = 1024 + p.stages * stage + outs;
  CUtensorMap tmX, tmW;
  if (!encode_u8_tmap_2d(&tmX, x, K, p.n, K, kBlk, p.a_rows) || !encode_u8_tmap_2d(&tmW, w, K, p.N, K, kBlk, BN))
    return EE_ERR_CUDA;
  {
    int dev = 0;
    const ee_status ds = current_device(&dev);
    if (ds != EE_OK) return ds;
    static std::mutex mu;
    static bool set[kMaxDevices] = {};
    std::lock_guard<std::mutex> lock(mu);
    if (!set[dev]) {
      EE_CUDA_OK(cudaFuncSetAttribute(fp8_linear_kernel<BN, kSplit>, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024));
      set[dev] = true;
    }
  }
  const int grid = kSplit ? tiles * p.ks : std::min(tiles, kNumSMs);
  EE_CUDA_OK(launch_pdl(fp8_linear_kernel<BN, kSplit>, dim3(grid), dim3(kThreads), smem, stream, (unsigned)p.ks, tmX, tmW, p));
  return EE_OK;
}

}  // namespace

extern "C" size_t ee_linear_workspace_size(void) { return ee::align_up(ee::kWorkspaceBytes, 256); }

extern "C" ee_status ee_fp8_linear(const uint8_t* x, const float* x_scale, const uint8_t* w, const float* w_scale,
                                   const ee_bf16* bias_or_null, int32_t n, int32_t K, int32_t N, ee_bf16* out,
                                   int64_t out_stride, void* ws, size_t ws_bytes, ee_stream_t stream) {
  if (n < 0 || K < 1 || N < 1) return EE_ERR_INVALID_ARG;
  if (K % 16 != 0 || K > (1 << 24) || N > (1 << 24) || n > (1 << 24)) return EE_ERR_UNSUPPORTED;
  if (n == 0) return EE_OK;
  if (!x || !x_scale || !w || !w_scale || !out || !ws || !ee::aligned(ws, 256) || !ee::aligned(x, 16) ||
      !ee::aligned(w, 16) || !ee::aligned(x_scale, 4) || !ee::aligned(w_scale, 4) || !ee::aligned(out, 2) ||
      !ee::aligned(bias_or_null, 2) || out_stride < N)
    return EE_ERR_INVALID_ARG;
  if (ws_bytes < ee_linear_workspace_size()) return EE_ERR_WORKSPACE;
  LinParams p;
  p.n = n;
  p.N = N;
  p.KB = (K + kBlk - 1) / kBlk;
  p.MT = (n + BM - 1) / BM;
  p.a_rows = std::min(BM, (n + 7) / 8 * 8);
  p.xs = x_scale;
  p.ws = w_scale;
  p.bias = reinterpret_cast<const __nv_bfloat16*>(bias_or_null);
  p.out = reinterpret_cast<__nv_bfloat16*>(out);
  p.out_stride = out_stride;
  p.vec = ee::aligned(out, 16) && out_stride % 8 == 0;
  p.err = ee::err_word(ws);
  const int64_t t128 = (int64_t)p.MT * ((N + 127) / 128), t256 = (int64_t)p.MT * ((N + 255) / 256);
  if (t256 > (1 << 30)) return EE_ERR_UNSUPPORTED;
  // Few tokens do without tiles where W is small: its call is over sooner, but its stream is slower.  (us without tiles and by
  // tiles, captured, weights from HBM, for 1, 8 and 16 tokens: 3,584 x 3,584 4.6 and 7.4, 5.1 and 8.3, 6.1 and 8.6; 14,336 x 3,584 11.7 and
  // 13.5, 12.8 and 14.1, 15.8 and 14.4; 18,944 x 3,584 14.5 and 14.7, 15.8 and 15.4; 28,672 x 3,584 20.2 and 20.3, 22.1 and 21.0, 28.3 and
  // 21.9; 76,032 x 3,584 47.6 and 42.3, 51.3 and 42.9.)
  if (n <= 16 && (int64_t)N * K < (n <= 8 ? 1 << 26 : (1 << 25) + 1)) {
    const auto kernel = n <= 8 ? fp8_linear_few_kernel<1> : fp8_linear_few_kernel<2>;
    EE_CUDA_OK(ee::launch_pdl(kernel, dim3((unsigned)((N + 15) / 16)), dim3(kFewWarps * 32), 0, (cudaStream_t)stream, 1, x, w, K, p));
    return EE_OK;
  }
  const cudaStream_t s = (cudaStream_t)stream;
  // Tiles of 128 or 256 weight rows, a tile's k-blocks split over ks CTAs.  What a call takes, in units of 0.12 us: 3 or 4
  // for a k-block (a wider tile brings x fewer times: 0.48 us for twice the 0.36), for a split
  // the way of its sums through the cluster.  (us, 28 blocks, 64 tokens: 3,584 rows as 28 tiles x 4 7.7, as 14 x 6 9.0,
  // unsplit 13.9; 10,752 rows as 42 x 3 11.6, as 84 14.4; 28,672 rows as 112 23.8, as 224 27.8.)
  const int rows = std::min(n, 128);
  int64_t best = INT64_MAX;
  bool wide = false;
  for (int ks = 1; ks <= 8; ++ks) {
    // a cluster's CTAs are on one GPC: of 5 and more fewer than the SMs would hold (18 clusters of 8 took two turns)
    if (ks == 7 || ks > p.KB) continue;
    const int64_t room = ks <= 4 ? ee::kNumSMs : ks == 5 ? 145 : 128;
    for (int w2 = 0; w2 < 2; ++w2) {
      const int64_t tiles = w2 ? t256 : t128;
      if (ks > 1 && tiles * ks > room) continue;
      const int64_t turns = ks > 1 ? 1 : (tiles + ee::kNumSMs - 1) / ee::kNumSMs;
      const int64_t cost = turns * ((p.KB + ks - 1) / ks) * (w2 ? 4 : 3) + (ks == 1 ? 0 : w2 ? 10 + rows / 7 : 4 + rows / 10);
      if (cost < best) {
        best = cost;
        p.ks = ks;
        wide = w2 != 0;
      }
    }
  }
  if (p.ks > 1) return wide ? launch<256, true>(x, w, K, p, s) : launch<128, true>(x, w, K, p, s);
  return wide ? launch<256, false>(x, w, K, p, s) : launch<128, false>(x, w, K, p, s);
}
