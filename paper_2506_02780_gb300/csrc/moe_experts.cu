// ee_moe_layer: a mixture-of-experts layer for the few tokens of a pass.  After the router (moe_route.cu)
// one persistent kernel runs the chosen experts:
//   gate tasks   h = silu(x Wg^T) * (x Wu^T)   128 columns of h for one token tile
//   down tasks   y = h Wd^T                    256 columns of y
//   the sum      out[t] = sum_j p[t][j] y[entry of t's j-th expert]
// The experts' weights are read once and bound the call; tokens are the MMA's M side, so that a
// few of them cost no more than 128 (block_mma.cuh).
//
// CTAs draw tasks from one queue, gate tasks first.  A down task waits for the gate tasks of its
// token tile; those were drawn before it by CTAs that are running, so no wait depends on
// a CTA that has not started.  Warp 0 draws, publishes the task to the other roles in a ring of
// shared memory and streams the operands (x's rows gathered by TMA); it runs ahead of the others across tasks, so
// that the stream does not stop between them.
#include <mutex>

#include "moe.cuh"

namespace {

using namespace ee;

constexpr int kThreads = 384;          // warp 0 tasks and TMA, 1 MMA, 2 TMEM, 3 none; 4..11 epilogue
constexpr int kEpiWarps = 8;           // two per TMEM lane quarter, half of the columns each
constexpr int kRegsAll = 168, kRegsEpi = 216, kRegsOther = 72;   // 256 * 216 + 128 * 72 = 384 * 168
constexpr int BN = 256, kHalf = 128;   // weight rows of a task: 128 of gate and up each, or 256 of down
constexpr int kBufs = 512 / BN;
constexpr int kRing = 4;               // tasks published and not yet taken by every role

struct MoeParams {
  int T, H, I, E, k, n;                // n = T k
  int KB1, KB2;                        // 128-byte blocks along H and I
  int IB, HT, HB;                      // gate tasks, down tasks of a token tile; scale blocks along H
  int a_rows, stages;
  MoeCtl* ctl;
  const MoeTile* tile;
  const int32_t* list;
  const int32_t* inv;
  const float* prob;
  const float* xs;                     // [blocks of H][T]
  const float* s1;                     // [E][2][IB][blocks of H]
  const float* s2;                     // [E][HB][blocks of I]
  void* h;                             // [n][I] codes or bf16
  float* hs;                           // [IB][n]
  float* y;                            // [n][H]
  __nv_bfloat16* out;
  int64_t out_stride;
  int vec;                             // rows of out are 8-byte aligned
  const int32_t* live;
  int32_t* err;
};

enum { kGate = 0, kDown = 1, kEnd = 2 };
struct Task {
  int kind, blk, expert, tile, entry, rows;   // column block; token tile, its first entry and their number
};

template <bool kFp8>
__global__ void __launch_bounds__(kThreads, 1)
moe_experts_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW1,
                   const __grid_constant__ CUtensorMap tmH, const __grid_constant__ CUtensorMap tmW2, const MoeParams p) {
  constexpr int kCols = kFp8 ? 128 : 64;        // elements in 128 bytes
  constexpr uint32_t kBoxBytes = 128 * 128;     // 128 weight rows
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  __shared__ __align__(8) uint64_t s_bars[2 * 8 + 2 * kBufs + 2 * kRing + 4 + 1];
  __shared__ Task s_task[kRing];
  __shared__ uint32_t s_top[2][2][128];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ int s_issued, s_consumed;

  pdl_allow_next();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int S = p.stages;
  const uint32_t aStage = ((uint32_t)p.a_rows * 128 + 1023) & ~1023u;
  const uint32_t stBytes = aStage + 2 * kBoxBytes;
  const uint32_t ring = smem_u32(smem);
  const uint32_t full0 = smem_u32(s_bars), empty0 = full0 + 8 * 8, tfull0 = empty0 + 8 * 8, tempty0 = tfull0 + 8 * kBufs,
                 qfull0 = tempty0 + 8 * kBufs, qempty0 = qfull0 + 8 * kRing, pair0 = qempty0 + 8 * kRing, drain = pair0 + 8 * 4;
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
    for (int a = 0; a < kRing; ++a) {
      mbar_init(qfull0 + 8 * a, 1);
      mbar_init(qempty0 + 8 * a, 1 + kEpiWarps);
    }
    for (int a = 0; a < 4; ++a) mbar_init(pair0 + 8 * a, 2);
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmX)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmW1)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmH)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmW2)) : "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
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
    const uint32_t tq = tmem + ((uint32_t)(32 * q) << 16);
    uint32_t it = 0, pairs = 0;                               // accumulators taken, meetings with the neighbour
    for (uint32_t nt = 0;; ++nt) {
      const uint32_t slot = nt % kRing;
      if (!__all_sync(0xffffffffu, mbar_wait(qfull0 + 8 * slot, (nt / kRing) & 1, &s_abort))) break;
      const Task t = s_task[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(qempty0 + 8 * slot);
      if (t.kind == kEnd) break;
      const bool gate = t.kind == kGate;
      const bool mine = 32 * q < t.rows;                      // the warp has something to keep
      const int entry = t.entry + min(r, t.rows - 1);
      // accumulator columns of this warp: 64 of gate and 64 of up, or 128 of down
      const uint32_t c0 = gate ? half * 64 : half * 128, c1 = gate ? 128 + half * 64 : half * 128 + 64;
      uint64_t acc[64];
      if constexpr (kFp8) {
        const int KB = gate ? p.KB1 : p.KB2;
        const int hb = min(t.blk * 2 + half, p.HB - 1);
        const float* ws0 = gate ? p.s1 + ((int64_t)(2 * t.expert) * p.IB + t.blk) * KB : p.s2 + ((int64_t)t.expert * p.HB + hb) * KB;
        const float* ws1 = gate ? ws0 + (int64_t)p.IB * KB : ws0;
        const int xstep = gate ? p.T : p.n;
        const float* xs = gate ? p.xs + p.list[entry] : p.hs + entry;
#pragma unroll
        for (int i = 0; i < 64; ++i) acc[i] = 0;
        bool ok = true;
        float sx = __ldcg(xs), sw0 = ws0[0], sw1 = ws1[0];
        for (int kb = 0; kb < KB; ++kb, ++it) {
          const uint32_t buf = it % kBufs, ph = (it / kBufs) & 1;
          const float f0 = sx * sw0, f1 = sx * sw1;
          if (kb + 1 < KB) {                                  // the next block's scales load behind this one
            sx = __ldcg(xs + (int64_t)(kb + 1) * xstep);
            sw0 = ws0[kb + 1];
            sw1 = ws1[kb + 1];
          }
          if (!__all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * buf, ph, &s_abort))) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (mine) promote_2x64(acc, tq + buf * BN + c0, tq + buf * BN + c1, f0, f1);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(tempty0 + 8 * buf);
        }
        if (!ok) break;
      } else {
        const uint32_t buf = it % kBufs, ph = (it / kBufs) & 1;
        ++it;
        if (!__all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * buf, ph, &s_abort))) break;
        tc_fence_after();
        if (mine) {
          uint32_t a[32], b[32];
          const uint32_t at0 = tq + buf * BN + c0, at1 = tq + buf * BN + c1;
          tc_ld32_nowait(at0, a);
          tc_ld32_nowait(at0 + 32, b);
          tc_wait_ld32(a);
          tc_pin32(b);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            acc[i] = f2_pack(a[2 * i], a[2 * i + 1]);
            acc[16 + i] = f2_pack(b[2 * i], b[2 * i + 1]);
          }
          tc_ld32_nowait(at1, a);
          tc_ld32_nowait(at1 + 32, b);
          tc_wait_ld32(a);
          tc_pin32(b);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            acc[32 + i] = f2_pack(a[2 * i], a[2 * i + 1]);
            acc[48 + i] = f2_pack(b[2 * i], b[2 * i + 1]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty0 + 8 * buf);
      }
      if (!mine) continue;
      if (gate) {
        const int i0 = t.blk * 128 + half * 64;               // first of 64 columns of h
        float h[64];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          uint32_t g0, g1, u0, u1;
          f2_unpack(acc[i], g0, g1);
          f2_unpack(acc[32 + i], u0, u1);
          h[2 * i] = silu_times(__uint_as_float(g0), __uint_as_float(u0));
          h[2 * i + 1] = silu_times(__uint_as_float(g1), __uint_as_float(u1));
        }
        if constexpr (kFp8) {
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (i0 + i < p.I) top = max(top, __float_as_uint(h[i]) & 0x7fffffffu);
          // the block's other 64 columns are the neighbour warp's; two places in turn, so that one meeting
          // a task is enough
          s_top[pairs & 1][half][r] = top;
          __syncwarp();
          if (lane == 0) mbar_arrive(pair0 + 8 * q);
          if (!__all_sync(0xffffffffu, mbar_wait(pair0 + 8 * q, pairs & 1, &s_abort))) break;
          top = max(top, s_top[pairs & 1][half ^ 1][r]);
          ++pairs;
          const BlockScale b = block_scale(__uint_as_float(top));
          if (r < t.rows) {
            uint8_t* o = static_cast<uint8_t*>(p.h) + (size_t)entry * p.I + i0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float* v = h + 16 * i + 4 * j;
                w[j] = pack_e4m3(to_code(v[0], b), to_code(v[1], b), to_code(v[2], b), to_code(v[3], b));
              }
              if (i0 + 16 * i < p.I) *reinterpret_cast<uint4*>(o + 16 * i) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            if (half == 0) p.hs[(size_t)t.blk * p.n + entry] = b.scale;
          }
        } else if (r < t.rows) {
          __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.h) + (size_t)entry * p.I + i0;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i0 + 8 * i < p.I)
              *reinterpret_cast<uint4*>(o + 8 * i) =
                  make_uint4(pack_bf16(h[8 * i], h[8 * i + 1]), pack_bf16(h[8 * i + 2], h[8 * i + 3]),
                             pack_bf16(h[8 * i + 4], h[8 * i + 5]), pack_bf16(h[8 * i + 6], h[8 * i + 7]));
        }
        // the down tasks read h by TMA
        asm volatile("fence.proxy.async;" ::: "memory");
        __syncwarp();
        if (lane == 0) red_inc_release(p.ctl->gate_done + t.tile, 0xffffffffu);
      } else {
        const int o0 = t.blk * BN + half * 128;
        if (r < t.rows) {
          float* o = p.y + (size_t)entry * p.H + o0;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            uint32_t x, y, z, w;
            f2_unpack(acc[2 * i], x, y);
            f2_unpack(acc[2 * i + 1], z, w);
            if (o0 + 4 * i < p.H) __stcg(reinterpret_cast<uint4*>(o + 4 * i), make_uint4(x, y, z, w));
          }
        }
        __syncwarp();
        if (lane == 0) red_inc_release(&p.ctl->down_done, 0xffffffffu);
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const int tiles = (int)p.ctl->tiles, gates = tiles * p.IB, total = gates + tiles * p.HT;
      int g = 0;
      if (lane == 0) g = (int)atomicAdd(&p.ctl->queue, 1u);
      g = __shfl_sync(0xffffffffu, g, 0);
      for (uint32_t nt = 0; ok; ++nt) {
        const uint32_t slot = nt % kRing;
        if (!__all_sync(0xffffffffu, mbar_wait(qempty0 + 8 * slot, ((nt / kRing) & 1) ^ 1, &s_abort))) break;
        if (g >= total) {
          if (lane == 0) {
            s_task[slot].kind = kEnd;
            mbar_arrive(qfull0 + 8 * slot);
          }
          break;
        }
        const bool gate = g < gates;
        const int per = gate ? p.IB : p.HT, at = gate ? g : g - gates;
        const MoeTile e = p.tile[at / per];
        const int local = at - e.first * per, mt = local % e.tiles, blk = local / e.tiles;
        const int entry = e.entry0 + mt * kMoeTile, rows = min(kMoeTile, e.count - mt * kMoeTile);
        int tok[4] = {0, 0, 0, 0};
        int wy0, wy1;                                         // the two boxes' first weight rows
        if (gate) {
#pragma unroll
          for (int j = 0; j < 4; ++j) tok[j] = p.list[entry + min(4 * lane + j, rows - 1)];
          wy0 = e.expert * 2 * p.I + blk * 128;
          wy1 = wy0 + p.I;
        } else {
          wy0 = e.expert * p.H + blk * BN;
          wy1 = wy0 + 128;
          const uint32_t want = (uint32_t)(p.IB * 2 * ((rows + 31) / 32));
          if (!__all_sync(0xffffffffu, wait_count_geq(p.ctl->gate_done + e.first + mt, want))) {
            s_abort = 1;
            break;
          }
          asm volatile("fence.proxy.async;" ::: "memory");
        }
        if (lane == 0) {                                      // (a down task after h is there: its scales are read by ordinary loads)
          Task t;
          t.kind = gate ? kGate : kDown;
          t.blk = blk;
          t.expert = e.expert;
          t.tile = e.first + mt;
          t.entry = entry;
          t.rows = rows;
          s_task[slot] = t;
          mbar_arrive(qfull0 + 8 * slot);
        }
        const int copies = gate ? (rows + 3) / 4 : (rows + 7) / 8;
        const uint32_t bytes = 2 * kBoxBytes + (uint32_t)copies * (gate ? 512u : 1024u);
        const int KB = gate ? p.KB1 : p.KB2;
        int next = 0;
        for (int kb = 0; kb < KB; ++kb) {
          if (!__all_sync(0xffffffffu, mbar_wait(empty0 + 8 * stage, phase ^ 1, &s_abort))) {
            ok = false;
            break;
          }
          const uint32_t fb = full0 + 8 * stage, sa = ring + (uint32_t)stage * stBytes, sw = sa + aStage;
          if (lane == 0) {
            mbar_expect_tx(fb, bytes);
            tma_load_2d(sw, gate ? &tmW1 : &tmW2, fb, kb * kCols, wy0);
            tma_load_2d(sw + kBoxBytes, gate ? &tmW1 : &tmW2, fb, kb * kCols, wy1);
            ++s_issued;
          }
          __syncwarp();
          if (lane < copies) {
            if (gate)
              tma_gather4(sa + lane * 512, &tmX, fb, kb * kCols, tok[0], tok[1], tok[2], tok[3]);
            else
              tma_load_2d(sa + lane * 1024, &tmH, fb, kb * kCols, entry + 8 * lane);
          }
          __syncwarp();
          if (kb == KB - 1 - min(KB - 1, 3) && lane == 0) next = (int)atomicAdd(&p.ctl->queue, 1u);
          if (++stage == S) {
            stage = 0;
            phase ^= 1;
          }
        }
        g = __shfl_sync(0xffffffffu, next, 0);
      }
    } else if (warp == 1) {
      constexpr uint32_t idesc = kFp8 ? idesc_e4m3(128, BN) : idesc_bf16(128, BN);
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      const uint64_t ad0 = smem_desc_sw128(__shfl_sync(0xffffffffu, ring, 0));
      int stage = 0, consumed = 0;
      uint32_t phase = 0, it = 0;
      bool ok = true;
      for (uint32_t nt = 0; ok; ++nt) {
        const uint32_t slot = nt % kRing;
        if (!__all_sync(0xffffffffu, mbar_wait(qfull0 + 8 * slot, (nt / kRing) & 1, &s_abort))) break;
        const int kind = s_task[slot].kind;
        __syncwarp();
        if (lane == 0) mbar_arrive(qempty0 + 8 * slot);
        if (kind == kEnd) break;
        const int KB = kind == kGate ? p.KB1 : p.KB2;
        for (int kb = 0; kb < KB; ++kb) {
          const uint32_t buf = it % kBufs, ph = (it / kBufs) & 1;
          if (((kFp8 || kb == 0) && !__all_sync(0xffffffffu, mbar_wait(tempty0 + 8 * buf, ph ^ 1, &s_abort))) ||
              !__all_sync(0xffffffffu, mbar_wait(full0 + 8 * stage, phase, &s_abort))) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (elect_one()) {
            const uint64_t ad = ad0 + (uint64_t)(stage * (stBytes >> 4));
            const uint64_t bd = ad + (uint64_t)(aStage >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) {                     // 32 bytes along K each
              if constexpr (kFp8)
                tc_mma_f8(tm + buf * BN, ad + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, k != 0 ? 1u : 0u);
              else
                tc_mma(tm + buf * BN, ad + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, kb + k != 0 ? 1u : 0u);
            }
            tc_commit(empty0 + 8 * stage);
            if (kFp8 || kb == KB - 1) tc_commit(tfull0 + 8 * buf);
          }
          __syncwarp();
          ++consumed;
          if (++stage == S) {
            stage = 0;
            phase ^= 1;
          }
          if (kFp8) ++it;
        }
        if (!kFp8) ++it;
      }
      if (lane == 0) s_consumed = consumed;
    }
  }

  // ---- the sum over a token's experts, all warps ------------------------------------
  // one code for all warps from here: as many registers as it was compiled for (a warpgroup has to
  // meet between two changes of its registers)
  __syncthreads();
  if (warp >= 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsAll));
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsAll));
  tc_fence_before();
  __syncthreads();
  if (!s_abort) {
    if (threadIdx.x == 0 && !wait_count_geq(&p.ctl->down_done, p.ctl->quarters * 2u * (uint32_t)p.HT)) s_abort = 1;
    __syncthreads();
  }
  if (!s_abort) {
    const int live = p.live ? max(0, min(p.T, ld_pinned(p.live))) : p.T;
    const int per = (p.H + 4 * kThreads - 1) / (4 * kThreads);
    for (int i = (int)blockIdx.x; i < live * per; i += (int)gridDim.x) {
      const int t = i / per, c = (i % per) * 4 * kThreads + 4 * (int)threadIdx.x;
      if (c >= p.H) continue;
      float f[4] = {0.f, 0.f, 0.f, 0.f};
      for (int j0 = 0; j0 < p.k; j0 += 4) {                   // four entries in flight
        float4 v[4];
        float pr[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j0 + j < p.k) {
            const int64_t at = (int64_t)t * p.k + j0 + j;
            pr[j] = p.prob[at];
            v[j] = __ldcg(reinterpret_cast<const float4*>(p.y + (size_t)p.inv[at] * p.H + c));
          }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j0 + j < p.k) {
            f[0] += pr[j] * v[j].x;
            f[1] += pr[j] * v[j].y;
            f[2] += pr[j] * v[j].z;
            f[3] += pr[j] * v[j].w;
          }
      }
      __nv_bfloat16* o = p.out + (int64_t)t * p.out_stride + c;
      if (p.vec) {
        *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = __float2bfloat16_rn(f[j]);
      }
    }
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

template <bool kFp8>
ee_status launch(const void* x, int64_t x_stride, const void* w1, const void* w2, MoeParams& p, cudaStream_t stream) {
  const uint64_t es = kFp8 ? 1 : 2;
  const size_t stage = (((size_t)p.a_rows * 128 + 1023) & ~(size_t)1023) + 2 * 128 * 128;
  p.stages = (int)std::min<size_t>(8, (size_t)(222 * 1024) / stage);
  const size_t smem = 1024 + p.stages * stage;
  CUtensorMap tmX, tmW1, tmH, tmW2;
  const auto encode = [](CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows, uint64_t stride, uint32_t box) {
    if constexpr (kFp8) return encode_u8_tmap_2d(m, base, cols, rows, stride, 128, box);
    const uint64_t dims[2] = {cols, rows}, strides[1] = {2 * stride};
    const uint32_t boxes[2] = {64, box};
    return encode_bf16_tmap(m, base, 2, dims, strides, boxes);
  };
  if (!encode(&tmX, x, p.H, p.T, x_stride, 1) || !encode(&tmW1, w1, p.H, (uint64_t)p.E * 2 * p.I, p.H, 128) ||
      !encode(&tmH, p.h, p.I, p.n, p.I, 8) || !encode(&tmW2, w2, p.I, (uint64_t)p.E * p.H, p.I, 128))
    return EE_ERR_CUDA;
  p.KB1 = (int)((p.H * es + 127) / 128);
  p.KB2 = (int)((p.I * es + 127) / 128);
  {
    int dev = 0;
    const ee_status ds = current_device(&dev);
    if (ds != EE_OK) return ds;
    static std::mutex mu;
    static bool set[kMaxDevices] = {};
    std::lock_guard<std::mutex> lock(mu);
    if (!set[dev]) {
      EE_CUDA_OK(cudaFuncSetAttribute(moe_experts_kernel<kFp8>, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024));
      set[dev] = true;
    }
  }
  EE_CUDA_OK(launch_pdl(moe_experts_kernel<kFp8>, dim3(kNumSMs), dim3(kThreads), smem, stream, 1, tmX, tmW1, tmH, tmW2, p));
  return EE_OK;
}

}  // namespace

extern "C" size_t ee_moe_workspace_size(int32_t T, int32_t H, int32_t I, int32_t E, int32_t k) {
  if (T < 0 || H < 1 || I < 1 || E < 1 || k < 1) return 0;
  return ee::moe_layout(T, H, I, E, k).total;
}

extern "C" ee_status ee_moe_layer(const ee_bf16* x, int64_t x_stride, const ee_bf16* router, const void* w1,
                                  const float* w1_scale_or_null, const void* w2, const float* w2_scale_or_null, int32_t T,
                                  int32_t H, int32_t I, int32_t E, int32_t k, int32_t renorm, const int32_t* live_or_null,
                                  ee_bf16* out, int64_t out_stride, int32_t* ids_or_null, float* probs_or_null, void* ws,
                                  size_t ws_bytes, ee_stream_t stream) {
  if (T < 0 || H < 1 || I < 1 || E < 1 || k < 1 || k > E) return EE_ERR_INVALID_ARG;
  if (H % 16 != 0 || I % 16 != 0 || H > (1 << 16) || I > (1 << 16) || E > kMoeMaxExperts || k > kMoeMaxTopK ||
      T > kMoeMaxTokens)
    return EE_ERR_UNSUPPORTED;
  if (T == 0) return EE_OK;
  if (!x || !router || !w1 || !w2 || !out || !ws || !w1_scale_or_null != !w2_scale_or_null) return EE_ERR_INVALID_ARG;
  if (!ee::aligned(ws, 256) || !ee::aligned(x, 16) || !ee::aligned(router, 16) || !ee::aligned(w1, 16) ||
      !ee::aligned(w2, 16) || !ee::aligned(w1_scale_or_null, 4) || !ee::aligned(w2_scale_or_null, 4) ||
      !ee::aligned(out, 2) || !ee::aligned(live_or_null, 4) || !ee::aligned(ids_or_null, 4) ||
      !ee::aligned(probs_or_null, 4))
    return EE_ERR_INVALID_ARG;
  if (x_stride < H || x_stride % 8 != 0 || out_stride < H) return EE_ERR_INVALID_ARG;
  const ee::MoeLayout l = ee::moe_layout(T, H, I, E, k);
  if (ws_bytes < l.total) return EE_ERR_WORKSPACE;
  char* const base = static_cast<char*>(ws);
  const bool fp8 = w1_scale_or_null != nullptr;
  ee::RouteParams r;
  r.x = reinterpret_cast<const __nv_bfloat16*>(x);
  r.x_stride = x_stride;
  r.router = reinterpret_cast<const __nv_bfloat16*>(router);
  r.live = live_or_null;
  r.T = T;
  r.H = H;
  r.E = E;
  r.k = k;
  r.renorm = renorm != 0;
  r.max_tiles = l.max_tiles;
  r.ctl = reinterpret_cast<ee::MoeCtl*>(base + l.ctl);
  r.tile = reinterpret_cast<ee::MoeTile*>(base + l.tile);
  r.ids = reinterpret_cast<int32_t*>(base + l.ids);
  r.prob = reinterpret_cast<float*>(base + l.prob);
  r.list = reinterpret_cast<int32_t*>(base + l.list);
  r.inv = reinterpret_cast<int32_t*>(base + l.inv);
  r.xq = fp8 ? reinterpret_cast<uint8_t*>(base + l.xq) : nullptr;
  r.xs = reinterpret_cast<float*>(base + l.xs);
  r.ids_out = ids_or_null;
  r.prob_out = probs_or_null;
  // the widest share of the hidden dimension that the SMs hold at once
  const int groups = (T + 15) / 16, blocks = (H + kBlk - 1) / kBlk;
  r.cl = 8;
  while (r.cl > 1 && (groups * r.cl > ee::kNumSMs || r.cl > blocks)) r.cl /= 2;
  MoeParams p;
  p.T = T;
  p.H = H;
  p.I = I;
  p.E = E;
  p.k = k;
  p.n = T * k;
  p.IB = (I + 127) / 128;
  p.HT = (H + BN - 1) / BN;
  p.HB = blocks;
  p.a_rows = std::min(128, (T + 7) / 8 * 8);
  p.ctl = r.ctl;
  p.tile = r.tile;
  p.list = r.list;
  p.inv = r.inv;
  p.prob = r.prob;
  p.xs = r.xs;
  p.s1 = w1_scale_or_null;
  p.s2 = w2_scale_or_null;
  p.h = base + l.h;
  p.hs = reinterpret_cast<float*>(base + l.hs);
  p.y = reinterpret_cast<float*>(base + l.y);
  p.out = reinterpret_cast<__nv_bfloat16*>(out);
  p.out_stride = out_stride;
  p.vec = ee::aligned(out, 8) && out_stride % 4 == 0;
  p.live = live_or_null;
  p.err = ee::err_word(ws);
  const ee_status st = ee::launch_moe_route(r, (cudaStream_t)stream);
  if (st != EE_OK) return st;
  return fp8 ? launch<true>(r.xq, H, w1, w2, p, (cudaStream_t)stream)
             : launch<false>(x, x_stride, w1, w2, p, (cudaStream_t)stream);
}
