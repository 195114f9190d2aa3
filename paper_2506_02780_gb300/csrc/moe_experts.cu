// ee_moe_layer: a mixture-of-experts layer for the few tokens of a pass.  After the router (moe_route.cu)
// one persistent kernel runs the chosen experts:
//   gate tasks   h = silu(x Wg^T) * (x Wu^T)   128 columns of h for one token tile
//   down tasks   y = h Wd^T                    256 columns of y
//   the sum      out[t] = sum_j p[t][j] y[entry of t's j-th expert]
// The experts' weights are read once and bound the call.  Weight rows are the MMA's M side (two tiles of
// 128: gate and up, or two of down), tokens its N side: a few tokens then cost the epilogue a few
// columns of every lane, where with tokens on the lanes two warps of eight would do all of its work (when it was turned, a draft
// tree's layer of 64 experts of 1280 x 3584 went from 194 us to 155).  A k-block of narrower weight tiles takes
// the same 0.4 us, so there are only those of 128 rows.
//
// On 8-bit weights tiles of 128 tokens have tokens on the lanes all the same: a token's scale is then one
// register, where the columns' scales come from shared memory, 128 of them a k-block and thread, whose reads
// bound such tiles (2,048 tokens at 4 of 16 experts 281 us, so 226).
//
// CTAs draw tasks from one queue, gate tasks first.  A down task waits for the gate tasks of its
// token tile; those were drawn before it by CTAs that are running, so no wait depends on
// a CTA that has not started.  Warp 0 draws, publishes the task to the other roles in a ring of
// shared memory and streams the operands (x's rows: warps 12..15); it runs ahead of the others across
// tasks, so that the stream does not stop between them.  Warp 2 puts products of scales into shared memory,
// warp 3 tells other CTAs what the epilogue warps 4..11 have stored (a release waits for the stores: it would hold them up
// for 2 us a task).
//
// Measured with the routing, 64 experts of 1280 x 3584, 6 a token: 64 tokens on 8-bit weights 133 to 137 us (845 MB; the
// experts' part 122 us, 6.9 TB/s), on bf16 ones 247 to 255 us; 534 tokens 171 to 175 and 292 to 300 us.
#include <mutex>

#include "moe.cuh"

namespace {

using namespace ee;

constexpr int kThreads = 512;          // warp 0 tasks and TMA, 1 MMA, 2 TMEM and scales, 3 publishing; 4..11 epilogue; 12..15 x
constexpr int kEpiWarps = 8;           // two per TMEM lane quarter, every other 16 tokens each
constexpr int kRegsAll = 128;          // a warp's at launch; the epilogue's take some of the others'
constexpr int kGatherWarps = 4;
constexpr int kTile = 128;             // rows of a weight tile
constexpr uint32_t kOutBytes = 32 * 16 * 4;   // of an epilogue warp: 32 rows of 16 columns of y on their way out
constexpr int kRing = 4;               // tasks published and not yet done with by every role
constexpr int kScRing = 8;             // k-blocks' scales
constexpr int kMaxStages = 6;

enum { kGate = 0, kDown = 1, kEnd = 2 };
struct Task {
  int kind, blk, expert, tile, entry, rows;   // column block; token tile, its first entry and their number
};

__device__ __forceinline__ void lds_2u64(uint32_t a, uint64_t& x, uint64_t& y) {
  asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(x), "=l"(y) : "r"(a) : "memory");
}
// acc += scale * 16 columns; scales of the columns at shared address a
__device__ __forceinline__ void add_scaled16(uint64_t (&acc)[8], const uint32_t (&r)[16], uint32_t a) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint64_t s0, s1;
    lds_2u64(a + 16 * i, s0, s1);
    acc[2 * i] = f2_fma(f2_pack(r[4 * i], r[4 * i + 1]), s0, acc[2 * i]);
    acc[2 * i + 1] = f2_fma(f2_pack(r[4 * i + 2], r[4 * i + 3]), s1, acc[2 * i + 1]);
  }
}

// NT: most tokens of a tile
template <bool kFp8, int NT>
__global__ void __launch_bounds__(kThreads, 1)
moe_experts_kernel(const __grid_constant__ CUtensorMap tmW1, const __grid_constant__ CUtensorMap tmH8,
                   const __grid_constant__ CUtensorMap tmH32, const __grid_constant__ CUtensorMap tmW2, const MoeParams p) {
  constexpr int kCols = kFp8 ? 128 : 64;        // elements in 128 bytes
  constexpr int kRegsEpi = NT == 128 ? 200 : 152, kRegsOther = 2 * kRegsAll - kRegsEpi;
  constexpr int kScBatch = NT == 128 ? 2 : 4;   // k-blocks whose scales' loads are in flight
  constexpr int kBufs = 512 / (2 * NT) < 8 ? 512 / (2 * NT) : 8;   // accumulators of two tiles
  constexpr bool kTok = kFp8 && NT == 128;      // tokens on the MMA's M side
  constexpr int kChunks = NT / 32;              // groups of 16 tokens of an epilogue warp
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages + 2 * 8 + 3 * kRing + 2 * kScRing + 4 + 1];
  __shared__ uint32_t s_top[kFp8 ? 2 : 1][4][NT];
  __shared__ __align__(16) float s_scale[kFp8 ? kScRing : 1][2][NT];
  __shared__ Task s_task[kRing];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ int s_issued, s_consumed;

  pdl_allow_next();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int S = p.stages;
  const uint32_t bStage = (uint32_t)p.b_rows * 128;            // tokens, then the weights' two tiles
  constexpr uint32_t kBoxBytes = kTile * 128;
  const uint32_t stBytes = bStage + 2 * kBoxBytes;
  const uint32_t ring = smem_u32(smem);
  const uint32_t full0 = smem_u32(s_bars), empty0 = full0 + 8 * kMaxStages, tfull0 = empty0 + 8 * kMaxStages,
                 tempty0 = tfull0 + 8 * 8, qfull0 = tempty0 + 8 * 8, qempty0 = qfull0 + 8 * kRing,
                 edone0 = qempty0 + 8 * kRing, sfull0 = edone0 + 8 * kRing, sempty0 = sfull0 + 8 * kScRing,
                 meet0 = sempty0 + 8 * kScRing, drain = meet0 + 8 * 4;
  if (threadIdx.x == 0) {
    s_abort = 0;
    s_issued = 0;
    s_consumed = 0;
    for (int s = 0; s < S; ++s) {
      mbar_init(full0 + 8 * s, 1 + kGatherWarps);
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int a = 0; a < kBufs; ++a) {
      mbar_init(tfull0 + 8 * a, 1);
      mbar_init(tempty0 + 8 * a, kEpiWarps);
    }
    for (int a = 0; a < kRing; ++a) {
      mbar_init(qfull0 + 8 * a, 1);
      mbar_init(qempty0 + 8 * a, kEpiWarps + kGatherWarps + (kFp8 ? 3 : 2));
      mbar_init(edone0 + 8 * a, kEpiWarps);
    }
    for (int a = 0; a < kScRing; ++a) {
      mbar_init(sfull0 + 8 * a, 1);
      mbar_init(sempty0 + 8 * a, kEpiWarps);
    }
    for (int a = 0; a < 4; ++a) mbar_init(meet0 + 8 * a, kTok ? 2 : 4);
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmH32)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmW1)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmH8)) : "memory");
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

  if (warp >= 4 && warp < 4 + kEpiWarps) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpi));
    const int q = warp & 3, half = (warp - 4) >> 2;
    const int r = 32 * q + lane;                              // row of both weight tiles
    const uint32_t tq = tmem + ((uint32_t)(32 * q) << 16);
    uint32_t it = 0, sc = 0, meets = 0;                       // accumulators and scales taken, blocks of h shared
    for (uint32_t nt = 0;; ++nt) {
      const uint32_t slot = nt % kRing;
      if (!__all_sync(0xffffffffu, mbar_wait(qfull0 + 8 * slot, (nt / kRing) & 1, &s_abort))) break;
      const Task t = s_task[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(qempty0 + 8 * slot);
      if (t.kind == kEnd) break;
      const bool gate = t.kind == kGate;
      const bool mine = half * 16 < t.rows;                   // the warp has something to keep
      if constexpr (kTok) {
        // this thread: token r; 64 columns of gate and of up, or 128 of down
        const int KB = gate ? p.KB1 : p.KB2;
        const bool some = 32 * q < t.rows;
        const uint32_t c0 = gate ? half * 64 : half * 128, c1 = gate ? 128 + half * 64 : half * 128 + 64;
        uint64_t acc[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) acc[i] = 0;
        bool ok = true;
        for (int kb = 0; kb < KB; ++kb, ++it, ++sc) {
          const uint32_t buf = it % kBufs, e = sc % kScRing;
          if (!__all_sync(0xffffffffu, mbar_wait(sfull0 + 8 * e, (sc / kScRing) & 1, &s_abort)) ||
              !__all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * buf, (it / kBufs) & 1, &s_abort))) {
            ok = false;
            break;
          }
          tc_fence_after();
          promote_2x64(acc, tq + buf * (2 * NT) + c0, tq + buf * (2 * NT) + c1, s_scale[e][gate ? 0 : half][r],
                       s_scale[e][gate ? 1 : half][r]);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(tempty0 + 8 * buf);
            mbar_arrive(sempty0 + 8 * e);
          }
        }
        if (!ok) break;
        if (some && gate) {
          const int i0 = t.blk * kTile + half * 64;
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            uint32_t h[2];
            acc[i] = silu_times2(acc[i], acc[32 + i]);
            f2_unpack(acc[i], h[0], h[1]);
#pragma unroll
            for (int d = 0; d < 2; ++d)
              if (i0 + 2 * i + d < p.I) top = max(top, h[d] & 0x7fffffffu);
          }
          // the block's other 64 columns are the neighbour warp's
          s_top[meets & 1][half][r] = top;
          __syncwarp();
          if (lane == 0) mbar_arrive(meet0 + 8 * q);
          if (!__all_sync(0xffffffffu, mbar_wait(meet0 + 8 * q, meets & 1, &s_abort))) break;
          const BlockScale s = block_scale(__uint_as_float(max(top, s_top[meets & 1][half ^ 1][r])));
          ++meets;
          if (r < t.rows) {
            uint8_t* o = static_cast<uint8_t*>(p.h) + (size_t)(t.entry + r) * p.I + i0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                uint32_t h[4];
                f2_unpack(acc[8 * i + 2 * j], h[0], h[1]);
                f2_unpack(acc[8 * i + 2 * j + 1], h[2], h[3]);
                w[j] = pack_e4m3(to_code(__uint_as_float(h[0]), s), to_code(__uint_as_float(h[1]), s),
                                 to_code(__uint_as_float(h[2]), s), to_code(__uint_as_float(h[3]), s));
              }
              if (i0 + 16 * i < p.I) *reinterpret_cast<uint4*>(o + 16 * i) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            if (half == 0) p.hs[(size_t)t.blk * p.n + t.entry + r] = s.scale;
          }
        } else if (some) {
          // 16 columns at a time through shared memory, so that a store is eight rows' 64 bytes
          const int col = t.blk * 2 * kTile + half * 128 + 4 * (lane & 3);
          const uint32_t out = ring + (uint32_t)S * stBytes + (uint32_t)(warp - 4) * kOutBytes;
#pragma unroll
          for (int h = 0; h < 8; ++h) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t v[4];
              f2_unpack(acc[8 * h + 2 * i], v[0], v[1]);
              f2_unpack(acc[8 * h + 2 * i + 1], v[2], v[3]);
              st_shared_u4(out + (uint32_t)lane * 64 + (uint32_t)((i ^ (lane >> 1 & 3)) << 4), make_uint4(v[0], v[1], v[2], v[3]));
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int rr = 8 * i + (lane >> 2);
              const uint4 v = ld_shared_u4(out + (uint32_t)rr * 64 + (uint32_t)(((lane & 3) ^ (rr >> 1 & 3)) << 4));
              if (32 * q + rr < t.rows && col + 16 * h < p.H)
                __stcg(reinterpret_cast<uint4*>(p.y + (size_t)(t.entry + 32 * q + rr) * p.H + col + 16 * h), v);
            }
            __syncwarp();
          }
        }
      } else {
        uint64_t acc0[kChunks][8], acc1[kChunks][8];            // tokens (2 j + half) 16 .. + 15 of the two tiles
#pragma unroll
        for (int j = 0; j < kChunks; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc0[j][i] = acc1[j][i] = 0;
        const int KB = kFp8 ? (gate ? p.KB1 : p.KB2) : 1;
        bool ok = true;
        for (int kb = 0; kb < KB; ++kb, ++it) {
          const uint32_t buf = it % kBufs, ph = (it / kBufs) & 1;
          if constexpr (kFp8)
            ok = __all_sync(0xffffffffu, mbar_wait(sfull0 + 8 * (sc % kScRing), (sc / kScRing) & 1, &s_abort));
          if (!ok || !__all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * buf, ph, &s_abort))) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (mine) {
            const uint32_t sa = smem_u32(&s_scale[kFp8 ? sc % kScRing : 0][0][0]);
#pragma unroll
            for (int j = 0; j < kChunks; ++j) {
              const int c = (2 * j + half) * 16;
              if (c < t.rows) {
                uint32_t a[16], b[16];
                tc_ld16_nowait(tq + buf * (2 * NT) + c, a);
                tc_ld16_nowait(tq + buf * (2 * NT) + NT + c, b);
                tc_wait_ld16x2(a, b);
                if constexpr (kFp8) {
                  add_scaled16(acc0[j], a, sa + 4 * c);
                  add_scaled16(acc1[j], b, sa + 4 * (NT + c));
                } else {
#pragma unroll
                  for (int i = 0; i < 8; ++i) {
                    acc0[j][i] = f2_pack(a[2 * i], a[2 * i + 1]);
                    acc1[j][i] = f2_pack(b[2 * i], b[2 * i + 1]);
                  }
                }
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(tempty0 + 8 * buf);
            if constexpr (kFp8) mbar_arrive(sempty0 + 8 * (sc % kScRing));
          }
          ++sc;
        }
        if (!ok) break;
        if (mine && gate) {
          const int col = t.blk * kTile + r;
          const bool in = col < p.I;
          uint32_t top[kChunks];                                // lane i: the largest |h| of token i in these 32 columns
#pragma unroll
          for (int j = 0; j < kChunks; ++j) {
            const int c = (2 * j + half) * 16;
            top[j] = 0;
            if (c >= t.rows) break;
            __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.h) + (size_t)(t.entry + c) * p.I + col;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              if (i % 2 == 0) acc0[j][i / 2] = silu_times2(acc0[j][i / 2], acc1[j][i / 2]);
              uint32_t h[2];
              f2_unpack(acc0[j][i / 2], h[0], h[1]);
              if constexpr (kFp8) {
                const uint32_t m = __reduce_max_sync(0xffffffffu, in ? h[i & 1] & 0x7fffffffu : 0u);
                if (lane == i) top[j] = m;
              } else if (in && c + i < t.rows) {
                o[(size_t)i * p.I] = __float2bfloat16_rn(__uint_as_float(h[i & 1]));
              }
            }
            if (kFp8 && lane < 16) s_top[meets & 1][q][c + lane] = top[j];
          }
          if constexpr (kFp8) {
            // the block's other columns are the three warps' of the same tokens
            __syncwarp();
            if (lane == 0) mbar_arrive(meet0 + 8 * half);
            if (!__all_sync(0xffffffffu, mbar_wait(meet0 + 8 * half, meets & 1, &s_abort))) break;
#pragma unroll
            for (int j = 0; j < kChunks; ++j) {
              const int c = (2 * j + half) * 16;
              if (c >= t.rows) break;
              uint32_t m = 0;
#pragma unroll
              for (int i = 0; i < 4; ++i) m = max(m, s_top[meets & 1][i][c + (lane & 15)]);
              const BlockScale mine_s = block_scale(__uint_as_float(m));
              if (q == 0 && lane < 16 && c + lane < t.rows) p.hs[(size_t)t.blk * p.n + t.entry + c + lane] = mine_s.scale;
              uint8_t* o = static_cast<uint8_t*>(p.h) + (size_t)(t.entry + c) * p.I + col;
#pragma unroll
              for (int i = 0; i < 16; i += 2) {
                uint32_t h[2];
                f2_unpack(acc0[j][i / 2], h[0], h[1]);
                float v[2];
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                  BlockScale s;
                  s.hi = __shfl_sync(0xffffffffu, mine_s.hi, i + d);
                  s.lo = __shfl_sync(0xffffffffu, mine_s.lo, i + d);
                  v[d] = to_code(__uint_as_float(h[d]), s);
                }
                const uint32_t code = pack_e4m3(v[0], v[1], 0.f, 0.f);
                if (in && c + i < t.rows) o[(size_t)i * p.I] = (uint8_t)code;
                if (in && c + i + 1 < t.rows) o[(size_t)(i + 1) * p.I] = (uint8_t)(code >> 8);
              }
            }
            ++meets;
          }
        } else if (mine) {
          const int col = t.blk * 2 * kTile + r;
          const bool in0 = col < p.H, in1 = col + kTile < p.H;
#pragma unroll
          for (int j = 0; j < kChunks; ++j) {
            const int c = (2 * j + half) * 16;
            if (c >= t.rows) break;
            float* o = p.y + (size_t)(t.entry + c) * p.H + col;
#pragma unroll
            for (int i = 0; i < 16; ++i, o += p.H) {
              uint32_t a[2], b[2];
              f2_unpack(acc0[j][i / 2], a[0], a[1]);
              f2_unpack(acc1[j][i / 2], b[0], b[1]);
              if (in0 && c + i < t.rows) __stcg(o, __uint_as_float(a[i & 1]));
              if (in1 && c + i < t.rows) __stcg(o + kTile, __uint_as_float(b[i & 1]));
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(edone0 + 8 * slot);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 0) {
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t u_full = __shfl_sync(0xffffffffu, full0, 0), u_ring = __shfl_sync(0xffffffffu, ring, 0);
      const int tiles = (int)p.ctl->tiles, gates = tiles * p.IB, total = gates + tiles * p.HT;
      // a task, worked out while the loads of the one before it wait for room in the ring: drawn at kDraw k-blocks
      // before that one's end, its tile looked up at kLook, whether h is there at kList
      constexpr int kDraw = 10, kLook = 7, kList = 4;
      int g = 0, blk = 0, entry = 0, rows = 0;
      uint32_t have = 0;
      const uint64_t policy = policy_evict_first();           // (h and y stay in L2)
      MoeTile e;
      const auto draw = [&]() {
        if (lane == 0) g = (int)atomicAdd(&p.ctl->queue, 1u);
      };
      const auto look = [&]() {
        g = __shfl_sync(0xffffffffu, g, 0);
        if (g < total) e = p.tile[(g < gates ? g : g - gates) / (g < gates ? p.IB : p.HT)];
      };
      int tile = 0;
      const auto list = [&]() {
        if (g >= total) return;
        const bool gate = g < gates;
        const int local = (gate ? g : g - gates) - e.first * (gate ? p.IB : p.HT), mt = local % e.tiles;
        blk = local / e.tiles;
        tile = e.first + mt;
        entry = e.entry0 + mt * NT;
        rows = min(NT, e.count - mt * NT);
        if (!gate) have = ld_acquire(p.ctl->gate_done + tile);
      };
      draw();
      look();
      list();
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
        const bool gate = __shfl_sync(0xffffffffu, (int)(g < gates), 0) != 0;
        const int at_entry = __shfl_sync(0xffffffffu, entry, 0), urows = __shfl_sync(0xffffffffu, rows, 0);
        const int h32 = gate ? 0 : urows / 32, h8 = gate ? 0 : (urows % 32 + 7) / 8;   // boxes of h
        int wy0, wy1;                                         // the two tiles' first weight rows
        if (gate) {
          wy0 = e.expert * 2 * p.I + blk * kTile;
          wy1 = wy0 + p.I;
        } else {
          wy0 = e.expert * p.H + blk * 2 * kTile;
          wy1 = wy0 + kTile;
          const uint32_t want = (uint32_t)p.IB;
          if (!__all_sync(0xffffffffu, have >= want || wait_count_geq(p.ctl->gate_done + tile, want))) {
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
          t.tile = tile;
          t.entry = entry;
          t.rows = rows;
          s_task[slot] = t;
          mbar_arrive(qfull0 + 8 * slot);
        }
        // (uniform values and an elected lane: copies whose operands the compiler has to move to uniform registers one by one
        // take 100 ns each to issue)
        wy0 = __shfl_sync(0xffffffffu, wy0, 0);
        wy1 = __shfl_sync(0xffffffffu, wy1, 0);
        const uint32_t bytes = 2 * kBoxBytes + (uint32_t)(4 * h32 + h8) * 1024u;
        const int KB = gate ? p.KB1 : p.KB2;
        for (int kb = 0; kb < KB; ++kb) {
          if (!__all_sync(0xffffffffu, mbar_wait(empty0 + 8 * stage, phase ^ 1, &s_abort))) {
            ok = false;
            break;
          }
          const uint32_t fb = u_full + 8 * stage, sb = u_ring + (uint32_t)stage * stBytes, sw = sb + bStage;
          if (elect_one()) {
            mbar_expect_tx(fb, bytes);
            if (gate) {
              tma_load_2d_hint(sw, &tmW1, fb, kb * kCols, wy0, policy);
              tma_load_2d_hint(sw + kBoxBytes, &tmW1, fb, kb * kCols, wy1, policy);
            } else {
              tma_load_2d_hint(sw, &tmW2, fb, kb * kCols, wy0, policy);
              tma_load_2d_hint(sw + kBoxBytes, &tmW2, fb, kb * kCols, wy1, policy);
              for (int i = 0; i < h32; ++i) tma_load_2d(sb + i * 4096, &tmH32, fb, kb * kCols, at_entry + 32 * i);
              for (int i = 0; i < h8; ++i) tma_load_2d(sb + h32 * 4096 + i * 1024, &tmH8, fb, kb * kCols, at_entry + 32 * h32 + 8 * i);
            }
          }
          __syncwarp();
          ++issued;
          if (kb == max(0, KB - kDraw)) draw();
          if (kb == max(0, KB - kLook)) look();
          if (kb == max(0, KB - kList)) list();
          if (++stage == S) {
            stage = 0;
            phase ^= 1;
          }
        }
      }
      if (lane == 0) s_issued = issued;
    } else if (warp == 1) {
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      const uint64_t bd0 = smem_desc_sw128(__shfl_sync(0xffffffffu, ring, 0));
      int stage = 0, consumed = 0;
      uint32_t phase = 0, it = 0;
      bool ok = true;
      for (uint32_t nt = 0; ok; ++nt) {
        const uint32_t slot = nt % kRing;
        if (!__all_sync(0xffffffffu, mbar_wait(qfull0 + 8 * slot, (nt / kRing) & 1, &s_abort))) break;
        const int kind = __shfl_sync(0xffffffffu, s_task[slot].kind, 0);
        const int rows = __shfl_sync(0xffffffffu, s_task[slot].rows, 0);
        if (lane == 0) mbar_arrive(qempty0 + 8 * slot);
        if (kind == kEnd) break;
        const int KB = kind == kGate ? p.KB1 : p.KB2;
        constexpr uint64_t tile2 = kBoxBytes >> 4;
        const int N = (rows + 15) & ~15;
        const uint32_t idesc = kTok ? idesc_e4m3(128, 2 * kTile) : kFp8 ? idesc_e4m3(128, N) : idesc_bf16(128, N);
        for (int kb = 0; kb < KB; ++kb) {
          const uint32_t buf = it % kBufs, ph = (it / kBufs) & 1;
          if (((kFp8 || kb == 0) && !__all_sync(0xffffffffu, mbar_wait(tempty0 + 8 * buf, ph ^ 1, &s_abort))) ||
              !__all_sync(0xffffffffu, mbar_wait(full0 + 8 * stage, phase, &s_abort))) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (elect_one()) {
            const uint64_t bd = bd0 + (uint64_t)(stage * (stBytes >> 4));
            const uint64_t ad = bd + (uint64_t)(bStage >> 4);
            const uint32_t d = tm + buf * (2 * NT);
#pragma unroll
            for (int k = 0; k < 4; ++k) {                     // 32 bytes along K each
              const uint32_t add = (kFp8 ? k : kb + k) != 0 ? 1u : 0u;
              if constexpr (kTok) {
                tc_mma_f8(d, bd + (uint64_t)(2 * k), ad + (uint64_t)(2 * k), idesc, add);
              } else if constexpr (kFp8) {
                tc_mma_f8(d, ad + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, add);
                tc_mma_f8(d + NT, ad + tile2 + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, add);
              } else {
                tc_mma(d, ad + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, add);
                tc_mma(d + NT, ad + tile2 + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, add);
              }
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
    } else if (warp == 2) {
      if constexpr (kFp8) {
        // scale of (k-block, token, weight tile): four tokens a lane, some k-blocks' loads at once
        uint32_t sc = 0;
        bool ok = true;
        for (uint32_t nt = 0; ok; ++nt) {
          const uint32_t slot = nt % kRing;
          if (!__all_sync(0xffffffffu, mbar_wait(qfull0 + 8 * slot, (nt / kRing) & 1, &s_abort))) break;
          const Task t = s_task[slot];
          __syncwarp();
          if (lane == 0) mbar_arrive(qempty0 + 8 * slot);
          if (t.kind == kEnd) break;
          const bool gate = t.kind == kGate;
          const int KB = gate ? p.KB1 : p.KB2;
          const float *ws0, *ws1;
          if (gate) {
            ws0 = p.s1 + ((int64_t)(2 * t.expert) * p.IB + t.blk) * KB;
            ws1 = ws0 + (int64_t)p.IB * KB;
          } else {
            ws0 = p.s2 + ((int64_t)t.expert * p.HB + min(t.blk * 2, p.HB - 1)) * KB;
            ws1 = p.s2 + ((int64_t)t.expert * p.HB + min(t.blk * 2 + 1, p.HB - 1)) * KB;
          }
          const float* xs = gate ? p.xs : p.hs;
          const int xstep = gate ? p.T : p.n;
          int at[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int e = t.entry + min(4 * lane + j, t.rows - 1);
            at[j] = gate ? p.list[e] : e;
          }
          for (int kb = 0; kb < KB && ok; kb += kScBatch) {
            float f[kScBatch][4], w0[kScBatch], w1[kScBatch];
#pragma unroll
            for (int b = 0; b < kScBatch; ++b)
              if (kb + b < KB) {
                const float* row = xs + (int64_t)(kb + b) * xstep;
#pragma unroll
                for (int j = 0; j < 4; ++j) f[b][j] = __ldcg(row + at[j]);
                w0[b] = ws0[kb + b];
                w1[b] = ws1[kb + b];
              }
#pragma unroll
            for (int b = 0; b < kScBatch; ++b)
              if (kb + b < KB && ok) {
                const uint32_t e = sc % kScRing;
                ok = __all_sync(0xffffffffu, mbar_wait(sempty0 + 8 * e, ((sc / kScRing) & 1) ^ 1, &s_abort));
                if (ok && 4 * lane < NT) {
                  *reinterpret_cast<float4*>(&s_scale[e][0][4 * lane]) =
                      make_float4(f[b][0] * w0[b], f[b][1] * w0[b], f[b][2] * w0[b], f[b][3] * w0[b]);
                  *reinterpret_cast<float4*>(&s_scale[e][1][4 * lane]) =
                      make_float4(f[b][0] * w1[b], f[b][1] * w1[b], f[b][2] * w1[b], f[b][3] * w1[b]);
                }
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(sfull0 + 8 * e);
                ++sc;
              }
          }
        }
      }
    } else if (warp >= 4 + kEpiWarps) {
      // x's rows of a tile, 16 bytes a copy, to where TMA's 128-byte swizzle would put them (gathered by TMA, four rows an
      // operation of 55 ns, they took longer than everything else for 40 tokens and more); a stage is
      // signalled kLag stages later, when its copies have landed, and at a task's end at once: the next
      // task may wait for this one
      constexpr int kLag = 2, kMine = NT / 16;
      const int gw = warp - 4 - kEpiWarps, ch = lane & 7, row0 = gw * 4 + (lane >> 3);
      const uint32_t to = (uint32_t)row0 * 128 + (uint32_t)((ch ^ (row0 & 7)) << 4);   // (16 rows on: the same place in a group of 8)
      const int x_bytes = p.H * (kFp8 ? 1 : 2);
      int stage = 0, sig = 0;                                 // stages filled and signalled
      uint32_t phase = 0;
      bool ok = true;
      const auto signal = [&]() {
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(full0 + 8 * sig);
        if (++sig == S) sig = 0;
      };
      for (uint32_t nt = 0; ok; ++nt) {
        const uint32_t slot = nt % kRing;
        if (!__all_sync(0xffffffffu, mbar_wait(qfull0 + 8 * slot, (nt / kRing) & 1, &s_abort))) break;
        const Task t = s_task[slot];
        __syncwarp();
        if (lane == 0) mbar_arrive(qempty0 + 8 * slot);
        if (t.kind == kEnd) break;
        const bool gate = t.kind == kGate;
        const int KB = gate ? p.KB1 : p.KB2;
        const uint8_t* src[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          src[i] = nullptr;
          if (gate && row0 + 16 * i < t.rows)
            src[i] = static_cast<const uint8_t*>(p.x) + (int64_t)p.list[t.entry + row0 + 16 * i] * p.x_stride * (kFp8 ? 1 : 2) + ch * 16;
        }
        for (int kb = 0; kb < KB; ++kb) {
          if (!__all_sync(0xffffffffu, mbar_wait(empty0 + 8 * stage, phase ^ 1, &s_abort))) {
            ok = false;
            break;
          }
          const uint32_t at = ring + (uint32_t)stage * stBytes + to;
          const uint32_t in = kb * 128 + ch * 16 < x_bytes ? 16u : 0u;   // (nothing is read where 0 bytes are)
#pragma unroll
          for (int i = 0; i < kMine; ++i)
            if (src[i]) cp_async16(at + i * 2048, src[i] + (in ? kb * 128 : 0), in);
          asm volatile("cp.async.commit_group;" ::: "memory");
          if (kb >= kLag) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kLag) : "memory");
            signal();
          }
          if (++stage == S) {
            stage = 0;
            phase ^= 1;
          }
        }
        cp_async_wait_all();
        if (ok)
          for (int i = 0; i < min(KB, kLag); ++i) signal();
      }
      cp_async_wait_all();
    } else {
      for (uint32_t nt = 0;; ++nt) {
        const uint32_t slot = nt % kRing;
        if (!__all_sync(0xffffffffu, mbar_wait(qfull0 + 8 * slot, (nt / kRing) & 1, &s_abort))) break;
        const Task t = s_task[slot];
        if (t.kind == kEnd) break;
        if (!__all_sync(0xffffffffu, mbar_wait(edone0 + 8 * slot, (nt / kRing) & 1, &s_abort))) break;
        if (lane == 0) mbar_arrive(qempty0 + 8 * slot);
        if (t.kind == kDown) {
          if (lane == 0) red_inc_release(&p.ctl->down_done, 0xffffffffu);
          continue;
        }
        asm volatile("fence.proxy.async;" ::: "memory");      // down tasks read h by TMA
        __syncwarp();
        if (lane == 0) red_inc_release(p.ctl->gate_done + t.tile, 0xffffffffu);
      }
    }
  }

  // one code for all warps from here: as many registers as it was compiled for (a warpgroup has to
  // meet between two changes of its registers)
  __syncthreads();
  if (warp >= 4 && warp < 4 + kEpiWarps) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsAll));
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsAll));
  tc_fence_before();
  __syncthreads();

  // ---- the sum over a token's experts, all warps ------------------------------------
  if (!s_abort) {
    if (threadIdx.x == 0 && !wait_count_geq(&p.ctl->down_done, p.ctl->tiles * (uint32_t)p.HT)) s_abort = 1;
    __syncthreads();
  }
  if (!s_abort) {
    const int live = p.live ? max(0, min(p.T, ld_pinned(p.live))) : p.T;
    // a warp takes 256 columns of a token: a round trip for the entries' numbers, one for 8 entries
    const int per = (p.H + 255) / 256, step = (int)gridDim.x * (kThreads / 32);
    for (int u = (int)blockIdx.x * (kThreads / 32) + warp; u < live * per; u += step) {
      const int t = u / per, c = u % per * 256 + 4 * lane;
      const bool in0 = c < p.H, in1 = c + 128 < p.H;
      int my_at = 0;
      float my_p = 0.f;
      if (lane < p.k) {
        my_at = p.inv[(int64_t)t * p.k + lane];
        my_p = p.prob[(int64_t)t * p.k + lane];
      }
      float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int j0 = 0; j0 < p.k; j0 += 8) {
        float4 v[8][2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float* y = p.y + (size_t)__shfl_sync(0xffffffffu, my_at, (j0 + j) & 31) * p.H + c;
          v[j][0] = v[j][1] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (j0 + j < p.k) {
            if (in0) v[j][0] = __ldcg(reinterpret_cast<const float4*>(y));
            if (in1) v[j][1] = __ldcg(reinterpret_cast<const float4*>(y + 128));
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float pr = __shfl_sync(0xffffffffu, my_p, (j0 + j) & 31);
          if (j0 + j < p.k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              f[4 * i] += pr * v[j][i].x;
              f[4 * i + 1] += pr * v[j][i].y;
              f[4 * i + 2] += pr * v[j][i].z;
              f[4 * i + 3] += pr * v[j][i].w;
            }
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (!(i ? in1 : in0)) continue;
        __nv_bfloat16* o = p.out + (int64_t)t * p.out_stride + c + 128 * i;
        if (p.vec) {
          *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(f[4 * i], f[4 * i + 1]), pack_bf16(f[4 * i + 2], f[4 * i + 3]));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] = __float2bfloat16_rn(f[4 * i + j]);
        }
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

template <bool kFp8, int NT>
ee_status launch(MoeParams& p, cudaStream_t stream) {
  const size_t stage = (size_t)p.b_rows * 128 + 2 * kTile * 128, outs = kFp8 && NT == 128 ? kEpiWarps * kOutBytes : 0;
  p.stages = (int)std::min<size_t>(kMaxStages, ((size_t)(213 * 1024) - outs) / stage);
  const size_t smem = 1024 + p.stages * stage + outs;
  CUtensorMap tmW1, tmH8, tmH32, tmW2;
  const auto encode = [](CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows, uint64_t stride, uint32_t box) {
    if constexpr (kFp8) return encode_u8_tmap_2d(m, base, cols, rows, stride, 128, box);
    const uint64_t dims[2] = {cols, rows}, strides[1] = {2 * stride};
    const uint32_t boxes[2] = {64, box};
    return encode_bf16_tmap(m, base, 2, dims, strides, boxes);
  };
  if (!encode(&tmW1, p.w1, p.H, (uint64_t)p.E * 2 * p.I, p.H, kTile) ||
      !encode(&tmH8, p.h, p.I, p.n, p.I, 8) || !encode(&tmH32, p.h, p.I, p.n, p.I, 32) || !encode(&tmW2, p.w2, p.I, (uint64_t)p.E * p.H, p.I, kTile))
    return EE_ERR_CUDA;
  {
    int dev = 0;
    const ee_status ds = current_device(&dev);
    if (ds != EE_OK) return ds;
    static std::mutex mu;
    static bool set[kMaxDevices] = {};
    std::lock_guard<std::mutex> lock(mu);
    if (!set[dev]) {
      EE_CUDA_OK(cudaFuncSetAttribute(moe_experts_kernel<kFp8, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, 214 * 1024));
      set[dev] = true;
    }
  }
  EE_CUDA_OK(launch_pdl(moe_experts_kernel<kFp8, NT>, dim3(kNumSMs), dim3(kThreads), smem, stream, 1, tmW1, tmH8, tmH32, tmW2, p));
  return EE_OK;
}

}  // namespace

// what both entry points take
static ee_status moe_sizes(int32_t T, int32_t H, int32_t I, int32_t E, int32_t k) {
  if (T < 0 || H < 1 || I < 1 || E < 1 || k < 1 || k > E) return EE_ERR_INVALID_ARG;
  if (H % 16 != 0 || I % 16 != 0 || H > (1 << 16) || I > (1 << 16) || E > kMoeMaxExperts || k > kMoeMaxTopK ||
      T > kMoeMaxTokens)
    return EE_ERR_UNSUPPORTED;
  return EE_OK;
}

extern "C" size_t ee_moe_workspace_size(int32_t T, int32_t H, int32_t I, int32_t E, int32_t k) {
  return moe_sizes(T, H, I, E, k) == EE_OK ? ee::moe_layout(T, H, I, E, k).total : 0;
}

extern "C" ee_status ee_moe_layer(const ee_bf16* x, int64_t x_stride, const ee_bf16* router, const void* w1,
                                  const float* w1_scale_or_null, const void* w2, const float* w2_scale_or_null, int32_t T,
                                  int32_t H, int32_t I, int32_t E, int32_t k, int32_t renorm, const int32_t* live_or_null,
                                  ee_bf16* out, int64_t out_stride, int32_t* ids_or_null, float* probs_or_null, void* ws,
                                  size_t ws_bytes, ee_stream_t stream) {
  const ee_status sizes = moe_sizes(T, H, I, E, k);
  if (sizes != EE_OK) return sizes;
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
  r.tile_rows = ee::moe_tile_rows(T, E, k, fp8);
  r.ctl = reinterpret_cast<ee::MoeCtl*>(base + l.ctl);
  r.tile = reinterpret_cast<ee::MoeTile*>(base + l.tile);
  size_t few_smem = 0;
  const bool few = ee::moe_few_stages(T, H, I, k, fp8, &few_smem) > 0;
  r.part = reinterpret_cast<float*>(base + l.part);
  r.few = few;
  r.ids = reinterpret_cast<int32_t*>(base + l.ids);
  r.prob = reinterpret_cast<float*>(base + l.prob);
  r.list = reinterpret_cast<int32_t*>(base + l.list);
  r.inv = reinterpret_cast<int32_t*>(base + l.inv);
  r.xq = fp8 ? reinterpret_cast<uint8_t*>(base + l.xq) : nullptr;
  r.xs = reinterpret_cast<float*>(base + l.xs);
  r.ids_out = ids_or_null;
  r.prob_out = probs_or_null;
  MoeParams p;
  p.T = T;
  p.H = H;
  p.I = I;
  p.E = E;
  p.k = k;
  p.n = T * k;
  p.KB1 = (H * (fp8 ? 1 : 2) + 127) / 128;
  p.KB2 = (I * (fp8 ? 1 : 2) + 127) / 128;
  p.IB = (I + kBlk - 1) / kBlk;
  p.HT = (H + 2 * kTile - 1) / (2 * kTile);
  p.HB = (H + kBlk - 1) / kBlk;
  const int nt = ee::moe_tile_rows(T, E, k, fp8);
  p.b_rows = std::min(nt, (T + 15) / 16 * 16);
  p.w1 = w1;
  p.w2 = w2;
  p.x = fp8 ? static_cast<const void*>(r.xq) : x;
  p.x_stride = fp8 ? H : x_stride;
  p.ctl = r.ctl;
  p.tile = r.tile;
  p.part = r.part;
  p.renorm = r.renorm;
  p.ids_out = ids_or_null;
  p.prob_out = probs_or_null;
  p.list = r.list;
  p.inv = r.inv;
  p.prob = r.prob;
  p.xs = r.xs;
  p.s1 = w1_scale_or_null;
  p.s2 = w2_scale_or_null;
  p.h = base + l.h;
  p.hf = reinterpret_cast<float*>(base + l.hf);
  p.hs = reinterpret_cast<float*>(base + l.hs);
  p.y = reinterpret_cast<float*>(base + l.y);
  p.out = reinterpret_cast<__nv_bfloat16*>(out);
  p.out_stride = out_stride;
  p.vec = ee::aligned(out, 8) && out_stride % 4 == 0;
  p.live = live_or_null;
  p.err = ee::err_word(ws);
  const ee_status st = ee::launch_moe_route(r, (cudaStream_t)stream);
  if (st != EE_OK) return st;
  p.cl = r.cl;
  const cudaStream_t s = (cudaStream_t)stream;
  if (few) return ee::launch_moe_few(p, fp8, s);
  if (fp8) return nt == 32 ? launch<true, 32>(p, s) : nt == 64 ? launch<true, 64>(p, s) : launch<true, 128>(p, s);
  return nt == 32 ? launch<false, 32>(p, s) : nt == 64 ? launch<false, 64>(p, s) : launch<false, 128>(p, s);
}
