// ee_moe_layer for up to 8 entries (tokens times chosen experts), after the router's product (moe_route.cu): one
// persistent kernel, a CTA an SM.  Every CTA adds up the product's parts and chooses the experts itself, which costs less than a way of the
// choice through memory.  So few experts make few tiles for the tensor cores (6 experts of 1280 x 3584 60 gate
// tasks for 152 SMs); here two groups of a producer warp and 8 consumer warps draw units from a queue:
//   gate unit    8 columns of h of one expert: a warp's MMAs take its 8 gate rows and its 8 up rows, so that a
//                lane holds both halves of silu(g) u
//   down unit    16 columns of out, over all chosen experts: their sums are weighted on the way, and no y is stored
// A group's producer streams its units' 16 weight rows in stages of up to 8 blocks of 128 bytes, one for
// each consumer (few.cuh), and runs ahead across units; the consumers add their sums at a unit's end.
// (Consumers that load their own weights spend more instructions on addresses than on products and reach 3 to
// 4.3 TB/s; here gate units run at 6.4.)  Between gate and down units lies one wait for the gate units of the other CTAs
// (all drawn before, by CTAs that are running), during which the first down units' weights are under way; then
// every CTA brings h into its own shared memory, as e4m3 codes for 8-bit weights.
// One token at 6 of 64 experts of 1280 x 3584, 8-bit: 29 us, by the tiles of moe_experts.cu 33; at 2 of 8 of 2560: 25 and 34; at
// 4 of 60 of 512 x 1024, bf16: 14 and 22; 8 tokens at 1 of 8 of 2560, 8-bit: 40 and 39.  8 entries are what an MMA's columns and the tables
// hold; more are those tiles'.
#include <mutex>

#include "moe.cuh"

namespace {

using namespace ee;

constexpr int kGroups = 2;
constexpr int kThreads = 32 * kGroups * (1 + kFewWarps);      // warps 0 and 1 produce
constexpr int kMaxDeep = 6;            // stages in a group's ring, at most
constexpr int kMinDeep = 3;
constexpr size_t kMostSmem = 204 * 1024;

// bytes of a row of x or h in shared memory: rows two by two on different banks
__host__ __device__ constexpr int row_stride(int KB) { return KB * 128 + 64; }
__host__ __device__ constexpr int stages_of(int KB) { return (KB + kFewWarps - 1) / kFewWarps; }
__host__ __device__ constexpr int blocks_of(int KB) { return (KB + stages_of(KB) - 1) / stages_of(KB); }   // of a stage

__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}

template <bool kFp8>
__global__ void __launch_bounds__(kThreads, 1)
moe_few_kernel(const __grid_constant__ CUtensorMap tmW1, const __grid_constant__ CUtensorMap tmW2, const MoeParams p) {
  constexpr int es = kFp8 ? 1 : 2, NT = kFewTokens;
  extern __shared__ uint8_t s_raw[];                           // the rings; rows of x, later of h; their scales
  uint8_t* const s_dyn = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(s_raw) + 127) & ~static_cast<uintptr_t>(127));
  __shared__ __align__(8) uint64_t s_bars[kGroups * (2 * kMaxDeep + 1) + 1];
  __shared__ float s_ws[kGroups][kMaxDeep][kFewWarps][2];      // scales of a stage's blocks: of rows 0 .. 7 and 8 .. 15
  __shared__ int s_unit[kGroups][kMaxDeep];
  __shared__ float s_part[kGroups][2][kFewWarps][16][kFewTokens];
  __shared__ float s_p[kFewEntries][kFewTokens];               // an active expert's weight for a token
  __shared__ int16_t s_map[kFewEntries][kFewTokens];           // ... and the entry, or -1
  __shared__ int s_exp[kFewEntries];
  __shared__ int s_ids[kFewEntries], s_active;                 // experts of a token's j-th place; how many different ones
  __shared__ float s_prob[kFewEntries];
  __shared__ int s_done[kGroups];                              // gate units of the group
  __shared__ volatile int s_abort;
  pdl_allow_next();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int D = p.stages;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int g = 0; g < kGroups; ++g) {
      const uint32_t b = smem_u32(s_bars) + 8 * (uint32_t)(g * (2 * kMaxDeep + 1));
      for (int i = 0; i < D; ++i) {
        mbar_init(b + 8 * i, kFp8 ? 1 + 2 * kFewWarps : 1);
        mbar_init(b + 8 * (kMaxDeep + i), kFewWarps);
      }
      mbar_init(b + 8 * 2 * kMaxDeep, kFewWarps);
    }
    mbar_init(smem_u32(s_bars) + 8 * (kGroups * (2 * kMaxDeep + 1)), kGroups * kFewWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmW1)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmW2)) : "memory");
  }
  pdl_wait();
  // All of a thread's loads are under way before the first is waited for.
  int first = 0;
  if (warp < kGroups && lane == 0) first = (int)atomicAdd(&p.ctl->queue, 1u);
  const int live = p.live ? max(0, min(p.T, ld_pinned(p.live))) : p.T;
  uint8_t* const s_rows = s_dyn + (size_t)kGroups * D * (16u * 128u * (uint32_t)max(blocks_of(p.KB1), blocks_of(p.KB2)));
  const int h_bytes = p.H * es, i_bytes = p.I * es, xs = row_stride(p.KB1);
  float* const s_xs = reinterpret_cast<float*>(s_rows + (size_t)p.T * xs);   // [T][KB1]
  const int chunks = p.KB1 * 8, logits = p.T * p.E;            // of 16 bytes; of tokens behind the live ones nobody looks at
  float part[kRouteParts];                                     // either
  uint4 v = make_uint4(0, 0, 0, 0);
  float sv = 0.f;
#pragma unroll
  for (int r = 0; r < kRouteParts; ++r)
    if (r < p.cl && (int)threadIdx.x < logits) part[r] = ld_pinned_f(p.part + (size_t)r * logits + threadIdx.x);
  const auto x_at = [&](int i) {                               // NULL: zeros
    const int t = i / chunks, c = i % chunks * 16;
    return t < p.T && c < h_bytes ? static_cast<const uint8_t*>(p.x) + (size_t)t * p.x_stride * es + c : nullptr;
  };
  if (const uint8_t* at = x_at((int)threadIdx.x)) v = ld_pinned16(at);
  const auto xs_at = [&](int i) { return p.xs + (size_t)(i % p.KB1) * p.T + i / p.KB1; };
  if (kFp8 && (int)threadIdx.x < p.T * p.KB1) sv = ld_pinned_f(xs_at((int)threadIdx.x));
  // the routing's parts of the logits in a fixed order
  float* const s_logit = &s_part[0][0][0][0][0];               // [T][E], in front of the units' sums
  static_assert(sizeof(s_part) >= kFewTokens * kMoeMaxExperts * sizeof(float));
  for (int i = threadIdx.x; i < logits; i += kThreads) {
    if (i >= kThreads)
#pragma unroll
      for (int r = 0; r < kRouteParts; ++r)
        if (r < p.cl) part[r] = ld_pinned_f(p.part + (size_t)r * logits + i);
    float f = part[0];
#pragma unroll
    for (int r = 1; r < kRouteParts; ++r)
      if (r < p.cl) f += part[r];
    s_logit[i] = f;
  }
  if (threadIdx.x < kFewEntries * NT) s_map[threadIdx.x / NT][threadIdx.x % NT] = -1;
  __syncthreads();
  if (warp < live) {                                           // a warp a token (live is at most 8)
    const MoeChoice c = choose_experts(s_logit + warp * p.E, p.E, p.k, p.renorm, lane);
    if (lane < p.k) {
      s_ids[warp * p.k + c.place] = c.expert;
      s_prob[warp * p.k + c.place] = c.p;
      const size_t at = (size_t)warp * p.k + c.place;
      if (blockIdx.x == 0 && p.ids_out) p.ids_out[at] = c.expert;
      if (blockIdx.x == 0 && p.prob_out) p.prob_out[at] = c.p;
    }
  }
  // x, and behind it the next barrier: a thread's first pieces are here by now
  for (int i = threadIdx.x; i < p.T * chunks; i += kThreads) {
    if (i >= kThreads) {
      const uint8_t* at = x_at(i);
      v = at ? ld_pinned16(at) : make_uint4(0, 0, 0, 0);
    }
    *reinterpret_cast<uint4*>(s_rows + (size_t)(i / chunks) * xs + i % chunks * 16) = v;
  }
  if constexpr (kFp8)
    for (int i = threadIdx.x; i < p.T * p.KB1; i += kThreads) s_xs[i] = i < kThreads ? sv : *xs_at(i);
  __syncthreads();
  if (warp == 0) {                                             // entries by expert, then by token; lane: an entry
    const int n = live * p.k;
    const int e = lane < n ? s_ids[lane] : 0x7fffffff, t = lane < n ? lane / p.k : 0;
    int pos = 0, active = 0;
    bool one = lane < n;                                       // the first of its expert
    for (int j = 0; j < n; ++j) {
      const int ej = __shfl_sync(0xffffffffu, e, j);
      pos += ej < e || (ej == e && j < lane);                  // (lanes are in the order of their tokens)
      if (ej == e && j < lane) one = false;
    }
    const uint32_t ones = __ballot_sync(0xffffffffu, one);
    for (int j = 0; j < n; ++j) active += (ones >> j & 1u) && __shfl_sync(0xffffffffu, e, j) < e;
    if (lane < n) {
      s_exp[active] = e;                                       // (the same from all of its entries)
      s_map[active][t] = (int16_t)pos;
      s_p[active][t] = s_prob[lane];
    }
    if (lane == 0) s_active = __popc(ones);
  }
  __syncthreads();
  const int na = s_active;
  const int per = p.I / 8, gates = na * per, total = gates + (na ? (p.H + 15) / 16 : 0);
  const int nst1 = stages_of(p.KB1), nst2 = stages_of(p.KB2), c1 = blocks_of(p.KB1), c2 = blocks_of(p.KB2);
  const uint32_t stBytes = 16u * 128u * (uint32_t)max(c1, c2);
  const int grp = warp < kGroups ? warp : (warp - kGroups) / kFewWarps;
  const uint32_t ring = smem_u32(s_dyn) + (uint32_t)(grp * D) * stBytes;
  const uint32_t full0 = smem_u32(s_bars) + 8 * (uint32_t)(grp * (2 * kMaxDeep + 1)), empty0 = full0 + 8 * kMaxDeep,
                 meet = empty0 + 8 * kMaxDeep, meet_all = smem_u32(s_bars) + 8 * (kGroups * (2 * kMaxDeep + 1));
  int slot = 0;
  uint32_t phase = 0;
  const auto advance = [&]() {
    if (++slot == D) {
      slot = 0;
      phase ^= 1;
    }
  };

  if (warp < kGroups) {
    // ---- producer ---------------------------------------------------------------------
    // (uniform values and an elected lane: see moe_experts.cu)
    const uint32_t u_ring = __shfl_sync(0xffffffffu, ring, 0), u_full = __shfl_sync(0xffffffffu, full0, 0);
    const int ug = __shfl_sync(0xffffffffu, grp, 0), una = __shfl_sync(0xffffffffu, na, 0);
    const int ugates = una * per, utotal = __shfl_sync(0xffffffffu, total, 0);
    const uint64_t policy = policy_evict_first();
    int issued = 0;
    bool ok = true;
    int u = __shfl_sync(0xffffffffu, first, 0);
    while (ok) {
      const bool end = u >= utotal, gate = u < ugates;
      int next = 0;
      if (!end && lane == 0) next = (int)atomicAdd(&p.ctl->queue, 1u);
      const int na_u = end || gate ? 1 : una, nst = end ? 1 : gate ? nst1 : nst2;
      const int col = gate ? u % per * 8 : (u - ugates) * 16;
      for (int i = 0; i < na_u && ok; ++i) {
        const int a = end ? 0 : gate ? u / per : i;
        const int e = __shfl_sync(0xffffffffu, s_exp[a], 0);
        const int y = gate ? e * 2 * p.I + col : e * p.H + col;
        for (int ch = 0; ch < nst; ++ch) {
          if (!__all_sync(0xffffffffu, mbar_wait(empty0 + 8 * slot, phase ^ 1, &s_abort))) {
            ok = false;
            break;
          }
          const uint32_t fb = u_full + 8 * slot, at = u_ring + (uint32_t)slot * stBytes;
          if (elect_one()) {
            s_unit[ug][slot] = u;
            if (end) {
              mbar_arrive(fb);
            } else if (gate) {
              mbar_expect_tx(fb, 16u * 128u * (uint32_t)c1);
              tma_load_2d_hint(at, &tmW1, fb, ch * c1 * 32, y, policy);
              tma_load_2d_hint(at + 8u * 128u * (uint32_t)c1, &tmW1, fb, ch * c1 * 32, y + p.I, policy);
            } else {
              mbar_expect_tx(fb, 16u * 128u * (uint32_t)c2);
              tma_load_2d_hint(at, &tmW2, fb, ch * c2 * 32, y, policy);
            }
          }
          if (kFp8 && lane < 2 * kFewWarps) {
            const int b = lane >> 1, which = lane & 1, kb = ch * (gate ? c1 : c2) + b;
            const uint32_t to = smem_u32(&s_ws[grp][slot][b][which]);
            if (!end && b < (gate ? c1 : c2) && kb < (gate ? p.KB1 : p.KB2)) {
              const float* ws = gate ? p.s1 + (((size_t)e * 2 + which) * p.IB + col / kBlk) * p.KB1 + kb
                                     : p.s2 + ((size_t)e * p.HB + col / kBlk) * p.KB2 + kb;
              asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(ws) : "memory");
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(fb) : "memory");
          }
          __syncwarp();
          if (!end) ++issued;
          advance();
        }
      }
      if (end) break;
      u = __shfl_sync(0xffffffffu, next, 0);
    }
    cp_async_wait_all();
    // the copies under way have to land before the CTA ends (a unit that says the end has taken the place of
    // the oldest, which was consumed)
    for (int k = max(0, issued - D + (ok ? 1 : 0)); k < issued; ++k)
      if (!mbar_wait_plain(full0 + 8 * (k % D), (uint32_t)((k / D) & 1))) break;
  } else {
    // ---- consumers --------------------------------------------------------------------
    const int w = (warp - kGroups) % kFewWarps, g = lane >> 2, tq = lane & 3;
    const int ct = (int)threadIdx.x - 32 * kGroups, gt = ct % (32 * kFewWarps);   // thread of all consumers, of the group
    const int hs = row_stride(p.KB2);
    float* const s_hs = reinterpret_cast<float*>(s_rows + (size_t)p.n * hs);   // [n][IB]
    uint32_t met = 0, met_all = 0;
    // a meeting of the group's consumers (or all): false when it was given up
    const auto meet_at = [&](uint32_t bar, uint32_t& count) {
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
      return (bool)__all_sync(0xffffffffu, mbar_wait(bar, count++ & 1, &s_abort));
    };
    bool ok = true;
    const int last = max(live, 1) - 1;
    const int t0 = min(2 * tq, last), t1 = min(2 * tq + 1, last);
    const uint32_t xrow = smem_u32(s_rows) + (uint32_t)(min(g, p.T - 1) * xs + tq * 16);
    const uint32_t wat = (uint32_t)(w * 128 + tq * 16);
    int done = 0, u = 0;
    while (ok) {
      ok = __all_sync(0xffffffffu, mbar_wait(full0 + 8 * slot, phase, &s_abort));
      if (!ok) break;
      u = s_unit[grp][slot];
      if (u >= gates) break;
      const int a = u / per, i8 = u % per, turn = done & 1;
      float acc[4] = {0.f, 0.f, 0.f, 0.f};
      for (int ch = 0; ch < nst1; ++ch) {
        if (ch > 0 && !__all_sync(0xffffffffu, mbar_wait(full0 + 8 * slot, phase, &s_abort))) {
          ok = false;
          break;
        }
        const int kb = ch * c1 + w;
        if (w < c1 && kb < p.KB1) {
          const uint32_t r0 = ring + (uint32_t)slot * stBytes + (uint32_t)(g * c1 * 128) + wat, r1 = r0 + (uint32_t)(8 * c1 * 128);
          FewFrag fa, fb;
          fa.lo = lds16(r0);
          fa.hi = lds16(r0 + 64);
          fb.lo = lds16(r1);
          fb.hi = lds16(r1 + 64);
          FewFrag fx;
          fx.lo = lds16(xrow + (uint32_t)kb * 128);            // (rows past T: a copy of the last one, not looked at)
          fx.hi = lds16(xrow + (uint32_t)kb * 128 + 64);
          if constexpr (kFp8) {
            const float x0 = s_xs[t0 * p.KB1 + kb], x1 = s_xs[t1 * p.KB1 + kb];
            const float w0 = s_ws[grp][slot][w][0], w1 = s_ws[grp][slot][w][1];
            float d[4] = {0.f, 0.f, 0.f, 0.f};
            few_block<true>(d, fa, fb, fx);
            acc[0] = __fmaf_rn(d[0], x0 * w0, acc[0]);
            acc[1] = __fmaf_rn(d[1], x1 * w0, acc[1]);
            acc[2] = __fmaf_rn(d[2], x0 * w1, acc[2]);
            acc[3] = __fmaf_rn(d[3], x1 * w1, acc[3]);
          } else {
            few_block<false>(acc, fa, fb, fx);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty0 + 8 * slot);
        advance();
      }
      if (!ok) break;
      float(*part)[16][NT] = s_part[grp][turn];
      *reinterpret_cast<float2*>(&part[w][g][2 * tq]) = make_float2(acc[0], acc[1]);
      *reinterpret_cast<float2*>(&part[w][g + 8][2 * tq]) = make_float2(acc[2], acc[3]);
      ok = meet_at(meet, met);
      if (!ok) break;
      ++done;
      constexpr int kSumWarps = NT * 8 / 32;                   // others in turn: token t, column o
      if (w / kSumWarps == done % (kFewWarps / kSumWarps)) {
        const int t = gt / 8 % NT, o = gt & 7;
        const int entry = s_map[a][t];
        if (entry >= 0) {
          float gs = part[0][o][t], us = part[0][o + 8][t];
#pragma unroll
          for (int i = 1; i < kFewWarps; ++i) {
            gs += part[i][o][t];
            us += part[i][o + 8][t];
          }
          const float h = silu_times(gs, us);
          const size_t at = (size_t)entry * p.I + i8 * 8 + o;
          if constexpr (kFp8) __stcg(p.hf + at, h);
          else static_cast<__nv_bfloat16*>(p.h)[at] = __float2bfloat16_rn(h);
        }
      }
    }
    if (gt == 0) s_done[grp] = done;

    // ---- h, once it is there: one release for all of this CTA's gate units --------------
    ok = ok && meet_at(meet_all, met_all);
    if (ok && ct == 0) {
      int n = 0;
      for (int i = 0; i < kGroups; ++i) n += s_done[i];
      red_add_release(&p.ctl->down_done, (uint32_t)n);
      if (!wait_count_geq(&p.ctl->down_done, (uint32_t)gates)) s_abort = 1;
    }
    ok = ok && meet_at(meet_all, met_all);
    const int n = live * p.k;
    if (ok) {
      if constexpr (kFp8) {
        constexpr int kAll = kGroups * kFewWarps;
        for (int i0 = ct >> 5; i0 < n * p.IB; i0 += kAll * 8) {   // a block a warp, eight loads in flight
          float4 v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * kAll, m = i / p.IB, col = i % p.IB * kBlk + 4 * lane;
            v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i < n * p.IB && col < p.I) v[j] = __ldcg(reinterpret_cast<const float4*>(p.hf + (size_t)m * p.I + col));
          }
          uint32_t my_top = 0;                                 // lane j: of the j-th block
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t k = 0x7fffffffu;
            const uint32_t top = __reduce_max_sync(0xffffffffu, max(max(__float_as_uint(v[j].x) & k, __float_as_uint(v[j].y) & k),
                                                                    max(__float_as_uint(v[j].z) & k, __float_as_uint(v[j].w) & k)));
            if (lane == j) my_top = top;
          }
          const BlockScale mine = block_scale(__uint_as_float(my_top));
          if (lane < 8 && i0 + lane * kAll < n * p.IB) s_hs[i0 + lane * kAll] = mine.scale;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * kAll, m = i / p.IB, b = i % p.IB;
            BlockScale s;
            s.hi = __shfl_sync(0xffffffffu, mine.hi, j);
            s.lo = __shfl_sync(0xffffffffu, mine.lo, j);
            if (i < n * p.IB)
              *reinterpret_cast<uint32_t*>(s_rows + (size_t)m * hs + b * kBlk + 4 * lane) =
                  pack_e4m3(to_code(v[j].x, s), to_code(v[j].y, s), to_code(v[j].z, s), to_code(v[j].w, s));
          }
        }
      } else {
        constexpr int kAll = 32 * kGroups * kFewWarps;
        const int chunks = p.KB2 * 8;                          // 16 bytes
        for (int i0 = ct; i0 < n * chunks; i0 += kAll * 4) {
          uint4 v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * kAll, m = i / chunks, b = i % chunks * 16;
            v[j] = make_uint4(0, 0, 0, 0);
            if (i < n * chunks && b < i_bytes)
              v[j] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.h) + (size_t)m * i_bytes + b));
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * kAll;
            if (i < n * chunks) *reinterpret_cast<uint4*>(s_rows + (size_t)(i / chunks) * hs + i % chunks * 16) = v[j];
          }
        }
      }
      ok = meet_at(meet_all, met_all);
    }

    while (ok) {
      ok = __all_sync(0xffffffffu, mbar_wait(full0 + 8 * slot, phase, &s_abort));
      if (!ok) break;
      u = s_unit[grp][slot];
      if (u >= total) break;
      const int o0 = (u - gates) * 16, turn = done & 1;
      float acc[4] = {0.f, 0.f, 0.f, 0.f};
      int a = 0, ch = 0;
      for (int i = 0; i < na * nst2; ++i) {
        if (i > 0 && !__all_sync(0xffffffffu, mbar_wait(full0 + 8 * slot, phase, &s_abort))) {
          ok = false;
          break;
        }
        const int kb = ch * c2 + w;
        if (w < c2 && kb < p.KB2) {
          const uint32_t r0 = ring + (uint32_t)slot * stBytes + (uint32_t)(g * c2 * 128) + wat, r1 = r0 + (uint32_t)(8 * c2 * 128);
          FewFrag fa, fb;
          fa.lo = lds16(r0);
          fa.hi = lds16(r0 + 64);
          fb.lo = lds16(r1);
          fb.hi = lds16(r1 + 64);
          const float ws = kFp8 ? s_ws[grp][slot][w][0] : 1.f;
          const int m = s_map[a][g], m0 = s_map[a][2 * tq], m1 = s_map[a][2 * tq + 1];
          FewFrag fx;
          fx.lo = fx.hi = make_uint4(0, 0, 0, 0);
          if (m >= 0) {
            const uint32_t r = smem_u32(s_rows) + (uint32_t)(m * hs + kb * 128 + tq * 16);
            fx.lo = lds16(r);
            fx.hi = lds16(r + 64);
          }
          float d[4] = {0.f, 0.f, 0.f, 0.f};
          few_block<kFp8>(d, fa, fb, fx);
          if (m0 >= 0) {                                       // (a token at other experts takes nothing, not even a NaN)
            const float f = kFp8 ? s_p[a][2 * tq] * (s_hs[m0 * p.IB + kb] * ws) : s_p[a][2 * tq];
            acc[0] = __fmaf_rn(d[0], f, acc[0]);
            acc[2] = __fmaf_rn(d[2], f, acc[2]);
          }
          if (m1 >= 0) {
            const float f = kFp8 ? s_p[a][2 * tq + 1] * (s_hs[m1 * p.IB + kb] * ws) : s_p[a][2 * tq + 1];
            acc[1] = __fmaf_rn(d[1], f, acc[1]);
            acc[3] = __fmaf_rn(d[3], f, acc[3]);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty0 + 8 * slot);
        advance();
        if (++ch == nst2) {
          ch = 0;
          ++a;
        }
      }
      if (!ok) break;
      float(*part)[16][NT] = s_part[grp][turn];
      *reinterpret_cast<float2*>(&part[w][g][2 * tq]) = make_float2(acc[0], acc[1]);
      *reinterpret_cast<float2*>(&part[w][g + 8][2 * tq]) = make_float2(acc[2], acc[3]);
      ok = meet_at(meet, met);
      if (!ok) break;
      ++done;
      const int t = gt >> 4, o = gt & 15;
      if (t < live && o0 + o < p.H) {                          // (live is at most 8)
        float f = part[0][o][t];
#pragma unroll
        for (int i = 1; i < kFewWarps; ++i) f += part[i][o][t];
        p.out[(int64_t)t * p.out_stride + o0 + o] = __float2bfloat16_rn(f);
      }
    }
    if (!ok && lane == 0) flag_error(p.err, EE_DEVERR_TIMEOUT);
  }
}

template <bool kFp8>
ee_status launch(const MoeParams& p, size_t smem, cudaStream_t stream) {
  constexpr uint64_t es = kFp8 ? 1 : 2;
  CUtensorMap tmW1, tmW2;
  if (!encode_u32_tmap_2d(&tmW1, p.w1, p.H * es / 4, (uint64_t)p.E * 2 * p.I, p.H * es, (uint32_t)blocks_of(p.KB1) * 32, 8) ||
      !encode_u32_tmap_2d(&tmW2, p.w2, p.I * es / 4, (uint64_t)p.E * p.H, p.I * es, (uint32_t)blocks_of(p.KB2) * 32, 16))
    return EE_ERR_CUDA;
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
  EE_CUDA_OK(launch_pdl(moe_few_kernel<kFp8>, dim3(kNumSMs), dim3(kThreads), smem, stream, 1, tmW1, tmW2, p));
  return EE_OK;
}

}  // namespace

namespace ee {

int moe_few_stages(int T, int H, int I, int k, bool fp8, size_t* smem) {
  if (T * k > kFewEntries) return 0;
  const size_t es = fp8 ? 1 : 2, KB1 = (H * es + 127) / 128, KB2 = (I * es + 127) / 128;
  const size_t x = (size_t)T * (row_stride((int)KB1) + 4 * KB1), h = (size_t)T * k * (row_stride((int)KB2) + 4 * KB2);
  const size_t rows = std::max(x, h), stage = 16 * 128 * (size_t)std::max(blocks_of((int)KB1), blocks_of((int)KB2));
  if (128 + rows + kGroups * kMinDeep * stage > kMostSmem) return 0;
  const size_t deep = std::min<size_t>(kMaxDeep, (kMostSmem - 128 - rows) / (kGroups * stage));
  *smem = 128 + rows + kGroups * deep * stage;
  return (int)deep;
}

ee_status launch_moe_few(MoeParams& p, bool fp8, cudaStream_t stream) {
  size_t smem = 0;
  p.stages = moe_few_stages(p.T, p.H, p.I, p.k, fp8, &smem);
  return fp8 ? launch<true>(p, smem, stream) : launch<false>(p, smem, stream);
}

}  // namespace ee
