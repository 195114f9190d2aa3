// First kernel of ee_moe_layer: the router's product, each token's experts and their
// probabilities, x as e4m3 codes (for 8-bit weights), and the tokens grouped by expert.
//
// A CTA takes 16 tokens, 8 or 64 experts and up to an eighth of the hidden dimension: an m16n8k16 MMA
// of bf16 a warp and 16 columns, operands straight from global memory (a lane takes 8
// neighbouring columns of its row of x and of the router; the order of the columns within
// a sum is free, so x's and the router's fragments need only agree).  2 T E H operations are too few for
// the tensor memory's set-up; what bounds the kernel is the chain of waits for memory, of its instructions, too, which
// weights of the layer in front have driven out: the loop over 64 experts alone takes 3 to 4 us then, over 8 1, so there are
// CTAs for every 8 experts as long as the SMs hold them at once.  Warps' sums are added in shared memory, CTAs' through a
// cluster's, or by the last of a token group's CTAs through global memory, always in the same order; then the experts are chosen.  The last
// CTA to finish groups the tokens: a bit for each expert and token, so that an entry's place is a count of bits and does not depend on who comes first.
// Of up to 8 entries only the CTAs' sums are made here (moe_few.cu).  CTAs of their own quantise x.
// Alone on cold caches: one token's sums 5 us, 64 tokens 11 to 12.5, 300 tokens 13.
#include <mutex>

#include "moe.cuh"

namespace {

using namespace ee;

constexpr int kTok = 16, kQuantUnits = 4, kWarps = 16, kThreads = 32 * kWarps;

__device__ __forceinline__ float ld_cluster_f(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// NT: groups of 8 experts of a CTA; kCluster: a token group's CTAs are a cluster
template <int NT, bool kCluster>
__global__ void __launch_bounds__(kThreads) moe_route_kernel(const RouteParams p, const int keep) {
  constexpr int EP = 8 * NT;
  extern __shared__ float s_red[];                 // [kWarps][kTok][EP]; the logits [kTok][E]
  __shared__ int s_last;
  __shared__ int s_ids[kTok * kMoeMaxTopK];        // of a single group's tokens
  __shared__ float s_prob[kTok * kMoeMaxTopK];
  __shared__ uint32_t s_bits[kMoeMaxExperts];      // ... a bit for each expert and token
  __shared__ uint32_t s_scan[kWarps];
  pdl_allow_next();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // the grid is CTAs that share the columns x those that share the experts x token groups, then those that quantise
  // (a division costs more than it looks where its instructions come from memory)
  const int groups = (p.T + kTok - 1) / kTok, parts = (int)(gridDim.x * gridDim.y);
  const int rank = (int)blockIdx.x, e0 = (int)blockIdx.y * EP, group = (int)blockIdx.z, t0 = group * kTok;
  const bool first = rank == 0 && e0 == 0;
  const bool alone = groups == 1;
  if (alone)
    for (int i = threadIdx.x; i < kMoeMaxExperts; i += kThreads) s_bits[i] = 0;
  if (t0 == 0) {      // this CTA's columns of the router, while the kernel in front still runs
    const int blocks = (p.H + kBlk - 1) / kBlk, c0 = blocks * rank / p.cl * kBlk, c1 = min(p.H, blocks * (rank + 1) / p.cl * kBlk);
    if (c0 < c1)
      for (int e = e0 + (int)threadIdx.x; e < min(p.E, e0 + EP); e += kThreads) prefetch_l2(p.router + (size_t)e * p.H + c0, (uint32_t)(c1 - c0) * 2);
  }
  pdl_wait();
  const int live = p.live ? max(0, min(p.T, ld_pinned(p.live))) : p.T;
  if (first && group == 0 && threadIdx.x == 0) {
    p.ctl->queue = 0;
    p.ctl->down_done = 0;
  }
  if (group >= groups) {                // x as codes: a warp and a block of one token, four at once
    const int blocks = (p.H + kBlk - 1) / kBlk, units = live * blocks;
    const int u0 = ((((group - groups) * (int)gridDim.y + (int)blockIdx.y) * p.cl + rank) * kWarps + warp) * kQuantUnits;
    uint2 v[kQuantUnits];
#pragma unroll
    for (int j = 0; j < kQuantUnits; ++j) {
      const int u = u0 + j, t = u / blocks, col = u % blocks * kBlk + lane * 4;
      v[j] = make_uint2(0, 0);
      if (u < units && col < p.H) v[j] = *reinterpret_cast<const uint2*>(p.x + t * p.x_stride + col);
    }
#pragma unroll
    for (int j = 0; j < kQuantUnits; ++j) {
      const int u = u0 + j, t = u / blocks, b = u % blocks, col = b * kBlk + lane * 4;
      if (u >= units) break;
      const uint32_t a = __vmaxu2(v[j].x & 0x7fff7fffu, v[j].y & 0x7fff7fffu);
      const uint32_t top = __reduce_max_sync(0xffffffffu, max(a & 0xffffu, a >> 16));
      const BlockScale s = block_scale(__uint_as_float(top << 16));
      if (col < p.H)
        *reinterpret_cast<uint32_t*>(p.xq + (size_t)t * p.H + col) =
            pack_e4m3(to_code(bf16_lo(v[j].x), s), to_code(bf16_hi(v[j].x), s), to_code(bf16_lo(v[j].y), s),
                      to_code(bf16_hi(v[j].y), s));
      if (lane == 0) p.xs[(size_t)b * p.T + t] = s.scale;
    }
    return;
  }
  if (t0 < live) {
    const int nb = (p.H + kBlk - 1) / kBlk;
    const int b0 = nb * rank / p.cl, b1 = nb * (rank + 1) / p.cl;
    const int g = lane >> 2, tq = lane & 3;
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int c = b0 * 4 + warp; c < b1 * 4; c += kWarps) {
      const int col = c * 32 + tq * 8;
      const bool in = col < p.H;
      uint4 xa = zero, xb = zero;
      if (in && t0 + g < live) xa = ld_pinned16(p.x + (t0 + g) * p.x_stride + col);
      if (in && t0 + g + 8 < live) xb = ld_pinned16(p.x + (t0 + g + 8) * p.x_stride + col);
      constexpr int kStep = NT < 8 ? NT : 8;
#pragma unroll
      for (int n0 = 0; n0 < NT; n0 += kStep) {
        uint4 w[kStep];
#pragma unroll
        for (int n = 0; n < kStep; ++n) {
          const int e = e0 + (n0 + n) * 8 + g;
          w[n] = zero;
          if (in && e < p.E) w[n] = ld_pinned16(p.router + (size_t)e * p.H + col);
        }
#pragma unroll
        for (int n = 0; n < kStep; ++n) {
          mma_16816(acc[n0 + n], xa.x, xb.x, xa.y, xb.y, w[n].x, w[n].y);
          mma_16816(acc[n0 + n], xa.z, xb.z, xa.w, xb.w, w[n].z, w[n].w);
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float* r = s_red + ((size_t)warp * kTok + g) * EP + n * 8 + 2 * tq;
      *reinterpret_cast<float2*>(r) = make_float2(acc[n][0], acc[n][1]);
      *reinterpret_cast<float2*>(r + 8 * EP) = make_float2(acc[n][2], acc[n][3]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kTok * EP; i += kThreads) {
      float s = s_red[i];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) s += s_red[w * kTok * EP + i];
      const int row = i / EP, e = e0 + i % EP;
      if (kCluster) s_red[i] = s;
      else if (t0 + row < live && e < p.E) p.part[((size_t)rank * p.T + t0 + row) * p.E + e] = s;
    }
    if (!kCluster && p.few) return;
    const int rows = min(kTok, live - t0);
    int row = warp;                                // a warp chooses a token's experts
    if constexpr (kCluster) {
      if (p.cl > 1) cluster_sync();
      else __syncthreads();
      // the cluster's CTAs take the tokens in turn, a single group's first CTA all of them
      row = !alone ? rank + p.cl * warp : rank == 0 ? warp : kTok;
    } else {                                       // the last of the group's CTAs all of them
      __syncthreads();
      if (threadIdx.x == 0) s_last = atom_add_acq_rel(&p.ctl->group_ticket[group], 1u) == (uint32_t)parts - 1;
      __syncthreads();
      if (!s_last) return;
      if (threadIdx.x == 0) p.ctl->group_ticket[group] = 0;
      for (int i = threadIdx.x; i < rows * p.E; i += kThreads) {
        float part[kRouteParts];
#pragma unroll
        for (int r = 0; r < kRouteParts; ++r)
          if (r < p.cl) part[r] = __ldcg(p.part + ((size_t)r * p.T + t0) * p.E + i);
        float f = part[0];
#pragma unroll
        for (int r = 1; r < kRouteParts; ++r)
          if (r < p.cl) f += part[r];
        s_red[i] = f;
      }
      __syncthreads();
    }
    if (row < rows) {
      const auto sum_of = [&](int e) {
        const uint32_t at = smem_u32(s_red + row * EP + e);
        float part[kRouteParts];
#pragma unroll
        for (int r = 0; r < kRouteParts; ++r)
          if (r < p.cl) part[r] = p.cl > 1 ? ld_cluster_f(map_cluster(at, r)) : s_red[row * EP + e];
        float f = part[0];
#pragma unroll
        for (int r = 1; r < kRouteParts; ++r)
          if (r < p.cl) f += part[r];
        return f;
      };
      MoeChoice ch;
      if constexpr (kCluster) ch = choose_of<(EP + 31) / 32>(sum_of, p.E, p.k, p.renorm, lane);
      else ch = choose_experts(s_red + row * p.E, p.E, p.k, p.renorm, lane);
      if (lane < p.k) {
        const size_t at = (size_t)(t0 + row) * p.k + ch.place;
        if (alone) {
          atomicOr(&s_bits[ch.expert], 1u << row);
          s_ids[at] = ch.expert;
          s_prob[at] = ch.p;
        } else {
          p.ids[at] = ch.expert;
          p.prob[at] = ch.p;
        }
        if (p.ids_out) p.ids_out[at] = ch.expert;
        if (p.prob_out) p.prob_out[at] = ch.p;
      }
    }
    // nobody leaves while a peer reads its sums; who groups a single cluster's tokens waits at its end
    if (kCluster && p.cl > 1) {
      asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
      if (!alone || rank != 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
  } else if (!kCluster && (p.few || !first)) {
    return;
  }

  // ---- the last CTA groups the tokens by expert --------------------------------------
  const int words = (live + 31) >> 5, n = live * p.k;
  uint32_t* mask = alone ? s_bits : reinterpret_cast<uint32_t*>(s_red);   // [E][words]
  uint16_t* pre = reinterpret_cast<uint16_t*>(reinterpret_cast<uint32_t*>(s_red) + p.E * words);   // bits in an expert's earlier words
  int* s_off = reinterpret_cast<int*>(pre + ((p.E * words + 1) & ~1));
  uint8_t* s_e = reinterpret_cast<uint8_t*>(s_off + p.E);                 // [n] expert of a token's j-th place (where keep)
  __syncthreads();
  if (alone) {
    if (kCluster && rank != 0) return;
  } else {
    if (threadIdx.x == 0)
      s_last = atom_add_acq_rel(&p.ctl->route_ticket, 1u) == (uint32_t)(kCluster ? groups * p.cl : groups) - 1;
    for (int i = threadIdx.x; i < p.E * words; i += kThreads) mask[i] = 0;
    __syncthreads();
    if (!s_last) return;
  }
  for (int i = threadIdx.x; i < p.max_tiles; i += kThreads) p.ctl->gate_done[i] = 0;
  if (threadIdx.x == 0) p.ctl->route_ticket = 0;
  constexpr int kAhead = 4;                        // entries of a thread whose loads are under way together
  for (int i0 = threadIdx.x; i0 < n && !alone; i0 += kThreads * kAhead) {
    int e[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = i0 + j * kThreads;
      if (i < n) e[j] = __ldcg(p.ids + i);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = i0 + j * kThreads, t = i / p.k;
      if (i < n) {
        atomicOr(&mask[e[j] * words + (t >> 5)], 1u << (t & 31));
        if (keep) s_e[i] = (uint8_t)e[j];
      }
    }
  }
  if (!alone) __syncthreads();
  int cnt = 0;                                     // (at most 256 experts: thread e counts expert e's)
  if ((int)threadIdx.x < p.E)
    for (int w = 0; w < words; ++w) {
      pre[threadIdx.x * words + w] = (uint16_t)cnt;
      cnt += __popc(mask[threadIdx.x * words + w]);
    }
  // running numbers of entries and tiles in one scan (at most 2^16 entries, 2^11 tiles)
  const int tiles = (cnt + p.tile_rows - 1) / p.tile_rows;
  const uint32_t own = (uint32_t)cnt | (uint32_t)tiles << 20;
  uint32_t incl = own;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) s_scan[warp] = incl;
  __syncthreads();
  for (int w = 0; w < warp; ++w) incl += s_scan[w];
  if ((int)threadIdx.x < p.E) {
    const uint32_t before = incl - own;
    MoeTile m;
    m.expert = (int)threadIdx.x;
    m.entry0 = (int)(before & 0xfffffu);
    m.count = cnt;
    m.first = (int)(before >> 20);
    m.tiles = tiles;
    m.pad[0] = m.pad[1] = m.pad[2] = 0;
    s_off[threadIdx.x] = m.entry0;
    for (int i = 0; i < tiles; ++i) p.tile[m.first + i] = m;
    if ((int)threadIdx.x == p.E - 1) p.ctl->tiles = incl >> 20;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int t = i / p.k, e = alone ? s_ids[i] : keep ? s_e[i] : __ldcg(p.ids + i), at = e * words + (t >> 5);
    const int pos = s_off[e] + pre[at] + __popc(mask[at] & ((1u << (t & 31)) - 1u));
    p.list[pos] = t;
    p.inv[i] = pos;
    if (alone) p.prob[i] = s_prob[i];
  }
  if (kCluster && alone && p.cl > 1 && live > 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int NT, bool kCluster>
ee_status launch(const RouteParams& p, cudaStream_t stream) {
  const size_t sums = std::max((size_t)kWarps * kTok * 8 * NT * 4, (size_t)kTok * p.E * 4);
  const size_t words = ((size_t)p.T + 31) / 32;
  size_t group = p.E * words * 6 + 4 + 4 * (size_t)p.E;
  const int keep = group + (size_t)p.T * p.k <= 220 * 1024;   // (4,096 tokens at 16 of 256 experts do not fit)
  if (keep) group += (size_t)p.T * p.k;
  const size_t smem = std::max(sums, group);
  {
    int dev = 0;
    const ee_status ds = current_device(&dev);
    if (ds != EE_OK) return ds;
    static std::mutex mu;
    static size_t have[kMaxDevices] = {};
    std::lock_guard<std::mutex> lock(mu);
    if (have[dev] < smem) {
      EE_CUDA_OK(cudaFuncSetAttribute(moe_route_kernel<NT, kCluster>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
      have[dev] = smem;
    }
  }
  const int sets = (p.E + 8 * NT - 1) / (8 * NT), units = p.xq ? p.T * ((p.H + kBlk - 1) / kBlk) : 0;
  const int per = p.cl * sets * kWarps * kQuantUnits;
  const dim3 grid(p.cl, sets, (p.T + kTok - 1) / kTok + (units + per - 1) / per);
  EE_CUDA_OK(launch_pdl(moe_route_kernel<NT, kCluster>, grid, dim3(kThreads), smem, stream, kCluster ? (unsigned)p.cl : 1u, p, keep));
  return EE_OK;
}

}  // namespace

namespace ee {
ee_status launch_moe_route(RouteParams& p, cudaStream_t stream) {
  const int groups = (p.T + kTok - 1) / kTok, blocks = (p.H + kBlk - 1) / kBlk;
  // Few experts a CTA where that leaves the hidden dimension to four of them or more (whole layers: 4 tokens, 60 experts 24.8 us and
  // 26.2, 4 tokens, 128 experts 39.5 and 42; 576 tokens, 64 experts even).  One CTA for all experts: sums through the cluster (16 tokens, 8
  // experts 17.9 us, through global memory 18.7); more: through global memory (1,500 tokens, 160 experts 180 us; by one CTA for all of them 236).
  const bool narrow = groups * ((p.E + 7) / 8) * 4 <= kRouteCtas || p.E <= 8 || p.few;
  const int sets = narrow ? (p.E + 7) / 8 : (p.E + 63) / 64, each = groups * sets;
  const bool clustered = sets == 1 && !p.few;
  // the widest share of the hidden dimension that the SMs hold at once (clusters: one CTA an SM, of two the layer took 310 us)
  p.cl = kRouteParts;
  while (p.cl > 1 && (each * p.cl > (clustered ? kNumSMs : kRouteCtas) || p.cl > blocks)) p.cl /= 2;
  if (clustered) return narrow ? launch<1, true>(p, stream) : launch<8, true>(p, stream);
  return narrow ? launch<1, false>(p, stream) : launch<8, false>(p, stream);
}
}  // namespace ee
