// ee_prompt_attn, ee_chunk_attn: causal attention of packed new tokens, whole
// prompts over their own K/V or chunks over the paged cache.
//
//   o_t = sum_{j <= p_t} softmax_j(scale q_t . k_j) v_j,   p_t = ctx + t
//
// in one pass over the keys with a running maximum m and sum l: a tile of 128 keys
// gives S = Q K^T, P = 2^(S scale log2e - m), O = O 2^(m_old - m) + P V, and the row
// ends as O / l.
//
// Rows and units.  A KV head serves g = n_q / n_kv query heads, so a row tile is the g
// heads of tpt = 128 / g consecutive tokens (row = token * g + head: one TMA box of Q,
// at most g - 1 rows empty, and a causal edge of tpt keys instead of 128).  A unit is
// two row tiles, A and B, of one sequence and KV head: they share every K/V tile, and
// while one's scores are in the softmax the tensor core works for the other.
//
// Work.  The keys of all units (plus a constant for each: a unit's start and end) are
// laid on one line, cut into equal shares, one for each CTA; one CTA runs on each SM.
// A share may begin and end inside a unit.  Such a unit's pieces leave (m, l) and the
// unnormalised O in the workspace, count their tiles done and, once all are, each
// merge a part of the rows and columns with weights 2^(m - max).  Every length follows
// from the device's offsets: long prompts, ragged batches and single tokens over long
// contexts are one case.  The launch is cooperative, so a wait for another CTA ends.
//
// Roles of a CTA's twelve warps; all walk the share's segments (tile ranges of units)
// by themselves, from a ring the scheduler fills:
//   0      streams K and V tiles by TMA into a ring of four 32 KB slots;
//   1      issues the MMAs: per tile and row tile P V of this one, then Q K^T of the
//          next (whose S takes the place of P: MMAs of one thread run in order);
//   2      finds the segments, streams Q;
//   3      cleans V where the causal edge or the sequence's end lies in a tile: the
//          MMA multiplies masked rows by P = 0, and 0 times a NaN is a NaN.  Rows past
//          the unit are zeroed, non-finite values of rows that some query must not see
//          are zeroed and added at the end for the queries that do;
//   4-7    softmax of row tile A, one row per thread; 8-11 of row tile B.
// TMEM: S/P of A and B, O of A and B, 128 columns each.
#include "ee_common.cuh"
#include "ee_ptx.cuh"

namespace {

using namespace ee;

constexpr int kD = EE_HEAD_DIM;
constexpr int kThreads = 384;
constexpr int kRows = 128;                    // rows of a row tile (MMA M)
constexpr int kKT = 128;                      // keys of a tile
constexpr int kRing = 4;                      // K/V slots, K and V tiles in turn
constexpr int kSegs = 4;                      // segments in flight
constexpr int kZones = 4;                     // cleaned V tiles in flight (at most kRing / 2)
constexpr int kMasks = 8;                     // page masks in flight (K runs at most 4 tiles ahead of the softmax)
constexpr uint32_t kHalf = kKT * 128;         // 64 of a tile's 128 columns
constexpr uint32_t kTile = 2 * kHalf;         // 32 KB
constexpr uint32_t kOffKV = 0, kOffQ = kRing * kTile, kOffBar = kOffQ + 2 * kTile;
constexpr uint32_t kNumBars = 2 * kRing + 4 + 8 + 2 * kSegs + kZones + 1;
constexpr uint32_t kSmemBytes = 1024 + kOffBar + 8 * kNumBars;
constexpr uint32_t kTmemCols = 512, kColO = 256;
constexpr float kRescaleLog2 = 8.0f;          // O is rescaled when a maximum grows by 2^8
// work in keys: a unit's own constant, and the smallest share of a CTA
constexpr int kUnitKeys = 3 * kKT, kMinShare = 5 * kKT;
constexpr int kWarpKV = 0, kWarpMma = 1, kWarpQ = 2, kWarpClean = 3, kWarpSoft = 4;
constexpr int kSegReaders = 3 + 8;            // warps 0, 1, 3 and the softmax warps
constexpr int kRegsLaunch = 168, kRegsSoft = 208, kRegsOther = 88;
static_assert(256 * kRegsSoft + 128 * kRegsOther <= kThreads * kRegsLaunch, "register split");
static_assert(kSmemBytes <= 227 * 1024 - 4096, "shared memory budget");
// counters of a split unit in the trailer of its first piece's slot, past the word
// that the verification attention keeps there
constexpr size_t kCntOff = kAttnCntOff + 64;

struct PromptParams {
  const __nv_bfloat16* v;       // V once more, for values the MMA must not see
  int64_t v_stride;
  const int32_t *block_table, *ctx_len, *tok_off;
  __nv_bfloat16* out;
  float* lse;
  uint8_t* part;
  int32_t* err;
  int B, total, num_pages, max_pages, n_q, n_kv, g, tpt;
  float scale, scale_log2;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t bf16x2_rn(float hi, float lo) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ float fmax3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// One sequence: first token, tokens, cached positions (T = 0: nothing to do).
struct Seq {
  int o, T, ctx;
};

template <bool kPaged>
__device__ __forceinline__ Seq load_seq(const PromptParams& p, int s, int& err) {
  Seq q;
  q.o = p.tok_off[s];
  const int end = p.tok_off[s + 1];
  q.ctx = kPaged ? p.ctx_len[s] : 0;
  q.T = end - q.o;
  if (q.o < 0 || end < q.o || end > p.total) {
    err |= EE_DEVERR_TREE;
    q.T = 0;
  } else if (kPaged && (q.ctx < 0 || (int64_t)q.ctx + q.T > (int64_t)p.max_pages * EE_PAGE)) {
    err |= EE_DEVERR_CTX;
    q.T = 0;
  }
  return q;
}

// The line of work.  Unit n of a sequence and KV head: tokens [n w, (n + 1) w), w = 2
// tpt, keys ctx + min(T, (n + 1) w); it takes that many places plus kUnitKeys + 64 (half
// a tile: the last one is rarely full).
constexpr int kUnitConst = kUnitKeys + kKT / 2;
__device__ __forceinline__ int num_units(int T, int w) { return (T + w - 1) / w; }
// places of a sequence and head before unit n (n below the number of units)
__device__ __forceinline__ int64_t places_before(int ctx, int w, int64_t n) {
  return n * ((int64_t)ctx + kUnitConst) + n * (n + 1) / 2 * w;
}
__device__ __forceinline__ int64_t head_places(int ctx, int T, int w) {
  if (T == 0) return 0;
  const int64_t P = num_units(T, w);
  return places_before(ctx, w, P - 1) + ctx + T + kUnitConst;
}
// tiles of a unit of n that lie before place y of it
__device__ __forceinline__ int tiles_before(int64_t y, int n) {
  const int64_t j = (y - kUnitKeys + kKT / 2) >> 7;
  return (int)min(max(j, (int64_t)0), (int64_t)n);
}
// start of CTA c's share of W places cut for N
__device__ __forceinline__ int64_t share_start(int64_t W, int N, int c) { return W * c / N; }

// A segment: tiles [j0, j1) of a unit.
struct Seg {
  int s, o, T, ctx;        // sequence
  int hk, tok0;            // KV head, the unit's first token
  int j0, j1, n_tiles;     // n_tiles: of the whole unit; j1 = 0: no more segments
  int nA, nB;              // tiles each row tile needs (B: 0 without tokens)
  int c0, c1;              // first and last CTA that may hold a piece
  int64_t X;               // the unit's first place
};

// Whether tile j of the unit holds keys that the first query must not see.
__device__ __forceinline__ bool in_zone(const Seg& s, int j) { return j * kKT + kKT - 1 > s.ctx + s.tok0; }
__device__ __forceinline__ bool active(const Seg& s, int st, int j) { return j < (st ? s.nB : s.nA); }

template <bool kPaged>
__device__ __forceinline__ const __nv_bfloat16* v_row(const PromptParams& p, const Seg& s, int key) {
  if constexpr (kPaged) {
    const int pg = p.block_table[(size_t)s.s * p.max_pages + key / EE_PAGE];
    if (pg < 0 || pg >= p.num_pages) return nullptr;
    return p.v + (((size_t)pg * p.n_kv + s.hk) * EE_PAGE + key % EE_PAGE) * kD;
  } else {
    return p.v + (size_t)(s.o + key) * p.v_stride + (size_t)s.hk * kD;
  }
}

__device__ __forceinline__ uint32_t nonfinite2(uint32_t x) {   // 0xffff in each half that is
  const uint32_t lo = (x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u;
  const uint32_t hi = (x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
  return lo | hi;
}

// Rows and columns of a split unit merged by one of its pieces: thread t of nthr.
// Items are (8-column group, row), the rows fastest, so that a warp's loads of a
// piece's slot (column-chunk major) are contiguous.
__device__ __forceinline__ void merge_piece(const PromptParams& p, const Seg& s, const int16_t* list, int K, int64_t lo,
                                            int64_t hi, int t, int nthr) {
  const int w = 2 * p.tpt;
  const int nt = min(w, s.T - s.tok0);                       // tokens of the unit
  const int rows_a = min(nt, p.tpt) * p.g, rows = nt * p.g;  // rows of A, of both
  for (int64_t i = lo + t; i < hi; i += nthr) {
    const int cg = (int)(i / rows), r = (int)(i - (int64_t)cg * rows);
    const int st = r >= rows_a, rr = st ? r - rows_a : r;
    float M = -INFINITY;
    for (int k = 0; k < K; ++k)
      if (list[k] >= 0)
        M = fmaxf(M, __ldcg(reinterpret_cast<const float2*>(
                                p.part + (size_t)(2 * list[k] + st) * kAttnPartBytes + kAttnMlOff) + rr).x);
    float a[8] = {}, L = 0.f;
#pragma unroll 4
    for (int k = 0; k < K; ++k) {
      if (list[k] < 0) continue;
      const uint8_t* slot = p.part + (size_t)(2 * list[k] + st) * kAttnPartBytes;
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(slot + kAttnMlOff) + rr);
      const float4* O = reinterpret_cast<const float4*>(slot) + (size_t)(2 * cg) * kRows + rr;
      // a row without keys in the piece has l = 0 and no O (a sum that is NaN has one)
      if (ml.y == 0.f) continue;
      const float4 u = __ldcg(O), v = __ldcg(O + kRows);
      const float f = ml.x == -INFINITY ? 1.f : ex2(ml.x - M);
      L = fmaf(f, ml.y, L);
      a[0] = fmaf(f, u.x, a[0]);
      a[1] = fmaf(f, u.y, a[1]);
      a[2] = fmaf(f, u.z, a[2]);
      a[3] = fmaf(f, u.w, a[3]);
      a[4] = fmaf(f, v.x, a[4]);
      a[5] = fmaf(f, v.y, a[5]);
      a[6] = fmaf(f, v.z, a[6]);
      a[7] = fmaf(f, v.w, a[7]);
    }
    const float il = L == 0.f ? 0.f : 1.f / L;
    const int tok = s.tok0 + (st ? p.tpt : 0) + rr / p.g, h = s.hk * p.g + rr % p.g;
    const size_t row = (size_t)(s.o + tok) * p.n_q + h;
    uint4 o;
    o.x = bf16x2_rn(a[1] * il, a[0] * il);
    o.y = bf16x2_rn(a[3] * il, a[2] * il);
    o.z = bf16x2_rn(a[5] * il, a[4] * il);
    o.w = bf16x2_rn(a[7] * il, a[6] * il);
    *reinterpret_cast<uint4*>(p.out + row * kD + 8 * cg) = o;
    if (cg == 0 && p.lse) p.lse[row] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
  }
}

template <bool kPaged>
__global__ void __launch_bounds__(kThreads, 1)
prompt_attn_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const PromptParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem =
      reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ Seg s_seg[kSegs];
  __shared__ int s_bad[kSegs];                   // V values taken out of the segment's tiles
  __shared__ uint32_t s_mask[kMasks];            // per tile: 16-key blocks in a valid page
  __shared__ int64_t s_scan[kThreads / 32];
  __shared__ int s_first;                        // the share's first sequence, and
  __shared__ int64_t s_firstX;                   // its first place
  __shared__ int s_kvissued[kRing], s_zissued[kZones], s_qissued[2];   // phases of copies started (-1: none)
  __shared__ Seg s_pc[2];                        // pieces of split units
  __shared__ int s_npc;
  __shared__ int16_t s_list[2][kNumSMsMax];      // their pieces' slot pairs (-1: empty)
  __shared__ int s_ready[2];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sbase = smem_u32(smem);
  const uint32_t sKV = sbase + kOffKV, sQ = sbase + kOffQ, bar0 = sbase + kOffBar;
  const uint32_t kv_full = bar0, kv_empty = kv_full + 8 * kRing;
  const uint32_t q_full = kv_empty + 8 * kRing, q_empty = q_full + 16;
  const uint32_t s_full = q_empty + 16, p_full = s_full + 16, pv_done = p_full + 16, o_free = pv_done + 16;
  const uint32_t seg_full = o_free + 16, seg_empty = seg_full + 8 * kSegs, z_full = seg_empty + 8 * kSegs;
  const uint32_t drain = z_full + 8 * kZones;

  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmQ)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmK)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmV)) : "memory");
    s_abort = 0;
    s_npc = 0;
    s_first = p.B;
    s_firstX = 0;
    for (int i = 0; i < kRing; ++i) {
      mbar_init(kv_full + 8 * i, 1);
      mbar_init(kv_empty + 8 * i, 1);
      s_kvissued[i] = -1;
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full + 8 * i, 1);
      mbar_init(q_empty + 8 * i, 1);
      mbar_init(s_full + 8 * i, 2);
      mbar_init(p_full + 8 * i, 4);
      mbar_init(pv_done + 8 * i, 2);
      mbar_init(o_free + 8 * i, 4);
      s_qissued[i] = -1;
    }
    for (int i = 0; i < kSegs; ++i) {
      mbar_init(seg_full + 8 * i, 1);
      mbar_init(seg_empty + 8 * i, kSegReaders);
    }
    for (int i = 0; i < kZones; ++i) {
      mbar_init(z_full + 8 * i, 1);
      s_zissued[i] = -1;
    }
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // rows of the Q tiles past g * tpt are never loaded
  for (int i = tid; i < 2 * 2 * (kRows - p.g * p.tpt) * 8; i += kThreads) {
    const int c = i & 7, r = i >> 3, per = kRows - p.g * p.tpt;
    *reinterpret_cast<uint4*>(smem + kOffQ + (r / per) * kHalf + (p.g * p.tpt + r % per) * 128 + 16 * c) =
        make_uint4(0, 0, 0, 0);
  }
  fence_async_smem();
  pdl_wait();   // no global access before the previous kernel's writes are visible

  // ---- the line of work: its length, this CTA's share and where that begins ----
  const int w = 2 * p.tpt;
  int64_t W, x0, x1;
  int N;
  {
    const int per = (p.B + kThreads - 1) / kThreads;
    const int b0 = min(tid * per, p.B), b1 = min(b0 + per, p.B);
    int64_t sum = 0;
    int err = 0;
    for (int s = b0; s < b1; ++s) {
      const Seq q = load_seq<kPaged>(p, s, err);
      sum += head_places(q.ctx, q.T, w) * p.n_kv;
    }
    if (err && blockIdx.x == 0) flag_error(p.err, err);
    int64_t incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t a = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += a;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    int64_t base = 0;
    W = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) {
      if (i < warp) base += s_scan[i];
      W += s_scan[i];
    }
    N = (int)min((int64_t)gridDim.x, max(W / kMinShare, (int64_t)1));
    const int c = blockIdx.x;
    x0 = c < N ? share_start(W, N, c) : W;
    x1 = c < N ? share_start(W, N, c + 1) : W;
    int64_t at = base + incl - sum;
    if (x0 < x1 && x0 >= at && x0 < at + sum) {
      for (int s = b0; s < b1; ++s) {
        const Seq q = load_seq<kPaged>(p, s, err);
        const int64_t n = head_places(q.ctx, q.T, w) * p.n_kv;
        if (x0 < at + n) {
          s_first = s;
          s_firstX = at;
          break;
        }
        at += n;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);

  auto wait = [&](uint32_t bar, int use) -> bool {
    return __all_sync(0xffffffffu, mbar_wait(bar, (uint32_t)(use & 1), &s_abort));
  };
  // segment i of the share (false: there is none, or a wait gave up)
  auto receive = [&](int i, Seg& s) -> bool {
    if (!wait(seg_full + 8 * (i % kSegs), i / kSegs)) return false;
    s = s_seg[i % kSegs];
    return s.j1 > 0;
  };
  auto release = [&](int i) {
    __syncwarp();
    if (lane == 0) mbar_arrive(seg_empty + 8 * (i % kSegs));
  };

  if (warp < kWarpSoft) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == kWarpKV) {
      // ---------------- K and V tiles ----------------
      // The V tiles that warp 3 cleans signal it, and it signals the MMA warp.
      Seg s;
      int tile = 0, zone = 0;
      bool go = true;
      for (int i = 0; go && receive(i, s); ++i) {
        // paged: lane l holds the page of 16-key block l % 8 of the (l / 8)-th of four tiles
        auto fetch = [&](int j) -> int32_t {
          const int key = (j + (lane >> 3)) * kKT + 16 * (lane & 7);
          const bool need = (j + (lane >> 3)) < s.j1 && key < s.ctx + s.T;
          return need ? max(ld_nc_pinned(p.block_table + (size_t)s.s * p.max_pages + key / EE_PAGE), -1) : INT32_MIN;
        };
        int32_t ids = INT32_MIN, ids_next = INT32_MIN;
        if constexpr (kPaged) ids_next = fetch(s.j0);
        for (int j = s.j0; j < s.j1 && go; ++j, ++tile) {
          int row[8];
          uint32_t okm = 0;
          if constexpr (kPaged) {
            const int q = (j - s.j0) & 3;
            if (q == 0) {
              ids = ids_next;
              ids_next = fetch(j + 4);
            }
            bool bad = false;
#pragma unroll
            for (int b = 0; b < 8; ++b) {
              const int32_t id = __shfl_sync(0xffffffffu, ids, 8 * q + b);
              const bool ok = id >= 0 && id < p.num_pages;
              // rows wholly out of range are filled with zeros
              row[b] = ok ? (id * p.n_kv + s.hk) * EE_PAGE : -EE_PAGE;
              okm |= ok ? 1u << b : 0u;
              bad |= !ok && id != INT32_MIN;
            }
            if (bad && lane == 0) flag_error(p.err, EE_DEVERR_PAGE);
          }
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const int idx = 2 * tile + kv, slot = idx % kRing, use = idx / kRing;
            go = go && wait(kv_empty + 8 * slot, use + 1);
            if (go && elect_one()) {
              const bool z = kv && in_zone(s, j);
              const uint32_t full = z ? z_full + 8 * (zone % kZones) : kv_full + 8 * slot;
              const uint32_t dst = sKV + slot * kTile;
              const CUtensorMap* tm = kv ? &tmV : &tmK;
              if (kPaged && kv == 0) s_mask[tile % kMasks] = okm;
              mbar_expect_tx(full, kTile);
              if constexpr (kPaged) {
#pragma unroll
                for (int b = 0; b < 8; ++b) {
                  tma_load_2d(dst + b * 2048, tm, full, 0, row[b]);
                  tma_load_2d(dst + kHalf + b * 2048, tm, full, 64, row[b]);
                }
              } else {
                tma_load_3d(dst, tm, full, 0, s.hk, s.o + j * kKT);
                tma_load_3d(dst + kHalf, tm, full, 64, s.hk, s.o + j * kKT);
              }
              if (z) s_zissued[zone % kZones] = zone / kZones;
              else s_kvissued[slot] = use;
            }
            __syncwarp();
          }
          zone += in_zone(s, j);
        }
        release(i);
      }
    } else if (warp == kWarpQ) {
      // ---------------- segments and Q ----------------
      // lane l holds sequence base + l, so that many short sequences cost one
      // round trip for 32 of them
      int base = s_first, err = 0;
      Seq mine{0, 0, 0};
      auto load32 = [&]() {
        mine = Seq{0, 0, 0};
        if (base + lane < p.B) mine = load_seq<kPaged>(p, base + lane, err);
      };
      load32();
      int s = base;
      int64_t X = x0 < x1 ? s_firstX : x1;   // the next unit's first place
      int o = 0, T = 0, ctx = 0, hk = 0, n = 0;
      auto take = [&]() {        // sequence s from its lane
        if (s - base >= 32) {
          base = s;
          load32();
        }
        o = __shfl_sync(0xffffffffu, mine.o, s - base);
        T = __shfl_sync(0xffffffffu, mine.T, s - base);
        ctx = __shfl_sync(0xffffffffu, mine.ctx, s - base);
      };
      if (x0 < x1) {
        take();
        const int64_t per_head = head_places(ctx, T, w);
        int64_t rem = x0 - X;
        hk = (int)(rem / per_head);
        rem -= hk * per_head;
        X += hk * per_head;
        int lo = 0, hi = num_units(T, w);
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (places_before(ctx, w, mid) <= rem) lo = mid; else hi = mid;
        }
        n = lo;
        X += places_before(ctx, w, n);
      }
      // the next non-empty segment of the share
      auto find = [&](Seg& g) -> bool {
        while (X < x1) {
          if (n >= num_units(T, w)) {          // next head, or next sequence with tokens
            n = 0;
            if (T == 0 || ++hk == p.n_kv) {
              hk = 0;
              if (++s >= p.B) break;
              take();
            }
            continue;
          }
          const int tok0 = n * w;
          const int keys = ctx + min(T, tok0 + w);
          const int tiles = (keys + kKT - 1) / kKT;
          const int64_t len = keys + kUnitConst;
          const int j0 = X < x0 ? tiles_before(x0 - X, tiles) : 0;
          const int j1 = x1 >= X + len ? tiles : tiles_before(x1 - X, tiles);
          g.X = X;
          X += len;
          ++n;
          if (j0 >= j1) continue;
          g.s = s;
          g.o = o;
          g.T = T;
          g.ctx = ctx;
          g.hk = hk;
          g.tok0 = tok0;
          g.j0 = j0;
          g.j1 = j1;
          g.n_tiles = tiles;
          g.nA = (ctx + min(T, tok0 + p.tpt) + kKT - 1) / kKT;
          g.nB = T > tok0 + p.tpt ? tiles : 0;
          g.c0 = g.c1 = 0;
          if (j1 - j0 < tiles) {
            // CTA c holds a first piece when its share starts before the second tile's
            // places do, and any piece when it starts before the last one's
            const int64_t y = g.X + kUnitKeys + kKT / 2;
            g.c0 = (int)((y * N + W - 1) / W) - 1;
            g.c1 = min((int)(((y + (int64_t)kKT * (tiles - 1)) * N + W - 1) / W) - 1, N - 1);
          }
          return true;
        }
        g.j1 = 0;
        return false;
      };
      auto publish = [&](int i, const Seg& g) -> bool {
        if (!wait(seg_empty + 8 * (i % kSegs), i / kSegs + 1)) return false;
        if (lane == 0) {
          s_seg[i % kSegs] = g;
          s_bad[i % kSegs] = 0;
          if (g.j1 - g.j0 < g.n_tiles && g.j1 > 0) {
            s_pc[s_npc & 1] = g;
            s_npc = s_npc + 1;
          }
          mbar_arrive(seg_full + 8 * (i % kSegs));
        }
        __syncwarp();
        return true;
      };
      Seg cur, nxt;
      bool more = find(cur);
      bool go = publish(0, cur);
      int uses[2] = {0, 0};
      for (int i = 0; more && go; ++i) {
        more = find(nxt);
        go = publish(i + 1, nxt);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          if (!go || !active(cur, st, cur.j0)) continue;
          go = wait(q_empty + 8 * st, uses[st] + 1);
          if (go && elect_one()) {
            const uint32_t full = q_full + 8 * st, dst = sQ + st * kTile;
            const int tok = cur.o + cur.tok0 + st * p.tpt;
            mbar_expect_tx(full, 2u * 128u * p.g * p.tpt);
            tma_load_3d(dst, &tmQ, full, 0, cur.hk * p.g, tok);
            tma_load_3d(dst + kHalf, &tmQ, full, 64, cur.hk * p.g, tok);
            s_qissued[st] = uses[st];
          }
          __syncwarp();
          ++uses[st];
        }
        cur = nxt;
      }
    } else if (warp == kWarpClean) {
      // ---------------- V where a query's last key or the unit's last lies inside a tile ----
      Seg s;
      int tile = 0, zone = 0;
      bool go = true;
      for (int i = 0; go && receive(i, s); ++i) {
        const int first = s.ctx + s.tok0, last = s.ctx + min(s.T, s.tok0 + w) - 1;
        for (int j = s.j0; j < s.j1 && go; ++j, ++tile) {
          if (!in_zone(s, j)) continue;
          const int slot = (2 * tile + 1) % kRing;
          go = wait(z_full + 8 * (zone % kZones), zone / kZones);
          if (!go) break;
          uint8_t* v = smem + kOffKV + slot * kTile;
          const int r0 = max(first + 1 - j * kKT, 0), r1 = min(last + 1 - j * kKT, kKT);
          uint32_t seen = 0;
          // a row's 128 bytes in each half are a permutation of its 16-byte chunks
          for (int c = r0 * 8 + lane; c < kKT * 8; c += 32) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint4* a = reinterpret_cast<uint4*>(v + h * kHalf + 16 * c);
              if ((c >> 3) >= r1) {
                *a = make_uint4(0, 0, 0, 0);
              } else {
                uint4 x = *a;
                const uint32_t m0 = nonfinite2(x.x), m1 = nonfinite2(x.y), m2 = nonfinite2(x.z), m3 = nonfinite2(x.w);
                if (m0 | m1 | m2 | m3) {
                  seen = 1;
                  x.x &= ~m0;
                  x.y &= ~m1;
                  x.z &= ~m2;
                  x.w &= ~m3;
                  *a = x;
                }
              }
            }
          }
          fence_async_smem();   // generic-proxy writes, read by the tensor core
          if (__any_sync(0xffffffffu, seen) && lane == 0) s_bad[i % kSegs] = 1;
          __syncwarp();
          if (lane == 0) mbar_arrive(kv_full + 8 * slot);
          ++zone;
        }
        release(i);
      }
    } else {
      // ---------------- MMAs ----------------
      const uint32_t id_qk = idesc_f16(kRows, kKT, 1, 1, 0), id_pv = idesc_f16(kRows, kD, 1, 1, 1);
      const uint64_t dq0 = smem_desc_sw128(__shfl_sync(0xffffffffu, sQ, 0));
      const uint64_t dk0 = smem_desc_sw128(__shfl_sync(0xffffffffu, sKV, 0));
      const uint64_t dv0 = smem_desc_sw128_mn(__shfl_sync(0xffffffffu, sKV, 0), kHalf, 1024);
      int q_uses[2] = {0, 0}, o_uses[2] = {0, 0}, p_uses[2] = {0, 0};
      // S = Q K^T of row tile st and tile j (the CTA's tile-th)
      auto qk = [&](const Seg& s, int st, int j, int tile) {
        if (elect_one()) {
          const uint64_t dk = dk0 + (uint64_t)(((2 * tile) % kRing) * (kTile >> 4));
          const uint64_t dq = dq0 + (uint64_t)(st * (kTile >> 4));
#pragma unroll
          for (int kk = 0; kk < kD / 16; ++kk) {
            const uint64_t off = ((kk >> 2) * kHalf + (kk & 3) * 32) >> 4;
            tc_mma(tmem + st * kKT, dq + off, dk + off, id_qk, kk > 0 ? 1u : 0u);
          }
          tc_commit(s_full + 8 * st);
          mbar_arrive(s_full + 8 * st);   // releases the tile's page mask (acquired with kv_full)
          if (j + 1 == s.j1 || !active(s, st, j + 1)) tc_commit(q_empty + 8 * st);
        }
        __syncwarp();
      };
      auto pv = [&](const Seg& s, int st, int j, int tile) {
        if (elect_one()) {
          const uint64_t dv = dv0 + (uint64_t)(((2 * tile + 1) % kRing) * (kTile >> 4));
#pragma unroll
          for (int kk = 0; kk < kKT / 16; ++kk)
            tc_mma_ts(tmem + kColO + st * kD, tmem + st * kKT + 8 * kk, dv + (uint64_t)(kk * (2048 >> 4)), id_pv,
                      (j > s.j0 || kk > 0) ? 1u : 0u);
          if (j + 1 == s.j1 || !active(s, st, j + 1)) {
            tc_commit(pv_done + 8 * st);
            mbar_arrive(pv_done + 8 * st);   // releases s_bad (acquired with kv_full)
          }
        }
        __syncwarp();
      };
      Seg s, nx;
      int i = 0, tile = 0;
      bool go = receive(0, s);
      int j = s.j0;
      if (go) {
        go = wait(kv_full, 0);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          if (!go || !active(s, st, j)) continue;
          go = wait(q_full + 8 * st, q_uses[st]++);
          tc_fence_after();
          if (go) qk(s, st, j, 0);
        }
        if (go && elect_one()) tc_commit(kv_empty);
        __syncwarp();
      }
      while (go) {
        nx = s;
        int jn = j + 1;
        bool has = true;
        const bool fresh = jn == s.j1;
        if (fresh) {
          has = receive(i + 1, nx);
          jn = nx.j0;
          if (s_abort) break;
        }
        const int vi = 2 * tile + 1, ki = 2 * tile + 2;
        go = wait(kv_full + 8 * (vi % kRing), vi / kRing);
        bool k_in = false;
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          if (go && active(s, st, j)) {
            go = wait(p_full + 8 * st, p_uses[st]++);
            if (go && j == s.j0) {
              if (o_uses[st] > 0) go = wait(o_free + 8 * st, o_uses[st] - 1);   // the last segment's O is read
              ++o_uses[st];
            }
            tc_fence_after();
            if (go) pv(s, st, j, tile);
          }
          if (go && has && active(nx, st, jn)) {
            if (!k_in) go = wait(kv_full + 8 * (ki % kRing), ki / kRing);
            k_in = true;
            if (go && fresh) go = wait(q_full + 8 * st, q_uses[st]++);
            tc_fence_after();
            if (go) qk(nx, st, jn, tile + 1);
          }
        }
        if (go && elect_one()) {
          tc_commit(kv_empty + 8 * (vi % kRing));
          if (has) tc_commit(kv_empty + 8 * (ki % kRing));
        }
        __syncwarp();
        if (!has) break;
        if (fresh) {
          release(i);
          ++i;
          s = nx;
        }
        j = jn;
        ++tile;
      }
    }

    // ---- drain on abort, free TMEM ----
    tc_fence_before();
    __syncthreads();
    pdl_allow_next();
    if (s_abort) {
      if (tid == 0) {
        flag_error(p.err, EE_DEVERR_TIMEOUT);
        for (int i = 0; i < kRing; ++i)
          if (s_kvissued[i] >= 0) mbar_wait_plain(kv_full + 8 * i, (uint32_t)(s_kvissued[i] & 1));
        for (int i = 0; i < kZones; ++i)
          if (s_zissued[i] >= 0) mbar_wait_plain(z_full + 8 * i, (uint32_t)(s_zissued[i] & 1));
        for (int i = 0; i < 2; ++i)
          if (s_qissued[i] >= 0) mbar_wait_plain(q_full + 8 * i, (uint32_t)(s_qissued[i] & 1));
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      if (warp == kWarpMma && elect_one()) {   // MMAs still in flight
        tc_commit(drain);
        mbar_wait_plain(drain, 0);
      }
      __syncwarp();
    }
    if (warp == kWarpMma) {
      tc_fence_after();
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(s_tmem), "r"(kTmemCols) : "memory");
    }
    return;
  }
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));

  // ---------------- softmax: one row per thread ----------------
  {
    const int st = (warp - kWarpSoft) >> 2, qd = warp & 3;
    const int r = qd * 32 + lane;
    const int tok_r = r / p.g, head = r - tok_r * p.g;
    const uint32_t lane_base = (uint32_t)(qd * 32) << 16;
    const uint32_t tS = tmem + lane_base + st * kKT, tO = tmem + lane_base + kColO + st * kD;
    const float sl2 = p.scale_log2;
    Seg s;
    int tile = 0, uses = 0, o_uses = 0;
    bool go = true;
    for (int i = 0; go && receive(i, s); ++i) {
      const int tok = s.tok0 + st * p.tpt + tok_r;
      const bool vrow = tok_r < p.tpt && tok < s.T;
      const bool warp_rows = __any_sync(0xffffffffu, vrow);
      const int pos = s.ctx + tok;                             // the row's last key
      const int tile_first = s.ctx + s.tok0 + st * p.tpt;      // the row tile's first row's
      const int j_end = min(s.j1, st ? s.nB : s.nA);
      float m = -INFINITY, l = 0.f;                            // m in raw score units (scale > 0)
      for (int j = s.j0; j < j_end; ++j) {
        go = wait(s_full + 8 * st, uses);
        if (!go) break;
        ++uses;
        if (warp_rows) {
          tc_fence_after();
          uint32_t sr[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) tc_ld32_nowait(tS + 32 * c, *reinterpret_cast<uint32_t(*)[32]>(&sr[32 * c]));
          const uint32_t pm = kPaged ? s_mask[(tile + j - s.j0) % kMasks] : 0xFFu;
          const int base = j * kKT;
          tc_wait_ld32(*reinterpret_cast<uint32_t(*)[32]>(&sr[0]));
#pragma unroll
          for (int c = 1; c < 4; ++c) tc_pin32(*reinterpret_cast<uint32_t(*)[32]>(&sr[32 * c]));
          if (base + kKT - 1 > tile_first || pm != 0xFFu) {
            const int nvis = pos + 1 - base;
#pragma unroll
            for (int c = 0; c < 128; ++c)
              if (c >= nvis || !((pm >> (c >> 4)) & 1u)) sr[c] = __float_as_uint(-INFINITY);
          }
          float mx[8];
#pragma unroll
          for (int k = 0; k < 8; ++k)
            mx[k] = fmaxf(__uint_as_float(sr[k]), __uint_as_float(sr[8 + k]));
#pragma unroll
          for (int c = 16; c < 128; c += 16)
#pragma unroll
            for (int k = 0; k < 8; ++k)
              mx[k] = fmax3(mx[k], __uint_as_float(sr[c + k]), __uint_as_float(sr[c + 8 + k]));
          const float tmax = fmax3(fmax3(mx[0], mx[1], mx[2]), fmax3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7]));
          const float m_new = fmaxf(m, tmax);
          const bool need = (m_new - m) * sl2 > kRescaleLog2;   // true when m = -inf < m_new
          if (j > s.j0 && __any_sync(0xffffffffu, need)) {
            // S of this tile was issued after P V of the one before: O holds it
            const float f = need ? ex2((m - m_new) * sl2) : 1.f;
#pragma unroll 1
            for (int c = 0; c < 8; ++c) {
              uint32_t ov[16];
              tc_ld16(tO + 16 * c, ov);
#pragma unroll
              for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * f);
              tc_st16_nowait(tO + 16 * c, ov);
            }
          }
          if (need) {
            l *= ex2((m - m_new) * sl2);
            m = m_new;
          }
          const float nms = m == -INFINITY ? 0.f : -m * sl2;
          const uint64_t sl2x2 = f2_pack(__float_as_uint(sl2), __float_as_uint(sl2));
          const uint64_t nmsx2 = f2_pack(__float_as_uint(nms), __float_as_uint(nms));
          uint64_t ls[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t pw[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int x = 32 * c + 2 * e;
              uint32_t y0, y1;
              f2_unpack(f2_fma(f2_pack(sr[x], sr[x + 1]), sl2x2, nmsx2), y0, y1);
              const float p0 = ex2(__uint_as_float(y0)), p1 = ex2(__uint_as_float(y1));
              const uint64_t pp = f2_pack(__float_as_uint(p0), __float_as_uint(p1));
              ls[e & 3] = c == 0 && e < 4 ? pp : f2_add(ls[e & 3], pp);
              pw[e] = bf16x2_rn(p1, p0);
            }
            tc_st16_nowait(tS + 16 * c, pw);
          }
          tc_wait_st();
          tc_fence_before();
          ls[0] = f2_add(f2_add(ls[0], ls[1]), f2_add(ls[2], ls[3]));
          uint32_t a0, a1;
          f2_unpack(ls[0], a0, a1);
          l += __uint_as_float(a0) + __uint_as_float(a1);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 8 * st);
      }
      tile += s.j1 - s.j0;
      if (!go) break;

      // ---- the segment's rows: O / l, or a partial ----
      const bool whole = s.j1 - s.j0 == s.n_tiles;
      const bool any = j_end > s.j0;
      if (any) {
        go = wait(pv_done + 8 * st, o_uses);
        if (!go) break;
        ++o_uses;
        tc_fence_after();
      }
      const bool bad = any && s_bad[i % kSegs] != 0;
      const float il = l == 0.f ? 0.f : 1.f / l;
      const size_t row = (size_t)(s.o + tok) * p.n_q + s.hk * p.g + head;
      const int slot = whole ? 0 : 2 * (2 * (int)blockIdx.x + (s.j0 == 0 ? 1 : 0)) + st;
      uint8_t* part = p.part + (size_t)slot * kAttnPartBytes;
      if (any && warp_rows) {
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t ov[32];
          tc_ld32_nowait(tO + 32 * c, ov);
          tc_wait_ld32(ov);
          if (bad && vrow) {
            const int k1 = min(pos, s.j1 * kKT - 1);
            for (int key = max(s.ctx + s.tok0 + 1, s.j0 * kKT); key <= k1; ++key) {
              const __nv_bfloat16* v = v_row<kPaged>(p, s, key);
              if (!v) continue;
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                const float x = __bfloat162float(v[32 * c + e]);
                if (!isfinite(x)) ov[e] = __float_as_uint(__uint_as_float(ov[e]) + x);
              }
            }
          }
          if (vrow && whole) {
            uint4* dst = reinterpret_cast<uint4*>(p.out + row * kD + 32 * c);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint4 x;
              x.x = bf16x2_rn(__uint_as_float(ov[8 * e + 1]) * il, __uint_as_float(ov[8 * e]) * il);
              x.y = bf16x2_rn(__uint_as_float(ov[8 * e + 3]) * il, __uint_as_float(ov[8 * e + 2]) * il);
              x.z = bf16x2_rn(__uint_as_float(ov[8 * e + 5]) * il, __uint_as_float(ov[8 * e + 4]) * il);
              x.w = bf16x2_rn(__uint_as_float(ov[8 * e + 7]) * il, __uint_as_float(ov[8 * e + 6]) * il);
              dst[e] = x;
            }
          } else if (vrow) {
            float4* dst = reinterpret_cast<float4*>(part) + (size_t)(8 * c) * kRows + r;
#pragma unroll
            for (int e = 0; e < 8; ++e)
              __stcg(dst + (size_t)e * kRows,
                     make_float4(__uint_as_float(ov[4 * e]), __uint_as_float(ov[4 * e + 1]),
                                 __uint_as_float(ov[4 * e + 2]), __uint_as_float(ov[4 * e + 3])));
          }
        }
        tc_fence_before();
      }
      if (vrow && whole && p.lse) p.lse[row] = l == 0.f ? -INFINITY : fmaf(m, p.scale, logf(l));
      if (vrow && !whole)
        __stcg(reinterpret_cast<float2*>(part + kAttnMlOff) + r, make_float2(m == -INFINITY ? m : m * sl2, l));
      __syncwarp();
      if (any && lane == 0) mbar_arrive(o_free + 8 * st);
      release(i);
    }
  }
  tc_fence_before();
  __syncthreads();
  pdl_allow_next();
  if (s_abort) return;

  // ---- pieces of split units: counted, waited for and merged ----
  const int npc = s_npc;
  if (npc == 0) return;
  const int nthr = npc == 2 ? 128 : 256;
  const int pi = (tid - 32 * kWarpSoft) / nthr, t = (tid - 32 * kWarpSoft) - pi * nthr;
  const Seg s = s_pc[pi];
  const int K = s.c1 - s.c0 + 1, mine = (int)blockIdx.x - s.c0;
  unsigned int* cnt =
      reinterpret_cast<unsigned int*>(p.part + (size_t)(2 * (2 * s.c0 + 1)) * kAttnPartBytes + kCntOff);
  if (t == 0) {
    atom_add_acq_rel(cnt, (unsigned)(s.j1 - s.j0));
    const bool ok = wait_count_geq(cnt, (unsigned)s.n_tiles);
    if (!ok) flag_error(p.err, EE_DEVERR_TIMEOUT);
    s_ready[pi] = ok;
  }
  for (int k = t; k < K; k += nthr) {
    const int c = s.c0 + k;
    const int j0 = k == 0 ? 0 : tiles_before(share_start(W, N, c) - s.X, s.n_tiles);
    const int j1 = tiles_before(share_start(W, N, c + 1) - s.X, s.n_tiles);
    s_list[pi][k] = j0 < j1 ? (int16_t)(2 * c + (k == 0 ? 1 : 0)) : (int16_t)-1;
  }
  asm volatile("bar.sync %0, %1;" ::"r"(2 + pi), "r"(nthr) : "memory");
  if (!s_ready[pi]) return;
  {
    const int64_t items = (int64_t)min(w, s.T - s.tok0) * p.g * (kD / 8);
    merge_piece(p, s, s_list[pi], K, items * mine / K, items * (mine + 1) / K, t, nthr);
  }
  // the last piece to have read the partials clears the counts for the next launch
  asm volatile("bar.sync %0, %1;" ::"r"(2 + pi), "r"(nthr) : "memory");
  if (t == 0) {
    const unsigned left = atom_add_acq_rel(cnt + 1, (unsigned)(s.j1 - s.j0)) + (unsigned)(s.j1 - s.j0);
    if (left == (unsigned)s.n_tiles) {
      cnt[0] = 0;
      cnt[1] = 0;
    }
  }
}

bool good_stride(int64_t stride, int heads) { return stride % 8 == 0 && stride >= (int64_t)heads * kD; }

// Dynamic shared memory and the CTAs the device holds at once, asked once per device.
ee_status resident_ctas(int dev, int* ctas) {
  static std::mutex mu;
  static int cached[kMaxDevices] = {};
  std::lock_guard<std::mutex> lock(mu);
  if (!cached[dev]) {
    int sms = 0, per = 0;
    EE_CUDA_OK(cudaFuncSetAttribute(prompt_attn_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes));
    EE_CUDA_OK(cudaFuncSetAttribute(prompt_attn_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes));
    EE_CUDA_OK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    EE_CUDA_OK(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, prompt_attn_kernel<true>, kThreads, kSmemBytes));
    if (per < 1) return EE_ERR_CUDA;
    cached[dev] = std::min(sms * per, kNumSMsMax);
  }
  *ctas = cached[dev];
  return EE_OK;
}

// The checks both calls share.
ee_status check(const ee_bf16* q, int64_t q_stride, const ee_bf16* k, const ee_bf16* v, const int32_t* tok_off,
                int32_t B, int32_t total, int32_t n_q, int32_t n_kv, int32_t head_dim, float scale, const ee_bf16* out,
                const float* lse, const void* ws, size_t ws_bytes) {
  if (B < 0 || total < 0 || n_q < 1 || n_kv < 1) return EE_ERR_INVALID_ARG;
  if (head_dim != EE_HEAD_DIM || n_q % n_kv != 0 || n_q / n_kv > kRows) return EE_ERR_UNSUPPORTED;
  if (!(scale > 0.f) || !std::isfinite(scale)) return EE_ERR_INVALID_ARG;
  if (B == 0 || total == 0) return EE_OK;
  if (!q || !k || !v || !tok_off || !out || !ws) return EE_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(lse, 4) ||
      !aligned(ws, 256))
    return EE_ERR_INVALID_ARG;
  if (!good_stride(q_stride, n_q)) return EE_ERR_INVALID_ARG;
  if (ws_bytes < ee_prompt_workspace_size()) return EE_ERR_WORKSPACE;
  return EE_OK;
}

// A map over [tokens][heads][128] with `rows` tokens x `heads_box` heads x 64 columns a box.
bool token_map(CUtensorMap* map, const void* base, int heads, int total, int64_t stride, int heads_box, int rows) {
  const uint64_t dims[3] = {(uint64_t)kD, (uint64_t)heads, (uint64_t)total};
  const uint64_t strides[2] = {(uint64_t)kD * 2, (uint64_t)stride * 2};
  const uint32_t box[3] = {64, (uint32_t)heads_box, (uint32_t)rows};
  return encode_bf16_tmap(map, base, 3, dims, strides, box);
}

template <bool kPaged>
ee_status launch(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const PromptParams& p,
                 int ctas, ee_stream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeCooperative;
  attr[1].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  EE_CUDA_OK(cudaLaunchKernelEx(&cfg, prompt_attn_kernel<kPaged>, tmQ, tmK, tmV, p));
  return EE_OK;
}

PromptParams params(const int32_t* tok_off, int B, int total, int n_q, int n_kv, float scale, ee_bf16* out, float* lse,
                    void* ws) {
  PromptParams p{};
  p.tok_off = tok_off;
  p.out = reinterpret_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.part = static_cast<uint8_t*>(ws) + kAttnPartOff;
  p.err = err_word(ws);
  p.B = B;
  p.total = total;
  p.n_q = n_q;
  p.n_kv = n_kv;
  p.g = n_q / n_kv;
  p.tpt = kRows / p.g;
  p.scale = scale;
  p.scale_log2 = scale * 1.4426950408889634f;
  return p;
}

}  // namespace

extern "C" size_t ee_prompt_workspace_size(void) {
  return kAttnPartOff + (size_t)4 * kNumSMsMax * kAttnPartBytes;
}

extern "C" ee_status ee_prompt_attn(const ee_bf16* q, int64_t q_stride, const ee_bf16* k, int64_t k_stride,
                                    const ee_bf16* v, int64_t v_stride, const int32_t* tok_off, int32_t B,
                                    int32_t total, int32_t n_q, int32_t n_kv, int32_t head_dim, float scale,
                                    ee_bf16* out, float* lse_or_null, void* ws, size_t ws_bytes,
                                    ee_stream_t stream) {
  const ee_status st = check(q, q_stride, k, v, tok_off, B, total, n_q, n_kv, head_dim, scale, out, lse_or_null, ws,
                             ws_bytes);
  if (st != EE_OK || B == 0 || total == 0) return st;
  if (!good_stride(k_stride, n_kv) || !good_stride(v_stride, n_kv)) return EE_ERR_INVALID_ARG;
  int dev = 0, ctas = 0;
  ee_status ds = current_device(&dev);
  if (ds == EE_OK) ds = resident_ctas(dev, &ctas);
  if (ds != EE_OK) return ds;
  PromptParams p = params(tok_off, B, total, n_q, n_kv, scale, out, lse_or_null, ws);
  p.v = reinterpret_cast<const __nv_bfloat16*>(v);
  p.v_stride = v_stride;
  CUtensorMap tmQ, tmK, tmV;
  if (!token_map(&tmQ, q, n_q, total, q_stride, p.g, p.tpt) || !token_map(&tmK, k, n_kv, total, k_stride, 1, kKT) ||
      !token_map(&tmV, v, n_kv, total, v_stride, 1, kKT))
    return EE_ERR_CUDA;
  return launch<false>(tmQ, tmK, tmV, p, ctas, stream);
}

extern "C" ee_status ee_chunk_attn(const ee_bf16* q, int64_t q_stride, const ee_bf16* k_cache, const ee_bf16* v_cache,
                                   int32_t num_pages, const int32_t* block_table, int32_t max_pages,
                                   const int32_t* ctx_len, const int32_t* tok_off, int32_t B, int32_t total,
                                   int32_t n_q, int32_t n_kv, int32_t head_dim, float scale, ee_bf16* out,
                                   float* lse_or_null, void* ws, size_t ws_bytes, ee_stream_t stream) {
  if (num_pages < 1 || max_pages < 1) return EE_ERR_INVALID_ARG;
  const ee_status st = check(q, q_stride, k_cache, v_cache, tok_off, B, total, n_q, n_kv, head_dim, scale, out,
                             lse_or_null, ws, ws_bytes);
  if (st != EE_OK || B == 0 || total == 0) return st;
  if (!block_table || !ctx_len) return EE_ERR_INVALID_ARG;
  if ((int64_t)num_pages * n_kv * EE_PAGE >= ((int64_t)1 << 31) || max_pages >= (1 << 27)) return EE_ERR_UNSUPPORTED;
  int dev = 0, ctas = 0;
  ee_status ds = current_device(&dev);
  if (ds == EE_OK) ds = resident_ctas(dev, &ctas);
  if (ds != EE_OK) return ds;
  PromptParams p = params(tok_off, B, total, n_q, n_kv, scale, out, lse_or_null, ws);
  p.v = reinterpret_cast<const __nv_bfloat16*>(v_cache);
  p.block_table = block_table;
  p.ctx_len = ctx_len;
  p.num_pages = num_pages;
  p.max_pages = max_pages;
  CUtensorMap tmQ, tmK, tmV;
  const uint64_t dims[2] = {(uint64_t)kD, (uint64_t)num_pages * n_kv * EE_PAGE};
  const uint64_t strides[1] = {(uint64_t)kD * 2};
  const uint32_t box[2] = {64, EE_PAGE};
  if (!token_map(&tmQ, q, n_q, total, q_stride, p.g, p.tpt) || !encode_bf16_tmap(&tmK, k_cache, 2, dims, strides, box) ||
      !encode_bf16_tmap(&tmV, v_cache, 2, dims, strides, box))
    return EE_ERR_CUDA;
  return launch<true>(tmQ, tmK, tmV, p, ctas, stream);
}
