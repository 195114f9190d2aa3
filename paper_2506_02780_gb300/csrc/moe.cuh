// ee_moe_layer's workspace and the launch of its first kernel (moe_route.cu).  Internal header.
//
// An ENTRY is a token at one of its experts; entries are numbered by expert, then by token.
// A token TILE is up to 32, 64 or 128 entries of one expert.
#pragma once
#include "few.cuh"

namespace ee {

constexpr int kMoeMaxTopK = 16;
constexpr int kMoeMaxExperts = 256;
constexpr int kMoeMaxTokens = 4096;
// Entries of a tile (moe_experts.cu): no more than a call's tokens, for an expert has no more.  On 8-bit weights tiles of 128 have tokens on the
// MMA's lanes, and empty lanes cost as much as full ones, so 64 is taken up to 64 entries an expert (us by 64 and by 128, 64 experts of
// 1,280 x 3,584 with so many entries each: 2 110 and 118, 6 136 and 146, 28 150 and 162, 54 179 and 185, 64 201 and 200, 94 255 and 228).  On
// bf16 ones an empty column costs nothing in either and a second tile a stream of weights from L2 (6 256 and 257, 28 276 and 277, 54 307 and
// 304, 94 366 and 337).
inline int moe_tile_rows(int64_t T, int64_t E, int64_t k, bool fp8) {
  return T <= 32 ? 32 : T <= 64 || (fp8 && T * k <= 64 * E) ? 64 : 128;
}

// counters in front of the workspace's arrays, set by the routing kernel
struct MoeCtl {
  uint32_t route_ticket;     // zero between calls
  uint32_t queue;            // next task of the experts' kernel
  uint32_t down_done;        // down tasks that stored their part of y (few tokens: gate tasks, of h)
  uint32_t tiles;            // token tiles
  uint32_t pad[4];
  uint32_t group_ticket[kMoeMaxTokens / 16];   // per 16 tokens; zero between calls
  uint32_t gate_done[1];     // per token tile: gate tasks that stored their part of h
};
struct __align__(32) MoeTile {   // a token tile's expert
  int expert, entry0, count;   // its first entry and their number
  int first, tiles;            // its first tile and their number
  int pad[3];
};
constexpr int kFewEntries = 8, kFewTokens = 8;   // what moe_few.cu takes
constexpr int kRouteParts = 8, kRouteCtas = 2 * kNumSMs;   // CTAs that share the hidden dimension, at most; so many in all

struct MoeLayout {
  size_t ctl, tile, part, ids, prob, list, inv, xq, xs, h, hf, hs, y, total;
  int max_tiles;             // token tiles of all experts, at most
};
inline MoeLayout moe_layout(int64_t T, int64_t H, int64_t I, int64_t E, int64_t k) {
  MoeLayout l;
  const int64_t n = T * k;
  l.max_tiles = (int)(std::min(E, n) + n / 64);   // (32 only where no expert can have more)
  size_t at = align_up(kWorkspaceBytes, 256);
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at = align_up(at + bytes, 256);
    return here;
  };
  l.ctl = take(sizeof(MoeCtl) + 4 * (size_t)l.max_tiles);
  l.tile = take(sizeof(MoeTile) * (size_t)l.max_tiles);
  l.part = take(4 * (size_t)(std::min<int64_t>(kRouteParts * T, 16 * kRouteCtas) * E));
  l.ids = take(4 * (size_t)n);
  l.prob = take(4 * (size_t)n);
  l.list = take(4 * (size_t)n);
  l.inv = take(4 * (size_t)n);
  l.xq = take((size_t)(T * H));
  l.xs = take(4 * (size_t)(T * ((H + kBlk - 1) / kBlk)));
  l.h = take(2 * (size_t)(n * I));
  l.hf = take(4 * (size_t)(kFewEntries * I));
  l.hs = take(4 * (size_t)(n * ((I + kBlk - 1) / kBlk)));
  l.y = take(4 * (size_t)(n * H));
  l.total = at;
  return l;
}

struct RouteParams {
  const __nv_bfloat16* x;
  int64_t x_stride;
  const __nv_bfloat16* router;
  const int32_t* live;       // or NULL
  int T, H, E, k, renorm, cl, max_tiles, tile_rows;
  MoeCtl* ctl;
  MoeTile* tile;
  float* part;               // [cl][T][E] sums over a CTA's columns
  int few;                   // moe_few.cu chooses itself
  int32_t* ids;              // [T][k] experts of a token, ascending
  float* prob;               // [T][k]
  int32_t* list;             // [T k] token of an entry
  int32_t* inv;              // [T][k] entry of a token's j-th expert
  uint8_t* xq;               // [T][H] codes of x (NULL: not wanted)
  float* xs;                 // [blocks][T]
  int32_t* ids_out;          // the caller's copies, or NULL
  float* prob_out;
};
ee_status launch_moe_route(RouteParams& p, cudaStream_t stream);   // sets cl

// larger key, better logit; at least 1: a NaN is the worst
__device__ __forceinline__ uint32_t logit_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return f != f ? 1u : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
// A warp chooses one token's k experts; lane holds those of number lane + 32 i.  Lane j < k: an expert, its weight
// and its place among the chosen ones in ascending order.
struct MoeChoice {
  int expert, place;
  float p;
};
template <int kPer, class Logit>
__device__ __forceinline__ MoeChoice choose_of(const Logit& logit, int E, int k, bool renorm, int lane) {
  float l[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) l[i] = lane + 32 * i < E ? logit(lane + 32 * i) : 0.f;
  uint32_t key[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) key[i] = lane + 32 * i < E ? logit_key(l[i]) : 0u;
  MoeChoice c;
  c.expert = 0x7fffffff;
  float my_l = 0.f, top = 0.f;
  for (int j = 0; j < k; ++j) {
    uint32_t best = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) best = max(best, key[i]);
    const uint32_t all = __reduce_max_sync(0xffffffffu, best);
    uint32_t e = 0xffffffffu;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i)
      if (key[i] == all) e = lane + 32 * i;
    e = __reduce_min_sync(0xffffffffu, e);         // of equal logits the lowest expert
    float le = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (e == (uint32_t)(lane + 32 * i)) {
        le = l[i];
        key[i] = 0;
      }
    le = __shfl_sync(0xffffffffu, le, e & 31);
    if (j == 0) top = le;
    if (lane == j) {
      c.expert = (int)e;
      my_l = le;
    }
  }
  float sum = 0.f;
  const float pe = lane < k ? expf(my_l - top) : 0.f;
  if (renorm) {
    sum = pe;
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (lane + 32 * i < E) sum += expf(l[i] - top);
  }
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  c.place = 0;
  for (int j = 0; j < k; ++j) c.place += __shfl_sync(0xffffffffu, c.expert, j) < c.expert;
  c.p = __fdiv_rn(pe, sum);
  return c;
}
__device__ __forceinline__ MoeChoice choose_experts(const float* logits, int E, int k, bool renorm, int lane) {
  const auto logit = [logits](int e) { return logits[e]; };
  return E <= 64 ? choose_of<2>(logit, E, k, renorm, lane) : choose_of<kMoeMaxExperts / 32>(logit, E, k, renorm, lane);
}

struct MoeParams {
  int T, H, I, E, k, n;                // n = T k
  int KB1, KB2;                        // 128-byte blocks along H and I
  int HT;                              // down tasks of a token tile
  int IB, HB;                          // blocks of 128 along I (gate tasks, too) and H
  int b_rows, stages;
  const void* w1;
  const void* w2;
  const void* x;                       // codes or bf16
  int64_t x_stride;
  MoeCtl* ctl;
  const MoeTile* tile;
  const float* part;                   // [cl][T][E] parts of the logits
  int cl, renorm;
  int32_t* ids_out;
  float* prob_out;
  const int32_t* list;
  const int32_t* inv;
  const float* prob;
  const float* xs;                     // [blocks of H][T]
  const float* s1;                     // [E][2][IB][blocks of H]
  const float* s2;                     // [E][HB][blocks of I]
  void* h;                             // [n][I] codes or bf16
  float* hf;                           // [n][I] h before it is quantised (few tokens)
  float* hs;                           // [IB][n]
  float* y;                            // [n][H]
  __nv_bfloat16* out;
  int64_t out_stride;
  int vec;                             // rows of out are 8-byte aligned
  const int32_t* live;
  int32_t* err;
};
// Up to 8 entries whose x and h fit in shared memory beside the rings (moe_few.cu): their depth and the bytes, or 0.
int moe_few_stages(int T, int H, int I, int k, bool fp8, size_t* smem);
ee_status launch_moe_few(MoeParams& p, bool fp8, cudaStream_t stream);

}  // namespace ee
