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
// while one's scores are in the softmax the tensor core works for the other.  (B sharing
// A's rows where a unit has one row tile only, each on every other key tile, gained nothing:
// such calls are bound by the cache.)
//
// Work.  The keys of all units (plus a constant for each: a unit's start and end) are
// laid on one line, cut into equal shares, one for each CTA; one CTA runs on each SM.
// A share may begin and end inside a unit.  Such a unit's pieces are joined with weights
// 2^(m - max): of up to kDirect pieces the last to finish joins the partials (m, l,
// unnormalised O) that the others left in the workspace to its own O on the way out,
// nobody waits; of more, all leave theirs, and the last to finish joins them or, in a
// call of few long units, all meet at a count and each join a part (such a call is
// launched cooperatively, so that the wait ends).  Every length follows from the device's
// offsets: long prompts, ragged batches and single tokens over long contexts are one case.
//
// Bound, and measured (captured / calls one after another, where the long ones run at the
// power cap).  Long rows: the tensor core, as far as the chain S -> P -> P V -> next S of
// the two row tiles keeps it busy: 128 keys of both take 2,700 cycles, of which the MMAs
// need 2,048 (S and P of both and both O fill tensor memory, so S of the next tile waits
// for P V of this one).  One prompt of 16384 tokens, 28 heads over 4: 1,156 / 1,250 us
// (1,660 / 1,540 TFLOP/s); a chunk of 2048 after 30720, 56 heads over 8: 1,135 / 1,230 us
// (1,640 / 1,515).  Ragged batches: also a segment's start and end, about 4,500 cycles that
// no product covers (the next segment's receipt, its first S, the last P V and the output
// follow one another), and the CTAs' imbalance (5%): 16 prompts of 33 to 4097 tokens 184 /
// 197 us, 1,250 / 1,165 TFLOP/s.  Single tokens: the cache, 64 sequences of 1024 to 16384
// keys 140 / 141 us, 5.6 TB/s, where loads of random pages alone reach 6.2.  One token over
// 4096 keys: latency, 12.0 / 14.4 us (4,000 cycles until the roles start, 5,000 until the
// first page is asked for, 7,000 for its tile, 6,000 to meet and join); a prompt of 37
// tokens, 8 heads over 2: 7.8 / 9.3 us.
//
// Roles of a CTA's twelve warps; all walk the share's segments (tile ranges of units)
// by themselves, from a ring the scheduler fills:
//   0      streams K and V tiles by TMA into a ring of four 32 KB slots;
//   1      issues the MMAs: per tile and row tile P V of this one, then Q K^T of the
//          next (whose S takes the place of P: MMAs of one thread run in order);
//   2      finds the segments, streams Q;
//   3      cleans V where the causal edge or the sequence's end lies in a tile: the
//          MMA multiplies masked rows by P = 0, and 0 times a NaN is a NaN.  Non-finite
//          values of rows that some query must not see are zeroed, and added at the end
//          (of a split unit: when its pieces are joined) for the queries that do;
//   4-7    softmax and output of row tile A, one row per thread; 8-11 of row tile B.
//          (Output by four warps of its own: 214 us instead of 190 for the 16 prompts.)
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
constexpr uint32_t kOffKV = 0, kOffQ = kRing * kTile, kOffOut = kOffQ + 2 * kTile;
constexpr uint32_t kOutBytes = 32 * 128;      // a softmax warp's rows x 64 columns of bf16, on their way out
constexpr uint32_t kOffBar = kOffOut + 8 * kOutBytes;
constexpr uint32_t kNumBars = 2 * kRing + 4 + 10 + 3 * kSegs + kZones + 1;
constexpr uint32_t kSmemBytes = 1024 + kOffBar + 8 * kNumBars;
constexpr uint32_t kTmemCols = 512, kColO = 256;
constexpr float kRescaleLog2 = 8.0f;          // O is rescaled when a maximum grows by 2^8
// Work in keys: the smallest share of a CTA, a unit's own constant, and how near (in tiles)
// a cut comes to a unit's start or end before it moves there, for calls of many rows and of
// few (see params).  Constants of 128 / 160 / 192 / 256 / 320 keys: 16 packed prompts take 200 /
// 187 / 182 / 185 / 189 us.
constexpr int kShareMany = 5 * kKT, kUnitMany = 192, kSnapMany = 2;
constexpr int kShareFew = kKT, kUnitFew = 128, kSnapFew = 1;
static_assert(kShareFew >= kKT, "every CTA between a unit's first and last piece holds one");
constexpr int kWarpKV = 0, kWarpMma = 1, kWarpQ = 2, kWarpClean = 3, kWarpSoft = 4;
constexpr int kVBox = 32;                     // packed V: rows of a box
constexpr int kSegReaders = 3 + 8;            // warps 0, 1, 3 and the softmax warps
static_assert(kRing == 4, "two slots each for K and V tiles");
static_assert(kSmemBytes <= 227 * 1024 - 1024, "shared memory budget");
// counts of a split unit's finished pieces, in the trailer of its first piece's slots
// past the word that the verification attention keeps there: one for each softmax
// warp (units of at most kDirect pieces), one for all (of more)
constexpr size_t kCntOff = kAttnCntOff + 64, kCntAllOff = kAttnCntOff + 128;
constexpr int kDirect = 3;

struct PromptParams {
  const __nv_bfloat16* v;       // V once more, for values the MMA must not see
  int64_t v_stride;
  const int32_t *block_table, *ctx_len, *tok_off;
  __nv_bfloat16* out;
  float* lse;
  uint8_t* part;
  int32_t* err;
  int B, total, num_pages, max_pages, n_q, n_kv, g, tpt;
  int units;                    // of the call, at most
  int min_share, coop;
  int unit_keys, snap;
  float scale, scale_log2;
};

// The code that a CTA runs over and over is kept small (loops over the two row tiles
// and over column blocks stay rolled): warps of six kinds share one instruction cache, and
// a segment's start and end run all of it (of its requests 4.5% miss in 16 packed prompts,
// 0.9% in a long one).
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

// The larger of m and 32 scores (a NaN is passed over).
__device__ __forceinline__ float max32(const uint32_t (&x)[32], float m) {
  float a = m, b = __uint_as_float(x[0]);
#pragma unroll
  for (int k = 1; k < 31; k += 4) {
    a = fmax3(a, __uint_as_float(x[k]), __uint_as_float(x[k + 1]));
    if (k + 3 < 32) b = fmax3(b, __uint_as_float(x[k + 2]), __uint_as_float(x[k + 3]));
  }
  return fmax3(a, b, __uint_as_float(x[31]));
}
// P = 2^(S sl2 + nms) of 32 scores, rounded to bf16 and packed; the fp32 values are added
// to ls.  Scale and shift and the sums take one packed instruction a pair.  P V takes P in
// one bf16 word (in two, as the verification attention has it, P V would take twice the
// tensor time and P all of S's columns): a probability is off by 2^-9 of itself at most,
// either way, and l is not, so that outputs are 1.05 to 1.4 times as far from 64 bits as
// with P in 32 bits, most of which is the output's own rounding to bf16.
__device__ __forceinline__ void exp32(const uint32_t (&x)[32], uint64_t sl2x2, uint64_t nmsx2, uint64_t (&ls)[2],
                                      uint32_t (&pw)[16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    uint32_t y0, y1;
    f2_unpack(f2_fma(f2_pack(x[2 * e], x[2 * e + 1]), sl2x2, nmsx2), y0, y1);
    const float p0 = ex2(__uint_as_float(y0)), p1 = ex2(__uint_as_float(y1));
    ls[e & 1] = f2_add(ls[e & 1], f2_pack(__float_as_uint(p0), __float_as_uint(p1)));
    pw[e] = bf16x2_rn(p1, p0);
  }
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
// tpt, keys ctx + min(T, (n + 1) w); it takes that many places plus `u`: unit_keys + 64
// (half a tile: the last one is rarely full).
__device__ __forceinline__ int num_units(int T, int w) { return (T + w - 1) / w; }
// places of a sequence and head before unit n (n below the number of units)
__device__ __forceinline__ int64_t places_before(int ctx, int w, int u, int64_t n) {
  return n * ((int64_t)ctx + u) + n * (n + 1) / 2 * w;
}
__device__ __forceinline__ int64_t head_places(int ctx, int T, int w, int u) {
  if (T == 0) return 0;
  const int64_t P = num_units(T, w);
  return places_before(ctx, w, u, P - 1) + ctx + T + u;
}
// tiles of a unit of n that lie before place y of it; a cut within `snap` tiles of the
// unit's start or end moves there
__device__ __forceinline__ int tiles_before(const PromptParams& p, int64_t y, int n) {
  const int64_t j = (y - p.unit_keys + kKT / 2) >> 7;
  return j < p.snap ? 0 : j > n - p.snap ? n : (int)j;
}
// the first places that tiles_before puts past the unit's start, and at its end
__device__ __forceinline__ int past_start(const PromptParams& p) { return p.unit_keys - kKT / 2 + p.snap * kKT; }
__device__ __forceinline__ int at_end(const PromptParams& p, int n) {
  return p.unit_keys - kKT / 2 + (n - p.snap + 1) * kKT;
}
// W places (below 2^56) cut for N CTAs: CTA c's share starts at floor(c W / N)
struct Shares {
  int64_t W, q;      // q = W / N, r = W mod N, by two 32-bit divisions
  int N, r;
  uint32_t inv;      // 2^32 / N rounded up: (x inv) >> 32 = x / N for x below 2^17
  __device__ __forceinline__ Shares(int64_t w, int n) : W(w), N(n), inv(0xFFFFFFFFu / (uint32_t)n + 1) {
    const uint32_t a = (uint32_t)(w >> 24), b = (uint32_t)w & 0xFFFFFFu;
    const uint32_t q1 = a / (uint32_t)n, lo = ((a - q1 * (uint32_t)n) << 24) + b, q0 = lo / (uint32_t)n;
    q = ((int64_t)q1 << 24) + q0;
    r = (int)(lo - q0 * (uint32_t)n);
  }
  __device__ __forceinline__ int64_t start(int c) const {
    return q * c + (N == 1 ? 0 : (int)__umulhi((uint32_t)(r * c), inv));
  }
  // the last CTA whose share starts before place y (y > 0)
  __device__ __forceinline__ int before(int64_t y) const {
    int c = min(max((int)(__fdividef((float)y, (float)W) * N), 0), N - 1);   // put right below
#pragma unroll 1
    while (start(c) >= y) --c;
#pragma unroll 1
    while (c + 1 < N && start(c + 1) < y) ++c;
    return c;
  }
};

// A segment: tiles [j0, j1) of a unit.
struct Seg {
  int s, o, T, ctx;        // sequence
  int hk, tok0;            // KV head, the unit's first token
  int j0, j1, n_tiles;     // n_tiles: of the whole unit; j1 = 0: no more segments
  int kA, kB;              // keys each row tile needs (B: 0 without tokens)
  int c0, c1;              // first and last CTA that hold a piece (a split unit: set after the rest)
  int64_t X;               // the unit's first place
};

// Whether tile j of the unit holds keys that the first query must not see.
__device__ __forceinline__ bool in_zone(const Seg& s, int j) { return j * kKT + kKT - 1 > s.ctx + s.tok0; }
__device__ __forceinline__ bool active(const Seg& s, int st, int j) { return j * kKT < (st ? s.kB : s.kA); }
// Halves of tile j that row tile st needs (of the last one half is often enough: the second
// half's exponentials and product are left out).
__device__ __forceinline__ int halves(const Seg& s, int st, int j) { return (st ? s.kB : s.kA) - j * kKT > kKT / 2 ? 2 : 1; }

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

// Non-finite values of V that warp 3 took out of the unit's tiles (keys past the first
// query's): a row that sees some gets them added once, unweighted, on its way out, whoever
// joins its pieces.  Partials do not hold them; a piece that met one says so by the sign of
// its l.
//
// To one row's output in memory.
template <bool kPaged>
__device__ __forceinline__ void add_nonfinite(const PromptParams& p, const Seg& s, int pos, __nv_bfloat16* out) {
#pragma unroll 1
  for (int key = s.ctx + s.tok0 + 1; key <= pos; ++key) {
    const __nv_bfloat16* v = v_row<kPaged>(p, s, key);
    if (!v) continue;
#pragma unroll 1
    for (int e = 0; e < kD; ++e) {
      const float x = __bfloat162float(v[e]);
      if (isfinite(x)) continue;
      volatile uint16_t* o = reinterpret_cast<volatile uint16_t*>(out) + e;
      *o = __bfloat16_as_ushort(__float2bfloat16_rn(__bfloat162float(__ushort_as_bfloat16(*o)) + x));
    }
  }
}
// To eight of one row's columns in registers.
template <bool kPaged>
__device__ __forceinline__ void add_nonfinite8(const PromptParams& p, const Seg& s, int pos, int col, float (&y)[8]) {
#pragma unroll 1
  for (int key = s.ctx + s.tok0 + 1; key <= pos; ++key) {
    const __nv_bfloat16* v = v_row<kPaged>(p, s, key);
    if (!v) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = __bfloat162float(v[col + e]);
      if (!isfinite(x)) y[e] += x;
    }
  }
}

__device__ __forceinline__ uint32_t nonfinite2(uint32_t x) {   // 0xffff in each half that is
  const uint32_t lo = (x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u;
  const uint32_t hi = (x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
  return lo | hi;
}

// A partial's (m, l): m is NaN where the piece has no tile of the row tile, and no O then
// (a row's own maximum is never NaN); l's sign says that values were taken out of V.
__device__ __forceinline__ float2 pack_ml(bool any, bool bad, float m, float l) {
  const uint32_t sign = bad ? 0x80000000u : 0u;
  return make_float2(any ? m : NAN, __uint_as_float((__float_as_uint(l) & 0x7fffffffu) | sign));
}
__device__ __forceinline__ bool no_tiles(float m) { return m != m; }
__device__ __forceinline__ bool took_out(float l) { return (int32_t)__float_as_uint(l) < 0; }

// (m, l, o) of one piece or lane joined to a running one
struct Joined {
  float M = -INFINITY, L = 0.f, a[8] = {};
  __device__ __forceinline__ void add(float m, float l, const float (&o)[8]) {
    const float m_new = fmaxf(M, m);
    const float fa = M == m_new ? 1.f : ex2(M - m_new), fb = m == m_new ? 1.f : ex2(m - m_new);
    M = m_new;
    L = fmaf(L, fa, l * fb);
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = fmaf(a[e], fa, o[e] * fb);
  }
};

// Items [lo, hi) of a split unit merged by one of its pieces: thread t of nthr.  An
// item is eight columns of a row, numbered rows fastest, so that a warp's loads of a
// slot (column-chunk major) are contiguous.  A thread loads from two pieces at a time (a
// round trip to L2 costs about 1,000 cycles).  With few items and many pieces 2^sub lanes
// share an item, each over every 2^sub-th piece.
template <bool kPaged>
__device__ __forceinline__ void merge_items(const PromptParams& p, const Seg& s, int lo, int hi, int t, int nthr) {
  const int K = s.c1 - s.c0 + 1;
  // (the sum's order depends on it: where any piece's CTA may be the one that joins, it must
  // not follow from how many units that one has)
  const int lanes = p.coop ? nthr : kThreads / 2;
  int sub = 0;
#pragma unroll 1
  while (sub < 5 && 1 << sub < K && (hi - lo) << (sub + 1) <= lanes) ++sub;
  const int nt = min(2 * p.tpt, s.T - s.tok0);               // tokens of the unit
  const int rows_a = min(nt, p.tpt) * p.g, rows = nt * p.g;  // rows of A, of both
  const int k0 = t & ((1 << sub) - 1);
  // whole warps walk together: the lanes of an item meet in shuffles
#pragma unroll 1
  for (int i0 = lo + (t >> sub); i0 - ((t & 31) >> sub) < hi; i0 += nthr >> sub) {
    const int i = min(i0, hi - 1), cg = i / rows, r = i - cg * rows;
    const int st = r >= rows_a, rr = st ? r - rows_a : r;
    Joined x;
    bool bad = false;
#pragma unroll 1
    for (int k = k0; k < K; k += 2 << sub) {
      float2 ml[2];
      float4 u[2], v[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int kk = min(k + (q << sub), K - 1), c = s.c0 + kk;   // CTA c's last segment, or its first
        const uint8_t* slot = p.part + (size_t)(2 * (2 * c + (kk == 0)) + st) * kAttnPartBytes;
        const float4* O = reinterpret_cast<const float4*>(slot) + (size_t)(2 * cg) * kRows + rr;
        ml[q] = __ldcg(reinterpret_cast<const float2*>(slot + kAttnMlOff) + rr);
        u[q] = __ldcg(O);
        v[q] = __ldcg(O + kRows);
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (k + (q << sub) >= K || no_tiles(ml[q].x)) continue;
        const float o[8] = {u[q].x, u[q].y, u[q].z, u[q].w, v[q].x, v[q].y, v[q].z, v[q].w};
        x.add(ml[q].x, fabsf(ml[q].y), o);
        bad |= took_out(ml[q].y);
      }
    }
#pragma unroll 1
    for (int d = 1; d < 1 << sub; d *= 2) {
      float o[8];
      const float Mo = __shfl_xor_sync(0xffffffffu, x.M, d), Lo = __shfl_xor_sync(0xffffffffu, x.L, d);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = __shfl_xor_sync(0xffffffffu, x.a[e], d);
      x.add(Mo, Lo, o);
      bad |= __shfl_xor_sync(0xffffffffu, (int)bad, d) != 0;
    }
    if (k0 != 0 || i0 >= hi) continue;
    const float il = x.L == 0.f ? 0.f : 1.f / x.L;
    const int tok = rr / p.g, h = rr - tok * p.g;
    const size_t row = (size_t)(s.o + s.tok0 + (st ? p.tpt : 0) + tok) * p.n_q + s.hk * p.g + h;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x.a[e] * il;
    if (bad) add_nonfinite8<kPaged>(p, s, s.ctx + s.tok0 + (st ? p.tpt : 0) + tok, 8 * cg, y);
    uint4 o;
    o.x = bf16x2_rn(y[1], y[0]);
    o.y = bf16x2_rn(y[3], y[2]);
    o.z = bf16x2_rn(y[5], y[4]);
    o.w = bf16x2_rn(y[7], y[6]);
    *reinterpret_cast<uint4*>(p.out + row * kD + 8 * cg) = o;
    if (cg == 0 && p.lse) p.lse[row] = x.L == 0.f ? -INFINITY : (x.M + log2f(x.L)) * 0.6931471805599453f;
  }
}

template <bool kPaged>
__global__ void __launch_bounds__(kThreads, 1)
prompt_attn_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PromptParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem =
      reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ Seg s_seg[kSegs];
  __shared__ int s_bad[kSegs];                   // V values taken out of the segment's tiles
  __shared__ uint32_t s_mask[kMasks];            // per tile: 16-key blocks in a valid page
  __shared__ int64_t s_scan[kThreads / 32];
  __shared__ int s_first;                        // the share's first sequence,
  __shared__ Seq s_firstseq;
  __shared__ int64_t s_firstX;                   // and its first place
  __shared__ int s_kvissued[kRing], s_zissued[kZones], s_qissued[2];   // phases of copies started (-1: none)
  __shared__ Seg s_pc[2];                        // pieces of split units
  __shared__ int s_npc;
  __shared__ int s_ready[2];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sbase = smem_u32(smem);
  const uint32_t sKV = sbase + kOffKV, sQ = sbase + kOffQ, bar0 = sbase + kOffBar;
  const uint32_t kv_full = bar0, kv_empty = kv_full + 8 * kRing;
  const uint32_t q_full = kv_empty + 8 * kRing, q_empty = q_full + 16;
  const uint32_t s_full = q_empty + 16, p_half = s_full + 16, p_full = p_half + 16;
  const uint32_t pv_done = p_full + 16, o_free = pv_done + 16;
  const uint32_t seg_full = o_free + 16, seg_empty = seg_full + 8 * kSegs, z_full = seg_empty + 8 * kSegs;
  const uint32_t drain = z_full + 8 * kZones, cut_full = drain + 8;

  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmQ)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmK)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmV)) : "memory");
    s_abort = 0;
    s_npc = 0;
#pragma unroll 1
    for (int i = 0; i < kRing; ++i) s_kvissued[i] = -1;
#pragma unroll 1
    for (int i = 0; i < kZones; ++i) s_zissued[i] = -1;
#pragma unroll 1
    for (int i = 0; i < 2; ++i) s_qissued[i] = -1;
  }
  if (warp == kWarpKV) {   // one barrier a lane
#pragma unroll 1
    for (int i = lane; i < (int)kNumBars; i += 32) {
      const uint32_t bar = bar0 + 8 * i;
      const uint32_t count = bar >= s_full && bar < p_half      ? kPaged + 1   // the commit (paged: and the page mask's release)
                             : bar >= p_half && bar < pv_done   ? 4            // warps
                             : bar >= pv_done && bar < o_free   ? 2            // the commit, and a release of s_bad
                             : bar >= o_free && bar < seg_full  ? 4
                             : bar >= seg_empty && bar < z_full ? kSegReaders
                                                                : 1;
      mbar_init(bar, count);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // rows of the Q tiles past g * tpt are never loaded
#pragma unroll 1
  for (int i = tid; i < 2 * 2 * (kRows - p.g * p.tpt) * 8; i += kThreads) {
    const int c = i & 7, r = i >> 3, per = kRows - p.g * p.tpt;
    *reinterpret_cast<uint4*>(smem + kOffQ + (r / per) * kHalf + (p.g * p.tpt + r % per) * 128 + 16 * c) =
        make_uint4(0, 0, 0, 0);
  }
  fence_async_smem();
  pdl_wait();   // no global access before the previous kernel's writes are visible

  // ---- the line of work: its length, this CTA's share and where that begins ----
  const int w = 2 * p.tpt, u = p.unit_keys + kKT / 2;
  int64_t W = 0;
  int64_t base = 0, sum = 0;
  const int per = (p.B + kThreads - 1) / kThreads;   // sequences of a thread
  const int b0 = min(tid * per, p.B), b1 = min(b0 + per, p.B);
  Seq sq{0, 0, 0};
  {
    int err = 0;
#pragma unroll 1
    for (int s = b0; s < b1; ++s) {
      sq = load_seq<kPaged>(p, s, err);
      sum += head_places(sq.ctx, sq.T, w, u) * p.n_kv;
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
    // (the first warps hold all sequences)
#pragma unroll 1
    for (int i = 0; i < min((p.B + 31) / 32, kThreads / 32); ++i) {
      if (i < warp) base += s_scan[i];
      W += s_scan[i];
    }
    base += incl - sum;
  }
  // as many CTAs as the units or the shortest share allow
  // (W past the grid's worth of the larger share changes nothing: 32-bit divisions)
  const uint32_t Wc = (uint32_t)min(W, (int64_t)gridDim.x * kShareMany);
  const int want = max((int)(Wc / (uint32_t)p.min_share), min((int)(Wc / kShareFew), p.units));
  const Shares sh(W, min((int)gridDim.x, max(want, 1)));
  const bool works = (int)blockIdx.x < sh.N && W > 0;
  const int64_t x0 = works ? sh.start(blockIdx.x) : W, x1 = works ? sh.start(blockIdx.x + 1) : W;
  if (works && x0 >= base && x0 < base + sum) {
    int s = b0;
    if (per > 1) {
      int err = 0;
#pragma unroll 1
      for (;; ++s) {
        sq = load_seq<kPaged>(p, s, err);
        const int64_t n = head_places(sq.ctx, sq.T, w, u) * p.n_kv;
        if (x0 < base + n) break;
        base += n;
      }
    }
    s_first = s;
    s_firstseq = sq;
    s_firstX = base;
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
    if (warp == kWarpKV) {
      // ---------------- K and V tiles ----------------
      // The V tiles that warp 3 cleans signal it, and it signals the MMA warp.
      Seg s;
      int tile = 0, zone = 0;
      bool go = true;
#pragma unroll 1
      for (int i = 0; go && receive(i, s); ++i) {
        // paged: lane l holds the page of 16-key block l % 8 of the (l / 8)-th of four tiles
        const int last = s.ctx + min(s.T, s.tok0 + w) - 1;
        auto fetch = [&](int j) -> int32_t {
          const int key = (j + (lane >> 3)) * kKT + 16 * (lane & 7);
          const bool need = (j + (lane >> 3)) < s.j1 && key <= last;
          return need ? max(ld_pinned(p.block_table + (size_t)s.s * p.max_pages + key / EE_PAGE), -1) : INT32_MIN;
        };
        int32_t ids = INT32_MIN, ids_next = INT32_MIN;
        if constexpr (kPaged) ids_next = fetch(s.j0);
#pragma unroll 1
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
              // (rows wholly out of range are filled with zeros)
              row[b] = ok ? (id * p.n_kv + s.hk) * EE_PAGE : -EE_PAGE;
              okm |= ok || id == INT32_MIN ? 1u << b : 0u;   // past the unit: masked as such
              bad |= !ok && id != INT32_MIN;
            }
            if (bad && lane == 0) flag_error(p.err, EE_DEVERR_PAGE);
          }
#pragma unroll 1
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
              } else if (kv == 0) {
                tma_load_3d(dst, tm, full, 0, s.hk, s.o + j * kKT);
                tma_load_3d(dst + kHalf, tm, full, 64, s.hk, s.o + j * kKT);
              } else {
#pragma unroll
                for (int b = 0; b < kKT / kVBox; ++b) {
                  // boxes past the unit are filled with zeros
                  const int at = j * kKT + kVBox * b <= last ? s.o + j * kKT + kVBox * b : p.total;
                  tma_load_3d(dst + b * kVBox * 128, tm, full, 0, s.hk, at);
                  tma_load_3d(dst + kHalf + b * kVBox * 128, tm, full, 64, s.hk, at);
                }
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
      int s = works ? s_first : p.B, base = 0, err = 0;   // (a CTA without a share: none is set)
      bool loaded = false;
      Seq mine{0, 0, 0};
      auto load32 = [&](int from) {
        base = from;
        loaded = true;
        mine = Seq{0, 0, 0};
        if (base + lane < p.B) mine = load_seq<kPaged>(p, base + lane, err);
      };
      int64_t X = works ? s_firstX : x1;                      // the next unit's first place
      int o = 0, T = 0, ctx = 0, hk = 0, n = 0;
      auto take = [&]() {        // sequence s from its lane
        if (!loaded || s - base >= 32) load32(s);
        o = __shfl_sync(0xffffffffu, mine.o, s - base);
        T = __shfl_sync(0xffffffffu, mine.T, s - base);
        ctx = __shfl_sync(0xffffffffu, mine.ctx, s - base);
      };
      if (works) {
        o = s_firstseq.o;
        T = s_firstseq.T;
        ctx = s_firstseq.ctx;
        const int64_t per_head = head_places(ctx, T, w, u);
        int64_t rem = x0 - X;
        hk = min((int)__fdividef((float)rem, (float)per_head), p.n_kv - 1);
        rem -= hk * per_head;
#pragma unroll 1
        for (; rem < 0; rem += per_head) --hk;
#pragma unroll 1
        for (; rem >= per_head; rem -= per_head) ++hk;
        X += hk * per_head;
        // the last unit that starts at or before rem: places_before(n) <= rem solved for n,
        // then put right (the root is off by a few units at most)
        const int units = num_units(T, w);
        if (units > 1) {
          const float b = (float)(ctx + u) + 0.5f * w;
          n = min(max((int)((sqrtf(b * b + 2.f * w * (float)rem) - b) / w), 0), units - 1);
#pragma unroll 1
          while (places_before(ctx, w, u, n) > rem) --n;
#pragma unroll 1
          while (n + 1 < units && places_before(ctx, w, u, n + 1) <= rem) ++n;
        }
        X += places_before(ctx, w, u, n);
      }
      // the next non-empty segment of the share
      auto find = [&](Seg& g) -> bool {
#pragma unroll 1
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
          const int64_t len = keys + u;
          const int j0 = X < x0 ? tiles_before(p, x0 - X, tiles) : 0;
          const int j1 = x1 >= X + len ? tiles : tiles_before(p, x1 - X, tiles);
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
          g.kA = ctx + min(T, tok0 + p.tpt);
          g.kB = T > tok0 + p.tpt ? keys : 0;
          g.c0 = g.c1 = 0;
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
          mbar_arrive(seg_full + 8 * (i % kSegs));
        }
        __syncwarp();
        return true;
      };
      // Which CTAs hold the unit's pieces, needed at the segment's end: after the segment and
      // its Q are on their way (it takes about 800 cycles)
      auto cut = [&](int i, Seg& g) {
        if (g.j1 - g.j0 < g.n_tiles) {
          // the first piece is that of the last CTA whose share starts before past_start,
          // the last piece that of the last whose share starts before at_end; shares are
          // no shorter than a tile, so every CTA between them holds one
          g.c0 = sh.before(g.X + past_start(p));
          g.c1 = sh.before(g.X + at_end(p, g.n_tiles));
        }
        if (lane == 0) {
          s_seg[i % kSegs].c0 = g.c0;
          s_seg[i % kSegs].c1 = g.c1;
          if (g.c1 - g.c0 >= kDirect) {
            s_pc[s_npc & 1] = g;
            s_npc = s_npc + 1;
          }
          mbar_arrive(cut_full + 8 * (i % kSegs));
        }
        __syncwarp();
      };
      // The first segment's Q is loaded at once; from then on segment i is published
      // before Q of segment i - 1, whose buffer may still be in use, is waited for.
      Seg cur, nxt;
      uint32_t q_phase = 3;      // bit st: parity that the row tile's Q buffer is free at
      bool go = true, more = true, pending = false;
#pragma unroll 1
      for (int i = 0; go && more; ++i) {
        more = find(nxt);
        go = publish(i, nxt);
        if (i == 0) cur = nxt;
#pragma unroll 1
        for (int st = 0; st < 2 && go && (pending || (i == 0 && more)); ++st) {
          if (!active(cur, st, cur.j0)) continue;
          go = wait(q_empty + 8 * st, q_phase >> st);
          if (go && elect_one()) {
            const uint32_t full = q_full + 8 * st, dst = sQ + st * kTile;
            const int tok = cur.o + cur.tok0 + st * p.tpt;
            mbar_expect_tx(full, 2u * 128u * p.g * p.tpt);
            tma_load_3d(dst, &tmQ, full, 0, cur.hk * p.g, tok);
            tma_load_3d(dst + kHalf, &tmQ, full, 64, cur.hk * p.g, tok);
            s_qissued[st] = (int)(~q_phase >> st & 1);
          }
          __syncwarp();
          q_phase ^= 1u << st;
        }
        if (go && more) cut(i, nxt);
        cur = nxt;
        pending = i > 0;
        if (!loaded && more) load32(s + 1);   // the sequences to come, beside the first segment's work
      }
    } else if (warp == kWarpClean) {
      // ---------------- V where a query's last key or the unit's last lies inside a tile ----
      Seg s;
      int tile = 0, zone = 0;
      bool go = true;
#pragma unroll 1
      for (int i = 0; go && receive(i, s); ++i) {
        const int first = s.ctx + s.tok0, last = s.ctx + min(s.T, s.tok0 + w) - 1;
#pragma unroll 1
        for (int j = s.j0; j < s.j1 && go; ++j, ++tile) {
          if (!in_zone(s, j)) continue;
          const int slot = (2 * tile + 1) % kRing;
          go = wait(z_full + 8 * (zone % kZones), zone / kZones);
          if (!go) break;
          uint8_t* v = smem + kOffKV + slot * kTile;
          // rows that some query must not see, and where those end that one does; past the
          // box that holds the last of them the tile is zero
          const int r0 = max(first + 1 - j * kKT, 0), r1 = min(last + 1 - j * kKT, kKT);
          const int r2 = kPaged ? (r1 + EE_PAGE - 1) / EE_PAGE * EE_PAGE : (r1 + kVBox - 1) / kVBox * kVBox;
          // a row's 128 bytes in each half are a permutation of its 16-byte chunks;
          // four loads in flight, and nothing to write as a rule
          bool seen = false, wrote = false;
#pragma unroll 1
          for (int c0 = r0 * 8 + lane; c0 < r2 * 8; c0 += 2 * 32) {
            uint4 x[4];
            uint32_t any = 0;      // (e + 1) << 7 reaches bit 15 where the exponent is all ones
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const int c = min(c0 + 32 * (u >> 1), r2 * 8 - 1);
              x[u] = *reinterpret_cast<const uint4*>(v + (u & 1) * kHalf + 16 * c);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
              any |= ((x[u].x & 0x7f807f80u) + 0x00800080u) | ((x[u].y & 0x7f807f80u) + 0x00800080u) |
                     ((x[u].z & 0x7f807f80u) + 0x00800080u) | ((x[u].w & 0x7f807f80u) + 0x00800080u);
            if (!(any & 0x80008000u)) continue;
            wrote = true;
#pragma unroll 1
            for (int u = 0; u < 4; ++u) {
              const int c = min(c0 + 32 * (u >> 1), r2 * 8 - 1);
              uint4* a = reinterpret_cast<uint4*>(v + (u & 1) * kHalf + 16 * c);
              const uint4 y = *a;
              const uint32_t m0 = nonfinite2(y.x), m1 = nonfinite2(y.y), m2 = nonfinite2(y.z), m3 = nonfinite2(y.w);
              seen |= (m0 | m1 | m2 | m3) != 0 && (c >> 3) < r1;
              *a = make_uint4(y.x & ~m0, y.y & ~m1, y.z & ~m2, y.w & ~m3);
            }
          }
          if (wrote) fence_async_smem();   // generic-proxy writes, read by the tensor core
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
      const uint64_t dv0 = smem_desc_sw128_mn(__shfl_sync(0xffffffffu, sKV + kTile, 0), kHalf, 1024);
      // (within elect_one) S = Q K^T of row tile st, K in its slot `odd`
      auto qk = [&](int st, uint32_t odd) {
        const uint64_t dk = dk0 + (uint64_t)(odd * (2 * kTile >> 4));
        const uint64_t dq = dq0 + (uint64_t)(st * (kTile >> 4));
#pragma unroll
        for (int kk = 0; kk < kD / 16; ++kk) {
          const uint64_t off = ((kk >> 2) * kHalf + (kk & 3) * 32) >> 4;
          tc_mma(tmem + st * kKT, dq + off, dk + off, id_qk, kk > 0 ? 1u : 0u);
        }
        tc_commit(s_full + 8 * st);
        if constexpr (kPaged) mbar_arrive(s_full + 8 * st);   // releases the page mask (acquired with kv_full)
      };
      // (within elect_one) O += P V for half of the keys, V in its slot `odd`
      auto pv = [&](int st, uint32_t odd, int half, bool acc) {
        const uint64_t dv = dv0 + (uint64_t)(odd * (2 * kTile >> 4));
#pragma unroll
        for (int k = 0; k < kKT / 32; ++k) {
          const int kk = half * (kKT / 32) + k;
          tc_mma_ts(tmem + kColO + st * kD, tmem + st * kKT + 8 * kk, dv + (uint64_t)(kk * (2048 >> 4)), id_pv,
                    (acc || kk > 0) ? 1u : 0u);
        }
      };
      // A wait without a vote: `go` is this lane's, voted on once a step.  (An MMA issued
      // after a wait gave up reads stale operands; the outputs are then undefined anyway.)
      bool go = true;
      auto meet = [&](uint32_t bar, uint32_t parity) { go = mbar_wait(bar, parity & 1, &s_abort) && go; };
      // K and V of tile t: slots 2 (t & 1) and 2 (t & 1) + 1, both in their (t >> 1)-th use
      auto k_bar = [&](int t) { return kv_full + 16 * (t & 1); };
      auto v_bar = [&](int t) { return kv_full + 16 * (t & 1) + 8; };
      Seg s;
      s.j0 = s.j1 = s.kA = s.kB = 0;
      int i = -1, j = -1, tile = -1;   // before the first tile: a step without P V
      uint32_t p_phase = 0, q_phase = 0, o_phase = 3;
      while (go) {
        // ---- tiles that both row tiles need, up to the last but one, past a segment's
        // first: a wait between two products costs the tensor core what it takes (about
        // 100 cycles; the queue holds a few MMAs), so there is one before each half of P V
        // and none before Q K^T, and K and V are looked at beside the first
        const int both = j > s.j0 ? min(s.j1, (min(s.kA, s.kB) + kKT - 1) / kKT) - 1 : j;
#pragma unroll 1
        for (; j < both && go; ++j, ++tile) {
          const uint32_t odd = tile & 1;
#pragma unroll 1
          for (int st = 0; st < 2; ++st) {
            const bool v_in = mbar_try(v_bar(tile), (tile >> 1) & 1);
            const bool k_in = mbar_try(k_bar(tile + 1), ((tile + 1) >> 1) & 1);
            meet(p_half + 8 * st, p_phase);
            if (!v_in) meet(v_bar(tile), tile >> 1);
            if (!k_in) meet(k_bar(tile + 1), (tile + 1) >> 1);
            tc_fence_after();
            if (elect_one()) pv(st, odd, 0, true);
            __syncwarp();
            meet(p_full + 8 * st, p_phase);
            tc_fence_after();
            if (elect_one()) {
              pv(st, odd, 1, true);
              qk(st, odd ^ 1);
              if (j + 2 == s.j1 || !active(s, st, j + 2)) tc_commit(q_empty + 8 * st);
            }
            __syncwarp();
            p_phase = (p_phase >> 1) | ((~p_phase & 1) << 1);   // the bits take turns, each inverted
          }
          if (elect_one()) {
            tc_commit(kv_empty + 16 * odd + 8);
            tc_commit(kv_empty + 16 * (odd ^ 1));
          }
          go = __all_sync(0xffffffffu, go);
        }
        if (!go) break;
        // ---- any other tile: a segment's first or last, or one that one row tile needs ----
        Seg nx = s;
        int jn = j + 1;
        const bool cur = i >= 0, fresh = jn >= s.j1;
        bool has = true;
        if (fresh) {
          has = receive(i + 1, nx);
          jn = nx.j0;
          if (s_abort || !(cur || has)) break;
        }
        const uint32_t odd = tile & 1;
        if (cur) meet(v_bar(tile), tile >> 1);
        if (has) meet(k_bar(tile + 1), (tile + 1) >> 1);
#pragma unroll 1
        for (int st = 0; st < 2; ++st) {
          if (cur && active(s, st, j)) {
            if (j == s.j0) {   // the last segment's O is read
              meet(o_free + 8 * st, o_phase >> st);
              o_phase ^= 1u << st;
            }
            meet(p_half + 8 * st, p_phase >> st);
            tc_fence_after();
            if (elect_one()) pv(st, odd, 0, j > s.j0);
            __syncwarp();
            meet(p_full + 8 * st, p_phase >> st);
            p_phase ^= 1u << st;
            tc_fence_after();
            if (elect_one()) {
              if (halves(s, st, j) == 2) pv(st, odd, 1, true);
              if (fresh || !active(s, st, jn)) {
                tc_commit(pv_done + 8 * st);
                mbar_arrive(pv_done + 8 * st);   // releases s_bad (acquired with kv_full)
              }
            }
            __syncwarp();
          }
          if (has && active(nx, st, jn)) {
            if (fresh) {
              meet(q_full + 8 * st, q_phase >> st);
              q_phase ^= 1u << st;
            }
            tc_fence_after();
            if (elect_one()) {
              qk(st, odd ^ 1);
              if (jn + 1 == nx.j1 || !active(nx, st, jn + 1)) tc_commit(q_empty + 8 * st);
            }
            __syncwarp();
          }
        }
        if (elect_one()) {
          if (cur) tc_commit(kv_empty + 16 * odd + 8);
          if (has) tc_commit(kv_empty + 16 * (odd ^ 1));
        }
        __syncwarp();
        go = __all_sync(0xffffffffu, go) && has;
        if (fresh) {
          if (cur) release(i);
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
#pragma unroll 1
        for (int i = 0; i < kRing; ++i)
          if (s_kvissued[i] >= 0) mbar_wait_plain(kv_full + 8 * i, (uint32_t)(s_kvissued[i] & 1));
#pragma unroll 1
        for (int i = 0; i < kZones; ++i)
          if (s_zissued[i] >= 0) mbar_wait_plain(z_full + 8 * i, (uint32_t)(s_zissued[i] & 1));
#pragma unroll 1
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
  } else {
    // ---------------- softmax: one row per thread ----------------
    const int st = (warp - kWarpSoft) >> 2, qd = warp & 3;
    const int r = qd * 32 + lane;
    const int tok_r = r / p.g, head = r - tok_r * p.g;
    const uint32_t lane_base = (uint32_t)(qd * 32) << 16;
    const uint32_t tS = tmem + lane_base + st * kKT, tO = tmem + lane_base + kColO + st * kD;
    const float sl2 = p.scale_log2;
    uint8_t* s_out = smem + kOffOut + (warp - kWarpSoft) * kOutBytes;
    Seg s;
    int tile = 0, uses = 0, o_uses = 0;
    bool go = true;
#pragma unroll 1
    for (int i = 0; go && receive(i, s); ++i) {
      const int tok = s.tok0 + st * p.tpt + tok_r;
      const bool vrow = tok_r < p.tpt && tok < s.T;
      const bool warp_rows = __any_sync(0xffffffffu, vrow);
      const int pos = s.ctx + tok;                             // the row's last key
      const int tile_first = s.ctx + s.tok0 + st * p.tpt;      // the row tile's first row's
      const int j_end = min(s.j1, ((st ? s.kB : s.kA) + kKT - 1) / kKT);
      float m = -INFINITY, l = 0.f;                            // m in raw score units (scale > 0)
#pragma unroll 1
      for (int j = s.j0; j < j_end; ++j) {
        go = wait(s_full + 8 * st, uses);
        if (!go) break;
        ++uses;
        if (warp_rows) {
          tc_fence_after();
          const uint32_t pm = kPaged ? s_mask[(tile + j - s.j0) % kMasks] : 0xFFu;
          const int base = j * kKT, nh = halves(s, st, j);
          if (base + kKT - 1 > tile_first || pm != 0xFFu) {
            // scores that a row must not see become -inf in tensor memory, from the first
            // 16-key block with one on
            const int nvis = pos + 1 - base;
#pragma unroll 1
            for (int c = pm != 0xFFu ? 0 : max(tile_first + 1 - base, 0) >> 4; c < nh * (kKT / 32); ++c) {
              const int nv = (pm >> c) & 1u ? nvis - 16 * c : 0;
              uint32_t sv[16];
              tc_ld16(tS + 16 * c, sv);
#pragma unroll
              for (int e = 0; e < 16; ++e) sv[e] = e < nv ? sv[e] : __float_as_uint(-INFINITY);
              tc_st16_nowait(tS + 16 * c, sv);
            }
            tc_wait_st();
          }
          // Two rolled passes over the tile's scores, 32 at a time with the next 32 on their
          // way: the tile's maximum, then the exponentials.  (All 128 in registers and the
          // passes unrolled is 7 KB of code: 3 cycles an instruction instead of 1.5.  A maximum
          // for each half instead, with the exponentials from the same registers: no faster
          // rolled, and unrolled 2% faster for long rows, 4% slower for short ones.)
          uint32_t xa[32], xb[32];
          float tmax = -INFINITY;
          tc_ld32_nowait(tS, xa);
#pragma unroll 1
          for (int c = 0; c < nh; ++c) {
            tc_wait_ld32(xa);
            tc_ld32_nowait(tS + 64 * c + 32, xb);
            tmax = max32(xa, tmax);
            tc_wait_ld32(xb);
            tc_ld32_nowait(tS + (c + 1 < nh ? 64 : 0), xa);   // (the second pass's first at last)
            tmax = max32(xb, tmax);
          }
          const bool need = (tmax - m) * sl2 > kRescaleLog2;   // true when m = -inf < tmax
          if (__any_sync(0xffffffffu, need)) {
            const float f = need ? ex2((m - tmax) * sl2) : 1.f;
            if (j > s.j0) {   // S of this tile was issued after P V of the one before: O holds it
#pragma unroll 1
              for (int c = 0; c < 8; ++c) {
                uint32_t ov[16];
                tc_ld16(tO + 16 * c, ov);
#pragma unroll
                for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * f);
                tc_st16_nowait(tO + 16 * c, ov);
              }
            }
            l *= f;
            m = need ? tmax : m;
          }
          const float nms = m == -INFINITY ? 0.f : -m * sl2;
          const uint64_t sl2x2 = f2_pack(__float_as_uint(sl2), __float_as_uint(sl2));
          const uint64_t nmsx2 = f2_pack(__float_as_uint(nms), __float_as_uint(nms));
          uint64_t ls[2] = {0ull, 0ull};
#pragma unroll 1
          for (int c = 0; c < nh; ++c) {
            // P of 64 keys goes to columns 32 c .. 32 c + 31, whose scores are in registers
            uint32_t pw[16];
            tc_wait_ld32(xa);
            tc_ld32_nowait(tS + 64 * c + 32, xb);
            exp32(xa, sl2x2, nmsx2, ls, pw);
            tc_st16_nowait(tS + 32 * c, pw);
            tc_wait_ld32(xb);
            if (c + 1 < nh) tc_ld32_nowait(tS + 64, xa);
            exp32(xb, sl2x2, nmsx2, ls, pw);
            tc_st16_nowait(tS + 32 * c + 16, pw);
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_half + 16 * c + 8 * st);   // (p_full follows p_half)
          }
          if (nh == 1 && lane == 0) mbar_arrive(p_full + 8 * st);
          ls[0] = f2_add(ls[0], ls[1]);
          uint32_t a0, a1;
          f2_unpack(ls[0], a0, a1);
          l += __uint_as_float(a0) + __uint_as_float(a1);
        } else if (lane == 0) {
          mbar_arrive(p_half + 8 * st);
          mbar_arrive(p_full + 8 * st);
        }
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
      // output rows: from the row tile's first, by token and head
      const size_t row0 = (size_t)(s.o + s.tok0 + st * p.tpt) * p.n_q + s.hk * p.g;
      const uint32_t orow = vrow ? (uint32_t)tok_r * p.n_q + head : UINT32_MAX;
      float M = m == -INFINITY ? m : m * sl2;             // of base-2 exponents
      bool bad = any && s_bad[i % kSegs];                 // values taken out of V: for the rows that see them
      bool fin = whole;
      if (!whole) {
        // Few pieces: a warp that finds its rows' other partials in place joins them to its own
        // O, in tensor memory, the others leave theirs (the first piece is its CTA's last
        // segment and the others' first, so that it is mostly the one that joins, and only it
        // looks before it leaves a partial).  The pieces are added in their order, whichever
        // warp adds them.  Many: see below.
        go = wait(cut_full + 8 * (i % kSegs), i / kSegs);
        if (!go) break;
        const int c0 = s_seg[i % kSegs].c0, K = s_seg[i % kSegs].c1 - c0 + 1, own = (int)blockIdx.x - c0;
        const bool direct = K <= kDirect;
        uint32_t* cnt =
            reinterpret_cast<uint32_t*>(p.part + (size_t)(2 * (2 * c0 + 1) + st) * kAttnPartBytes + kCntOff) + qd;
        if (direct && own == 0) fin = __shfl_sync(0xffffffffu, lane == 0 && ld_acquire(cnt) == (uint32_t)(K - 1), 0);
        // partial slot of piece k: the first is its CTA's second
        auto slot = [&](int k) { return p.part + (size_t)(2 * (2 * (c0 + k) + (k == 0)) + st) * kAttnPartBytes; };
        if (!fin) {
          uint8_t* part = slot(own);
          if (any && warp_rows) {
            float4* o = reinterpret_cast<float4*>(part) + r;
#pragma unroll 1
            for (int c = 0; c < 8; ++c) {
              uint32_t ov[16];
              tc_ld16(tO + 16 * c, ov);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (vrow)
                  __stcg(o + (size_t)(4 * c + e) * kRows,
                         make_float4(__uint_as_float(ov[4 * e]), __uint_as_float(ov[4 * e + 1]),
                                     __uint_as_float(ov[4 * e + 2]), __uint_as_float(ov[4 * e + 3])));
            }
          }
          if (vrow) __stcg(reinterpret_cast<float2*>(part + kAttnMlOff) + r, pack_ml(any, bad, M, l));
          __syncwarp();
          if (direct) {
            const uint32_t before = lane == 0 ? atom_inc_acq_rel(cnt, (uint32_t)(K - 1)) : 0u;
            fin = __shfl_sync(0xffffffffu, before, 0) == (uint32_t)(K - 1);
          }
        } else if (lane == 0) {
          *cnt = 0;              // for the next launch
        }
        __syncwarp();            // lane 0 acquired the count: a shuffle hands its value on, not its order
        if (fin && warp_rows) {
          float2 ml[kDirect];
          const float2 ml_own = pack_ml(any, bad, M, l);
#pragma unroll
          for (int k = 0; k < kDirect; ++k) {
            ml[k] = k == own ? ml_own : make_float2(NAN, 0.f);
            if (k < K && k != own && vrow) ml[k] = __ldcg(reinterpret_cast<const float2*>(slot(k) + kAttnMlOff) + r);
            M = fmaxf(M, ml[k].x);
            bad |= took_out(ml[k].y);
          }
          float f[kDirect];      // NaN: no O (the weight of one that has an O may well be 0)
          l = 0.f;
          static_assert(kDirect == 3, "f by number");
#pragma unroll
          for (int k = 0; k < kDirect; ++k) {
            f[k] = ml[k].x == M ? 1.f : ex2(ml[k].x - M);
            if (!no_tiles(ml[k].x)) l = fmaf(fabsf(ml[k].y), f[k], l);
          }
          // 64 columns of a piece in flight at a time (a round trip to L2 costs about 1,000 cycles)
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            float acc[64] = {};
#pragma unroll 1
            for (int k = 0; k < K; ++k) {
              const float fk = k == 0 ? f[0] : k == 1 ? f[1] : f[2];
              uint32_t xa[32], xb[32];
              if (k == own) {
                tc_ld32_nowait(tO + 64 * c, xa);
                tc_ld32_nowait(tO + 64 * c + 32, xb);
                tc_wait_ld32(xa);
                tc_wait_ld32(xb);
              } else {
                const uint4* o = reinterpret_cast<const uint4*>(slot(k)) + (size_t)(16 * c) * kRows + r;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const uint4 y = __ldcg(o + e * kRows);
                  uint32_t* x = e < 8 ? xa + 4 * e : xb + 4 * (e - 8);
                  x[0] = y.x;
                  x[1] = y.y;
                  x[2] = y.z;
                  x[3] = y.w;
                }
              }
              if (fk == fk) {
#pragma unroll
                for (int e = 0; e < 64; ++e)
                  acc[e] = fmaf(__uint_as_float(e < 32 ? xa[e] : xb[e - 32]), fk, acc[e]);
              }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t y[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(acc[16 * q + e]);
              tc_st16_nowait(tO + 64 * c + 16 * q, y);
            }
          }
          tc_wait_st();
        }
      }
      if (fin && warp_rows) {
        // Two rolled steps of 64 columns, 32 on their way while 32 are rounded (a wait for
        // each load costs 400 cycles).  Through shared memory: a row's 128 bytes leave from
        // eight neighbouring lanes (one lane a row touches 32 lines with each store).
        const float il = l == 0.f ? 0.f : 1.f / l;
        uint32_t xa[32], xb[32];
        tc_ld32_nowait(tO, xa);
        auto put = [&](const uint32_t (&x)[32], int at) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint4 y;
            y.x = bf16x2_rn(__uint_as_float(x[8 * e + 1]) * il, __uint_as_float(x[8 * e]) * il);
            y.y = bf16x2_rn(__uint_as_float(x[8 * e + 3]) * il, __uint_as_float(x[8 * e + 2]) * il);
            y.z = bf16x2_rn(__uint_as_float(x[8 * e + 5]) * il, __uint_as_float(x[8 * e + 4]) * il);
            y.w = bf16x2_rn(__uint_as_float(x[8 * e + 7]) * il, __uint_as_float(x[8 * e + 6]) * il);
            *reinterpret_cast<uint4*>(s_out + lane * 128 + (((at + e) ^ (lane & 7)) << 4)) = y;
          }
        };
        uint32_t dst[8];         // the output rows whose pieces this lane carries out
#pragma unroll
        for (int e = 0; e < 8; ++e) dst[e] = __shfl_sync(0xffffffffu, orow, 4 * e + (lane >> 3));
        __nv_bfloat16* out = p.out + row0 * kD + 8 * (lane & 7);
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          tc_wait_ld32(xa);
          tc_ld32_nowait(tO + 64 * c + 32, xb);
          put(xa, 0);
          tc_wait_ld32(xb);
          if (c == 0) tc_ld32_nowait(tO + 64, xa);
          put(xb, 4);
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int rr = 4 * e + (lane >> 3);
            const uint4 x = *reinterpret_cast<const uint4*>(s_out + rr * 128 + (((lane ^ rr) & 7) << 4));
            if (dst[e] != UINT32_MAX) *reinterpret_cast<uint4*>(out + (size_t)dst[e] * kD + 64 * c) = x;
          }
          __syncwarp();
        }
        if (vrow && p.lse) p.lse[row0 + orow] = l == 0.f ? -INFINITY : (M + log2f(l)) * 0.6931471805599453f;
        if (bad && vrow) add_nonfinite<kPaged>(p, s, pos, p.out + (row0 + orow) * kD);
      }
      tc_fence_before();
      __syncwarp();
      if (any && lane == 0) mbar_arrive(o_free + 8 * st);
      release(i);
    }
    tc_fence_before();
    __syncthreads();
    pdl_allow_next();
  }
  if (s_abort) return;

  // ---- pieces of units split among many: counted, waited for and merged ----
  const int npc = s_npc;
  if (npc == 0) return;
  const int nthr = npc == 2 ? kThreads / 2 : kThreads;
  const int pi = tid >= nthr, t = tid - pi * nthr;
  const Seg s = s_pc[pi];
  const int K = s.c1 - s.c0 + 1, mine = (int)blockIdx.x - s.c0;
  const int items = min(w, s.T - s.tok0) * p.g * (kD / 8);
  int lo = items * mine / K, hi = items * (mine + 1) / K;
  if (t == 0) {
    // the count wraps to zero with the last arrival: nothing resets it
    uint32_t* cnt = reinterpret_cast<uint32_t*>(p.part + (size_t)(2 * (2 * s.c0 + 1)) * kAttnPartBytes + kCntAllOff);
    bool ready;
    if (p.coop) {                // every CTA is resident: wait, and join a share
      red_inc_release(cnt, (uint32_t)(K - 1));
      ready = wait_count_zero(cnt);
      if (!ready) flag_error(p.err, EE_DEVERR_TIMEOUT);
    } else {                     // the last to arrive joins everything
      ready = atom_inc_acq_rel(cnt, (uint32_t)(K - 1)) == (uint32_t)(K - 1);
    }
    s_ready[pi] = ready;
  }
  if (!p.coop) {
    lo = 0;
    hi = items;
  }
  asm volatile("bar.sync %0, %1;" ::"r"(2 + pi), "r"(nthr) : "memory");
  if (s_ready[pi]) merge_items<kPaged>(p, s, lo, hi, t, nthr);
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
  if (head_dim != EE_HEAD_DIM || n_q % n_kv != 0 || n_q / n_kv > kRows || total > (1 << 30)) return EE_ERR_UNSUPPORTED;
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
  cfg.numAttrs = p.coop ? 2 : 1;
  EE_CUDA_OK(cudaLaunchKernelEx(&cfg, prompt_attn_kernel<kPaged>, tmQ, tmK, tmV, p));
  return EE_OK;
}

// max_keys: no unit has more.
PromptParams params(const int32_t* tok_off, int B, int total, int64_t max_keys, int n_q, int n_kv, float scale,
                    ee_bf16* out, float* lse, void* ws) {
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
  // Units of the call, at most (a sequence's last one may be partial; one without tokens has
  // none, which the host does not know: its lengths are on the device).  Where they are fewer
  // than a third of the SMs and may be long (for chunks, by the block table's width), they
  // are split among many CTAs, whose partials
  // all of them join, which needs a cooperative launch.  Measured with and without, captured
  // / back to back: one token over 4096 keys 12.0 / 14.4 us and 17.3 / 17.4, 100 tokens after
  // 8000 27 / 30 and 66 / 66; but 16 tokens over 1024 to 16384 keys (64 units) 49.9 / 52.8 and
  // 49.1 / 49.7, a prompt of 300 tokens 12.2 / 14.5 and 12.2 / 12.1.
  const int w = 2 * p.tpt;
  p.units = (int)std::min<int64_t>((int64_t)n_kv * std::min<int64_t>((int64_t)total / w + B, total), INT32_MAX);
  p.coop = p.units < kNumSMs / 3 && max_keys > kDirect * kShareMany ? 1 : 0;
  // Few rows a sequence, idle ones counted: their partials cost little to leave and to join.
  // With the shares of few and of many rows: one token over 4096 keys 12.0 and 17.7 us, 4 tokens 12.7 and 17.8;
  // 100 tokens after 8000 28.4 and 27.0, a prompt of 300 15.2 and 12.2.
  const bool few = (int64_t)total * p.g <= 32 * (int64_t)B;
  p.min_share = few ? kShareFew : kShareMany;
  p.unit_keys = few ? kUnitFew : kUnitMany;
  p.snap = few ? kSnapFew : kSnapMany;
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
  PromptParams p = params(tok_off, B, total, total, n_q, n_kv, scale, out, lse_or_null, ws);
  p.v = reinterpret_cast<const __nv_bfloat16*>(v);
  p.v_stride = v_stride;
  CUtensorMap tmQ, tmK, tmV;
  if (!token_map(&tmQ, q, n_q, total, q_stride, p.g, p.tpt) || !token_map(&tmK, k, n_kv, total, k_stride, 1, kKT) ||
      !token_map(&tmV, v, n_kv, total, v_stride, 1, kVBox))
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
  // (positions are int32, and what is formed of them runs ahead by a few tiles)
  if ((int64_t)num_pages * n_kv * EE_PAGE >= ((int64_t)1 << 31) || max_pages > (1 << 27) - 256)
    return EE_ERR_UNSUPPORTED;
  int dev = 0, ctas = 0;
  ee_status ds = current_device(&dev);
  if (ds == EE_OK) ds = resident_ctas(dev, &ctas);
  if (ds != EE_OK) return ds;
  PromptParams p =
      params(tok_off, B, total, (int64_t)max_pages * EE_PAGE, n_q, n_kv, scale, out, lse_or_null, ws);
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
