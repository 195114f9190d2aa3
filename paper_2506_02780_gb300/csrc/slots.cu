// ee_prompt_slots: cache pages, positions and slots of new tokens, from lengths
// that live on the device.
//
// One launch.  With t_s new tokens and n_s = ceil((ctx + t + reserve) / 16) -
// held_s pages to give (as far as the table has columns), everything follows from
// the exclusive sums of t and n over the sequences: token i's sequence is found in
// the first by bisection, and the k-th given page is the k-th from the end of the
// free list.  Every CTA forms both sums over all (at most 4096) sequences by
// itself, in shared memory: a second launch or a grid-wide barrier for one scan
// would cost more than the repeated reads, which come from L2.  Then the CTAs share
// the tokens and the new table entries; a token on a page given in this call takes
// it from the free list directly, so no CTA reads what another writes.
//
// Bound by latency: the reads of the lengths, the scan, the bisections in shared memory
// and the reads of the pages follow one another.  A thread takes four neighbouring tokens,
// mostly of one sequence and page, and all its reads precede its writes (four tokens a
// grid apart, each written before the next is read: 9.7 us for 1024 sequences).  Measured:
// 8 sequences with a token each 3.8 us; 1024 sequences of up to 2048 new tokens, 2.6 MB in
// all, 7.3 us.  512 threads: with 256 the latter takes 8.9 us, with 1024 the former 5.6 us.
#include "ee_common.cuh"
#include "ee_ptx.cuh"

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kTokens = 4;   // neighbouring tokens of a thread: mostly one bisection, one page, one store

struct SlotParams {
  const int32_t *ctx_len, *new_len, *held;
  int32_t* block_table;
  const int32_t *free_pages, *free_cnt;
  int32_t *tok_off, *pos, *slot, *ctx_out, *held_out, *free_out, *err;
  int B, total, reserve, max_pages, n_free, num_pages;
  bool vec;                    // pos and slot take 16-byte stores
};

// One sequence's share: tokens it gets and pages it is given (0 and 0 when its
// lengths are out of range).
__device__ __forceinline__ bool seq_share(const SlotParams& p, int s, int& ctx, int& held, int& t, int& give) {
  ctx = ee::ld_pinned(p.ctx_len + s);
  held = ee::ld_pinned(p.held + s);
  t = ee::ld_pinned(p.new_len + s);
  give = 0;
  const int64_t cap = (int64_t)p.max_pages * EE_PAGE;
  const int64_t end = (int64_t)ctx + t, want = min(end + p.reserve, cap);   // the reserve ends with the table
  if (ctx < 0 || t < 0 || held < 0 || held > p.max_pages || ctx > (int64_t)held * EE_PAGE || end > cap) {
    t = 0;
    return false;
  }
  if (end > 0) give = max((int)((want + EE_PAGE - 1) / EE_PAGE) - held, 0);
  return true;
}

// the last s in [lo, B) with off[s] <= i
__device__ __forceinline__ int seq_of(const int* off, int lo, int B, int i) {
  int hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kThreads) prompt_slots_kernel(const SlotParams p) {
  extern __shared__ int s_dyn[];
  int* s_tok = s_dyn;               // [B + 1] exclusive sums: tokens (capped at `total`)
  int* s_give = s_tok + p.B + 1;    // [B + 1] pages given
  int* s_ctx = s_give + p.B + 1;    // [B]
  int* s_held = s_ctx + p.B;        // [B]
  __shared__ int64_t s_wt[kWarps], s_wg[kWarps];
  ee::pdl_allow_next();
  ee::pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cnt = *p.free_cnt;

  // the sums, in 64 bits: thread i takes sequences [per i, per i + per)
  const int per = (p.B + kThreads - 1) / kThreads;
  const int s0 = min(tid * per, p.B), s1 = min(s0 + per, p.B);
  int64_t ts = 0, gs = 0;
  bool good = true;
#pragma unroll 4
  for (int s = s0; s < s1; ++s) {
    int ctx, held, t, give;
    good &= seq_share(p, s, ctx, held, t, give);
    s_ctx[s] = ctx;
    s_held[s] = held;
    s_tok[s] = t;
    s_give[s] = give;
    ts += t;
    gs += give;
  }
  int64_t ti = ts, gi = gs;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t a = __shfl_up_sync(0xffffffffu, ti, d), b = __shfl_up_sync(0xffffffffu, gi, d);
    if (lane >= d) {
      ti += a;
      gi += b;
    }
  }
  if (lane == 31) {
    s_wt[warp] = ti;
    s_wg[warp] = gi;
  }
  __syncthreads();
  int64_t tbase = 0, gbase = 0, tall = 0, gall = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) {
      tbase += s_wt[w];
      gbase += s_wg[w];
    }
    tall += s_wt[w];
    gall += s_wg[w];
  }
  const int avail = min(max(cnt, 0), p.n_free);
  const bool enough = cnt >= 0 && cnt <= p.n_free && gall <= avail;
  int64_t to = tbase + ti - ts, go = gbase + gi - gs;
  for (int s = s0; s < s1; ++s) {
    const int t = s_tok[s], give = s_give[s];
    s_tok[s] = (int)min(to, (int64_t)p.total);
    s_give[s] = enough ? (int)go : 0;
    if (blockIdx.x == 0) {
      p.tok_off[s] = s_tok[s];
      const int placed = (int)min(to + t, (int64_t)p.total) - s_tok[s];   // tokens past `total` are dropped
      p.ctx_out[s] = s_ctx[s] + (enough ? placed : 0);
      p.held_out[s] = s_held[s] + (enough ? give : 0);
    }
    to += t;
    go += give;
  }
  const int n_tok = (int)min(tall, (int64_t)p.total);
  const int n_give = enough ? (int)gall : 0;
  if (!good && blockIdx.x == 0) ee::flag_error(p.err, EE_DEVERR_CTX);
  if (tid == 0) {
    s_tok[p.B] = n_tok;
    s_give[p.B] = n_give;
    if (blockIdx.x == 0) {
      p.tok_off[p.B] = n_tok;
      *p.free_out = cnt - n_give;
      if (tall != p.total) ee::flag_error(p.err, EE_DEVERR_CTX);
      if (!enough) ee::flag_error(p.err, EE_DEVERR_PAGE);
    }
  }
  __syncthreads();

  // a free page by its number in this call (-1: no page of the cache)
  auto fresh = [&](int n) -> int {
    const int pg = p.free_pages[cnt - 1 - n];
    return pg >= 0 && pg < p.num_pages ? pg : -1;
  };
  bool bad_page = false;
  const int step = gridDim.x * kThreads;
  // the new entries of the table, 32 of a warp, dealt to all CTAs' first warps, second warps, ...
  for (int n = (warp * gridDim.x + blockIdx.x) * 32 + lane; n < n_give; n += step) {
    const int s = seq_of(s_give, 0, p.B, n);
    const int pg = fresh(n);
    bad_page |= pg < 0;
    p.block_table[(size_t)s * p.max_pages + s_held[s] + (n - s_give[s])] = pg;
  }
  // the tokens: all reads before the writes, so that they are in flight together
  for (int64_t base = (int64_t)kTokens * (blockIdx.x * kThreads + tid); base < p.total; base += (int64_t)kTokens * step) {
    const int i0 = (int)base;
    int pos[kTokens], slot[kTokens], pg[kTokens];
    int s = i0 < n_tok ? seq_of(s_tok, 0, p.B, i0) : 0;
#pragma unroll
    for (int k = 0; k < kTokens; ++k) {
      const int i = i0 + k;
      pos[k] = -1;
      pg[k] = -1;
      if (i >= n_tok) continue;
      if (i >= s_tok[s + 1]) s = seq_of(s_tok, s + 1, p.B, i);
      pos[k] = s_ctx[s] + (i - s_tok[s]);
      const int j = pos[k] / EE_PAGE, h = s_held[s];
      if (enough) {
        const int32_t* at = j < h ? p.block_table + (size_t)s * p.max_pages + j
                                  : p.free_pages + (cnt - 1 - (s_give[s] + j - h));
        pg[k] = *at;
      }
    }
#pragma unroll
    for (int k = 0; k < kTokens; ++k) {
      const bool ok = pg[k] >= 0 && pg[k] < p.num_pages;
      bad_page |= enough && pos[k] >= 0 && !ok;
      slot[k] = ok ? pg[k] * EE_PAGE + pos[k] % EE_PAGE : -1;
    }
    static_assert(kTokens == 4, "one 16-byte store");
    if (p.vec && i0 + kTokens <= p.total) {
      *reinterpret_cast<int4*>(p.pos + i0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      *reinterpret_cast<int4*>(p.slot + i0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
    } else {
#pragma unroll
      for (int k = 0; k < kTokens; ++k)
        if (i0 + k < p.total) {
          p.pos[i0 + k] = pos[k];
          p.slot[i0 + k] = slot[k];
        }
    }
  }
  if (bad_page) ee::flag_error(p.err, EE_DEVERR_PAGE);
}

constexpr size_t smem_bytes(int B) { return sizeof(int) * (4 * (size_t)B + 2); }

// The largest batch's sums pass 48 KB: raise the limit once per device.
cudaError_t set_attrs(int dev) {
  static std::mutex mu;
  static bool done[ee::kMaxDevices] = {};
  std::lock_guard<std::mutex> lock(mu);
  if (done[dev]) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(prompt_slots_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)smem_bytes(EE_MAX_SEQS));
  done[dev] = e == cudaSuccess;
  return e;
}

}  // namespace

extern "C" ee_status ee_prompt_slots(const int32_t* ctx_len, const int32_t* new_len, const int32_t* held, int32_t B,
                                     int32_t total, int32_t reserve, int32_t* block_table, int32_t max_pages,
                                     const int32_t* free_pages, int32_t n_free, const int32_t* free_cnt,
                                     int32_t num_pages, int32_t* tok_off, int32_t* pos, int32_t* slot,
                                     int32_t* ctx_out, int32_t* held_out, int32_t* free_out, void* ws,
                                     size_t ws_bytes, ee_stream_t stream) {
  constexpr int kMaxPages = 1 << 27;   // positions and slots are int32
  if (B < 1 || total < 0 || reserve < 0 || max_pages < 1 || n_free < 0 || num_pages < 1) return EE_ERR_INVALID_ARG;
  if (B > EE_MAX_SEQS || max_pages >= kMaxPages || num_pages >= kMaxPages || total > (1 << 30) || reserve > (1 << 30))
    return EE_ERR_UNSUPPORTED;
  if (!ctx_len || !new_len || !held || !block_table || (n_free > 0 && !free_pages) || !free_cnt || !tok_off ||
      (total > 0 && (!pos || !slot)) || !ctx_out || !held_out || !free_out || !ws || !ee::aligned(ws, 256))
    return EE_ERR_INVALID_ARG;
  if (ctx_out == ctx_len || held_out == held || free_out == free_cnt) return EE_ERR_INVALID_ARG;
  if (ws_bytes < ee::kWorkspaceBytes) return EE_ERR_WORKSPACE;
  int dev = 0;
  const ee_status ds = ee::current_device(&dev);
  if (ds != EE_OK) return ds;
  EE_CUDA_OK(set_attrs(dev));
  SlotParams p{ctx_len, new_len, held,     block_table, free_pages, free_cnt,        tok_off, pos,    slot,
               ctx_out, held_out, free_out, ee::err_word(ws), B,    total, reserve, max_pages, n_free, num_pages,
               ee::aligned(pos, 16) && ee::aligned(slot, 16)};
  // a CTA per round of its threads, two per SM at most: beyond that the scans repeat
  const int64_t want = ((int64_t)total + kThreads * kTokens - 1) / (kThreads * kTokens);
  const int grid = (int)std::min<int64_t>(std::max<int64_t>(want, 1), 2 * ee::kNumSMs);
  EE_CUDA_OK(ee::launch_pdl(prompt_slots_kernel, dim3(grid), dim3(kThreads), smem_bytes(B), (cudaStream_t)stream, 1, p));
  return EE_OK;
}
