// ee_prompt_attn, ee_chunk_attn: causal attention of packed new tokens, whole
// prompts over their own K/V or chunks over the paged cache.
//
// One warp per (token, query head): a lane holds four of the 128 dimensions and
// the warp walks the visible keys with a running maximum and sum.
#include "ee_common.cuh"

namespace {

using namespace ee;

constexpr int kD = EE_HEAD_DIM;

struct PromptParams {
  const __nv_bfloat16 *q, *k, *v;   // (paged: k, v = this layer's cache)
  int64_t q_stride, k_stride, v_stride;
  const int32_t *block_table, *ctx_len, *tok_off;
  __nv_bfloat16* out;
  float* lse;
  int32_t* err;
  int B, total, num_pages, max_pages, n_q, n_kv, g;
  float scale;
};

__device__ __forceinline__ float4 load4(const __nv_bfloat16* a) {
  const uint2 u = *reinterpret_cast<const uint2*>(a);
  const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
  const float2 y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
  return make_float4(x.x, x.y, y.x, y.y);
}

template <bool kPaged>
__global__ void __launch_bounds__(128) prompt_attn_kernel(const PromptParams p) {
  const int lane = threadIdx.x & 31;
  const int s = blockIdx.z, h = blockIdx.y;
  const int o = p.tok_off[s], T = p.tok_off[s + 1] - o;
  if (T < 0 || o < 0 || (int64_t)o + T > p.total) {
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) flag_error(p.err, EE_DEVERR_TREE);
    return;
  }
  int ctx = 0;
  if constexpr (kPaged) {
    ctx = p.ctx_len[s];
    if (ctx < 0 || (int64_t)ctx + T > (int64_t)p.max_pages * EE_PAGE) {
      if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) flag_error(p.err, EE_DEVERR_CTX);
      return;
    }
  }
  const int hk = h / p.g;
  for (int i = blockIdx.x * 4 + (threadIdx.x >> 5); i < T; i += gridDim.x * 4) {
    const float4 q = load4(p.q + (size_t)(o + i) * p.q_stride + (size_t)h * kD + 4 * lane);
    float m = -INFINITY, l = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int j = 0; j <= ctx + i; ++j) {
      size_t ko, vo;
      if constexpr (kPaged) {
        const int pg = p.block_table[(size_t)s * p.max_pages + j / EE_PAGE];
        if (pg < 0 || pg >= p.num_pages) {
          if (lane == 0) flag_error(p.err, EE_DEVERR_PAGE);
          continue;
        }
        ko = vo = (((size_t)pg * p.n_kv + hk) * EE_PAGE + j % EE_PAGE) * kD;
      } else {
        ko = (size_t)(o + j) * p.k_stride + (size_t)hk * kD;
        vo = (size_t)(o + j) * p.v_stride + (size_t)hk * kD;
      }
      const float4 k = load4(p.k + ko + 4 * lane), v = load4(p.v + vo + 4 * lane);
      float x = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, q.w * k.w)));
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
      x *= p.scale;
      const float mn = fmaxf(m, x);
      const float f = m == -INFINITY ? 0.f : expf(m - mn);
      const float e = x == -INFINITY ? 0.f : expf(x - mn);
      m = mn;
      l = fmaf(l, f, e);
      a.x = fmaf(a.x, f, e * v.x);
      a.y = fmaf(a.y, f, e * v.y);
      a.z = fmaf(a.z, f, e * v.z);
      a.w = fmaf(a.w, f, e * v.w);
    }
    const float il = l == 0.f ? 0.f : 1.f / l;
    const size_t row = (size_t)(o + i) * p.n_q + h;
    const __nv_bfloat162 u = __floats2bfloat162_rn(a.x * il, a.y * il), w = __floats2bfloat162_rn(a.z * il, a.w * il);
    uint2 st;
    st.x = *reinterpret_cast<const uint32_t*>(&u);
    st.y = *reinterpret_cast<const uint32_t*>(&w);
    *reinterpret_cast<uint2*>(p.out + row * kD + 4 * lane) = st;
    if (lane == 0 && p.lse) p.lse[row] = l == 0.f ? -INFINITY : m + logf(l);
  }
}

bool good_stride(int64_t stride, int heads) { return stride % 8 == 0 && stride >= (int64_t)heads * kD; }

// The checks both calls share.
ee_status check(const ee_bf16* q, int64_t q_stride, const ee_bf16* k, const ee_bf16* v, const int32_t* tok_off,
                int32_t B, int32_t total, int32_t n_q, int32_t n_kv, int32_t head_dim, float scale, const ee_bf16* out,
                const float* lse, const void* ws, size_t ws_bytes) {
  if (B < 0 || total < 0 || n_q < 1 || n_kv < 1) return EE_ERR_INVALID_ARG;
  if (head_dim != EE_HEAD_DIM || n_q % n_kv != 0 || n_q / n_kv > 128) return EE_ERR_UNSUPPORTED;
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
  PromptParams p{};
  p.q = reinterpret_cast<const __nv_bfloat16*>(q);
  p.k = reinterpret_cast<const __nv_bfloat16*>(k);
  p.v = reinterpret_cast<const __nv_bfloat16*>(v);
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.tok_off = tok_off;
  p.out = reinterpret_cast<__nv_bfloat16*>(out);
  p.lse = lse_or_null;
  p.err = err_word(ws);
  p.B = B;
  p.total = total;
  p.n_q = n_q;
  p.n_kv = n_kv;
  p.g = n_q / n_kv;
  p.scale = scale;
  prompt_attn_kernel<false><<<dim3(std::min((total + 3) / 4, 1024), n_q, B), 128, 0, (cudaStream_t)stream>>>(p);
  EE_LAUNCH_OK();
  return EE_OK;
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
  if ((int64_t)num_pages * n_kv * EE_PAGE >= ((int64_t)1 << 31)) return EE_ERR_UNSUPPORTED;
  PromptParams p{};
  p.q = reinterpret_cast<const __nv_bfloat16*>(q);
  p.k = reinterpret_cast<const __nv_bfloat16*>(k_cache);
  p.v = reinterpret_cast<const __nv_bfloat16*>(v_cache);
  p.q_stride = q_stride;
  p.block_table = block_table;
  p.ctx_len = ctx_len;
  p.tok_off = tok_off;
  p.out = reinterpret_cast<__nv_bfloat16*>(out);
  p.lse = lse_or_null;
  p.err = err_word(ws);
  p.B = B;
  p.total = total;
  p.num_pages = num_pages;
  p.max_pages = max_pages;
  p.n_q = n_q;
  p.n_kv = n_kv;
  p.g = n_q / n_kv;
  p.scale = scale;
  prompt_attn_kernel<true><<<dim3(std::min((total + 3) / 4, 1024), n_q, B), 128, 0, (cudaStream_t)stream>>>(p);
  EE_LAUNCH_OK();
  return EE_OK;
}
