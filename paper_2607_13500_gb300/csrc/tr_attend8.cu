// Attention of new tokens over the paged cache held in 8 bits
// (tr_cache8_attend): o = sum_j p_j v_j, p = softmax over the visible keys of
// scale q . k_j, with k_j = c_j 2^e(j) and v_j alike.
//
// One warp per row (token and query head), four channels a lane: 32 keys'
// scores at a time, one after another, then their values.
#include <cmath>

#include "tr_attend8.cuh"

namespace tr {
namespace {

using namespace attend8;

__device__ __forceinline__ float4 values4(const uint8_t *codes, float scale) {
  const uint32_t w = *reinterpret_cast<const uint32_t *>(codes);
  const uint32_t lo = halves((uint16_t)w), hi = halves((uint16_t)(w >> 16));
  const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&lo)), b = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
  return make_float4(a.x * scale, a.y * scale, b.x * scale, b.y * scale);
}

template <typename T>
__global__ void __launch_bounds__(128) k_attend8_rows(const __grid_constant__ AttendArgs g, const __grid_constant__ Scales sc) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= (long long)g.c.total_new * g.q_heads) return;
  const int t = (int)(row / g.q_heads), h = (int)(row - (long long)t * g.q_heads), hk = h / g.group;
  const bool holds = 4 * lane < g.c.d;
  const NewToken own = find_token(g.c, t);
  float m = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f), q = acc;
  if (holds) q = load4<T>(g.q + 2 * ((long long)t * g.q_tok + (long long)h * g.q_head + 4 * lane));
  const float f = g.negate ? -g.scale : g.scale;
  int lo = 0, hi = 0;
  if (own.seq >= 0) {
    const int len = cache_len(g.c, own.seq);
    hi = g.causal ? min(len, own.key + 1) : len;
    lo = g.window > 0 ? window_start(own.key, g.window) : 0;
  }
  for (int j = lo; j < hi; ++j) {
    const int page = page_of(g.c, own.seq, j);
    float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
    if (page < 0) {
      if (lane == 0) flag(g, TR_CACHE_ERR_PAGE);
    } else {
      const int slot = j & (g.c.page - 1);
      const long long off = (((long long)page * g.c.heads + hk) * g.c.page + slot) * g.c.d + 4 * lane, s = scale_at(g.c, page, hk, slot);
      if (holds) {
        k = values4(static_cast<const uint8_t *>(g.c.k) + off, pow2(exp_of(sc.k[s])));
        v = values4(static_cast<const uint8_t *>(g.c.v) + off, pow2(exp_of(sc.v[s])));
      }
    }
    float s = q.x * k.x + q.y * k.y + (q.z * k.z + q.w * k.w);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    s *= f;
    const float mn = fmaxf(m, s), down = m == mn ? 1.f : exp2_fast(m - mn), p = s == -INFINITY ? 0.f : exp2_fast(s - mn);
    m = mn;
    l = l * down + p;
    acc.x = acc.x * down + p * v.x, acc.y = acc.y * down + p * v.y, acc.z = acc.z * down + p * v.z, acc.w = acc.w * down + p * v.w;
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  if (holds)
    reinterpret_cast<uint2 *>(g.o + 2 * ((long long)t * g.o_tok + (long long)h * g.o_head))[lane] =
        make_uint2(Bits<T>::pack(acc.x * inv, acc.y * inv), Bits<T>::pack(acc.z * inv, acc.w * inv));
  if (g.lse && lane == 0) g.lse[row] = l > 0.f || l != l ? m * 0.693147180559945309f + logf(l) : -INFINITY;
}

}  // namespace
}  // namespace tr

using namespace tr;

extern "C" {

size_t tr_cache8_attend_workspace_bytes(const tr_cache8 *c, int32_t q_heads, int32_t window, int32_t max_new,
                                        int32_t max_len) {
  if (check_cache8(c) != TR_OK || q_heads <= 0 || q_heads % c->c.heads || window < 0 || max_new < 0 || max_len < 0)
    return 0;
  return few_takes(&c->c, q_heads, max_new) ? few_workspace_bytes(c->c.head_dim, sm_count() > 0 ? sm_count() : 1) : 0;
}

tr_status tr_cache8_attend(const tr_cache8 *c8, const tr_heads *q, const tr_heads *o, float *lse, float scale,
                           int32_t causal, int32_t window, int32_t max_new, int32_t max_len, void *ws,
                           size_t ws_bytes, int32_t *d_error, void *stream) {
  tr_status rc = check_cache8(c8);
  if (rc != TR_OK) return rc;
  const tr_cache *c = &c8->c;
  if (!q || !o || max_new < 0 || max_len < 0 || window < 0 || !std::isfinite(scale)) return TR_ERR_ARG;
  if ((rc = check_heads(q, 2)) != TR_OK || (rc = check_heads(o, 2)) != TR_OK) return rc;
  if (q->heads != o->heads || q->heads % c->heads) return TR_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(lse) & 3u) return TR_ERR_ALIGN;
  if ((long long)c->total_new * q->heads > INT_MAX - 65536) return TR_ERR_UNSUPPORTED;
  if (c->heads > 65535) return TR_ERR_UNSUPPORTED;
  if (c->total_new == 0) return TR_OK;
  AttendArgs g{};
  g.c = cache_view(c);
  g.q = static_cast<const char *>(q->p);
  g.o = static_cast<char *>(o->p);
  g.q_tok = q->token_stride, g.q_head = q->head_stride;
  g.o_tok = o->token_stride, g.o_head = o->head_stride;
  g.q_heads = q->heads, g.group = q->heads / c->heads;
  g.lse = lse;
  // (not zero: masked scores are -inf, and -inf * 0 would be NaN)
  g.scale = fmaxf(fabsf(scale) * 1.44269504088896341f, 1e-30f);
  g.negate = scale < 0.f;
  g.causal = causal, g.window = window;
  g.err = d_error;
  const Scales sc{c8->k_scale, c8->v_scale};
  const long long rows = (long long)c->total_new * q->heads;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  while ((1 << g.page_log2) < c->page) ++g.page_log2;
  if (few_takes(c, q->heads, max_new)) {
    g.ctas = sm_count() > 0 ? sm_count() : 1;
    const size_t need = few_workspace_bytes(c->head_dim, g.ctas);
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < need) return TR_ERR_WORKSPACE;
    CUtensorMap mk{}, mv{};
    const long long keys = (long long)c->pages * c->heads * c->page;
    const int box = c->page < kTile ? c->page : kTile, wide = c->head_dim <= 64 ? 64 : 128;
    // an empty cache keeps one row in the maps' extents: no page id is valid, so nothing reads it
    if (!make_map_bytes(&mk, c->k, keys > 0 ? keys : 1, c->head_dim, box, wide) ||
        !make_map_bytes(&mv, c->v, keys > 0 ? keys : 1, c->head_dim, box, wide))
      return TR_ERR_CUDA;
    Attend8Args p{g, sc};
    return launch_few8(mk, mv, p, c->dtype == TR_BF16, ws, st) == cudaSuccess ? TR_OK : TR_ERR_CUDA;
  }
  const dim3 grid((unsigned)((rows + 3) / 4));
  const cudaError_t err = c->dtype == TR_BF16 ? launch_kernel(k_attend8_rows<__nv_bfloat16>, grid, dim3(128), 0, st, false, g, sc)
                                              : launch_kernel(k_attend8_rows<__half>, grid, dim3(128), 0, st, false, g, sc);
  return err == cudaSuccess ? TR_OK : TR_ERR_CUDA;
}

}  // extern "C"
