// Attention of new tokens over the paged cache (tr_cache_attend):
//   o = sum_j p_j v_j,  p = softmax over the visible keys of scale q . k_j.
#include <climits>
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tr_cache.cuh"

namespace tr {
namespace {

struct AttendArgs {
  CacheView c;
  const char *q;
  char *o;
  long long q_tok, q_head, o_tok, o_head;  // elements
  int q_heads, group;                      // group: query heads of a key head
  float *lse;
  float scale;
  int causal, window;
  int32_t *err;
};

template <typename T>
__device__ __forceinline__ float4 load4(const char *p) {
  const uint2 v = *reinterpret_cast<const uint2 *>(p);
  const T *h = reinterpret_cast<const T *>(&v);
  return make_float4((float)h[0], (float)h[1], (float)h[2], (float)h[3]);
}

// One warp per row (token, query head): four channels a lane, one key at a
// time, the running maximum and sum of the softmax in registers.
template <typename T>
__global__ void __launch_bounds__(128) k_attend_rows(const __grid_constant__ AttendArgs g) {
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= (long long)g.c.total_new * g.q_heads) return;
  const int t = (int)(row / g.q_heads), h = (int)(row - (long long)t * g.q_heads);
  const NewToken at = find_token(g.c, t);
  int lo = 0, hi = 0;
  if (at.seq >= 0) {
    hi = cache_len(g.c, at.seq);
    if (g.causal) hi = min(hi, at.key + 1);
    if (g.window > 0) lo = max(0, at.key - g.window + 1);
  }
  const int d = g.c.d, ch = 4 * lane, hk = h / g.group;
  const bool holds = ch < d;
  float4 q = make_float4(0.f, 0.f, 0.f, 0.f), acc = q;
  if (holds) q = load4<T>(g.q + 2 * ((long long)t * g.q_tok + (long long)h * g.q_head + ch));
  float m = -INFINITY, l = 0.f;
  for (int j = lo; j < hi; ++j) {
    const int page = page_of(g.c, at.seq, j);
    float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
    if (page >= 0) {
      if (holds) {
        const long long off =
            2 * ((((long long)page * g.c.heads + hk) * g.c.page + (j & (g.c.page - 1))) * d + ch);
        k = load4<T>(static_cast<const char *>(g.c.k) + off);
        v = load4<T>(static_cast<const char *>(g.c.v) + off);
      }
    } else if (g.err && lane == 0) {
      atomicOr(g.err, TR_CACHE_ERR_PAGE);
    }
    float s = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    s *= g.scale;
    const float mn = fmaxf(m, s);
    const float f = m == mn ? 1.f : __expf(m - mn), p = s == -INFINITY ? 0.f : __expf(s - mn);
    m = mn;
    l = l * f + p;
    acc.x = acc.x * f + p * v.x;
    acc.y = acc.y * f + p * v.y;
    acc.z = acc.z * f + p * v.z;
    acc.w = acc.w * f + p * v.w;
  }
  const float inv = hi > lo ? 1.f / l : 0.f;
  if (holds) {
    T out[4] = {(T)(acc.x * inv), (T)(acc.y * inv), (T)(acc.z * inv), (T)(acc.w * inv)};
    *reinterpret_cast<uint2 *>(g.o + 2 * ((long long)t * g.o_tok + (long long)h * g.o_head + ch)) =
        *reinterpret_cast<uint2 *>(out);
  }
  if (g.lse && lane == 0) g.lse[(long long)t * g.q_heads + h] = hi > lo ? m + logf(l) : -INFINITY;
}

}  // namespace
}  // namespace tr

using namespace tr;

extern "C" {

size_t tr_cache_attend_workspace_bytes(const tr_cache *c, int32_t q_heads, int32_t max_new, int32_t max_len) {
  if (check_cache(c) != TR_OK || q_heads <= 0 || q_heads % c->heads || max_new < 0 || max_len < 0) return 0;
  return 0;
}

tr_status tr_cache_attend(const tr_cache *c, const tr_heads *q, const tr_heads *o, float *lse, float scale,
                          int32_t causal, int32_t window, int32_t max_new, int32_t max_len, void *ws,
                          size_t ws_bytes, int32_t *d_error, void *stream) {
  tr_status rc = check_cache(c);
  if (rc != TR_OK) return rc;
  if (!q || !o || max_new < 0 || max_len < 0 || window < 0 || !std::isfinite(scale)) return TR_ERR_ARG;
  if ((rc = check_heads(q, 2)) != TR_OK || (rc = check_heads(o, 2)) != TR_OK) return rc;
  if (q->heads != o->heads || q->heads % c->heads) return TR_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(lse) & 3u) return TR_ERR_ALIGN;
  if ((long long)c->total_new * q->heads > INT_MAX) return TR_ERR_UNSUPPORTED;
  if (c->total_new == 0 || c->batch == 0) return TR_OK;
  AttendArgs g{};
  g.c = cache_view(c);
  g.q = static_cast<const char *>(q->p);
  g.o = static_cast<char *>(o->p);
  g.q_tok = q->token_stride, g.q_head = q->head_stride;
  g.o_tok = o->token_stride, g.o_head = o->head_stride;
  g.q_heads = q->heads, g.group = q->heads / c->heads;
  g.lse = lse;
  g.scale = scale;
  g.causal = causal, g.window = window;
  g.err = d_error;
  const int grid = (int)(((long long)c->total_new * q->heads + 3) / 4);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t err = c->dtype == TR_BF16
                              ? launch_kernel(k_attend_rows<__nv_bfloat16>, dim3(grid), dim3(128), 0, st, false, g)
                              : launch_kernel(k_attend_rows<__half>, dim3(grid), dim3(128), 0, st, false, g);
  return err == cudaSuccess ? TR_OK : TR_ERR_CUDA;
}

}  // extern "C"
