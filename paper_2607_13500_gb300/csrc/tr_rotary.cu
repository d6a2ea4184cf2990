// Rotary positions with several axes, with the RMS norm of each head in the
// same pass (tr_rotary_apply, tr_rotary_backward), and the append of keys and
// values to the paged cache with both applied on the way (tr_cache_append).
//
// Per head row x of d channels: n = x r w with r = 1 / sqrt(mean(x^2) + eps)
// (or n = x), then each pair (a, b) of n turns by its angle:
//   y_a = n_a cos - n_b sin,  y_b = n_b cos + n_a sin.
// Backward, with g = the gradient dy turned by the opposite angle:
//   dw = sum g x r,  dx = r (w g) - x r^3 mean(x w g).
//
// All of it is bound by memory: each row is read once and written once.  A
// row belongs to a group of lanes, each of which holds both halves of V
// pairs (two vector loads), so the rotation needs no exchange and the norm a
// few shuffles.  The angles of a token are shared by all its heads: a CTA
// takes a few tokens, computes their cosines and sines once into shared
// memory and then streams the rows of all heads.
#include <climits>
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tr_cache.cuh"
#include "tr_internal.cuh"

namespace tr {
namespace {

constexpr int kRotThreads = 256;
constexpr int kMaxTokens = 8;                       // tokens of one CTA at most
constexpr int kMaxTrig = kRotThreads;               // angles a CTA holds (tokens x frequencies)

struct Rows {
  const char *in;   // NULL: segment absent
  char *out;        // NULL: into the cache
  long long in_tok, in_head, out_tok, out_head;  // elements
  int heads;
  const float *w;   // norm weight or NULL
  int turn;         // rows are rotated
  int cache;        // 0: out, 1: the cache's keys, 2: its values
};

struct RotArgs {
  const unsigned long long *turns;
  const int32_t *axis;
  const int32_t *pos;
  int d, half, axes, tokens, tokens_per_cta;
  int lanes_log2;   // lanes of a row's group
  int slots;        // lanes of it that hold channels: d / (2 V)
  float sign;       // -1 turns backwards
  float eps;
  Rows seg[3];      // queries, keys, values
  CacheView cache;
  int32_t *err;
};

// ---------------------------------------------------------------- elements
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t v);
template <>
__device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 unpack2<__half>(uint32_t v) {
  __half2 h;
  *reinterpret_cast<uint32_t *>(&h) = v;
  return __half22float2(h);
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
  __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t *>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<uint32_t *>(&h);
}

// V consecutive elements as raw words: one 16- or 8-byte access.
template <typename T, int V>
struct Chunk {
  static constexpr int kWords = V * (int)sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const char *p) {
    if (kWords == 4) {
      const uint4 v = __ldcs(reinterpret_cast<const uint4 *>(p));
      w[0] = v.x, w[1] = v.y, w[kWords - 2] = v.z, w[kWords - 1] = v.w;
    } else {
      const uint2 v = __ldcs(reinterpret_cast<const uint2 *>(p));
      w[0] = v.x, w[1] = v.y;
    }
  }
  __device__ __forceinline__ void store(char *p) const {
    if (kWords == 4)
      *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[kWords - 2], w[kWords - 1]);
    else
      *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
  }
  __device__ __forceinline__ void get(float (&f)[V]) const {
#pragma unroll
    for (int i = 0; i < V / (4 / (int)sizeof(T)); ++i) {
      if constexpr (sizeof(T) == 4) {
        f[i] = __uint_as_float(w[i]);
      } else {
        const float2 t = unpack2<T>(w[i]);
        f[2 * i] = t.x, f[2 * i + 1] = t.y;
      }
    }
  }
  __device__ __forceinline__ void set(const float (&f)[V]) {
#pragma unroll
    for (int i = 0; i < V / (4 / (int)sizeof(T)); ++i) {
      if constexpr (sizeof(T) == 4)
        w[i] = __float_as_uint(f[i]);
      else
        w[i] = pack2<T>(f[2 * i], f[2 * i + 1]);
    }
  }
};

// The slot's two chunks: first halves and second halves of V pairs
// (TR_ROTARY_HALF), or 2 V neighbouring channels (TR_ROTARY_PAIRS, and the
// channels past rot_dim).
struct SlotPlace {
  int a, b;      // first channel of each chunk
  bool turns;
};
template <int V, bool PAIRS>
__device__ __forceinline__ SlotPlace slot_place(int slot, int half) {
  SlotPlace p;
  p.turns = slot * V < half;
  if (!PAIRS && p.turns) {
    p.a = slot * V;
    p.b = half + slot * V;
  } else {
    p.a = slot * 2 * V;
    p.b = p.a + V;
  }
  return p;
}

// Turns the slot's pairs in place by (c, s); with PAIRS a pair is two
// neighbours of the 2 V channels, else the same place in both chunks.
template <int V, bool PAIRS>
__device__ __forceinline__ void turn(float (&x)[V], float (&y)[V], const float *c, const float *s) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float &a = PAIRS ? (2 * i < V ? x[2 * i % V] : y[2 * i % V]) : x[i];
    float &b = PAIRS ? (2 * i < V ? x[(2 * i + 1) % V] : y[(2 * i + 1) % V]) : y[i];
    const float a0 = a, b0 = b;
    a = a0 * c[i] - b0 * s[i];
    b = b0 * c[i] + a0 * s[i];
  }
}

// Cosines and sines of the CTA's tokens into shared memory.  position *
// turns modulo 2^64 is the angle as a fraction of a turn, exactly; its top 32
// bits, signed, are the angle in units of pi / 2^31.
__device__ __forceinline__ void fill_trig(const RotArgs &g, int t0, int nt, float *cs, float *sn) {
  for (int i = threadIdx.x; i < nt * g.half; i += kRotThreads) {
    const int lt = i / g.half, f = i - lt * g.half;
    const int ax = __ldg(g.axis + f);
    const long long p = (unsigned)ax < (unsigned)g.axes ? (long long)__ldg(g.pos + (long long)ax * g.tokens + t0 + lt) : 0;
    const unsigned long long frac = (unsigned long long)p * __ldg(g.turns + f);
    float s, c;
    sincospif((float)(int)(frac >> 32) * 0x1p-31f, &s, &c);
    cs[i] = c;
    sn[i] = s * g.sign;
  }
}

template <typename T, int V, bool PAIRS, bool NORM>
__global__ void __launch_bounds__(kRotThreads) k_rotate(const __grid_constant__ RotArgs g) {
  __shared__ __align__(16) float cs[kMaxTrig], sn[kMaxTrig];
  __shared__ long long home[kMaxTokens];  // the token's first key row in the cache (head 0), or -1
  pdl_wait();  // q, k, v come from the kernel before
  const int t0 = blockIdx.x * g.tokens_per_cta;
  const int nt = min(g.tokens_per_cta, g.tokens - t0);
  fill_trig(g, t0, nt, cs, sn);
  if (g.cache.k && (int)threadIdx.x < nt) {
    const NewToken at = find_token(g.cache, t0 + threadIdx.x);
    long long row = -1;
    if (at.seq >= 0 && at.key >= 0) {
      const int page = page_of(g.cache, at.seq, at.key);
      if (page >= 0)
        row = (long long)page * g.cache.heads * g.cache.page + (at.key & (g.cache.page - 1));
      else if (g.err)
        atomicOr(g.err, TR_CACHE_ERR_PAGE);
    } else if (at.seq >= 0 && g.err) {
      atomicOr(g.err, TR_CACHE_ERR_PAGE);
    }
    home[threadIdx.x] = row;
  }
  __syncthreads();
  const int slot = threadIdx.x & ((1 << g.lanes_log2) - 1);
  const int group = threadIdx.x >> g.lanes_log2, groups = kRotThreads >> g.lanes_log2;
  const bool holds = slot < g.slots;
  const SlotPlace at = slot_place<V, PAIRS>(slot, g.half);
  const int q_heads = g.seg[0].heads, k_heads = g.seg[1].heads;
  const int heads = q_heads + k_heads + g.seg[2].heads;
  const int rows = nt * heads;
  constexpr int kU = 2;  // rows in flight per group
  for (int r0 = 0; r0 < rows; r0 += kU * groups) {  // the same trips for every lane of a warp
    Chunk<T, V> ca[kU], cb[kU];
    int tok[kU], head[kU], which[kU];
    bool live[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int r = r0 + u * groups + group;
      live[u] = holds && r < rows;
      tok[u] = r / heads;
      int h = r - tok[u] * heads;
      which[u] = h < q_heads ? 0 : h < q_heads + k_heads ? 1 : 2;
      head[u] = which[u] == 0 ? h : which[u] == 1 ? h - q_heads : h - q_heads - k_heads;
      if (live[u]) {
        const Rows &s = g.seg[which[u]];
        const char *src =
            s.in + (long long)sizeof(T) * ((long long)(t0 + tok[u]) * s.in_tok + (long long)head[u] * s.in_head);
        ca[u].load(src + sizeof(T) * at.a);
        cb[u].load(src + sizeof(T) * at.b);
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const Rows &s = g.seg[which[u]];
      if (NORM || s.turn) {
        float x[V], y[V];
        ca[u].get(x);
        cb[u].get(y);
        if (NORM) {
          float ss = 0.f;
          if (live[u]) {
#pragma unroll
            for (int i = 0; i < V; ++i) ss += x[i] * x[i] + y[i] * y[i];
          }
          for (int o = 1 << g.lanes_log2 >> 1; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          if (s.w && live[u]) {
            const float r = rsqrtf(ss / (float)g.d + g.eps);
#pragma unroll
            for (int i = 0; i < V; i += 4) {
              const float4 wa = __ldg(reinterpret_cast<const float4 *>(s.w + at.a + i));
              const float4 wb = __ldg(reinterpret_cast<const float4 *>(s.w + at.b + i));
              x[i] *= r * wa.x, x[i + 1] *= r * wa.y, x[i + 2] *= r * wa.z, x[i + 3] *= r * wa.w;
              y[i] *= r * wb.x, y[i + 1] *= r * wb.y, y[i + 2] *= r * wb.z, y[i + 3] *= r * wb.w;
            }
          }
        }
        if (live[u]) {
          if (s.turn && at.turns) turn<V, PAIRS>(x, y, cs + tok[u] * g.half + slot * V, sn + tok[u] * g.half + slot * V);
          if (s.turn || s.w) {  // values pass bit for bit
            ca[u].set(x);
            cb[u].set(y);
          }
        }
      }
      if (live[u]) {
        char *dst;
        if (s.cache == 0) {
          dst = s.out + (long long)sizeof(T) * ((long long)(t0 + tok[u]) * s.out_tok + (long long)head[u] * s.out_head);
        } else {
          const long long row = home[tok[u]];
          if (row < 0) continue;
          dst = static_cast<char *>(s.cache == 1 ? g.cache.k : g.cache.v) +
                (long long)sizeof(T) * (row + (long long)head[u] * g.cache.page) * g.d;
        }
        ca[u].store(dst + sizeof(T) * at.a);
        cb[u].store(dst + sizeof(T) * at.b);
      }
    }
  }
}

// ---------------------------------------------------------------- backward with the norm
struct RotBackArgs {
  RotArgs g;          // seg[].in = dy, seg[].out = dx
  const char *x[2];   // the forward inputs
  long long x_tok[2], x_head[2];
  float *part;        // [CTAs][2][d]
  int ctas;
};

// The weights' gradients stay in registers (a lane's channels never change)
// over all the rows a CTA takes, are summed over its groups once at the end
// and leave as one row per CTA and weight; k_rotate_weight_sum adds those in
// a fixed order.
template <typename T, int V, bool PAIRS>
__global__ void __launch_bounds__(kRotThreads) k_rotate_back(const __grid_constant__ RotBackArgs a) {
  __shared__ __align__(16) float cs[kMaxTrig], sn[kMaxTrig];
  __shared__ float sums[kRotThreads / 32][TR_ROTARY_MAX_DIM];
  const RotArgs &g = a.g;
  pdl_wait();
  const int slot = threadIdx.x & ((1 << g.lanes_log2) - 1);
  const int group = threadIdx.x >> g.lanes_log2, groups = kRotThreads >> g.lanes_log2;
  const bool holds = slot < g.slots;
  const SlotPlace at = slot_place<V, PAIRS>(slot, g.half);
  float wa[2][V], wb[2][V], da[2][V], db[2][V];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool have = holds && g.seg[s].w;
      wa[s][i] = have ? __ldg(g.seg[s].w + at.a + i) : 0.f;
      wb[s][i] = have ? __ldg(g.seg[s].w + at.b + i) : 0.f;
      da[s][i] = db[s][i] = 0.f;
    }
  for (int t0 = blockIdx.x * g.tokens_per_cta; t0 < g.tokens; t0 += gridDim.x * g.tokens_per_cta) {
    const int nt = min(g.tokens_per_cta, g.tokens - t0);
    __syncthreads();  // the last tokens' angles are used up
    fill_trig(g, t0, nt, cs, sn);
    __syncthreads();
#pragma unroll
    for (int sg = 0; sg < 2; ++sg) {
      const Rows &s = g.seg[sg];
      const int rows = nt * s.heads;
      for (int r0 = 0; r0 < rows; r0 += groups) {
        const int r = r0 + group;
        const bool live = holds && r < rows;
        const int tok = live ? r / s.heads : 0, head = live ? r - tok * s.heads : 0;
        Chunk<T, V> ga, gb, xa, xb;
        float x[V], y[V], p[V], q[V];
        float ss = 0.f, dot = 0.f;
        if (live) {
          const char *src = s.in + (long long)sizeof(T) * ((long long)(t0 + tok) * s.in_tok + (long long)head * s.in_head);
          ga.load(src + sizeof(T) * at.a);
          gb.load(src + sizeof(T) * at.b);
          if (s.w) {
            const char *xs = a.x[sg] +
                             (long long)sizeof(T) * ((long long)(t0 + tok) * a.x_tok[sg] + (long long)head * a.x_head[sg]);
            xa.load(xs + sizeof(T) * at.a);
            xb.load(xs + sizeof(T) * at.b);
          }
          ga.get(p);
          gb.get(q);
          if (at.turns) turn<V, PAIRS>(p, q, cs + tok * g.half + slot * V, sn + tok * g.half + slot * V);
          if (s.w) {
            xa.get(x);
            xb.get(y);
#pragma unroll
            for (int i = 0; i < V; ++i) {
              ss += x[i] * x[i] + y[i] * y[i];
              dot += x[i] * (wa[sg][i] * p[i]) + y[i] * (wb[sg][i] * q[i]);
            }
          }
        }
        if (s.w) {
          for (int o = 1 << g.lanes_log2 >> 1; o; o >>= 1) {
            ss += __shfl_xor_sync(0xffffffffu, ss, o);
            dot += __shfl_xor_sync(0xffffffffu, dot, o);
          }
          if (live) {
            const float r1 = rsqrtf(ss / (float)g.d + g.eps);
            const float k = r1 * r1 * r1 * (dot / (float)g.d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
              da[sg][i] += p[i] * (x[i] * r1);
              db[sg][i] += q[i] * (y[i] * r1);
              p[i] = r1 * (wa[sg][i] * p[i]) - x[i] * k;
              q[i] = r1 * (wb[sg][i] * q[i]) - y[i] * k;
            }
          }
        }
        if (live) {
          ga.set(p);
          gb.set(q);
          char *dst = s.out + (long long)sizeof(T) * ((long long)(t0 + tok) * s.out_tok + (long long)head * s.out_head);
          ga.store(dst + sizeof(T) * at.a);
          gb.store(dst + sizeof(T) * at.b);
        }
      }
    }
  }
  // over the groups of each warp by shuffles, over the warps through shared memory
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int sg = 0; sg < 2; ++sg) {
    if (!g.seg[sg].w) continue;
#pragma unroll
    for (int i = 0; i < V; ++i)
      for (int o = 1 << g.lanes_log2; o < 32; o <<= 1) {
        da[sg][i] += __shfl_xor_sync(0xffffffffu, da[sg][i], o);
        db[sg][i] += __shfl_xor_sync(0xffffffffu, db[sg][i], o);
      }
    __syncthreads();
    if (holds && lane < 1 << g.lanes_log2)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        sums[warp][at.a + i] = da[sg][i];
        sums[warp][at.b + i] = db[sg][i];
      }
    __syncthreads();
    if ((int)threadIdx.x < g.d) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < kRotThreads / 32; ++w) t += sums[w][threadIdx.x];
      a.part[((long long)blockIdx.x * 2 + sg) * g.d + threadIdx.x] = t;
    }
  }
}

// dw[c] = the sum of the CTAs' rows: 1024 / 32 slices of rows for 32 channels
// per CTA, each slice in order, then the slices in order.
__global__ void __launch_bounds__(1024) k_rotate_weight_sum(const float *part, int ctas, int d, float *dq, float *dk) {
  __shared__ float sums[32][33];
  pdl_wait();
  const int sg = blockIdx.y, c = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  float *out = sg ? dk : dq;
  if (!out) return;
  float t = 0.f;
  if (c < d)
    for (int i = slice; i < ctas; i += 32) t += part[((long long)i * 2 + sg) * d + c];
  sums[slice][threadIdx.x & 31] = t;
  __syncthreads();
  if (slice == 0 && c < d) {
    float all = 0.f;
    for (int i = 0; i < 32; ++i) all += sums[i][threadIdx.x];
    out[c] = all;
  }
}

// ---------------------------------------------------------------- host side
bool misaligned16(const void *p) { return p && (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

tr_status check_rotary(const tr_rotary *r) {
  if (!r || r->head_dim <= 0 || r->rot_dim < 0 || r->rot_dim > r->head_dim || r->axes < 0) return TR_ERR_ARG;
  if (r->layout != TR_ROTARY_HALF && r->layout != TR_ROTARY_PAIRS) return TR_ERR_ARG;
  if (r->head_dim > TR_ROTARY_MAX_DIM) return TR_ERR_UNSUPPORTED;
  if (r->head_dim % 8 || r->rot_dim % 8) return TR_ERR_ALIGN;
  if (r->rot_dim && (!r->turns || !r->axis || r->axes < 1)) return TR_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(r->turns) & 7u) || (reinterpret_cast<uintptr_t>(r->axis) & 3u)) return TR_ERR_ALIGN;
  return TR_OK;
}

// Shape of the lane groups: V pairs a lane, 8 where the halves and the rest
// of the row are whole numbers of such slots, else 4.
int pairs_per_lane(int dtype, int d, int rot) {
  return dtype != TR_F32 && rot % 16 == 0 && d % 16 == 0 ? 8 : 4;
}

void shape(RotArgs &g, int dtype, int d, int rot, int tokens) {
  const int v = pairs_per_lane(dtype, d, rot);
  g.d = d;
  g.half = rot / 2;
  g.tokens = tokens;
  g.slots = d / (2 * v);
  g.lanes_log2 = 0;
  while ((1 << g.lanes_log2) < g.slots) ++g.lanes_log2;
  // A few tokens a CTA share the angles' cost and keep every thread busy
  // with them; fewer when the GPU would not be filled.
  const int sms = sm_count();
  int per = kMaxTrig / (g.half > 32 ? g.half : 32);
  if (per > kMaxTokens) per = kMaxTokens;
  const int fill = sms > 0 ? tokens / (4 * sms) : 1;
  g.tokens_per_cta = fill < 1 ? 1 : fill < per ? fill : per;
}

template <typename T, int V, bool PAIRS>
cudaError_t launch_rotate_t(const RotArgs &g, cudaStream_t st) {
  const dim3 grid((g.tokens + g.tokens_per_cta - 1) / g.tokens_per_cta);
  const bool norm = g.seg[0].w || g.seg[1].w;
  return norm ? launch_kernel(k_rotate<T, V, PAIRS, true>, grid, dim3(kRotThreads), 0, st, false, g)
              : launch_kernel(k_rotate<T, V, PAIRS, false>, grid, dim3(kRotThreads), 0, st, false, g);
}

cudaError_t launch_rotate(const RotArgs &g, int dtype, int rot, int layout, cudaStream_t st) {
  const bool wide = pairs_per_lane(dtype, g.d, rot) == 8, pairs = layout == TR_ROTARY_PAIRS;
  if (dtype == TR_F32) return pairs ? launch_rotate_t<float, 4, true>(g, st) : launch_rotate_t<float, 4, false>(g, st);
  if (dtype == TR_BF16) {
    if (wide)
      return pairs ? launch_rotate_t<__nv_bfloat16, 8, true>(g, st) : launch_rotate_t<__nv_bfloat16, 8, false>(g, st);
    return pairs ? launch_rotate_t<__nv_bfloat16, 4, true>(g, st) : launch_rotate_t<__nv_bfloat16, 4, false>(g, st);
  }
  if (wide) return pairs ? launch_rotate_t<__half, 8, true>(g, st) : launch_rotate_t<__half, 8, false>(g, st);
  return pairs ? launch_rotate_t<__half, 4, true>(g, st) : launch_rotate_t<__half, 4, false>(g, st);
}

template <typename T, int V, bool PAIRS>
cudaError_t launch_back_t(const RotBackArgs &a, cudaStream_t st) {
  return launch_kernel(k_rotate_back<T, V, PAIRS>, dim3(a.ctas), dim3(kRotThreads), 0, st, false, a);
}

cudaError_t launch_back(const RotBackArgs &a, int dtype, int rot, int layout, cudaStream_t st) {
  const bool wide = pairs_per_lane(dtype, a.g.d, rot) == 8, pairs = layout == TR_ROTARY_PAIRS;
  if (dtype == TR_F32) return pairs ? launch_back_t<float, 4, true>(a, st) : launch_back_t<float, 4, false>(a, st);
  if (dtype == TR_BF16) {
    if (wide) return pairs ? launch_back_t<__nv_bfloat16, 8, true>(a, st) : launch_back_t<__nv_bfloat16, 8, false>(a, st);
    return pairs ? launch_back_t<__nv_bfloat16, 4, true>(a, st) : launch_back_t<__nv_bfloat16, 4, false>(a, st);
  }
  if (wide) return pairs ? launch_back_t<__half, 8, true>(a, st) : launch_back_t<__half, 8, false>(a, st);
  return pairs ? launch_back_t<__half, 4, true>(a, st) : launch_back_t<__half, 4, false>(a, st);
}

Rows rows_of(const tr_heads *in, const tr_heads *out, const float *w, int turn, int cache) {
  Rows r{};
  if (!in || !in->p) return r;
  r.in = static_cast<const char *>(in->p);
  r.in_tok = in->token_stride;
  r.in_head = in->head_stride;
  r.heads = in->heads;
  if (out) {
    r.out = static_cast<char *>(out->p);
    r.out_tok = out->token_stride;
    r.out_head = out->head_stride;
  }
  r.w = w;
  r.turn = turn;
  r.cache = cache;
  return r;
}

// in and out together, or neither; the same heads.
tr_status check_pair(const tr_heads *in, const tr_heads *out, const float *w, int es, bool required) {
  const bool have = in && in->p;
  if (!have) return required || (out && out->p) ? TR_ERR_ARG : TR_OK;
  if (!out || !out->p || in->heads != out->heads) return TR_ERR_ARG;
  tr_status rc = check_heads(in, es);
  if (rc == TR_OK) rc = check_heads(out, es);
  if (rc == TR_OK && misaligned16(w)) rc = TR_ERR_ALIGN;
  return rc;
}

int back_ctas(int tokens) {
  const int sms = sm_count();
  const int most = 4 * (sms > 0 ? sms : 1);  // four resident CTAs per SM
  return tokens < most ? tokens : most;
}

}  // namespace
}  // namespace tr

using namespace tr;

extern "C" {

tr_status tr_rotary_turns(const double *h_freq, int32_t n, uint64_t *h_turns) {
  if (n < 0 || (n && (!h_freq || !h_turns))) return TR_ERR_ARG;
  for (int32_t i = 0; i < n; ++i)
    if (!std::isfinite(h_freq[i])) return TR_ERR_ARG;
  for (int32_t i = 0; i < n; ++i) {
    const double turn = h_freq[i] / 6.283185307179586476925287;
    const double part = turn - std::floor(turn);  // [0, 1]: turns modulo one
    const double scaled = part * 0x1p64;
    h_turns[i] = scaled >= 0x1p64 ? 0 : static_cast<uint64_t>(scaled);
  }
  return TR_OK;
}

tr_status tr_rotary_apply(const tr_rotary *r, int32_t dtype, int32_t tokens, const int32_t *pos, const tr_heads *q,
                          const float *q_weight, const tr_heads *q_out, const tr_heads *k, const float *k_weight,
                          const tr_heads *k_out, float eps, void *stream) {
  tr_status rc = check_rotary(r);
  if (rc != TR_OK) return rc;
  if (dtype != TR_F32 && dtype != TR_BF16 && dtype != TR_F16) return TR_ERR_DTYPE;
  if (tokens < 0 || (r->rot_dim && !pos)) return TR_ERR_ARG;
  const int es = elem_bytes(dtype);
  if ((rc = check_pair(q, q_out, q_weight, es, true)) != TR_OK) return rc;
  if ((rc = check_pair(k, k_out, k_weight, es, false)) != TR_OK) return rc;
  if (reinterpret_cast<uintptr_t>(pos) & 3u) return TR_ERR_ALIGN;
  if (tokens == 0) return TR_OK;
  RotArgs g{};
  shape(g, dtype, r->head_dim, r->rot_dim, tokens);
  g.turns = reinterpret_cast<const unsigned long long *>(r->turns);
  g.axis = r->axis;
  g.axes = r->axes;
  g.pos = pos;
  g.sign = 1.f;
  g.eps = eps;
  g.seg[0] = rows_of(q, q_out, q_weight, 1, 0);
  g.seg[1] = rows_of(k, k_out, k_weight, 1, 0);
  return launch_rotate(g, dtype, r->rot_dim, r->layout, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TR_OK
                                                                                                          : TR_ERR_CUDA;
}

size_t tr_rotary_backward_workspace_bytes(const tr_rotary *r, int32_t tokens) {
  if (check_rotary(r) != TR_OK || tokens < 0) return 0;
  return align_up((size_t)back_ctas(tokens) * 2 * r->head_dim * sizeof(float), 256);
}

tr_status tr_rotary_backward(const tr_rotary *r, int32_t dtype, int32_t tokens, const int32_t *pos,
                             const tr_heads *dq, const tr_heads *q, const float *q_weight, const tr_heads *dq_out,
                             float *dq_weight, const tr_heads *dk, const tr_heads *k, const float *k_weight,
                             const tr_heads *dk_out, float *dk_weight, float eps, void *ws, size_t ws_bytes,
                             void *stream) {
  tr_status rc = check_rotary(r);
  if (rc != TR_OK) return rc;
  if (dtype != TR_F32 && dtype != TR_BF16 && dtype != TR_F16) return TR_ERR_DTYPE;
  if (tokens < 0 || (r->rot_dim && !pos)) return TR_ERR_ARG;
  const int es = elem_bytes(dtype);
  if ((rc = check_pair(dq, dq_out, q_weight, es, true)) != TR_OK) return rc;
  if ((rc = check_pair(dk, dk_out, k_weight, es, false)) != TR_OK) return rc;
  if (reinterpret_cast<uintptr_t>(pos) & 3u) return TR_ERR_ALIGN;
  if (q_weight) {
    if (!dq_weight || !q || !q->p || q->heads != dq->heads) return TR_ERR_ARG;
    if ((rc = check_heads(q, es)) != TR_OK) return rc;
  } else if (dq_weight) {
    return TR_ERR_ARG;
  }
  if (k_weight) {
    if (!dk || !dk->p || !dk_weight || !k || !k->p || k->heads != dk->heads) return TR_ERR_ARG;
    if ((rc = check_heads(k, es)) != TR_OK) return rc;
  } else if (dk_weight) {
    return TR_ERR_ARG;
  }
  if ((reinterpret_cast<uintptr_t>(dq_weight) & 3u) || (reinterpret_cast<uintptr_t>(dk_weight) & 3u)) return TR_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  RotBackArgs a{};
  RotArgs &g = a.g;
  const bool norm = q_weight || k_weight;
  if (norm && tokens > 0 &&
      (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < tr_rotary_backward_workspace_bytes(r, tokens)))
    return TR_ERR_WORKSPACE;
  if (tokens == 0) {  // no rows: the weights' gradients are empty sums
    if (dq_weight && cudaMemsetAsync(dq_weight, 0, sizeof(float) * r->head_dim, st) != cudaSuccess) return TR_ERR_CUDA;
    if (dk_weight && cudaMemsetAsync(dk_weight, 0, sizeof(float) * r->head_dim, st) != cudaSuccess) return TR_ERR_CUDA;
    return TR_OK;
  }
  shape(g, dtype, r->head_dim, r->rot_dim, tokens);
  g.turns = reinterpret_cast<const unsigned long long *>(r->turns);
  g.axis = r->axis;
  g.axes = r->axes;
  g.pos = pos;
  g.sign = -1.f;
  g.eps = eps;
  g.seg[0] = rows_of(dq, dq_out, q_weight, 1, 0);
  g.seg[1] = rows_of(dk, dk_out, k_weight, 1, 0);
  if (!norm)  // a rotation's gradient is the rotation back
    return launch_rotate(g, dtype, r->rot_dim, r->layout, st) == cudaSuccess ? TR_OK : TR_ERR_CUDA;
  a.ctas = back_ctas(tokens);
  a.part = static_cast<float *>(ws);
  if (q_weight) a.x[0] = static_cast<const char *>(q->p), a.x_tok[0] = q->token_stride, a.x_head[0] = q->head_stride;
  if (k_weight) a.x[1] = static_cast<const char *>(k->p), a.x_tok[1] = k->token_stride, a.x_head[1] = k->head_stride;
  if (launch_back(a, dtype, r->rot_dim, r->layout, st) != cudaSuccess) return TR_ERR_CUDA;
  return launch_kernel(k_rotate_weight_sum, dim3((r->head_dim + 31) / 32, 2), dim3(1024), 0, st, false,
                       (const float *)a.part, a.ctas, (int)r->head_dim, dq_weight, dk_weight) == cudaSuccess
             ? TR_OK
             : TR_ERR_CUDA;
}

tr_status tr_cache_append(const tr_cache *c, const tr_heads *k, const tr_heads *v, const tr_rotary *r,
                          const int32_t *pos, const float *k_weight, const tr_heads *q, const float *q_weight,
                          const tr_heads *q_out, float eps, int32_t *d_error, void *stream) {
  tr_status rc = check_cache(c);
  if (rc != TR_OK) return rc;
  if (r) {
    if ((rc = check_rotary(r)) != TR_OK) return rc;
    if (r->head_dim != c->head_dim || (r->rot_dim && !pos)) return TR_ERR_ARG;
  }
  if (!k || !k->p || !v || !v->p || k->heads != c->heads || v->heads != c->heads) return TR_ERR_ARG;
  if ((rc = check_heads(k, 2)) != TR_OK || (rc = check_heads(v, 2)) != TR_OK) return rc;
  if (misaligned16(k_weight) || (reinterpret_cast<uintptr_t>(pos) & 3u)) return TR_ERR_ALIGN;
  if ((rc = check_pair(q, q_out, q_weight, 2, false)) != TR_OK) return rc;
  if (c->total_new == 0 || c->batch == 0) return TR_OK;
  const int rot = r ? r->rot_dim : 0;
  RotArgs g{};
  shape(g, c->dtype, c->head_dim, rot, c->total_new);
  if (rot) {
    g.turns = reinterpret_cast<const unsigned long long *>(r->turns);
    g.axis = r->axis;
    g.axes = r->axes;
    g.pos = pos;
  }
  g.sign = 1.f;
  g.eps = eps;
  g.seg[0] = rows_of(q, q_out, q_weight, rot > 0, 0);
  g.seg[1] = rows_of(k, nullptr, k_weight, rot > 0, 1);
  g.seg[2] = rows_of(v, nullptr, nullptr, 0, 2);
  g.cache = cache_view(c);
  g.err = d_error;
  return launch_rotate(g, c->dtype, rot, r ? r->layout : TR_ROTARY_HALF, static_cast<cudaStream_t>(stream)) ==
                 cudaSuccess
             ? TR_OK
             : TR_ERR_CUDA;
}

}  // extern "C"
