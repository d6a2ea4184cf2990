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
// Each row is read once and written once.  Measured on GB300, bf16, graphs of
// calls over inputs larger than L2: 12288 tokens x 64 heads of 128 66.6 us (6.0
// TB/s of the measured 6.77 copy: memory); with the norm 6272 tokens x 32 heads
// 23.3 us (4.4 TB/s), their gradients 44.0 us (3.5 TB/s, two launches), 29.6k
// tokens appended 109 us (4.9 TB/s).  There neither memory (30 to 55 % busy) nor
// instruction issue (47 to 58 %) is full: with two rows in flight per lane
// group, latency is the limit.  fp32: 128, 37.4 and 66.9 us.  A row belongs to a group of lanes, each of which holds both halves of V
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
#include "tr_pack.cuh"

namespace tr {
namespace {

constexpr int kRotThreads = 256;
constexpr int kMaxTokens = 32;                      // tokens a CTA takes at a time at most
constexpr int kMaxTrig = 4 * kRotThreads;           // angles it holds (tokens x frequencies)

using pack::f2;

struct Rows {
  const char *in;   // NULL: segment absent
  char *out;        // NULL: into the cache
  int in_tok, in_head, out_tok, out_head;  // elements
  int heads;
  const float *w;   // norm weight or NULL
  int turn;         // rows are rotated
  int cache;        // 0: out, 1: the cache's keys, 2: its values
  int tokens;       // that a CTA takes at a time
  int toks, rest;   // a step of one row per lane group: whole tokens, and heads
  int cta0;         // first CTA of the segment
};

struct RotArgs {
  const unsigned long long *turns;
  const int32_t *axis;
  const int32_t *pos;
  int d, half, axes, tokens;
  int lanes_log2;   // lanes of a row's group
  int slots;        // lanes of it that hold channels: d / (2 V)
  int trig_toks, trig_rest;  // a step of kRotThreads angles
  float sign;       // -1 turns backwards
  float eps, inv_d;
  Rows seg[3];      // queries, keys, values
  CacheView cache;
  int32_t *err;
};

// ---------------------------------------------------------------- elements
template <typename T>
__device__ __forceinline__ long long row_bytes(int tok, int tok_stride, int head, int head_stride) {
  return (long long)sizeof(T) * ((long long)tok * tok_stride + (long long)head * head_stride);
}
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
  __device__ __forceinline__ void get(f2 (&f)[V / 2]) const {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      if constexpr (sizeof(T) == 4) {
        f[i] = pack::make(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
      } else {
        const float2 t = unpack2<T>(w[i]);
        f[i] = pack::make(t.x, t.y);
      }
    }
  }
  __device__ __forceinline__ void set(const f2 (&f)[V / 2]) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const float2 t = pack::split(f[i]);
      if constexpr (sizeof(T) == 4)
        w[2 * i] = __float_as_uint(t.x), w[2 * i + 1] = __float_as_uint(t.y);
      else
        w[i] = pack2<T>(t.x, t.y);
    }
  }
};

// 2 V floats of a vector at the slot's channels, as pairs.
template <int V>
__device__ __forceinline__ void get_weights(const float *w, int a, int b, f2 (&wa)[V / 2], f2 (&wb)[V / 2]) {
#pragma unroll
  for (int i = 0; i < V; i += 4) {
    const float4 x = __ldg(reinterpret_cast<const float4 *>(w + a + i)), y = __ldg(reinterpret_cast<const float4 *>(w + b + i));
    wa[i / 2] = pack::make(x.x, x.y), wa[i / 2 + 1] = pack::make(x.z, x.w);
    wb[i / 2] = pack::make(y.x, y.y), wb[i / 2 + 1] = pack::make(y.z, y.w);
  }
}

// Sum over the 2^log2 lanes of a row's group.
__device__ __forceinline__ float group_sum(float v, int log2) {
#pragma unroll
  for (int i = 0; i < 5; ++i)
    if (i < log2) v += __shfl_xor_sync(0xffffffffu, v, 1 << i);
  return v;
}

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

// Turns the slot's pairs in place by V angles (16-byte aligned in shared
// memory); with PAIRS a pair is two neighbours of the 2 V channels, else the
// same place in both chunks.
template <int V, bool PAIRS>
__device__ __forceinline__ void turn(f2 (&x)[V / 2], f2 (&y)[V / 2], const float *cs, const float *sn) {
#pragma unroll
  for (int j = 0; j < V; j += 4) {
    const float4 c = *reinterpret_cast<const float4 *>(cs + j), s = *reinterpret_cast<const float4 *>(sn + j);
    if (PAIRS) {
      const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f2 &v = j + k < V / 2 ? x[(j + k) % (V / 2)] : y[(j + k) % (V / 2)];
        const float2 t = pack::split(v);
        v = pack::fma(v, pack::make(cc[k], cc[k]), pack::mul(pack::make(t.y, t.x), pack::make(-ss[k], ss[k])));
      }
    } else {
      const f2 c2[2] = {pack::make(c.x, c.y), pack::make(c.z, c.w)}, s2[2] = {pack::make(s.x, s.y), pack::make(s.z, s.w)};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f2 a = x[j / 2 + k], b = y[j / 2 + k];
        x[j / 2 + k] = pack::sub(pack::mul(a, c2[k]), pack::mul(b, s2[k]));
        y[j / 2 + k] = pack::fma(b, c2[k], pack::mul(a, s2[k]));
      }
    }
  }
}

// A group's walk over the rows (token, head) of its CTA, `groups` rows on
// each time.
struct RowWalk {
  int tok, head;
  __device__ __forceinline__ RowWalk(int r, int heads) : tok(r < heads ? 0 : r / heads), head(r - tok * heads) {}
  __device__ __forceinline__ void step(int toks, int rest, int heads) {
    tok += toks;
    head += rest;
    if (head >= heads) head -= heads, ++tok;
  }
};

// Cosines and sines of the CTA's tokens into shared memory.  position *
// turns modulo 2^64 is the angle as a fraction of a turn, exactly; its top 32
// bits, signed, are the angle in units of pi / 2^31.
__device__ __forceinline__ void fill_trig(const RotArgs &g, int t0, int nt, float *cs, float *sn) {
  if (!g.half) return;
  RowWalk w(threadIdx.x, g.half);
  for (int i = threadIdx.x; i < nt * g.half; i += kRotThreads, w.step(g.trig_toks, g.trig_rest, g.half)) {
    const int lt = w.tok, f = w.head;
    const int ax = __ldg(g.axis + f);
    const long long p = (unsigned)ax < (unsigned)g.axes ? (long long)__ldg(g.pos + (long long)ax * g.tokens + t0 + lt) : 0;
    const unsigned long long frac = (unsigned long long)p * __ldg(g.turns + f);
    float s, c;
    sincospif((float)(int)(frac >> 32) * 0x1p-31f, &s, &c);
    cs[i] = c;
    sn[i] = s * g.sign;
  }
}

// Two (normed) or four rows per lane group in flight, the first asked for
// before the angles: a CTA has few rows per group, so the latency of its
// first loads would otherwise stand alone.
// (Rows of all three segments in one CTA took far more instructions -- which
// segment, whose weight, where to: a third more time, 26.3 us against 20.0 us,
// for 6272 tokens x 32 normed heads when both were tried, on inputs in L2.)
template <typename T, int V, bool PAIRS, bool NORM>
__global__ void __launch_bounds__(kRotThreads, V == 8 ? 3 : 4) k_rotate(const __grid_constant__ RotArgs g) {
  __shared__ __align__(16) float cs[kMaxTrig], sn[kMaxTrig];
  __shared__ long long home[kMaxTokens];  // the token's first key row in the cache (head 0), or -1
  pdl_wait();  // q, k, v come from the kernel before
  const int sg = (int)blockIdx.x < g.seg[1].cta0 ? 0 : (int)blockIdx.x < g.seg[2].cta0 ? 1 : 2;
  const Rows &s = sg == 0 ? g.seg[0] : sg == 1 ? g.seg[1] : g.seg[2];
  const int heads = s.heads, t0 = (blockIdx.x - s.cta0) * s.tokens;
  const int nt = min(s.tokens, g.tokens - t0), rows = nt * heads;
  const int slot = threadIdx.x & ((1 << g.lanes_log2) - 1);
  const int group = threadIdx.x >> g.lanes_log2, groups = kRotThreads >> g.lanes_log2;
  const bool holds = slot < g.slots;
  const SlotPlace at = slot_place<V, PAIRS>(slot, g.half);
  const char *src = s.in + (long long)sizeof(T) * ((long long)t0 * s.in_tok + at.a);
  const int ab = (int)sizeof(T) * (at.b - at.a);
  constexpr int kU = NORM ? 2 : 4;
  Chunk<T, V> na[kU], nb[kU];
  RowWalk ahead(group, heads);
  auto ask = [&]() {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (holds && ahead.tok < nt) {
        const char *p = src + row_bytes<T>(ahead.tok, s.in_tok, ahead.head, s.in_head);
        na[u].load(p);
        nb[u].load(p + ab);
      }
      ahead.step(s.toks, s.rest, heads);
    }
  };
  ask();
  if (s.turn) fill_trig(g, t0, nt, cs, sn);
  if (s.cache) {  // a warp per token
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x >> 5; i < nt; i += kRotThreads / 32) {
      const int t = t0 + i;
      int b = -1;  // the last sequence that starts at or before the token
      for (int i0 = 0; i0 < g.cache.batch; i0 += 32) {
        const bool before = i0 + lane < g.cache.batch && __ldg(g.cache.cu_new + i0 + lane) <= t;
        const unsigned m = __ballot_sync(0xffffffffu, before);
        b += __popc(m);
        if (m != 0xffffffffu) break;
      }
      if (lane == 0) {
        long long row = -1;
        const int end = b >= 0 ? __ldg(g.cache.cu_new + b + 1) : 0;
        if (t < end) {
          const int key = max(__ldg(g.cache.lens + b), 0) - end + t;
          const int page = key >= 0 ? page_of(g.cache, b, key) : -1;
          if (page >= 0)
            row = (long long)page * g.cache.heads * g.cache.page + (key & (g.cache.page - 1));
          else if (g.err)
            atomicOr(g.err, TR_CACHE_ERR_PAGE);
        }
        home[i] = row;
      }
    }
  }
  f2 wa[V / 2] = {}, wb[V / 2] = {};
  if (NORM && s.w && holds) get_weights<V>(s.w, at.a, at.b, wa, wb);
  __syncthreads();
  RowWalk now(group, heads);
  for (int r0 = 0; r0 < rows; r0 += kU * groups) {  // the same trips for every lane of a warp
    if (r0) ask();
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const bool live = holds && now.tok < nt;
      if (s.w || s.turn) {  // (values pass bit for bit)
        f2 x[V / 2], y[V / 2];
        na[u].get(x);
        nb[u].get(y);
        if (NORM && s.w) {
          f2 s2 = 0ull;
#pragma unroll
          for (int i = 0; i < V / 2; ++i) s2 = pack::fma(x[i], x[i], pack::fma(y[i], y[i], s2));
          const float2 t = pack::split(s2);
          float ss = live ? t.x + t.y : 0.f;
          ss = group_sum(ss, g.lanes_log2);
          const float f = rsqrtf(ss * g.inv_d + g.eps);
          const f2 f2f = pack::make(f, f);
#pragma unroll
          for (int i = 0; i < V / 2; ++i) {
            x[i] = pack::mul(x[i], pack::mul(f2f, wa[i]));
            y[i] = pack::mul(y[i], pack::mul(f2f, wb[i]));
          }
        }
        if (live && s.turn && at.turns)
          turn<V, PAIRS>(x, y, cs + now.tok * g.half + slot * V, sn + now.tok * g.half + slot * V);
        na[u].set(x);
        nb[u].set(y);
      }
      if (live) {
        char *dst;
        bool there = true;
        if (s.cache == 0) {
          dst = s.out + row_bytes<T>(t0 + now.tok, s.out_tok, now.head, s.out_head);
        } else {
          const long long row = home[now.tok];
          there = row >= 0;
          dst = static_cast<char *>(s.cache == 1 ? g.cache.k : g.cache.v) +
                (long long)sizeof(T) * ((row + now.head * g.cache.page) * g.d);
        }
        if (there) {
          na[u].store(dst + sizeof(T) * at.a);
          nb[u].store(dst + sizeof(T) * at.b);
        }
      }
      now.step(s.toks, s.rest, heads);
    }
  }
}

// ---------------------------------------------------------------- backward with the norm
struct RotBackArgs {
  RotArgs g;          // seg[].in = dy, seg[].out = dx
  const char *x[2];   // the forward inputs
  int x_tok[2], x_head[2];
  float *part;        // [CTAs][d]
  int ctas, q_ctas;   // the first q_ctas take the queries' rows, the others the keys'
};

// A CTA takes the rows of one of the two segments, so that a lane's weights
// and its share of their gradients (its channels never change) stay in
// registers over all of them; the gradients are summed over the CTA once at
// the end and leave as one row per CTA, which k_rotate_weight_sum adds in a
// fixed order.  The next row is asked for before the present one is worked
// on.
template <typename T, int V, bool PAIRS>
__global__ void __launch_bounds__(kRotThreads, 2) k_rotate_back(const __grid_constant__ RotBackArgs a) {
  __shared__ __align__(16) float cs[kMaxTrig], sn[kMaxTrig];
  __shared__ float sums[kRotThreads / 32][TR_ROTARY_MAX_DIM];
  const RotArgs &g = a.g;
  pdl_wait();
  const int sg = (int)blockIdx.x < a.q_ctas ? 0 : 1;
  const int cta = sg ? blockIdx.x - a.q_ctas : blockIdx.x, ctas = sg ? a.ctas - a.q_ctas : a.q_ctas;
  const Rows &s = sg ? g.seg[1] : g.seg[0];
  const bool normed = s.w != nullptr;
  const int slot = threadIdx.x & ((1 << g.lanes_log2) - 1);
  const int group = threadIdx.x >> g.lanes_log2, groups = kRotThreads >> g.lanes_log2;
  const bool holds = slot < g.slots;
  const SlotPlace at = slot_place<V, PAIRS>(slot, g.half);
  f2 wa[V / 2] = {}, wb[V / 2] = {}, da[V / 2] = {}, db[V / 2] = {};
  if (normed && holds) get_weights<V>(s.w, at.a, at.b, wa, wb);
  Chunk<T, V> ga, gb, xa, xb;
  const int heads = s.heads, toks = s.toks, rest = s.rest;
  for (int t0 = cta * s.tokens; t0 < g.tokens; t0 += ctas * s.tokens) {
    const int nt = min(s.tokens, g.tokens - t0), rows = nt * heads;
    RowWalk ahead(group, heads), now = ahead;
    auto ask = [&]() {
      const int tok = ahead.tok, head = ahead.head;
      ahead.step(toks, rest, heads);
      if (!holds || tok >= nt) return;
      const char *src = s.in + row_bytes<T>(t0 + tok, s.in_tok, head, s.in_head);
      ga.load(src + sizeof(T) * at.a);
      gb.load(src + sizeof(T) * at.b);
      if (normed) {
        const char *xs = (sg ? a.x[1] : a.x[0]) + row_bytes<T>(t0 + tok, sg ? a.x_tok[1] : a.x_tok[0], head,
                                                               sg ? a.x_head[1] : a.x_head[0]);
        xa.load(xs + sizeof(T) * at.a);
        xb.load(xs + sizeof(T) * at.b);
      }
    };
    ask();
    __syncthreads();  // the last tokens' angles are used up
    fill_trig(g, t0, nt, cs, sn);
    __syncthreads();
    for (int r0 = 0; r0 < rows; r0 += groups) {
      const int tok = now.tok, head = now.head;
      const bool live = holds && tok < nt;
      now.step(toks, rest, heads);
      f2 x[V / 2], y[V / 2], p[V / 2], q[V / 2];
      ga.get(p);
      gb.get(q);
      xa.get(x);
      xb.get(y);
      ask();
      if (live && at.turns) turn<V, PAIRS>(p, q, cs + tok * g.half + slot * V, sn + tok * g.half + slot * V);
      if (normed) {
        f2 s2 = 0ull, d2 = 0ull;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          s2 = pack::fma(x[i], x[i], pack::fma(y[i], y[i], s2));
          d2 = pack::fma(x[i], pack::mul(wa[i], p[i]), pack::fma(y[i], pack::mul(wb[i], q[i]), d2));
        }
        const float2 st = pack::split(s2), dt = pack::split(d2);
        float ss = live ? st.x + st.y : 0.f, dot = live ? dt.x + dt.y : 0.f;
        ss = group_sum(ss, g.lanes_log2);
        dot = group_sum(dot, g.lanes_log2);
        if (live) {
          const float r1 = rsqrtf(ss * g.inv_d + g.eps);
          const float k = r1 * r1 * r1 * (dot * g.inv_d);
          const f2 r2 = pack::make(r1, r1), k2 = pack::make(k, k);
#pragma unroll
          for (int i = 0; i < V / 2; ++i) {
            da[i] = pack::fma(p[i], pack::mul(x[i], r2), da[i]);
            db[i] = pack::fma(q[i], pack::mul(y[i], r2), db[i]);
            p[i] = pack::sub(pack::mul(r2, pack::mul(wa[i], p[i])), pack::mul(x[i], k2));
            q[i] = pack::sub(pack::mul(r2, pack::mul(wb[i], q[i])), pack::mul(y[i], k2));
          }
        }
      }
      if (live) {
        Chunk<T, V> oa, ob;
        oa.set(p);
        ob.set(q);
        char *dst = s.out + row_bytes<T>(t0 + tok, s.out_tok, head, s.out_head);
        oa.store(dst + sizeof(T) * at.a);
        ob.store(dst + sizeof(T) * at.b);
      }
    }
  }
  if (!normed) return;
  // over the groups of each warp by shuffles, over the warps through shared memory
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < V / 2; ++i) {
    float2 u = pack::split(da[i]), v = pack::split(db[i]);
    for (int o = 1 << g.lanes_log2; o < 32; o <<= 1) {
      u.x += __shfl_xor_sync(0xffffffffu, u.x, o);
      u.y += __shfl_xor_sync(0xffffffffu, u.y, o);
      v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
      v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if (holds && lane < 1 << g.lanes_log2) {
      sums[warp][at.a + 2 * i] = u.x, sums[warp][at.a + 2 * i + 1] = u.y;
      sums[warp][at.b + 2 * i] = v.x, sums[warp][at.b + 2 * i + 1] = v.y;
    }
  }
  __syncthreads();
  if ((int)threadIdx.x < g.d) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kRotThreads / 32; ++w) t += sums[w][threadIdx.x];
    a.part[(long long)blockIdx.x * g.d + threadIdx.x] = t;
  }
}

// dw[c] = the sum of the CTAs' rows: 1024 / 32 slices of rows for 32 channels
// per CTA, each slice in order, then the slices in order.
__global__ void __launch_bounds__(1024)
    k_rotate_weight_sum(const float *part, int q_ctas, int ctas, int d, float *dq, float *dk) {
  __shared__ float sums[32][33];
  pdl_wait();
  const int sg = blockIdx.y, c = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  float *out = sg ? dk : dq;
  if (!out) return;
  float t = 0.f;
  if (c < d)
    for (int i = (sg ? q_ctas : 0) + slice; i < (sg ? ctas : q_ctas); i += 32) t += part[(long long)i * d + c];
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
  g.inv_d = 1.f / (float)d;
  g.half = rot / 2;
  g.tokens = tokens;
  g.slots = d / (2 * v);
  g.lanes_log2 = 0;
  while ((1 << g.lanes_log2) < g.slots) ++g.lanes_log2;
  if (g.half) g.trig_toks = kRotThreads / g.half, g.trig_rest = kRotThreads % g.half;
}

void set_steps(RotArgs &g) {
  const int groups = kRotThreads >> g.lanes_log2;
  for (Rows &s : g.seg)
    if (s.heads) s.toks = groups / s.heads, s.rest = groups % s.heads;
}

// The tokens that a CTA takes of each segment: four rows for every lane
// group, all asked for at once (12288 tokens x 64 heads: with sixteen a quarter
// more time), eight where they are normed, so that what a CTA costs besides its
// rows (addresses, weights) is spread over more; fewer when the three CTAs an
// SM holds would not all get some, and within the room for angles.  Returns
// the CTAs of all segments.
int cut_segments(RotArgs &g) {
  const bool norm = g.seg[0].w || g.seg[1].w;
  const int sms = sm_count() > 0 ? sm_count() : 1, groups = kRotThreads >> g.lanes_log2;
  int room = g.half ? kMaxTrig / g.half : kMaxTokens;
  if (room > kMaxTokens) room = kMaxTokens;
  long long all = 0;
  for (int i = 0; i < 3; ++i) all += (long long)g.tokens * g.seg[i].heads;
  long long rows = all / (3 * sms);
  if (rows < groups) rows = groups;
  const int most = norm ? 8 * groups : 4 * groups;
  if (rows > most) rows = most;
  set_steps(g);
  int ctas = 0;
  for (int i = 0; i < 3; ++i) {
    Rows &s = g.seg[i];
    s.cta0 = ctas;
    if (!s.in) continue;
    const long long n = rows / s.heads;
    s.tokens = n < 1 ? 1 : n > room ? room : (int)n;
    ctas += (g.tokens + s.tokens - 1) / s.tokens;
  }
  return ctas;
}

template <typename T, int V, bool PAIRS>
cudaError_t launch_rotate_t(RotArgs &g, cudaStream_t st) {
  const int ctas = cut_segments(g);
  return g.seg[0].w || g.seg[1].w
             ? launch_kernel(k_rotate<T, V, PAIRS, true>, dim3(ctas), dim3(kRotThreads), 0, st, false, g)
             : launch_kernel(k_rotate<T, V, PAIRS, false>, dim3(ctas), dim3(kRotThreads), 0, st, false, g);
}

cudaError_t launch_rotate(RotArgs &g, int dtype, int rot, int layout, cudaStream_t st) {
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
  r.in_tok = (int)in->token_stride;
  r.in_head = (int)in->head_stride;
  r.heads = in->heads;
  if (out) {
    r.out = static_cast<char *>(out->p);
    r.out_tok = (int)out->token_stride;
    r.out_head = (int)out->head_stride;
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

// CTAs of the backward pass: one wave of two per SM, at least one for each
// segment.
int back_ctas() {
  const int sms = sm_count();
  return 2 * (sms > 0 ? sms : 1);
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
  return align_up((size_t)back_ctas() * r->head_dim * sizeof(float), 256);
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
  // tokens a CTA takes at a time: as many as the angles' room holds, fewer
  // when the CTAs would not all get some
  const int q_heads = g.seg[0].heads, k_heads = g.seg[1].heads;
  a.ctas = back_ctas();
  a.q_ctas = k_heads ? (int)((long long)a.ctas * q_heads / (q_heads + k_heads)) : a.ctas;
  if (a.q_ctas < 1) a.q_ctas = 1;
  if (k_heads && a.q_ctas == a.ctas) --a.q_ctas;
  int per = g.half ? kMaxTrig / g.half : kMaxTokens;
  if (per > kMaxTokens) per = kMaxTokens;
  for (int i = 0; i < 2; ++i) {
    // equal rounds: n tokens for each CTA in as few rounds as the room allows
    const int ctas = i ? (a.ctas - a.q_ctas > 0 ? a.ctas - a.q_ctas : 1) : a.q_ctas;
    const int n = (tokens + ctas - 1) / ctas, rounds = (n + per - 1) / per;
    g.seg[i].tokens = (n + rounds - 1) / rounds;
  }
  a.part = static_cast<float *>(ws);
  set_steps(g);
  if (q_weight) a.x[0] = static_cast<const char *>(q->p), a.x_tok[0] = (int)q->token_stride, a.x_head[0] = (int)q->head_stride;
  if (k_weight) a.x[1] = static_cast<const char *>(k->p), a.x_tok[1] = (int)k->token_stride, a.x_head[1] = (int)k->head_stride;
  if (launch_back(a, dtype, r->rot_dim, r->layout, st) != cudaSuccess) return TR_ERR_CUDA;
  return launch_kernel(k_rotate_weight_sum, dim3((r->head_dim + 31) / 32, 2), dim3(1024), 0, st, true,
                       (const float *)a.part, a.q_ctas, a.ctas, (int)r->head_dim, dq_weight, dk_weight) == cudaSuccess
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
  if (c->total_new == 0) return TR_OK;
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
