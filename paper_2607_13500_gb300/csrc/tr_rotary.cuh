// The norm and the rotation of heads' rows as the kernels that apply them
// share them (tr_rotary.cu, tr_append8.cu): elements, angles, a CTA's rows, and
// the host's checks and cuts.
#pragma once

#include <climits>
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tr_cache.cuh"
#include "tr_internal.cuh"
#include "tr_pack.cuh"

namespace tr {
namespace rotary {

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
// (threads: a half of the CTA's may take tokens of its own.)
__device__ __forceinline__ void fill_trig(const RotArgs &g, int t0, int nt, float *cs, float *sn, int threads = kRotThreads) {
  if (!g.half) return;
  const int tid = threadIdx.x & (threads - 1);
  const int toks = threads == kRotThreads ? g.trig_toks : threads / g.half, rest = threads == kRotThreads ? g.trig_rest : threads - toks * g.half;
  RowWalk w(tid, g.half);
  for (int i = tid; i < nt * g.half; i += threads, w.step(toks, rest, g.half)) {
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
// (cs, sn: kMaxTrig floats of shared memory each; home: kMaxTokens keys' rows.)
template <typename T, int V, bool PAIRS, bool NORM, int kU = NORM ? 2 : 4>
__device__ __forceinline__ void rotate_rows(const RotArgs &g, int block, float *cs, float *sn, long long *home) {
  const int sg = block < g.seg[1].cta0 ? 0 : block < g.seg[2].cta0 ? 1 : 2;
  const Rows &s = sg == 0 ? g.seg[0] : sg == 1 ? g.seg[1] : g.seg[2];
  const int heads = s.heads, t0 = (block - s.cta0) * s.tokens;
  const int nt = min(s.tokens, g.tokens - t0), rows = nt * heads;
  const int slot = threadIdx.x & ((1 << g.lanes_log2) - 1);
  const int group = threadIdx.x >> g.lanes_log2, groups = kRotThreads >> g.lanes_log2;
  const bool holds = slot < g.slots;
  const SlotPlace at = slot_place<V, PAIRS>(slot, g.half);
  const char *src = s.in + (long long)sizeof(T) * ((long long)t0 * s.in_tok + at.a);
  const int ab = (int)sizeof(T) * (at.b - at.a);
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

// ---------------------------------------------------------------- host side
inline bool misaligned16(const void *p) { return p && (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline tr_status check_rotary(const tr_rotary *r) {
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
inline int pairs_per_lane(int dtype, int d, int rot) {
  return dtype != TR_F32 && rot % 16 == 0 && d % 16 == 0 ? 8 : 4;
}

inline void shape(RotArgs &g, int dtype, int d, int rot, int tokens) {
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

inline void set_steps(RotArgs &g) {
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
inline int cut_segments(RotArgs &g) {
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

inline Rows rows_of(const tr_heads *in, const tr_heads *out, const float *w, int turn, int cache) {
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
inline tr_status check_pair(const tr_heads *in, const tr_heads *out, const float *w, int es, bool required) {
  const bool have = in && in->p;
  if (!have) return required || (out && out->p) ? TR_ERR_ARG : TR_OK;
  if (!out || !out->p || in->heads != out->heads) return TR_ERR_ARG;
  tr_status rc = check_heads(in, es);
  if (rc == TR_OK) rc = check_heads(out, es);
  if (rc == TR_OK && misaligned16(w)) rc = TR_ERR_ALIGN;
  return rc;
}

}  // namespace rotary
}  // namespace tr
