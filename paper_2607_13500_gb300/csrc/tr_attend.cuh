// What the attention kernels share: their arguments, the rows and keys of a
// block, the loads of K and V tiles, and what becomes of values that are not
// finite and not seen by every row.
#pragma once

#include <cfloat>
#include <climits>
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tr_cache.cuh"
#include "tr_map.cuh"
#include "tr_tc.cuh"

namespace tr {
namespace attend {

constexpr int kTile = 128;  // keys of a tile, rows of a block

struct AttendArgs {
  CacheView c;
  const char *q;
  char *o;
  long long q_tok, q_head, o_tok, o_head;  // elements
  int q_heads, group;                      // group: query heads of a key head
  float *lse;
  float scale;      // |scale| log2(e), never zero
  int negate;       // scale < 0: the queries enter negated
  int causal, window;
  int splits;       // parts of the keys, each a CTA's: split_tiles tiles (the last: the rest)
  int split_tiles;
  float *part;      // splits > 1: [splits][total_new * q_heads][d] unnormalised sums,
  float2 *part_ml;  //             [splits][total_new * q_heads] (maximum, sum)
  int page_log2;
  int ctas;         // few rows: CTAs that share the work; part [2 ctas][16][d], part_ml [2 ctas][16]
  int32_t *err;
};

template <typename T>
struct Bits;
template <>
struct Bits<__nv_bfloat16> {
  static constexpr bool kBf16 = true;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  // a * 0 + b of a pair: b, or NaN where a is not finite
  static __device__ __forceinline__ uint32_t fma0(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(0u), "r"(b));
    return r;
  }
};
template <>
struct Bits<__half> {
  static constexpr bool kBf16 = false;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  static __device__ __forceinline__ uint32_t fma0(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(0u), "r"(b));
    return r;
  }
};

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// ---------------------------------------------------------------- where a CTA works
// Sequence b's row blocks occupy the slots from floor(cu_new[b] group / R) + b
// on (R rows a block), which leaves room for all of them whatever cu_new
// holds; the last slot of a sequence may stay empty.  The tokens behind the
// last sequence's, which belong to none, have the slots behind its own.
struct Block {
  int seq, first;     // sequence, first row (token * group + head) of the block
  int rows;           // rows of the sequence: new tokens * group
  int tok0;           // first new token of the sequence
  int base;           // key of new token 0
  int len;            // keys of the sequence
  int end;            // the last sequence's slots and those behind: first token of no sequence (others: total_new)
};

// All lanes of a warp together; seq = -1 for an empty slot.
__device__ __forceinline__ Block find_block(const AttendArgs &g, int slot, int rows_per_block) {
  const int lane = threadIdx.x & 31;
  const CacheView &c = g.c;
  int b = 0;  // sequences whose slots start at or before this one, less one
  for (int i0 = 0; i0 < c.batch; i0 += 32) {
    const int i = i0 + lane;
    const bool before =
        i < c.batch && ((long long)__ldg(c.cu_new + i) * g.group) / rows_per_block + i <= (long long)slot;
    const unsigned m = __ballot_sync(0xffffffffu, before);
    b += __popc(m);
    if (m != 0xffffffffu) break;
  }
  b -= 1;
  Block k;
  k.seq = -1;
  k.rows = k.first = k.tok0 = k.base = k.len = 0;
  k.end = c.batch ? c.total_new : 0;
  if (b < 0) return k;
  const int t0 = __ldg(c.cu_new + b), t1 = min(__ldg(c.cu_new + b + 1), c.total_new);
  const int n = t1 > t0 ? t1 - t0 : 0;
  const long long start = ((long long)t0 * g.group) / rows_per_block + b;
  if (b + 1 == c.batch) k.end = max(t1, 0);
  k.first = (int)((slot - start) * rows_per_block);
  k.rows = n * g.group;
  if (t0 < 0 || k.first < 0 || k.first >= k.rows) return k;
  k.seq = b;
  k.tok0 = t0;
  k.len = cache_len(c, b);
  k.base = max(__ldg(c.lens + b), 0) - n;
  return k;
}

// First key of the window that ends with key `own`.
__device__ __forceinline__ int window_start(int own, int window) { return own >= window ? own - window + 1 : 0; }

// Keys [lo, hi) that some row of [r0, r1) sees.
struct Range {
  int lo, hi;
};
__device__ __forceinline__ Range keys_of_rows(const AttendArgs &g, const Block &k, int r0, int r1) {
  Range r{0, 0};
  if (r0 >= r1) return r;
  r.hi = g.causal ? min(k.len, k.base + (r1 - 1) / g.group + 1) : k.len;
  r.lo = g.window > 0 ? window_start(k.base + r0 / g.group, g.window) : 0;
  if (r.hi <= r.lo) r.lo = r.hi = 0;
  return r;
}

// Keys [lo, hi) are seen by every row of [r0, r1).  A tile with others is
// open: in the product over it, a row gets 0 * v of a value v that it does not
// see, which is NaN where v is not finite.  So values that are not finite are
// taken out of open tiles before the product and added to the results of the
// rows that do see them after it.  A block has a few open tiles at most (at
// its own tokens and where its windows begin), however long the sequence is.
struct Edges {
  int lo, hi, len;
  __device__ __forceinline__ bool open(int t) const {
    return t * kTile < lo || min(t * kTile + kTile, len) > hi;
  }
};
__device__ __forceinline__ Edges edges_of_rows(const AttendArgs &g, int base, int len, int r0, int r1) {
  Edges e;
  e.lo = g.window > 0 ? window_start(base + (r1 - 1) / g.group, g.window) : 0;
  e.hi = g.causal ? min(len, base + r0 / g.group + 1) : len;
  e.len = len;
  return e;
}

template <typename T>
__device__ __forceinline__ float4 load4(const char *p) {
  const uint2 v = *reinterpret_cast<const uint2 *>(p);
  const T *h = reinterpret_cast<const T *>(&v);
  return make_float4((float)h[0], (float)h[1], (float)h[2], (float)h[3]);
}
__device__ __forceinline__ bool finite1(float v) { return fabsf(v) <= FLT_MAX; }
__device__ __forceinline__ bool finite4(const float4 &v) {
  return finite1(v.x) && finite1(v.y) && finite1(v.z) && finite1(v.w);
}
// Zeros in the place of what is not finite in a pair; whether there was any.
template <typename T>
__device__ __forceinline__ bool clean_pair(uint32_t &v) {
  constexpr uint32_t kExp = Bits<T>::kBf16 ? 0x7f80u : 0x7c00u;
  const bool lo = (v & kExp) == kExp, hi = (v >> 16 & kExp) == kExp;
  if (lo) v &= 0xffff0000u;
  if (hi) v &= 0x0000ffffu;
  return lo || hi;
}
// Offset in bytes of key j's row in the cache, -1 when its page is bad (then
// it reads as zeros).
__device__ __forceinline__ long long key_offset(const AttendArgs &g, int seq, int hk, int j) {
  const int page = page_of(g.c, seq, j);
  return page < 0 ? -1 : 2 * ((((long long)page * g.c.heads + hk) * g.c.page + (j & (g.c.page - 1))) * g.c.d);
}
// Whether the values there (-1: none) are finite.
template <typename T>
__device__ __forceinline__ bool values_finite(const AttendArgs &g, long long off) {
  bool ok = true;
  if (off >= 0)
    for (int ch = 0; ch < g.c.d; ch += 4) ok &= finite4(load4<T>(static_cast<const char *>(g.c.v) + off + 2 * ch));
  return ok;
}
// The values of the open tiles among [t0, t1) that are not finite, by a warp:
// add(j, bad) for every key j that has any, with zeros for the finite ones
// (four channels a lane, for all lanes together).  Those of keys that every
// row sees are in the results already; once more makes no difference.
template <typename T, typename F>
__device__ __forceinline__ void for_bad_values(const AttendArgs &g, const Edges &e, int seq, int hk, int t0, int t1, F add) {
  const int lane = threadIdx.x & 31;
  for (int t = t0; t < t1; ++t) {
    if (!e.open(t)) continue;
    for (int j0 = t * kTile; j0 < min((t + 1) * kTile, e.len); j0 += 32) {
      const long long off = j0 + lane < e.len ? key_offset(g, seq, hk, j0 + lane) : -1;
      unsigned keys = __ballot_sync(0xffffffffu, !values_finite<T>(g, off));
      while (keys) {
        const int i = __ffs(keys) - 1;
        keys &= keys - 1;
        const long long from = __shfl_sync(0xffffffffu, off, i);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (4 * lane < g.c.d) v = load4<T>(static_cast<const char *>(g.c.v) + from + 8 * lane);
        if (finite1(v.x)) v.x = 0.f;
        if (finite1(v.y)) v.y = 0.f;
        if (finite1(v.z)) v.z = 0.f;
        if (finite1(v.w)) v.w = 0.f;
        add(j0 + i, v);
      }
    }
  }
}
// Adds to four channels of a row of 16-bit or of fp32 results.
template <typename T>
__device__ __forceinline__ void add_to_row(char *row16, float *row32, const float4 &v) {
  const int ch = 4 * (threadIdx.x & 31);
  if (finite4(v)) return;  // zeros
  if (row32) {
    float4 *p = reinterpret_cast<float4 *>(row32 + ch);
    const float4 x = *p;
    *p = make_float4(x.x + v.x, x.y + v.y, x.z + v.z, x.w + v.w);
  } else {
    const float4 x = load4<T>(row16 + 2 * ch);
    *reinterpret_cast<uint2 *>(row16 + 2 * ch) = make_uint2(Bits<T>::pack(x.x + v.x, x.y + v.y), Bits<T>::pack(x.z + v.z, x.w + v.w));
  }
}

// Whether the values of keys [lo, hi) are finite, by a warp.
template <typename T>
__device__ __forceinline__ bool hidden_values_finite(const AttendArgs &g, int seq, int hk, int lo, int hi) {
  bool ok = true;
  for (int j = lo + (int)(threadIdx.x & 31); j < hi; j += 32) ok &= values_finite<T>(g, key_offset(g, seq, hk, j));
  return __all_sync(0xffffffffu, ok);
}
// The product of two pairs, summed.
template <typename T>
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b) {
  const T *x = reinterpret_cast<const T *>(&a), *y = reinterpret_cast<const T *>(&b);
  return (float)x[0] * (float)y[0] + (float)x[1] * (float)y[1];
}
// One row by one warp on the plain cores: the running maximum (powers of two),
// sum and weighted values (four channels a lane) over the keys [lo, hi), 32 at
// a time.  A lane takes the whole score of one key, so that a run of keys
// costs one wait for its pages, keys and values each and one exchange.
template <typename T>
__device__ __forceinline__ float4 row_by_warp(const AttendArgs &g, int seq, int hk, const char *q, int lo, int hi, float &m,
                                           float &l) {
  const int d = g.c.d, lane = threadIdx.x & 31;
  const bool holds = 4 * lane < d;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  const float sc = g.negate ? -g.scale : g.scale;
  m = -INFINITY;
  l = 0.f;
  for (int j0 = lo; j0 < hi; j0 += 32) {
    const int n = min(hi - j0, 32);
    const long long off = lane < n ? key_offset(g, seq, hk, j0 + lane) : -1;
    float s = 0.f;
    for (int c0 = 0; c0 < d; c0 += 64) {
      uint4 k[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        k[i] = make_uint4(0u, 0u, 0u, 0u);
        if (off >= 0 && c0 + 8 * i < d)
          k[i] = *reinterpret_cast<const uint4 *>(static_cast<const char *>(g.c.k) + off + 2 * c0 + 16 * i);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c0 + 8 * i < d) {
          const uint4 x = *reinterpret_cast<const uint4 *>(q + 2 * c0 + 16 * i);
          s += dot2<T>(x.x, k[i].x) + dot2<T>(x.y, k[i].y) + (dot2<T>(x.z, k[i].z) + dot2<T>(x.w, k[i].w));
        }
    }
    s = lane < n ? s * sc : -INFINITY;
    float mn = fmaxf(m, s);
#pragma unroll
    for (int o = 16; o; o >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
    const float f = m == mn ? 1.f : exp2_fast(m - mn), p = s == -INFINITY ? 0.f : exp2_fast(s - mn);
    float sum = p;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    m = mn;
    l = l * f + sum;
    float4 run = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < n; i0 += 16) {
      float4 v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const long long oi = __shfl_sync(0xffffffffu, off, i0 + i);
        v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (oi >= 0 && holds) v[i] = load4<T>(static_cast<const char *>(g.c.v) + oi + 8 * lane);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float pi = __shfl_sync(0xffffffffu, p, i0 + i);
        run.x += pi * v[i].x, run.y += pi * v[i].y, run.z += pi * v[i].z, run.w += pi * v[i].w;
      }
    }
    acc.x = acc.x * f + run.x, acc.y = acc.y * f + run.y, acc.z = acc.z * f + run.z, acc.w = acc.w * f + run.w;
  }
  return acc;
}

__device__ __forceinline__ void flag(const AttendArgs &g, int bit) {
  if (g.err) atomicOr(g.err, bit);
}

// ---------------------------------------------------------------- K and V tiles
// A ring of 128-key tiles (D / 64 halves of 128 rows x 128 bytes, 128-byte
// swizzle), the first kK of them for K, the others for V, each kind filled by
// a warp of its own (positions that both filled in turn would need one warp
// to follow the other's laps: a barrier tells only two phases apart).  A tile
// is loaded page by page, the halves apart; the lanes of the warp issue its
// loads (one warp for both kinds took 3 us a tile of 16-key pages).
// CHECKED: value tiles that are open or hold the sequence's end pass through
// check_values before they are handed on -- values there that are not finite
// (stale memory behind the end may hold NaN) would reach every row of a
// product that reads the tile from shared memory.  Consumers that read the
// tile into registers see to those values themselves.
template <int D, int STAGES, bool CHECKED>
struct TileRing {
  static constexpr int kHalves = D / 64;
  static constexpr uint32_t kBytes = kTile * D * 2;
  static constexpr int kK = (STAGES + 1) / 2;
  uint32_t base, full0, empty0, raw0;
  int kv = 0, stage = 0;  // 0: K, 1: V; position of the next tile
  Range seen;             // keys that some row sees: a bad page is only an error there
  Edges edges;            // CHECKED
  uint32_t phase = 0, filled = 0, parity = 0;

  __device__ __forceinline__ void take(int kind) {
    kv = kind;
    stage = first(kind);
  }
  // The positions of a kind, and the walk over them.
  static __device__ __forceinline__ int first(int kind) { return kind ? kK : 0; }
  static __device__ __forceinline__ void on(int kind, int &st, uint32_t &ph) {
    if (++st == (kind ? STAGES : kK)) {
      st = first(kind);
      ph ^= 1u;
    }
  }
  __device__ __forceinline__ uint32_t full(int s) const { return full0 + 8u * s; }
  __device__ __forceinline__ uint32_t empty(int s) const { return empty0 + 8u * s; }
  __device__ __forceinline__ uint32_t raw(int s) const { return raw0 + 8u * (s - kK); }  // value tiles, before the check
  __device__ __forceinline__ bool checked(int t) const { return edges.open(t) || (t + 1) * kTile > edges.len; }

  // The page id that this lane's part of tile t needs (part: one half of
  // the rows of one page).  Asked for one tile ahead of its load, so that
  // the table's latency is not in the loads' way.
  __device__ __forceinline__ int page_id(const AttendArgs &g, int seq, int len, int t) const {
    const int piece = min(g.c.page, kTile), key = t * kTile + (int)(threadIdx.x & 31) % (kTile / piece) * piece;
    const int i = key >> g.page_log2;
    return key < len && i < g.c.max_pages ? __ldg(g.c.table + (long long)seq * g.c.max_pages + i) : -1;
  }
  // Tile t of the sequence; false when a wait timed out.
  __device__ __forceinline__ bool load(const AttendArgs &g, const CUtensorMap *map, int id, int len, int hk, int t) {
    const int lane = threadIdx.x & 31;
    const int page = g.c.page, piece = min(page, kTile);  // keys of one load
    const int key0 = t * kTile, left = min(len - key0, kTile);
    const int pieces = (left + piece - 1) / piece;
    const int pc = lane % (kTile / piece), half = lane / (kTile / piece);
    const bool mine = pc < pieces && half < kHalves;
    int row = max(1, g.c.pages * g.c.heads * page);  // a row past the cache: reads as zeros
    if (mine) {
      if ((unsigned)id < (unsigned)g.c.pages) row = (id * g.c.heads + hk) * page + ((key0 + pc * piece) & (page - 1));
      else if (key0 + pc * piece < seen.hi && key0 + (pc + 1) * piece > seen.lo) flag(g, TR_CACHE_ERR_PAGE);
    }
    const uint32_t bytes = (uint32_t)pieces * piece * 128u * kHalves;
    if (!tc::mbar_wait_warp(empty(stage), phase ^ 1u)) return false;
    const uint32_t dst = base + stage * kBytes;
    const uint32_t bar = CHECKED && kv == 1 && checked(t) ? raw(stage) : full(stage);
    if (lane == 0) tc::mbar_expect_tx(bar, bytes);
    __syncwarp();
    if (mine) tc::tma_load_2d(dst + half * (kTile * 128) + pc * piece * 128, map, half * 64, row, bar);
    filled |= 1u << stage;
    parity = (parity & ~(1u << stage)) | (phase << stage);
    on(kv, stage, phase);
    return true;
  }
  // The value tiles [t0, t1) that need it, checked by a warp of its own (so
  // that loads go on meanwhile) before their consumers get them: rows past the
  // sequence's end become zeros, and so does, in an open tile, what is not
  // finite of the keys that some row does not see; then *bad is set.  A product
  // with zero tells, the places are looked for only where there are any.  False when
  // a wait timed out.
  template <typename T>
  __device__ __forceinline__ bool check_values(int t0, int t1, int *bad) {
    const int lane = threadIdx.x & 31;
    uint32_t raw_parity = 0;
    take(1);
    for (int t = t0; t < t1; ++t, on(1, stage, phase)) {
      if (!checked(t)) continue;
      if (!tc::mbar_wait_warp(raw(stage), raw_parity >> stage & 1u)) return false;
      raw_parity ^= 1u << stage;
      const uint32_t tile = base + stage * kBytes;
      const int left = min(edges.len - t * kTile, kTile);
      // keys [0, below) are before some row's window, keys [above, left) after some row's own
      const int below = min(max(edges.lo - t * kTile, 0), left), above = max(min(edges.hi - t * kTile, left), below);
#pragma unroll 1
      for (int part = 0; part < 2; ++part) clean_rows<T>(tile, part ? above : 0, part ? left : below, bad);
      for (int i = lane + left * 8; i < kTile * 8; i += 32)
#pragma unroll
        for (int h = 0; h < kHalves; ++h) tc::st_shared_v4(tile + h * (kTile * 128) + i * 16, 0, 0, 0, 0);
      tc::fence_async_shared();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(full(stage));
    }
    return true;
  }
  template <typename T>
  __device__ __forceinline__ void clean_rows(uint32_t tile, int r0, int r1, int *bad) {
    if (r0 >= r1) return;
    const int lane = threadIdx.x & 31;
    uint32_t s0 = 0u, s1 = 0u;
#pragma unroll 2
    for (int i = r0 * 8 + lane; i < r1 * 8; i += 32)
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const uint4 v = tc::ld_shared_v4(tile + h * (kTile * 128) + i * 16);
        s0 = Bits<T>::fma0(v.y, Bits<T>::fma0(v.x, s0)), s1 = Bits<T>::fma0(v.w, Bits<T>::fma0(v.z, s1));
      }
    if (!__any_sync(0xffffffffu, ((s0 | s1) & 0x7fff7fffu) != 0u)) return;
#pragma unroll 1
    for (int h = 0; h < kHalves; ++h)
#pragma unroll 1
      for (int i = r0 * 8 + lane; i < r1 * 8; i += 32) {
        const uint32_t at = tile + h * (kTile * 128) + i * 16;
        uint4 v = tc::ld_shared_v4(at);
        clean_pair<T>(v.x), clean_pair<T>(v.y), clean_pair<T>(v.z), clean_pair<T>(v.w);
        tc::st_shared_v4(at, v.x, v.y, v.z, v.w);
      }
    if (lane == 0) *bad = 1;
  }
  // The loads already issued land before the CTA may exit.
  __device__ __forceinline__ void drain() const {
    for (int s = 0; s < STAGES; ++s)
      if (filled >> s & 1u) tc::mbar_wait_warp(full(s), parity >> s & 1u);
  }
};

// ---------------------------------------------------------------- chunks (tr_attend.cu, tr_attend8.cu)
__device__ __forceinline__ float max3(float a, uint32_t b, uint32_t c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
  return r;
}

// The block of tokens that belong to no sequence (first: their first) in this
// slot: zeros, lse -inf.
inline __device__ __noinline__ void clear_block(const AttendArgs &g, int first, int slot, int rows_per_block, int hk) {
  const int rows = (g.c.total_new - first) * g.group;
  const int block = slot - ((int)((long long)first * g.group / rows_per_block) + g.c.batch);
  if (block < 0) return;  // an empty slot of the last sequence
  const int r0 = block * rows_per_block, chunks = g.c.d / 8;
  for (int i = threadIdx.x; i < min(rows - r0, rows_per_block) * chunks; i += blockDim.x) {
    const int r = r0 + i / chunks, c = i % chunks;
    const long long t = first + r / g.group;
    const int head = hk * g.group + r % g.group;
    *reinterpret_cast<uint4 *>(g.o + 2 * (t * g.o_tok + (long long)head * g.o_head) + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
    if (c == 0 && g.lse) g.lse[t * g.q_heads + head] = -INFINITY;
  }
}

constexpr float kFar = 0x1p-126f;

// Joins the splits of each row: one warp per row, in the splits' order.
// NORMED: the splits' values are divided by their sums.
template <typename T, bool NORMED>
__global__ void __launch_bounds__(128) k_attend_join(const __grid_constant__ AttendArgs g) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long rows = (long long)g.c.total_new * g.q_heads;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const int t = (int)(row / g.q_heads), h = (int)(row - (long long)t * g.q_heads);
  char *orow = g.o + 2 * ((long long)t * g.o_tok + (long long)h * g.o_head);
  const bool holds = 4 * lane < g.c.d;
  float m = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (find_token(g.c, t).seq >= 0) {
    for (int s = 0; s < g.splits; ++s) m = fmaxf(m, g.part_ml[s * rows + row].x);
    for (int s = 0; s < g.splits; ++s) {
      const float2 ml = g.part_ml[s * rows + row];
      if (ml.y == 0.f) continue;  // saw no key
      const float f = exp2_fast(ml.x - m);
      l += ml.y * f;
      if (!NORMED && holds) {
        const float4 v = reinterpret_cast<const float4 *>(g.part + (s * rows + row) * g.c.d)[lane];
        acc.x += v.x * f, acc.y += v.y * f, acc.z += v.z * f, acc.w += v.w * f;
      }
    }
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  if (NORMED) {
    // weighed by their shares of the sum, 1 at most, so that values near the end of fp32 stay below it; shares under
    // 2^-126 in two factors, of which kFar is one: a value may outweigh its small probability
    for (int s = 0; l != 0.f && s < g.splits; ++s) {
      const float2 ml = g.part_ml[s * rows + row];
      if (ml.y == 0.f || !holds) continue;
      float4 v = reinterpret_cast<const float4 *>(g.part + (s * rows + row) * g.c.d)[lane];
      const bool far = ml.x - m < -126.f;
      if (far) v.x *= kFar, v.y *= kFar, v.z *= kFar, v.w *= kFar;
      const float w = ml.y * exp2_fast(far ? ml.x - m + 126.f : ml.x - m) * inv;
      acc.x += v.x * w, acc.y += v.y * w, acc.z += v.z * w, acc.w += v.w * w;
    }
  } else {
    acc.x *= inv, acc.y *= inv, acc.z *= inv, acc.w *= inv;
  }
  if (holds)
    reinterpret_cast<uint2 *>(orow)[lane] =
        make_uint2(Bits<T>::pack(acc.x, acc.y), Bits<T>::pack(acc.z, acc.w));
  if (g.lse && lane == 0) g.lse[row] = l > 0.f || l != l ? m * 0.693147180559945309f + logf(l) : -INFINITY;
}

// ---------------------------------------------------------------- few rows (tr_attend_few.cu)
constexpr int kFewRows = 16;         // rows of a block there
constexpr int kFewItemCost = 2;      // units that an item counts besides its tiles
constexpr int kFewMaxBatch = 8192;   // sequences its unit count handles
// Whether that kernel takes a call: its units, tiles of all blocks and key
// heads, are counted in 31 bits.
inline bool few_takes(const tr_cache *c, int q_heads, int max_new, int item_cost = kFewItemCost, int rows = kFewRows) {
  const int group = q_heads / c->heads;
  const long long most = (long long)(max_new < c->total_new ? max_new : c->total_new) * group;
  const long long blocks16 = (long long)c->total_new * group / kFewRows + c->batch;
  const long long table_tiles = ((long long)c->max_pages * c->page + kTile - 1) / kTile + item_cost;
  return most <= rows && c->batch <= kFewMaxBatch && blocks16 * c->heads <= INT_MAX / table_tiles;
}
// Workspace bytes, and the launch (work and join kernels); g.part and
// g.part_ml are carved from ws by the launch.
size_t few_workspace_bytes(int d, int ctas);
cudaError_t launch_few(const CUtensorMap &mk, const CUtensorMap &mv, AttendArgs g, bool bf16, void *ws, cudaStream_t st);

}  // namespace attend
}  // namespace tr
