// What the attention kernels share: their arguments, the rows and keys of a
// block, the loads of K and V tiles, and the slow exact path of one row.
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
};
template <>
struct Bits<__half> {
  static constexpr bool kBf16 = false;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
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

// One row by one warp on the plain cores, four channels a lane: the running
// maximum (powers of two), sum and weighted values over the keys [lo, hi).
template <typename T>
__device__ __forceinline__ float4 load4(const char *p) {
  const uint2 v = *reinterpret_cast<const uint2 *>(p);
  const T *h = reinterpret_cast<const T *>(&v);
  return make_float4((float)h[0], (float)h[1], (float)h[2], (float)h[3]);
}
__device__ __forceinline__ bool finite4(const float4 &v) {
  return fabsf(v.x) <= FLT_MAX && fabsf(v.y) <= FLT_MAX && fabsf(v.z) <= FLT_MAX && fabsf(v.w) <= FLT_MAX;
}
template <typename T>
__device__ __forceinline__ bool hidden_values_finite(const AttendArgs &g, int seq, int hk, int lo, int hi) {
  const int ch = 4 * (threadIdx.x & 31);
  bool ok = true;
  for (int j = lo; j < hi; ++j) {
    const int page = page_of(g.c, seq, j);
    if (page >= 0 && ch < g.c.d)
      ok &= finite4(load4<T>(static_cast<const char *>(g.c.v) +
                             2 * ((((long long)page * g.c.heads + hk) * g.c.page + (j & (g.c.page - 1))) * g.c.d + ch)));
  }
  return __all_sync(0xffffffffu, ok);
}
template <typename T>
__device__ __forceinline__ float4 row_by_warp(const AttendArgs &g, int seq, int hk, const char *q, int lo, int hi, float &m,
                                           float &l) {
  const int d = g.c.d, ch = 4 * (threadIdx.x & 31);
  const bool holds = ch < d;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f), acc = x;
  if (holds) x = load4<T>(q + 2 * ch);
  const float sc = g.negate ? -g.scale : g.scale;
  m = -INFINITY;
  l = 0.f;
  for (int j = lo; j < hi; ++j) {
    const int page = page_of(g.c, seq, j);
    float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
    if (page >= 0 && holds) {
      const long long off = 2 * ((((long long)page * g.c.heads + hk) * g.c.page + (j & (g.c.page - 1))) * d + ch);
      k = load4<T>(static_cast<const char *>(g.c.k) + off);
      v = load4<T>(static_cast<const char *>(g.c.v) + off);
    }
    float s = x.x * k.x + x.y * k.y + x.z * k.z + x.w * k.w;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    s *= sc;
    const float mn = fmaxf(m, s);
    const float f = m == mn ? 1.f : exp2_fast(m - mn), p = s == -INFINITY ? 0.f : exp2_fast(s - mn);
    m = mn;
    l = l * f + p;
    acc.x = acc.x * f + p * v.x;
    acc.y = acc.y * f + p * v.y;
    acc.z = acc.z * f + p * v.z;
    acc.w = acc.w * f + p * v.w;
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
// ZERO_TAIL: value rows past the sequence's end are zeroed before the tile is
// handed on -- stale memory may hold NaN there, and 0 * NaN would reach every
// row of a product that reads the tile from shared memory.  That waits for
// the tile, so it suits a CTA that ends with it; consumers that read the
// tile into registers drop those rows themselves.
template <int D, int STAGES, bool ZERO_TAIL>
struct TileRing {
  static constexpr int kHalves = D / 64;
  static constexpr uint32_t kBytes = kTile * D * 2;
  static constexpr int kK = (STAGES + 1) / 2;
  uint32_t base, full0, empty0, tail;
  int kv = 0, stage = 0;  // 0: K, 1: V; position of the next tile
  Range seen;             // keys that some row sees: a bad page is only an error there
  uint32_t phase = 0, tails = 0, filled = 0, parity = 0;

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
    const bool cut = ZERO_TAIL && kv == 1 && left < kTile;  // the sequence ends inside this value tile
    const uint32_t bar = cut ? tail : full(stage);
    if (lane == 0) tc::mbar_expect_tx(bar, bytes);
    __syncwarp();
    if (mine) tc::tma_load_2d(dst + half * (kTile * 128) + pc * piece * 128, map, half * 64, row, bar);
    bool ok = true;
    if (cut) {
      ok = __all_sync(0xffffffffu, tc::mbar_wait(tail, tails));
      tails ^= 1u;
      for (int i = lane + left * 8; i < kTile * 8; i += 32)
#pragma unroll
        for (int h = 0; h < kHalves; ++h) tc::st_shared_v4(dst + h * (kTile * 128) + i * 16, 0, 0, 0, 0);
      tc::fence_async_shared();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(full(stage));
    }
    filled |= 1u << stage;
    parity = (parity & ~(1u << stage)) | (phase << stage);
    on(kv, stage, phase);
    return ok;
  }
  // The loads already issued land before the CTA may exit.
  __device__ __forceinline__ void drain() const {
    for (int s = 0; s < STAGES; ++s)
      if (filled >> s & 1u) tc::mbar_wait_warp(full(s), parity >> s & 1u);
  }
};

// ---------------------------------------------------------------- few rows (tr_attend_few.cu)
constexpr int kFewRows = 16;         // rows of a block there
constexpr int kFewItemCost = 2;      // units that an item counts besides its tiles
constexpr int kFewMaxBatch = 8192;   // sequences its unit count handles
// Workspace bytes, and the launch (work and join kernels); g.part and
// g.part_ml are carved from ws by the launch.
size_t few_workspace_bytes(int d, int ctas);
cudaError_t launch_few(const CUtensorMap &mk, const CUtensorMap &mv, AttendArgs g, bool bf16, void *ws, cudaStream_t st);

}  // namespace attend
}  // namespace tr
