// What the attention kernels over the 8-bit cache share: their arguments, the
// loads of tiles of codes, codes that stand for no number.
#pragma once

#include "tr_attend.cuh"
#include "tr_cache8.cuh"

namespace tr {
namespace attend8 {

using namespace attend;
using namespace cache8;

struct Attend8Args {
  AttendArgs a;
  Scales scale;
};

// ---------------------------------------------------------------- codes that stand for no number
// Zeros in the place of NaN among four codes; whether there was any.
__device__ __forceinline__ bool clean_codes(uint32_t &w) {
  const uint32_t bad = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;  // a byte of 0x7f carries
  if (!bad) return false;
  w &= ~((bad >> 7) * 0xffu);
  return true;
}
__device__ __forceinline__ bool has_bad_codes(const uint4 &v) {
  uint32_t bad = 0u;
  bad |= (v.x & 0x7f7f7f7fu) + 0x01010101u;
  bad |= (v.y & 0x7f7f7f7fu) + 0x01010101u;
  bad |= (v.z & 0x7f7f7f7fu) + 0x01010101u;
  bad |= (v.w & 0x7f7f7f7fu) + 0x01010101u;
  return (bad & 0x80808080u) != 0u;
}
// As for_bad_values: the values of the open tiles among [t0, t1) that are no
// numbers, by a warp: add(j, bad) for every key j that has any, with zeros for
// the others (four channels a lane).
template <typename F>
__device__ __forceinline__ void for_bad_codes(const AttendArgs &g, const Edges &e, int seq, int hk, int t0, int t1, F add) {
  const int lane = threadIdx.x & 31;
  const uint8_t *codes = static_cast<const uint8_t *>(g.c.v);
  for (int t = t0; t < t1; ++t) {
    if (!e.open(t)) continue;
    for (int j0 = t * kTile; j0 < min((t + 1) * kTile, e.len); j0 += 32) {
      long long off = j0 + lane < e.len ? key_offset(g, seq, hk, j0 + lane) : -1;
      if (off >= 0) off /= 2;  // (codes: a byte each)
      bool bad = false;
      if (off >= 0)
        for (int ch = 0; ch < g.c.d; ch += 16) bad |= has_bad_codes(*reinterpret_cast<const uint4 *>(codes + off + ch));
      unsigned keys = __ballot_sync(0xffffffffu, bad);
      while (keys) {
        const int i = __ffs(keys) - 1;
        keys &= keys - 1;
        const long long from = __shfl_sync(0xffffffffu, off, i);
        const uint32_t w = 4 * lane < g.c.d ? *reinterpret_cast<const uint32_t *>(codes + from + 4 * lane) : 0u;
        const float nan = __int_as_float(0x7fc00000);
        add(j0 + i, make_float4((w & 0x7fu) == 0x7fu ? nan : 0.f, (w >> 8 & 0x7fu) == 0x7fu ? nan : 0.f,
                                (w >> 16 & 0x7fu) == 0x7fu ? nan : 0.f, (w >> 24 & 0x7fu) == 0x7fu ? nan : 0.f));
      }
    }
  }
}

// ---------------------------------------------------------------- tiles of codes
// A ring of tiles of 128 keys, D bytes a key (64- or 128-byte swizzle: a
// row's 16-byte pieces change places by its number), the first kK for K, the
// others for V, as TileRing: each kind filled by a warp of its own.
template <int D, int STAGES>
struct CodeRing {
  static_assert(D == 64 || D == 128, "");
  static constexpr uint32_t kBytes = kTile * D;
  static constexpr int kK = (STAGES + 1) / 2;
  uint32_t base, full0, empty0;
  int kv = 0, stage = 0;
  Range seen;
  uint32_t phase = 0, filled = 0, parity = 0;

  static __device__ __forceinline__ int first(int kind) { return kind ? kK : 0; }
  static __device__ __forceinline__ void on(int kind, int &st, uint32_t &ph) {
    if (++st == (kind ? STAGES : kK)) {
      st = first(kind);
      ph ^= 1u;
    }
  }
  // Byte offset of 16-byte piece c of row r in a tile.
  static __device__ __forceinline__ uint32_t piece(int r, int c) {
    return (uint32_t)(r * D + ((c ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4));
  }
  __device__ __forceinline__ void take(int kind) {
    kv = kind;
    stage = first(kind);
  }
  __device__ __forceinline__ uint32_t full(int s) const { return full0 + 8u * s; }
  __device__ __forceinline__ uint32_t empty(int s) const { return empty0 + 8u * s; }

  // The page id that this lane's part of tile t needs (part: the rows of one
  // page), asked for one tile ahead of its load.
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
    const bool mine = lane < pieces;
    int row = max(1, g.c.pages * g.c.heads * page);  // a row past the cache: reads as zeros
    if (mine) {
      if ((unsigned)id < (unsigned)g.c.pages) row = (id * g.c.heads + hk) * page + ((key0 + lane * piece) & (page - 1));
      else if (key0 + lane * piece < seen.hi && key0 + (lane + 1) * piece > seen.lo) flag(g, TR_CACHE_ERR_PAGE);
    }
    if (!tc::mbar_wait_warp(empty(stage), phase ^ 1u)) return false;
    if (lane == 0) tc::mbar_expect_tx(full(stage), (uint32_t)pieces * piece * D);
    __syncwarp();
    if (mine) tc::tma_load_2d(base + stage * kBytes + lane * piece * D, map, 0, row, full(stage));
    filled |= 1u << stage;
    parity = (parity & ~(1u << stage)) | (phase << stage);
    on(kv, stage, phase);
    return true;
  }
  // The loads already issued land before the CTA may exit.
  __device__ __forceinline__ void drain() const {
    for (int s = 0; s < STAGES; ++s)
      if (filled >> s & 1u) tc::mbar_wait_warp(full(s), parity >> s & 1u);
  }
};

// The scales of key block j / 16 of the sequence, as held: keys' (low byte) and
// values'; kNoScales where there is no such block (its keys read as zeros).
constexpr uint32_t kNoScales = 0xff7fu;
__device__ __forceinline__ uint32_t scales_at(const Attend8Args &p, long long i) {
  return (uint32_t)min((int)__ldg(p.scale.k + i), 254) | (uint32_t)min((int)__ldg(p.scale.v + i), 254) << 8;
}
__device__ __forceinline__ uint32_t block_scales(const Attend8Args &p, int seq, int hk, int len, int j) {
  const AttendArgs &g = p.a;
  const int i = j >> g.page_log2;
  const int page = j < len && i < g.c.max_pages ? __ldg(g.c.table + (long long)seq * g.c.max_pages + i) : -1;
  return (unsigned)page < (unsigned)g.c.pages ? scales_at(p, scale_at(g.c, page, hk, j & (g.c.page - 1))) : kNoScales;
}

// A query's numbers as halves: fp16 as they are; bf16 times a power of two
// that brings the row's largest finite magnitude to [2^14, 2^15), so that what
// is left of them below is 2^-40 of it.  Returns the exponent of what it was
// divided by.
__device__ __forceinline__ int query_exp(uint32_t top) { return max((int)(top >> 23) - 127 - 14, -113); }
__device__ __forceinline__ uint32_t query_pair(uint32_t bf16x2, float f) {
  return Bits<__half>::pack(__uint_as_float(bf16x2 << 16) * f, __uint_as_float(bf16x2 & 0xffff0000u) * f);
}
// The largest finite magnitude of a pair, as fp32 bits.
__device__ __forceinline__ uint32_t top_of_pair(uint32_t bf16x2) {
  const uint32_t lo = bf16x2 << 16 & 0x7fffffffu, hi = bf16x2 & 0x7fff0000u;
  return max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u);
}

// What a block's products are multiplied by to become scores, in units of log 2:
// within bounds, so that -inf and 0 times it stay what they are.  A product that
// is not zero is 2^-33 at least and 2^31 at most, so beyond the bounds a score
// would be 2^66 and more, where none is defined, or under 2^-68: zero to the
// exponential.
__device__ __forceinline__ float block_factor(float row, float key) { return fminf(fmaxf(row * key, 1e-30f), 1e30f); }

constexpr int kItemCost = 5;  // few rows: an item's own cost in tiles (see units_of); 3 and 7: 61.4 and 61.2 us against 59.3 for 64 requests' tokens
// Rows that go there: 32 in two blocks, the second's keys from L2, where there
// are more than 8 tiles (21 rows of 64 sequences over 255 to 16000 keys 104 us,
// by chunks 156; 32 of one over 20000 keys 23 and 30; 28 of 32 over 1000 to
// 12000 keys 63 and 65, but over 16384 each 188 and 183; 32 of 64 over 100 to
// 300 keys 37 and 26).
constexpr int kMostFew = 32, kMinTilesFew = 9;
// Few rows (tr_attend8_few.cu): the launch (work and join kernels).
cudaError_t launch_few8(const CUtensorMap &mk, const CUtensorMap &mv, Attend8Args p, bool bf16, void *ws, cudaStream_t st);

}  // namespace attend8
}  // namespace tr
