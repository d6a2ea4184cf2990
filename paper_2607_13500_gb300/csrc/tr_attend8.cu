// Attention of new tokens over the paged cache held in 8 bits
// (tr_cache8_attend) on the 5th-generation tensor cores:
//   o = sum_j p_j v_j,  p = softmax over the visible keys of scale q . k_j,
//   k_j = c_j 2^e(j) and v_j alike, with e4m3 codes c and an exponent e for each
//   16 keys.
//
// The products take both operands in one type, and four bits of mantissa are
// too few for queries and probabilities, so codes become halves on their way:
// rows, products and softmax are those of tr_attend.cu, and between the TMA
// loads and the products stand four warps that turn a tile of codes in shared
// memory into a tile of halves, exactly, an instruction for two values.  They
// also put zeros in the place of the keys past the sequence's end and of codes
// that are no numbers in tiles that some row does not see all of (Edges in
// tr_attend.cuh).  bf16 queries enter as halves, each row divided by a power of
// two.
//
// The scales enter in the softmax, where they cost eight numbers a row and
// tile (a product of halves for each pair of codes, in the warps that turn
// them, took longer than the tile's products: 2048 tokens over 32768 keys 758
// us, here 701):
//   keys    a factor of the block's 16 scores;
//   values  d = e - R, R one exponent of the CTA's, is added to the block's 16
//           scores, and the softmax's maximum is that of these sums: what
//           enters the second product is p 2^d.  R enters the results, and the
//           sum of the p is taken block by block, times 2^-d (kLeast says how
//           far the d may lie apart for that, and what is done beyond).
// So what enters the second product, 2^14 at most, is rounded to halves: it
// keeps its bits down to 2^-20 of what the row's greatest key adds, and what is
// lost below is 2^-31 of it.  Sums and everything else are fp32.
//
// Two blocks of 128 rows share a turned tile (MT = 2); where the rows are few
// enough for one, a CTA is one block with two score buffers.  A tile of MT = 2
// takes 3700 clocks: its codes are read (32 KB), written as halves (64 KB) and
// read by each block's products (112 KB a block), 320 KB at some 90 B a clock,
// and the chain of a block's scores, softmax and second product has one score
// buffer (with heads of 64 channels, half the bytes, a tile takes 0.86 of it).
//
// 28 heads of 128 over 4: 2048 tokens over 32768 keys 700 us (1.33 PFLOP/s, 0.70
// of the measured cuBLAS); 5 tokens of 32 sequences over 1000 to 12000 keys (35
// rows a key head, MT = 1) 67 us; chunks of 784 tokens of 4 sequences over 1000
// to 6272 keys, in fp16, 84 us, where each CTA's start and end, 11 us, tell.
#include <atomic>
#include <cmath>

#include "tr_attend8.cuh"
#include "tr_pack.cuh"

namespace tr {
namespace {

using namespace attend8;

template <int D, int MT>
struct Shape8 {
  static_assert(MT == 2 || MT == 1, "");
  static constexpr int kTileBytes = kTile * D * 2;   // one K or V tile of halves, or one block's Q
  static constexpr int kCodeBytes = kTile * D;       // one tile of codes
  static constexpr int kBudget = 224 * 1024;          // shared memory less barriers and alignment
  static constexpr int kFit = (kBudget - (MT + 4) * kTileBytes) / kCodeBytes;
  static constexpr int kStages = kFit < 12 ? kFit : 12;  // of codes; two tiles of halves of each kind
  static constexpr int kSBuf = MT == 1 ? 2 : 1;      // score buffers of a block
  // Warpgroups: softmax (MT), loads and products, codes to halves.  Registers
  // move to the softmax, where a thread holds a row of scores (128): of 128 at
  // launch (MT = 2) 200 and 56 for the rest, of 168 (MT = 1) 216 and 144.
  static constexpr int kThreads = 128 * (MT + 2);
  static constexpr int kColO = 256;  // tensor-memory columns: scores below, sums from here
  static constexpr int kCols = 512;
  static constexpr size_t kSmem = (size_t)(MT + 4) * kTileBytes + (size_t)kStages * kCodeBytes + 1024 + 512;
  static_assert(kStages >= 2 && kSmem <= 227 * 1024, "");
  static_assert(kColO + MT * D <= kCols && kColO >= MT * kSBuf * kTile, "scores and sums fit the tensor memory");
};

constexpr float kLift8 = 6.f;   // probabilities are taken times 2^6 (and grow by 2^8 at most)
// R is the largest exponent of the CTA's blocks, and the sum's way through 2^-d
// holds for kLeast <= d <= 0: a probability that leaves the exponential as zero,
// because it is 2^-132 of the greatest times its 2^d, is then 2^-52 of another
// at most, and the sums, up to 2^94 a key, are fp32 numbers.  Where the exponents
// lie further apart (but for blocks of zeros: a wide CTA) the sum is taken from
// exponentials of its own, against the maximum of the scores alone
// (softmax_wide: 2048 tokens over 32768 keys 1820 us, else 700).
constexpr int kLeast = -80;
constexpr int kZeros = -117;  // the exponent of a block of zeros, as the append leaves it; but it may hold small values too

// What the softmax needs of a tile's blocks.
struct TileScales {
  float k[8];     // 2^e of keys
  float v[8];     // d of values
  float undo[8];  // 2^-d (wide CTAs: none)
};

// The values taken out of open tiles among [t0, t1) to those rows of the warp
// that see them.  (Not inline: it would cost the softmax registers.)
template <typename T>
__device__ __noinline__ void put_back8(const AttendArgs &g, int seq, int tok0, int base, int len, int rows, int first, int block,
                                       int hk, int split, int warp, int t0, int t1) {
  const Edges e = edges_of_rows(g, base, len, first, min(first + block, rows));
  for_bad_codes(g, e, seq, hk, t0, t1, [&](int j, const float4 &v) {
    for (int r = first + 32 * warp; r < min(first + 32 * warp + 32, rows); ++r) {
      const int tok = r / g.group, head = hk * g.group + r % g.group, own = base + tok;
      if ((g.causal && j > own) || (g.window > 0 && j < window_start(own, g.window))) continue;
      const long long t = tok0 + tok;
      add_to_row<T>(g.o + 2 * (t * g.o_tok + (long long)head * g.o_head),
                    g.splits > 1 ? g.part + (((long long)split * g.c.total_new + t) * g.q_heads + head) * g.c.d : nullptr, v);
    }
  });
}

__device__ __forceinline__ void rows_sync(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }
__device__ __forceinline__ void rows_arrive(int threads) { asm volatile("bar.arrive 1, %0;" ::"r"(threads) : "memory"); }
// The warps that turn codes into halves.
__device__ __forceinline__ void codes_sync() { asm volatile("bar.sync 2, 128;" ::: "memory"); }

// Codes to halves: 32 rows (from row0, a multiple of 32) of a tile by a warp;
// rows from `left` on become zeros; CLEAN: so do codes that are no numbers.  Returns whether there
// were any.
// The eight lanes of a phase of shared memory take the same half of rows r and
// r ^ 5: their 16-byte pieces lie in different banks on both sides.
// AT_ONCE pieces are loaded before any is turned.
template <int D, bool CLEAN, int AT_ONCE>
__device__ __forceinline__ bool to_halves(uint32_t codes, uint32_t tile, int row0, int left) {
  const int lane = threadIdx.x & 31;
  bool found = false;
  constexpr int kSteps = D / 16;  // of 4 (D = 128) or 8 rows
  static_assert(kSteps % AT_ONCE == 0, "");
  auto place = [&](int i, int &r, int &c) {
    if (D == 128) {
      const int x = 2 * (i & 1) + (lane >> 3 & 1);
      r = row0 + 8 * (i >> 1) + (lane & 4 ? x ^ 5 : x);
      c = (lane & 3) | (lane >> 4) << 2;
    } else {
      r = row0 + 8 * i + (lane >> 2);
      c = lane & 3;
    }
  };
#pragma unroll
  for (int i0 = 0; i0 < kSteps; i0 += AT_ONCE) {
    uint4 v[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      int r, c;
      place(i0 + i, r, c);
      v[i] = tc::ld_shared_v4(codes + CodeRing<D, 2>::piece(r, c));
    }
    if (row0 + 32 > left)
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        int r, c;
        place(i0 + i, r, c);
        if (r >= left) v[i] = make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      int r, c;
      place(i0 + i, r, c);
      if (CLEAN) found |= clean_codes(v[i].x) | clean_codes(v[i].y) | clean_codes(v[i].z) | clean_codes(v[i].w);
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      uint32_t h[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) halves4(w[k], h[2 * k], h[2 * k + 1]);
      const uint32_t at = tile + (c >> 2) * (kTile * 128) + r * 128;
      const int chunk = 2 * (c & 3), flip = r & 7;
      tc::st_shared_v4(at + ((chunk ^ flip) << 4), h[0], h[1], h[2], h[3]);
      tc::st_shared_v4(at + (((chunk + 1) ^ flip) << 4), h[4], h[5], h[6], h[7]);
    }
  }
  return found;
}

// Whether some of the key blocks from, from + 128, .. (a warp's 32 each time)
// whose exponent is kZeros or less hold anything but zeros, by a warp.  (With
// every second page of 32768 keys zeros, 2048 tokens take 962 us, without zeros
// 700; taking them for small values, as a wide CTA, would be 1820.)
__device__ __noinline__ bool holds_small_values(const Attend8Args &p, int seq, int hk, int len, int from, int blocks) {
  const AttendArgs &g = p.a;
  const uint8_t *codes = static_cast<const uint8_t *>(g.c.v);
  for (int i0 = from; i0 < blocks; i0 += 128) {
    const int i = i0 + (int)(threadIdx.x & 31);
    const uint32_t s = i < blocks ? block_scales(p, seq, hk, len, kBlock * i) : kNoScales;
    uint32_t any = 0u;
    if (s != kNoScales && (int)(s >> 8) - 127 <= kZeros) {
      // (the rows of a block lie one after the other)
      const uint4 *v = reinterpret_cast<const uint4 *>(codes + key_offset(g, seq, hk, kBlock * i) / 2);
      const int n = min(len - kBlock * i, kBlock) * (g.c.d / 16);
#pragma unroll 8
      for (int j = 0; j < n; ++j) any |= v[j].x | v[j].y | v[j].z | v[j].w;
    }
    if (__any_sync(0xffffffffu, (any & 0x7f7f7f7fu) != 0u)) return true;
  }
  return false;
}

// The softmax of a row's tiles in a wide CTA (see kLeast), by the warps of a
// block, as in k_attend8 but for the sum and for maxima that are whole numbers,
// so that their difference is exact.  It stands by itself, 32 scores at a time,
// because the same in the loop there took registers and order from the others
// (long 703 -> 757 us; as a second loop beside it drafts 66 -> 70).  False when a
// wait timed out.
struct WideRow {
  uint32_t s_col, o_col;            // tensor memory: scores (the first buffer's) and sums
  uint32_t s_full, p_full, o_done;  // barriers (the first buffer's)
  uint32_t scale_full, scales;      // barriers and numbers of the tiles' scales, four slots
  int t0, ta, tb, lo, hi;           // first tile of the CTA; tiles of the block; keys of the row
  float row_scale;
  float mx, top, sum;               // maxima of scores + d and of scores; the sum, against top
  bool live;
};
template <int D, int BUFS>
__device__ __noinline__ bool softmax_wide(WideRow &row) {
  WideRow w = row;  // (in registers: 4800 us without)
  bool ok = true;
  for (int t = w.ta; t < w.tb; ++t) {
    const int n = t - w.ta, ts = t - w.t0, buf = BUFS == 2 ? n & 1 : 0;
    const uint32_t par = BUFS == 2 ? (uint32_t)(n >> 1) & 1u : (uint32_t)n & 1u;
    if (!__all_sync(0xffffffffu, tc::mbar_wait(w.s_full + 8u * buf, par) &&
                                     tc::mbar_wait(w.scale_full + 8u * (ts & 3), (uint32_t)(ts >> 2) & 1u))) {
      ok = false;
      break;
    }
    tc::fence_after_sync();
    if (w.live) {
      const uint32_t s_col = w.s_col + buf * kTile, at = w.scales + (ts & 3) * (uint32_t)sizeof(TileScales);
      // scores 32 c and on, in units of log 2 (-inf: not seen); their blocks' d
      auto load = [&](int c, float (&s)[32], float (&d)[2]) {
        uint32_t x[32];
        tc::tmem_ld32_issue(s_col + 32 * c, x);
        tc::tmem_ld32_wait(x);
        float f[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f[b]) : "r"(at + 4 * (2 * c + b)));
          asm volatile("ld.shared.f32 %0, [%1];" : "=f"(d[b]) : "r"(at + 32 + 4 * (2 * c + b)));
          f[b] = block_factor(w.row_scale, f[b]);
        }
        const int key0 = t * kTile + 32 * c;
#pragma unroll
        for (int i = 0; i < 32; ++i)
          s[i] = key0 + i < w.lo || key0 + i >= w.hi ? -INFINITY : __uint_as_float(x[i]) * f[i / 16];
      };
      float now = -INFINITY, peak = -INFINITY;
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        float s[32], d[2];
        load(c, s, d);
#pragma unroll
        for (int i = 0; i < 32; ++i) peak = fmaxf(peak, s[i]), now = fmaxf(now, s[i] + d[i / 16]);
      }
      now = ceilf(now), peak = ceilf(peak);
      if (peak > w.top) w.sum *= exp2_fast(w.top - peak), w.top = peak;
      if (n == 0) {
        w.mx = now;
      } else if (__any_sync(0xffffffffu, now > w.mx + 8.f)) {  // the products so far move to the new maximum
        const bool more = now > w.mx + 8.f;
        const float down = more ? exp2_fast(w.mx - now) : 1.f;
        if (BUFS == 2) {
          if (!__all_sync(0xffffffffu, tc::mbar_wait(w.o_done, (uint32_t)(n - 1) & 1u))) {
            ok = false;
            break;
          }
          tc::fence_after_sync();
        }
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          tc::tmem_ld32_issue(w.o_col + c, o);
          tc::tmem_ld32_wait(o);
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * down);
          tc::tmem_st32(w.o_col + c, o);
        }
        tc::tmem_st_wait();
        if (more) w.mx = now;
      }
      const float less = w.top == -INFINITY ? 0.f : -w.top, neg = w.mx == -INFINITY ? 0.f : kLift8 - w.mx;
      // (probabilities of 64 keys take the 32 columns whose scores were read first)
#pragma unroll 1
      for (int c = 0; c < 4; c += 2) {
        uint32_t p[32];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float s[32], d[2];
          load(c + h, s, d);
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            acc[i / 2 & 3] += exp2_fast(s[i] + less) + exp2_fast(s[i + 1] + less);
            const float e = neg + d[i / 16];
            p[16 * h + i / 2] = Bits<__half>::pack(exp2_fast(s[i] + e), exp2_fast(s[i + 1] + e));
          }
          w.sum += (acc[0] + acc[1]) + (acc[2] + acc[3]);
        }
        tc::tmem_st32(s_col + 16 * c, p);
      }
      tc::tmem_st_wait();
    }
    tc::fence_before_sync();
    tc::mbar_arrive(w.p_full + 8u * buf);
  }
  row = w;
  return ok;
}

template <typename T, int D, int MT>
__global__ void __launch_bounds__(Shape8<D, MT>::kThreads, 1)
    k_attend8(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
              const __grid_constant__ Attend8Args p) {
  using S = Shape8<D, MT>;
  using Ring = CodeRing<D, S::kStages>;
  constexpr int kRows = kTile * MT;
  const AttendArgs &g = p.a;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t sbase = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;  // the swizzle atom
  const uint32_t k16 = sbase + MT * S::kTileBytes, v16 = k16 + 2 * S::kTileBytes, ring = v16 + 2 * S::kTileBytes;
  const uint32_t bars = ring + S::kStages * S::kCodeBytes;
  auto code_full = [&](int s) { return bars + 8u * s; };
  auto code_empty = [&](int s) { return bars + 8u * (S::kStages + s); };
  const uint32_t half_bars = bars + 16u * S::kStages;
  auto half_full = [&](int kind, int s) { return half_bars + 8u * (2 * kind + s); };
  auto half_empty = [&](int kind, int s) { return half_bars + 8u * (4 + 2 * kind + s); };
  const uint32_t row_bars = half_bars + 64u;
  auto q_full = [&](int m) { return row_bars + 8u * m; };
  auto s_full = [&](int m, int b) { return row_bars + 8u * (MT + m * S::kSBuf + b); };
  auto p_full = [&](int m, int b) { return row_bars + 8u * (MT + MT * S::kSBuf + m * S::kSBuf + b); };
  auto o_done = [&](int m) { return row_bars + 8u * (MT + 2 * MT * S::kSBuf + m); };
  auto o_last = [&](int m) { return row_bars + 8u * (2 * MT + 2 * MT * S::kSBuf + m); };
  const uint32_t scale_bars = row_bars + 8u * (3 * MT + 2 * MT * S::kSBuf);
  auto scale_full = [&](int s) { return scale_bars + 8u * s; };
  const uint32_t tmem_slot = scale_bars + 32u;
  __shared__ int bad_values;     // some were taken out of the tiles
  __shared__ int top_of[4], low_of[4], tiny_of[4], ref, wide_sum;  // largest and smallest exponents, R, whether they lie far apart
  __shared__ bool small_of[4];
  // Of tile t in slot t % 4: when the codes of tile t + 4 are turned, the
  // scores of tile t + 2 are done, and with them the softmax of tile t.
  __shared__ __align__(16) TileScales tile_scales[4];

  // (the warp's index by shuffle: the compiler then knows it to be uniform)
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  pdl_wait();  // q and the cache come from the kernels before
  // Causal chunks: the longest key ranges first, of all heads (head by head, the
  // last head's longest began last: chunks of 784 tokens 104.7 us).
  const int hk = blockIdx.x % g.c.heads, slot = (gridDim.x - 1 - blockIdx.x) / g.c.heads, split = blockIdx.y;
  const Block k = find_block(g, slot, kRows);
  if (k.seq < 0) {  // (with parts of the keys the join sees to the tokens of no sequence)
    if (k.end < g.c.total_new && g.splits == 1) clear_block(g, k.end, slot, kRows, hk);
    return;
  }

  // tiles of the whole CTA and of each 128-row block, cut to this split
  int t0, t1, a[MT], b[MT];
  {
    const Range r = keys_of_rows(g, k, k.first, min(k.first + kRows, k.rows));
    const int u0 = r.lo / kTile, u1 = (r.hi + kTile - 1) / kTile;
    t0 = min(u0 + split * g.split_tiles, u1);
    t1 = split + 1 < g.splits ? min(t0 + g.split_tiles, u1) : u1;
    int lo = INT_MAX, hi = 0;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const Range q = keys_of_rows(g, k, k.first + m * kTile, min(k.first + (m + 1) * kTile, k.rows));
      a[m] = max(t0, q.lo / kTile);
      b[m] = min(t1, (q.hi + kTile - 1) / kTile);
      if (b[m] <= a[m]) a[m] = b[m] = t0;
      else lo = min(lo, a[m]), hi = max(hi, b[m]);
    }
    t0 = lo < hi ? lo : 0;
    t1 = lo < hi ? hi : 0;
  }

  if (t0 < t1) {
    if (threadIdx.x == 0) {
      for (int s = 0; s < S::kStages; ++s) {
        tc::mbar_init(code_full(s), 1);
        tc::mbar_init(code_empty(s), 4);
      }
      for (int i = 0; i < 4; ++i) {
        tc::mbar_init(half_full(i >> 1, i & 1), 4);
        tc::mbar_init(half_empty(i >> 1, i & 1), 1);
      }
      for (int m = 0; m < MT; ++m) {
        tc::mbar_init(q_full(m), kTile);
        for (int i = 0; i < S::kSBuf; ++i) {
          tc::mbar_init(s_full(m, i), 1);
          tc::mbar_init(p_full(m, i), kTile);
        }
        tc::mbar_init(o_done(m), 1);
        tc::mbar_init(o_last(m), 1);
      }
      for (int s = 0; s < 4; ++s) tc::mbar_init(scale_full(s), 4);
      bad_values = 0;
      tc::mbar_fence_init();
      tc::tma_prefetch_map(&map_k);
      tc::tma_prefetch_map(&map_v);
    }
    if (warp == 4 * MT) {
      tc::tmem_alloc(tmem_slot, S::kCols);
      tc::tmem_relinquish();
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
  }
  const Edges edges = edges_of_rows(g, k.base, k.len, k.first, min(k.first + kRows, k.rows));
  const bool opens = t0 < t1 && (edges.open(t0) || edges.open(t1 - 1));  // (those between are open only if one of these is)
  uint32_t tmem = 0;
  if (t0 < t1) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));

  if (warp >= 4 * MT) {
    if (MT == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 144;");
    if (warp == 4 * MT || warp == 4 * MT + 2) {
      // ---------------------------------------------------------------- TMA producers
      Ring tiles;
      tiles.base = ring, tiles.full0 = code_full(0), tiles.empty0 = code_empty(0);
      tiles.take(warp == 4 * MT ? 0 : 1);
      tiles.seen = keys_of_rows(g, k, k.first, min(k.first + kRows, k.rows));
      const CUtensorMap *map = warp == 4 * MT ? &map_k : &map_v;
      bool ok = true;
      int id = t0 < t1 ? tiles.page_id(g, k.seq, k.len, t0) : -1;
      for (int t = t0; t < t1 && ok; ++t) {
        const int next = t + 1 < t1 ? tiles.page_id(g, k.seq, k.len, t + 1) : -1;
        ok = tiles.load(g, map, id, k.len, hk, t);
        id = next;
      }
      if (!ok && lane == 0) flag(g, TR_CACHE_ERR_WAIT);
      tiles.drain();
    } else if (warp >= 4 * MT + 4) {
      // ---------------------------------------------------------------- codes to halves
      const int w = warp - 4 * MT - 4;  // its rows: 32 w to 32 w + 31 of each tile
      int top = -127, low = 127, tiny = 127;
      // (from the first block that some row sees: those before a window may be given away and hold any scale)
      const int first = max(8 * t0, keys_of_rows(g, k, k.first, min(k.first + kRows, k.rows)).lo / kBlock) + 32 * w;
      const int blocks = min(8 * t1, (k.len + kBlock - 1) / kBlock);
#pragma unroll 4
      for (int i = first + lane; i < blocks; i += 128) {
        const uint32_t s = block_scales(p, k.seq, hk, k.len, kBlock * i);
        const int e = s != kNoScales ? (int)(s >> 8) - 127 : -127;
        top = max(top, e);
        if (e > kZeros) low = min(low, e);
        else if (s != kNoScales) tiny = min(tiny, e);
      }
      top = __reduce_max_sync(0xffffffffu, top), low = __reduce_min_sync(0xffffffffu, low);
      tiny = __reduce_min_sync(0xffffffffu, tiny);
      int r = 0;  // R
      bool wide = false;
      if (t0 < t1) {
        if (lane == 0) top_of[w] = top, low_of[w] = low, tiny_of[w] = tiny;
        codes_sync();
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, top_of[i]), low = min(low, low_of[i]), tiny = min(tiny, tiny_of[i]);
        if (tiny < top + kLeast && top + kLeast <= low) {  // only these are so far off: if they hold more than zeros
          const bool small = holds_small_values(p, k.seq, hk, k.len, first, blocks);
          if (lane == 0) small_of[w] = small;
          codes_sync();
          if (small_of[0] | small_of[1] | small_of[2] | small_of[3]) low = tiny;
        }
        r = top, wide = low < top + kLeast;
        if (w == 0 && lane == 0) ref = r, wide_sum = wide;
      }
      // scales of 16 tiles at a time, this warp's two blocks of one tile in two lanes
      auto scales = [&](int t) {
        const int i = t + (lane >> 1);
        return block_scales(p, k.seq, hk, i < t1 ? k.len : 0, i * kTile + 32 * w + 16 * (lane & 1));
      };
      uint32_t held = scales(t0), ahead = scales(t0 + 16);
      int st[2] = {Ring::first(0), Ring::first(1)}, held0 = t0;  // held0: first tile of `held`
      uint32_t ph[2] = {0u, 0u};
      bool found = false;
      auto turn = [&](int kind, int t) {
        const int n = t - t0, buf = n & 1;
        const int kst = kind ? st[1] : st[0];
        if (!tc::mbar_wait_warp(code_full(kst), kind ? ph[1] : ph[0])) return false;
        if (!tc::mbar_wait_warp(half_empty(kind, buf), (n >> 1 & 1) ^ 1)) return false;
        const uint32_t from = ring + kst * S::kCodeBytes, to = (kind ? v16 : k16) + buf * S::kTileBytes;
        if (!kind) {  // the tile's scales, for the softmax
          const int at = 2 * (t - held0 & 15) + (lane & 1);
          const uint32_t s0 = __shfl_sync(0xffffffffu, held, at), s1 = __shfl_sync(0xffffffffu, ahead, at);
          const uint32_t s = t - held0 < 16 ? s0 : s1;
          if (lane < 2) {
            TileScales &out = tile_scales[n & 3];
            int d = (s >> 8 < 255u ? (int)(s >> 8) - 127 : -127) - r;
            if (!wide) d = min(max(d, kLeast), 0);  // (above 0: seen by no row)
            out.k[2 * w + lane] = pow2((int)(s & 0xffu) - 127);
            out.v[2 * w + lane] = (float)d;
            out.undo[2 * w + lane] = wide ? 0.f : pow2(-d);
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(scale_full(n & 3));
        }
        constexpr int kAtOnce = 2;  // (4 and 8 crowd the products' reads of shared memory: 712 us for 2048 tokens over 32768 keys, 1 leaves waits: 702, here 701)
        if (kind && edges.open(t)) found |= to_halves<D, true, kAtOnce>(from, to, 32 * w, k.len - t * kTile);
        else to_halves<D, false, kAtOnce>(from, to, 32 * w, k.len - t * kTile);
        tc::fence_async_shared();
        __syncwarp();
        if (lane == 0) {
          tc::mbar_arrive(code_empty(kst));
          tc::mbar_arrive(half_full(kind, buf));
        }
        if (kind) Ring::on(1, st[1], ph[1]);
        else Ring::on(0, st[0], ph[0]);
        return true;
      };
      // in the order of the products: the scores of a tile come before the
      // second product of the tile before it
      bool ok = t0 < t1 ? turn(0, t0) : true;
      for (int t = t0; t < t1 && ok; ++t) {
        if (t + 1 < t1) ok = turn(0, t + 1);
        if (ok) ok = turn(1, t);
        if (t - held0 == 15) {
          held = ahead;
          held0 += 16;
          ahead = scales(held0 + 16);
        }
      }
      if (!ok && lane == 0) flag(g, TR_CACHE_ERR_WAIT);
      if (__any_sync(0xffffffffu, found) && lane == 0) bad_values = 1;
      if (opens) rows_arrive(kTile * MT + 128);
    } else if (warp == 4 * MT + 1) {
      // ---------------------------------------------------------------- MMA issuer (as in tr_attend.cu)
      const uint32_t lead = tc::elect_lane();
      const uint32_t idesc_s = tc::idesc_16(kTile, kTile, false, false);
      const uint32_t idesc_o = tc::idesc_16(kTile, g.c.d, false, true);
      const int ksteps = g.c.d / 16;
      const uint64_t q_desc = tc::sw128_desc(sbase), k_desc = tc::sw128_desc(k16),
                     v_desc = tc::sw128_desc_mn(v16, kTile * 128);
      constexpr uint32_t kStep = S::kTileBytes >> 4;  // a tile on, in a descriptor's address field
      uint32_t sn[MT], pn[MT];  // products issued so far, of each kind
      bool ok = true, have_q[MT];
#pragma unroll
      for (int m = 0; m < MT; ++m) sn[m] = pn[m] = 0, have_q[m] = false;
      // S_m = Q_m K^T of the tile of halves st
      auto scores = [&](int m, int st) {
        const uint64_t qd = q_desc + (uint64_t)(m * kStep), kd = k_desc + (uint64_t)((uint32_t)st * kStep);
        const int buf = S::kSBuf == 2 ? (int)(sn[m] & 1u) : 0;
        const uint32_t dst = tmem + (uint32_t)((MT == 1 ? buf : m) * kTile);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
          if (i < ksteps) {
            const uint64_t off = (uint64_t)(((i >> 2) * (kTile * 128) + (i & 3) * 32) >> 4);
            tc::mma_16_warp(dst, qd + off, kd + off, idesc_s, i > 0, lead);
          }
        tc::mma_commit_warp(s_full(m, buf), lead);
        ++sn[m];
      };
      // O_m (+)= P_m V of the tile of halves st
      auto values = [&](int m, int st, bool last) {
        const uint64_t vd = v_desc + (uint64_t)((uint32_t)st * kStep);
        const int buf = S::kSBuf == 2 ? (int)(pn[m] & 1u) : 0;
        const uint32_t pa = tmem + (uint32_t)((MT == 1 ? buf : m) * kTile), dst = tmem + (uint32_t)(S::kColO + m * D);
        const uint32_t more = pn[m] > 0;
#pragma unroll
        for (int i = 0; i < kTile / 16; ++i)
          tc::mma_16_ta_warp(dst, pa + 8 * i, vd + (uint64_t)(2048 * i >> 4), idesc_o, i > 0 ? 1u : more, lead);
        // one score buffer: the next scores, issued after this product, say as much
        if (last) tc::mma_commit_warp(o_last(m), lead);
        else if (S::kSBuf == 2) tc::mma_commit_warp(o_done(m), lead);
        ++pn[m];
      };
      for (int t = t0; t <= t1; ++t) {
        const int n = t - t0, kst = n & 1, vst = (n - 1) & 1;
        if (t > t0) ok &= tc::mbar_wait_warp(half_full(1, vst), (uint32_t)((n - 1) >> 1) & 1u);
        if (t < t1) ok &= tc::mbar_wait_warp(half_full(0, kst), (uint32_t)(n >> 1) & 1u);
        if (!ok) break;
        tc::fence_after_sync();
        if (S::kSBuf == 2 && t < t1) {
          if (!have_q[0]) ok &= tc::mbar_wait_warp(q_full(0), 0), have_q[0] = true;
          if (!ok) break;
          scores(0, kst);
          tc::mma_commit_warp(half_empty(0, kst), lead);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          if (S::kSBuf == 1 && t >= a[m] && t < b[m] && !have_q[m]) ok &= tc::mbar_wait_warp(q_full(m), 0), have_q[m] = true;
          if (t > a[m] && t <= b[m]) {
            ok &= tc::mbar_wait_warp(p_full(m, S::kSBuf == 2 ? (int)(pn[m] & 1u) : 0),
                                S::kSBuf == 2 ? pn[m] >> 1 & 1u : pn[m] & 1u);
            if (!ok) break;
            tc::fence_after_sync();
            values(m, vst, t == b[m]);
          }
          if (!ok) break;
          if (S::kSBuf == 1 && t >= a[m] && t < b[m]) scores(m, kst);
        }
        if (!ok) break;
        if (t > t0) tc::mma_commit_warp(half_empty(1, vst), lead);
        if (S::kSBuf == 1 && t < t1) tc::mma_commit_warp(half_empty(0, kst), lead);
      }
      if (!ok && lane == 0) flag(g, TR_CACHE_ERR_WAIT);
      __syncwarp();
    }
  } else {
    if (MT == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ---------------------------------------------------------------- softmax
    const int m = MT == 1 ? 0 : warp >> 2, quarter = warp & 3;
    const int row = 32 * quarter + lane, r = k.first + m * kTile + row;  // row of the block, of the sequence
    const bool valid = r < k.rows;
    const int tok = valid ? r / g.group : 0, head = hk * g.group + (valid ? r - tok * g.group : 0);
    const char *qrow = g.q + 2 * ((long long)(k.tok0 + tok) * g.q_tok + (long long)head * g.q_head);
    const int own = k.base + tok;
    // keys this row sees; rows that do not exist mask nothing and are dropped at the end
    const int hi = !valid ? INT_MAX : g.causal ? min(k.len, own + 1) : k.len;
    const int lo = valid && g.window > 0 ? window_start(own, g.window) : 0;
    const bool live = __any_sync(0xffffffffu, valid);
    const int ta = MT > 1 && m == 1 ? a[MT - 1] : a[0], tb = MT > 1 && m == 1 ? b[MT - 1] : b[0];
    float mx = -INFINITY, top = -INFINITY, sum = 0.f;  // maxima of scores + d and (wide) of scores
    bool ok = true, wide = false;
    const uint32_t lane_col = (uint32_t)(32 * quarter) << 16;
    const uint32_t o_col = tmem + lane_col + (uint32_t)(S::kColO + m * D);
    if (ta < tb) {
      // The warp's 32 rows of Q, as halves, into the swizzled layout that TMA
      // would write; D / 8 neighbouring lanes take a row, so that a load reads
      // whole lines.
      const uint32_t dst = sbase + m * S::kTileBytes + 32 * quarter * 128;
      const uint32_t flip = g.negate ? 0x80008000u : 0u;
      constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
      const int c = lane % kLanes;
      const long long qoff = valid ? qrow - g.q : -1;
      constexpr int kLoads = 32 / kAtOnce, kBatch = kLoads < 8 ? kLoads : 8;  // all loads of a batch before its stores
      int eq = 0;  // exponent that this thread's row was divided by
#pragma unroll 1
      for (int i0 = 0; i0 < kLoads; i0 += kBatch) {
        uint4 v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const long long off = __shfl_sync(0xffffffffu, qoff, (i0 + i) * kAtOnce + lane / kLanes);
          v[i] = make_uint4(0u, 0u, 0u, 0u);
          if (off >= 0 && 8 * c < g.c.d) v[i] = *reinterpret_cast<const uint4 *>(g.q + off + 16 * c);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int r1 = (i0 + i) * kAtOnce + lane / kLanes;
          if (Bits<T>::kBf16) {
            uint32_t most = max(max(top_of_pair(v[i].x), top_of_pair(v[i].y)), max(top_of_pair(v[i].z), top_of_pair(v[i].w)));
#pragma unroll
            for (int o = 1; o < kLanes; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
            const int e = query_exp(most);
            const float down = pow2(-e);
            v[i].x = query_pair(v[i].x, down), v[i].y = query_pair(v[i].y, down);
            v[i].z = query_pair(v[i].z, down), v[i].w = query_pair(v[i].w, down);
            const int from = __shfl_sync(0xffffffffu, e, lane % kAtOnce * kLanes);
            if (lane / kAtOnce == i0 + i) eq = from;
          }
          tc::st_shared_v4(dst + (c >> 3) * (kTile * 128) + r1 * 128 + (((c & 7) ^ (r1 & 7)) << 4), v[i].x ^ flip,
                           v[i].y ^ flip, v[i].z ^ flip, v[i].w ^ flip);
        }
      }
      tc::fence_async_shared();
      tc::mbar_arrive(q_full(m));
      // what a score of the row is multiplied by, its key's scale apart
      const float row_scale = g.scale * pow2(eq);

      // Whether the CTA is wide is known with the scales of its first tile.  (Their
      // barrier has no second phase yet: that is the fifth tile's, turned after
      // the third tile's scores, and those come after this block's first tile,
      // the CTA's first or second.  With one block and few tiles this wait before
      // that for the scores would take a microsecond: there it is read after it.)
      if (MT == 2) {
        ok = __all_sync(0xffffffffu, tc::mbar_wait(scale_full(0), 0));
        wide = ok && wide_sum;
      }
      for (int t = ta; !wide && t < tb && ok; ++t) {
        const int n = t - ta;
        const int buf = S::kSBuf == 2 ? n & 1 : 0;
        const uint32_t s_par = S::kSBuf == 2 ? (uint32_t)(n >> 1) & 1u : (uint32_t)n & 1u;
        const int ts = t - t0;
        ok = __all_sync(0xffffffffu, tc::mbar_wait(s_full(m, buf), s_par) && tc::mbar_wait(scale_full(ts & 3), (uint32_t)(ts >> 2) & 1u));
        if (!ok) break;
        if (MT == 1 && n == 0 && wide_sum) {
          wide = true;
          break;
        }
        tc::fence_after_sync();
        if (live) {
          const uint32_t s_col = tmem + lane_col + (uint32_t)((MT == 1 ? buf : m) * kTile);
          uint32_t s[kTile];
#pragma unroll
          for (int i = 0; i < kTile; i += 32) tc::tmem_ld32_issue(s_col + i, s + i);
          // (the scales while the scores are on their way)
          float f[8], dv[8], undo[8];
          {
            const uint32_t at = tc::smem_u32(&tile_scales[ts & 3]);
#pragma unroll
            for (int b = 0; b < 8; b += 4) {
              const uint4 x = tc::ld_shared_v4(at + 4 * b), y = tc::ld_shared_v4(at + 32 + 4 * b), z = tc::ld_shared_v4(at + 64 + 4 * b);
              f[b] = __uint_as_float(x.x), f[b + 1] = __uint_as_float(x.y), f[b + 2] = __uint_as_float(x.z), f[b + 3] = __uint_as_float(x.w);
              dv[b] = __uint_as_float(y.x), dv[b + 1] = __uint_as_float(y.y), dv[b + 2] = __uint_as_float(y.z), dv[b + 3] = __uint_as_float(y.w);
              undo[b] = __uint_as_float(z.x), undo[b + 1] = __uint_as_float(z.y), undo[b + 2] = __uint_as_float(z.z), undo[b + 3] = __uint_as_float(z.w);
            }
#pragma unroll
            for (int b = 0; b < 8; ++b) f[b] = block_factor(row_scale, f[b]);
          }
#pragma unroll
          for (int i = 0; i < kTile; i += 32) tc::tmem_ld32_wait(s + i);
          const int key0 = t * kTile;
          if (__any_sync(0xffffffffu, lo > key0 || hi < key0 + kTile)) {
            const int c0 = lo - key0, c1 = hi - key0;
#pragma unroll
            for (int i = 0; i < kTile; ++i)
              if (i < c0 || i >= c1) s[i] = 0xff800000u;  // -inf
          }
          float tops[8];
#pragma unroll
          for (int b = 0; b < 8; ++b) {
            float top0 = max3(__uint_as_float(s[16 * b]), s[16 * b + 1], s[16 * b + 2]), top1 = __uint_as_float(s[16 * b + 3]);
#pragma unroll
            for (int i = 4; i < 16; i += 4) top0 = max3(top0, s[16 * b + i], s[16 * b + i + 1]), top1 = max3(top1, s[16 * b + i + 2], s[16 * b + i + 3]);
            tops[b] = fmaf(fmaxf(top0, top1), f[b], dv[b]);
          }
          const float now = fmaxf(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), fmaxf(fmaxf(tops[4], tops[5]), fmaxf(tops[6], tops[7])));
          if (n == 0) {
            mx = now;
          } else if (__any_sync(0xffffffffu, now > mx + 8.f)) {
            // the sums so far (all products up to the last tile's are in) move to the new maximum
            const bool more = now > mx + 8.f;
            const float down = more ? exp2_fast(mx - now) : 1.f;
            if (S::kSBuf == 2) {  // (one buffer: these scores came after the last tile's product)
              ok = __all_sync(0xffffffffu, tc::mbar_wait(o_done(m), (uint32_t)(n - 1) & 1u));
              if (!ok) break;
              tc::fence_after_sync();
            }
#pragma unroll 1
            for (int c1 = 0; c1 < D; c1 += 32) {
              uint32_t o[32];
              tc::tmem_ld32_issue(o_col + c1, o);
              tc::tmem_ld32_wait(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * down);
              tc::tmem_st32(o_col + c1, o);
            }
            tc::tmem_st_wait();
            if (more) mx = now;
            sum *= down;
          }
          const float neg = mx == -INFINITY ? 0.f : kLift8 - mx;  // a row that has seen nothing: exp2(-inf) = 0
#pragma unroll
          for (int b = 0; b < 8; ++b) {
            const float d = neg + dv[b];
            const pack::f2 f2b = pack::make(f[b], f[b]), d2 = pack::make(d, d);
            float e[16];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              const float2 x = pack::split(pack::fma(pack::make(__uint_as_float(s[16 * b + i]), __uint_as_float(s[16 * b + i + 1])), f2b, d2));
              e[i] = x.x, e[i + 1] = x.y;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) e[i] = exp2_fast(e[i]);
#pragma unroll
            for (int i = 0; i < 16; i += 2) s[(16 * b + i) >> 1] = Bits<__half>::pack(e[i], e[i + 1]);
            pack::f2 acc = pack::add(pack::add(pack::add(pack::make(e[0], e[1]), pack::make(e[2], e[3])), pack::add(pack::make(e[4], e[5]), pack::make(e[6], e[7]))),
                                     pack::add(pack::add(pack::make(e[8], e[9]), pack::make(e[10], e[11])), pack::add(pack::make(e[12], e[13]), pack::make(e[14], e[15]))));
            const float2 x = pack::split(acc);
            sum = fmaf(x.x + x.y, undo[b], sum);
          }
          tc::tmem_st32(s_col, s);
          tc::tmem_st32(s_col + 32, s + 32);
          tc::tmem_st_wait();
        }
        tc::fence_before_sync();
        tc::mbar_arrive(p_full(m, buf));
      }
      if (wide) {
        WideRow w{tmem + lane_col + (uint32_t)((MT == 1 ? 0 : m) * kTile), o_col, s_full(m, 0), p_full(m, 0), o_done(m), scale_full(0),
                  tc::smem_u32(tile_scales), t0, ta, tb, lo, hi, row_scale, -INFINITY, -INFINITY, 0.f, live};
        ok = softmax_wide<D, S::kSBuf>(w);
        mx = w.mx, top = w.top, sum = w.sum;
      }
      // A barrier of its own: of one that every product completes, a thread
      // that comes late could not tell the last phase from the one before.
      if (ok) ok = __all_sync(0xffffffffu, tc::mbar_wait(o_last(m), 0));
      tc::fence_after_sync();
      if (!ok && lane == 0) flag(g, TR_CACHE_ERR_WAIT);
    }

    // ---------------------------------------------------------------- the rows' results
    if (live && ok) {
      const long long out_row = (long long)(k.tok0 + tok) * g.q_heads + head;
      char *orow = g.o + 2 * ((long long)(k.tok0 + tok) * g.o_tok + (long long)head * g.o_head);
      const bool parts = g.splits > 1;
      const long long all_rows = (long long)g.c.total_new * g.q_heads;
      float *prow = g.part + ((long long)split * all_rows + out_row) * g.c.d;
      // divided by the sum before V's scale, up to 2^127, enters (wide: with what the sum was taken against, in two
      // steps, because it may be 2^-140)
      const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
      const float half = top == -INFINITY ? 0.f : exp2_fast(0.5f * (mx - kLift8 + (ta < tb ? (float)ref : 0.f) - top));
      const float up0 = wide ? half : ta < tb ? pow2(ref) : 0.f, up1 = wide ? half : 1.f;
      // staged in the place of this row's queries, whose products are done
      const uint32_t stage_row = sbase + m * S::kTileBytes + row * 128;
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        if (ta < tb) {
          tc::tmem_ld32_issue(o_col + c, o);
          tc::tmem_ld32_wait(o);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0u;
        }
        if (valid && (ta < tb || !parts)) {
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            if (c + i >= g.c.d) break;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(o[i + j]) * inv * up0 * up1;
            if (parts) {
              *reinterpret_cast<float4 *>(prow + c + i) = make_float4(v[0], v[1], v[2], v[3]);
              *reinterpret_cast<float4 *>(prow + c + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
            } else {
              const int ch = (c + i) >> 3;
              tc::st_shared_v4(stage_row + (ch >> 3) * (kTile * 128) + (((ch & 7) ^ (row & 7)) << 4),
                               Bits<T>::pack(v[0], v[1]), Bits<T>::pack(v[2], v[3]), Bits<T>::pack(v[4], v[5]),
                               Bits<T>::pack(v[6], v[7]));
            }
          }
        }
      }
      if (!parts) {  // rows leave as whole lines, as they came
        __syncwarp();
        constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
        const int c = lane % kLanes;
        const long long ooff = valid ? orow - g.o : -1;
#pragma unroll 4
        for (int i = 0; i < 32; i += kAtOnce) {
          const int r1 = i + lane / kLanes;
          const long long off = __shfl_sync(0xffffffffu, ooff, r1);
          const uint32_t src = sbase + m * S::kTileBytes + (32 * quarter + r1) * 128 + (c >> 3) * (kTile * 128) +
                               (((c & 7) ^ (r1 & 7)) << 4);
          if (off >= 0 && 8 * c < g.c.d) *reinterpret_cast<uint4 *>(g.o + off + 16 * c) = tc::ld_shared_v4(src);
        }
        __syncwarp();
      }
      if (valid) {
        const float against = wide ? top : mx - kLift8;  // what the sum was taken against
        const bool any = sum > 0.f;  // (the parts' sums, of any size, join as exponents)
        if (parts) g.part_ml[(long long)split * all_rows + out_row] = any ? make_float2(against + log2f(sum), 1.f) : make_float2(against, sum);
        else if (g.lse) g.lse[out_row] = any || sum != sum ? against * 0.693147180559945309f + logf(sum) : -INFINITY;
      }
    }
    if (opens) {
      rows_sync(kTile * MT + 128);  // the tiles are checked, and the rows' results are in
      if (bad_values && ok) put_back8<T>(g, k.seq, k.tok0, k.base, k.len, k.rows, k.first, kRows, hk, split, warp, ta, tb);
    }
  }

  if (t0 < t1) {
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 4 * MT) {
      tc::fence_after_sync();
      tc::tmem_dealloc(tmem, S::kCols);
    }
  }
}

// ---------------------------------------------------------------- host side
struct Plan8 {
  bool few;                 // tr_attend8_few.cu's kernel
  int mt, slots;            // else blocks of 128 mt rows
  int splits, split_tiles;  // and the parts of the keys, in tiles
  size_t part_ml, total;    // workspace
};

// Parts of the keys: as many as finish earliest on `sms` SMs.  A CTA costs its
// tiles and about kCtaTiles more (its start and end, 11 us); with parts there
// is the join, of which kJoinRows rows take the time of a tile.  The host knows
// the longest of the lengths alone, so the time is the mean of what they take
// if all are so long (in waves) and if they are spread below it (the SMs' even
// shares and the last CTAs' end).  Of 18 cases measured with 1 to 8 parts, even and ragged,
// the choice is 3 % above the best (all lengths the same: 10 %): 5 tokens of 32
// sequences over 1000 to 12000 keys, 2 parts, 65 us, in one 93, in three 75.
int choose_parts8(double blocks, int tiles, int sms, double rows, bool one) {
  constexpr double kCtaTiles = 6.0, kJoinRows = 8192.0;
  double best = 0;
  int parts = 1;
  for (int s = 1; s <= 64 && s <= (tiles > 1 ? tiles : 1); ++s) {
    const double cta = (tiles + s - 1) / s + kCtaTiles;
    const double even = std::ceil(blocks * s / sms) * cta;
    const double spread = one                ? even
                          : blocks * s <= sms ? cta
                                              : std::fmax(cta, blocks * (0.5 * tiles + kCtaTiles * 0.5 * (s + 1)) / sms + 0.25 * cta);
    const double t = 0.5 * (even + spread) + (s > 1 ? kCtaTiles + rows * s / kJoinRows : 0.0);
    if (s == 1 || t < best) best = t, parts = s;
  }
  return parts;
}

Plan8 plan8_of(const tr_cache *c, int q_heads, int window, int max_new, int max_len) {
  Plan8 p{};
  const int group = q_heads / c->heads;
  const long long most = (long long)(max_new < c->total_new ? max_new : c->total_new) * group;
  const int sms = sm_count() > 0 ? sm_count() : 1;
  const long long cap = (long long)c->max_pages * c->page;
  long long keys = max_len < cap ? max_len : cap;
  if (window > 0 && keys > (long long)window + max_new) keys = (long long)window + max_new;
  const int tiles = (int)((keys + kTile - 1) / kTile);
  if (few_takes(c, q_heads, max_new, kItemCost, tiles < kMinTilesFew ? kFewRows : kMostFew)) {
    p.few = true;
    p.total = few_workspace_bytes(c->head_dim, sms);
    return p;
  }
  p.mt = most <= kTile ? 1 : 2;
  p.slots = (int)((long long)c->total_new * group / (kTile * p.mt)) + c->batch + 1;  // (tokens of no sequence: one more)
  const double blocks = most <= kTile ? c->batch : std::fmin(p.slots - 1, (double)c->total_new * group / (kTile * p.mt) + 0.5 * c->batch);
  p.splits = choose_parts8(blocks * c->heads, tiles, sms, (double)c->total_new * q_heads, c->batch == 1);
  p.split_tiles = (tiles + p.splits - 1) / p.splits;
  if (p.splits > 1) {
    const size_t r = (size_t)c->total_new * q_heads * p.splits;
    p.part_ml = align_up(r * c->head_dim * sizeof(float), 256);
    p.total = p.part_ml + align_up(r * sizeof(float2), 256);
  }
  return p;
}

std::atomic<int> g_attend8_smem_set[64];

template <typename T, int D, int MT>
cudaError_t launch_attend8_t(const CUtensorMap &mk, const CUtensorMap &mv, const Attend8Args &p, int slots, cudaStream_t st) {
  using S = Shape8<D, MT>;
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  const int bit = 1 << (Bits<T>::kBf16 * 4 + (D == 128) * 2 + (MT - 1));
  if (!(g_attend8_smem_set[dev & 63].load() & bit)) {
    err = cudaFuncSetAttribute(k_attend8<T, D, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
    if (err != cudaSuccess) return err;
    g_attend8_smem_set[dev & 63].fetch_or(bit);
  }
  return launch_kernel(k_attend8<T, D, MT>, dim3((unsigned)slots * p.a.c.heads, p.a.splits), dim3(S::kThreads), S::kSmem, st, false, mk,
                       mv, p);
}

template <typename T>
cudaError_t launch_attend8(const CUtensorMap &mk, const CUtensorMap &mv, const Attend8Args &p, const Plan8 &plan,
                           cudaStream_t st) {
  const bool narrow = p.a.c.d <= 64;
  const cudaError_t err = plan.mt == 1 ? narrow ? launch_attend8_t<T, 64, 1>(mk, mv, p, plan.slots, st)
                                                : launch_attend8_t<T, 128, 1>(mk, mv, p, plan.slots, st)
                          : narrow     ? launch_attend8_t<T, 64, 2>(mk, mv, p, plan.slots, st)
                                       : launch_attend8_t<T, 128, 2>(mk, mv, p, plan.slots, st);
  if (err != cudaSuccess || p.a.splits == 1) return err;
  const long long rows = (long long)p.a.c.total_new * p.a.q_heads;
  return launch_kernel(k_attend_join<T, true>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, true, p.a);
}

}  // namespace
}  // namespace tr

using namespace tr;

extern "C" {

size_t tr_cache8_attend_workspace_bytes(const tr_cache8 *c, int32_t q_heads, int32_t window, int32_t max_new,
                                        int32_t max_len) {
  if (check_cache8(c) != TR_OK || q_heads <= 0 || q_heads % c->c.heads || window < 0 || max_new < 0 || max_len < 0)
    return 0;
  return plan8_of(&c->c, q_heads, window, max_new, max_len).total;
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
  if (c->heads > 65535) return TR_ERR_UNSUPPORTED;  // as tr_cache_attend
  if (c->total_new == 0) return TR_OK;
  const Plan8 plan = plan8_of(c, q->heads, window, max_new, max_len);
  if ((long long)plan.slots * c->heads > INT_MAX) return TR_ERR_UNSUPPORTED;
  if (plan.total && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < plan.total)) return TR_ERR_WORKSPACE;
  Attend8Args p{};
  AttendArgs &g = p.a;
  g.c = cache_view(c);
  g.q = static_cast<const char *>(q->p);
  g.o = static_cast<char *>(o->p);
  g.q_tok = q->token_stride, g.q_head = q->head_stride;
  g.o_tok = o->token_stride, g.o_head = o->head_stride;
  g.q_heads = q->heads, g.group = q->heads / c->heads;
  g.lse = lse;
  g.scale = fabsf(scale) * 1.44269504088896341f;
  g.negate = scale < 0.f;
  g.causal = causal, g.window = window;
  g.splits = plan.splits;
  g.split_tiles = plan.split_tiles;
  while ((1 << g.page_log2) < c->page) ++g.page_log2;
  g.part = static_cast<float *>(ws);
  g.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(ws) + plan.part_ml);
  g.err = d_error;
  p.scale = Scales{c8->k_scale, c8->v_scale};
  CUtensorMap mk{}, mv{};
  const long long keys = (long long)c->pages * c->heads * c->page;
  const int box = c->page < kTile ? c->page : kTile, wide = c->head_dim <= 64 ? 64 : 128;
  // an empty cache keeps one row in the maps' extents: no page id is valid, so nothing reads it
  if (!make_map_bytes(&mk, c->k, keys > 0 ? keys : 1, c->head_dim, box, wide) ||
      !make_map_bytes(&mv, c->v, keys > 0 ? keys : 1, c->head_dim, box, wide))
    return TR_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (plan.few) {
    g.ctas = sm_count() > 0 ? sm_count() : 1;
    return launch_few8(mk, mv, p, c->dtype == TR_BF16, ws, st) == cudaSuccess ? TR_OK : TR_ERR_CUDA;
  }
  const cudaError_t err = c->dtype == TR_BF16 ? launch_attend8<__nv_bfloat16>(mk, mv, p, plan, st)
                                              : launch_attend8<__half>(mk, mv, p, plan, st);
  return err == cudaSuccess ? TR_OK : TR_ERR_CUDA;
}

}  // extern "C"
