// Attention of new tokens over the paged cache (tr_cache_attend) on the
// 5th-generation tensor cores:
//   o = sum_j p_j v_j,  p = softmax over the visible keys of scale q . k_j,
// in one pass over the keys with the running maximum and sum of the softmax.
//
// The query heads of one key head and the new tokens of one sequence make up
// the rows of a block (row r: token r / group, head r % group), so a page is
// read once for the whole group, and a single token of a grouped layer still
// fills several rows.  A CTA takes 128 MT rows of one sequence and key head
// and walks the keys in tiles of 128:
//   softmax warps   one warpgroup per 128 rows, one thread per row: scores
//                   from tensor memory, mask, maximum, exponentials; the
//                   probabilities go back to tensor memory as the A operand
//                   of the second product, in the place of the scores;
//   producer warps  TMA loads of K (one warp) and V (another) tiles, page by
//                   page, into a ring of 128-byte-swizzled tiles;
//   checking warp   value rows past the sequence's end become zeros (stale
//                   memory there may hold NaN), and values that are not finite
//                   leave the tiles that some row does not see all of (Edges
//                   in tr_attend.cuh);
//   MMA warp        S = Q K^T and O += P V from one thread.  The products of
//                   the two 128-row blocks alternate, so one block's softmax
//                   runs while the tensor cores work on the other.
//
// The maximum that the exponentials are taken against is only renewed (and
// O rescaled) when it has grown by more than 8 powers of two: p <= 2^8 is as
// exact as p <= 1 in floating point, and the rescaling, which reads and
// writes all of O, almost never runs after the first tiles.
//
// Probabilities are rounded to the cache's 16-bit type for the second
// product (the tensor cores take both operands in one type); their sum is
// taken before that rounding, and everything else is fp32.
//
// Bound by the tensor cores where there are many keys: 2048 tokens over 32768
// keys, 28/4 heads of 128, bf16, 615 us on GB300 (1.52 PFLOP/s, 0.79 of the
// measured cuBLAS rate).  A 128 x 128 x 16 product reads 8 KB of shared
// memory, or 4 KB and tensor memory, in the 64 cycles it could take.
#include <cfloat>
#include <climits>
#include <cmath>

#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tr_attend.cuh"
#include "tr_pack.cuh"

namespace tr {
namespace {

using namespace attend;

// MT blocks of 128 rows a CTA.  PAIRED (MT = 1): two CTAs share an SM, each
// with room for little more than the tile in use, so that one's start and
// end run beside the other's work: for keys of a few tiles, where a CTA is
// mostly start and end (16 prompts of 227 tokens, 32 heads: 49 us; MT = 2 took
// 54 us when it was left).
template <int D, int MT, bool PAIRED>
struct Shape {
  static_assert(MT == 2 || MT == 1, "");
  static constexpr int kTileBytes = kTile * D * 2;   // one K or V tile, or one block's Q
  static constexpr int kBudget = 227 * 1024 - 2048;  // shared memory less barriers and alignment
  static constexpr int kFit = (kBudget - MT * kTileBytes) / kTileBytes;
  static constexpr int kStages = PAIRED ? (D == 128 ? 2 : 4) : kFit < 12 ? kFit : 12;
  static constexpr int kSBuf = MT == 1 && !PAIRED ? 2 : 1;  // score buffers of a block
  // Whole warpgroups, so that registers can move between them where a thread
  // would have too few for a row of scores (128): of 168 at launch (MT = 2)
  // 216 for the softmax and 56 for the rest, of 128 (PAIRED) 200 and 48.
  static constexpr int kThreads = MT == 2 ? 384 : 256;
  static constexpr bool kMove = MT == 2 || PAIRED;
  static constexpr int kColO = PAIRED ? 128 : 256;  // tensor-memory columns: scores below, sums from here
  static constexpr int kCols = PAIRED ? 256 : 512;
  static constexpr size_t kSmem = (size_t)(MT + kStages) * kTileBytes + 1024 + 512;
  static_assert(kColO + MT * D <= kCols && kColO >= MT * kSBuf * kTile, "scores and sums fit the tensor memory");
  static_assert(!PAIRED || 2 * (kSmem + 1024) <= 228 * 1024, "two CTAs fit an SM");
};

__device__ __forceinline__ float max3(float a, uint32_t b, uint32_t c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
  return r;
}

// The block of tokens that belong to no sequence (first: their first) in this
// slot: zeros, lse -inf.
__device__ __noinline__ void clear_block(const AttendArgs &g, int first, int slot, int rows_per_block, int hk) {
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

// The values taken out of open tiles among [t0, t1) to those rows of the warp
// that see them.  (Not inline: it would cost the softmax registers.)
template <typename T>
__device__ __noinline__ void put_back(const AttendArgs &g, int seq, int tok0, int base, int len, int rows, int first, int block,
                                      int hk, int split, int warp, int t0, int t1) {
  const Edges e = edges_of_rows(g, base, len, first, min(first + block, rows));
  for_bad_values<T>(g, e, seq, hk, t0, t1, [&](int j, const float4 &v) {
    for (int r = first + 32 * warp; r < min(first + 32 * warp + 32, rows); ++r) {
      const int tok = r / g.group, head = hk * g.group + r % g.group, own = base + tok;
      if ((g.causal && j > own) || (g.window > 0 && j < window_start(own, g.window))) continue;
      const long long t = tok0 + tok;
      add_to_row<T>(g.o + 2 * (t * g.o_tok + (long long)head * g.o_head),
                    g.splits > 1 ? g.part + (((long long)split * g.c.total_new + t) * g.q_heads + head) * g.c.d : nullptr, v);
    }
  });
}

__device__ __forceinline__ void named_sync(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }
__device__ __forceinline__ void named_arrive(int threads) { asm volatile("bar.arrive 1, %0;" ::"r"(threads) : "memory"); }

template <typename T, int D, int MT, bool PAIRED>
__global__ void __launch_bounds__(Shape<D, MT, PAIRED>::kThreads, PAIRED ? 2 : 1)
    k_attend(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
             const __grid_constant__ AttendArgs g) {
  using S = Shape<D, MT, PAIRED>;
  constexpr int kRows = kTile * MT;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t sbase = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;  // the swizzle atom
  const uint32_t ring = sbase + MT * S::kTileBytes;
  const uint32_t bars = ring + S::kStages * S::kTileBytes;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (S::kStages + s); };
  auto q_full = [&](int m) { return bars + 8u * (2 * S::kStages + m); };
  auto s_full = [&](int m, int b) { return bars + 8u * (2 * S::kStages + MT + m * S::kSBuf + b); };
  auto p_full = [&](int m, int b) { return bars + 8u * (2 * S::kStages + MT + MT * S::kSBuf + m * S::kSBuf + b); };
  auto o_done = [&](int m) { return bars + 8u * (2 * S::kStages + MT + 2 * MT * S::kSBuf + m); };
  auto o_last = [&](int m) { return bars + 8u * (2 * S::kStages + 2 * MT + 2 * MT * S::kSBuf + m); };
  using Ring = TileRing<D, S::kStages, true>;
  const uint32_t raw0 = bars + 8u * (2 * S::kStages + 3 * MT + 2 * MT * S::kSBuf);
  const uint32_t tmem_slot = raw0 + 8u * (S::kStages - Ring::kK);
  __shared__ int bad_values;  // some were taken out of the tiles

  // (the warp's index by shuffle: the compiler then knows it to be uniform)
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  pdl_wait();  // q and the cache come from the kernels before
  const int slot = gridDim.x - 1 - blockIdx.x;  // causal chunks: the longest key ranges first
  const int hk = blockIdx.y, split = blockIdx.z;
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
        tc::mbar_init(full(s), 1);
        tc::mbar_init(empty(s), 1);
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
      for (int s = 0; s < S::kStages - Ring::kK; ++s) tc::mbar_init(raw0 + 8u * s, 1);
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
  // (PAIRED: no tile counts as open, see the rows' results)
  const Edges edges = PAIRED ? Edges{0, k.len, k.len} : edges_of_rows(g, k.base, k.len, k.first, min(k.first + kRows, k.rows));
  const bool opens = !PAIRED && t0 < t1 && (edges.open(t0) || edges.open(t1 - 1));  // (those between are open only if one of these is)
  uint32_t tmem = 0;
  if (t0 < t1) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));

  if (warp >= 4 * MT) {
  if (S::kMove) {
    if (PAIRED) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  }
  Ring tiles;
  tiles.base = ring, tiles.full0 = full(0), tiles.empty0 = empty(0), tiles.raw0 = raw0;
  tiles.edges = edges;
  if (warp == 4 * MT || warp == 4 * MT + 2) {
    // ---------------------------------------------------------------- TMA producers
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
  } else if (warp == 4 * MT + 3) {
    // ---------------------------------------------------------------- values that not every row sees
    if (!tiles.template check_values<T>(t0, t1, &bad_values) && lane == 0) flag(g, TR_CACHE_ERR_WAIT);
    if (opens) named_arrive(kTile * MT + 32);
  } else if (warp == 4 * MT + 1) {
    // ---------------------------------------------------------------- MMA issuer
    {
      const uint32_t lead = tc::elect_lane();
      // The tensor cores hold only a product or two beyond the one they run,
      // so every cycle this warp spends between two products is theirs
      // too: descriptors are sums with constants, ring positions are
      // counted, and what can be waited for early is.
      const uint32_t idesc_s = tc::idesc_16(kTile, kTile, Bits<T>::kBf16, false);
      const uint32_t idesc_o = tc::idesc_16(kTile, g.c.d, Bits<T>::kBf16, true);
      const int ksteps = g.c.d / 16;
      const uint64_t q_desc = tc::sw128_desc(sbase), k_desc = tc::sw128_desc(ring),
                     v_desc = tc::sw128_desc_mn(ring, kTile * 128);
      constexpr uint32_t kStep = S::kTileBytes >> 4;  // a tile on, in a descriptor's address field
      uint32_t sn[MT], pn[MT];  // products issued so far, of each kind
      bool ok = true, have_q[MT];
#pragma unroll
      for (int m = 0; m < MT; ++m) sn[m] = pn[m] = 0, have_q[m] = false;
      // S_m = Q_m K^T of the tile in ring position st
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
      // O_m (+)= P_m V of the tile in ring position st
      auto values = [&](int m, int st, bool last) {
        const uint64_t vd = v_desc + (uint64_t)((uint32_t)st * kStep);
        const int buf = S::kSBuf == 2 ? (int)(pn[m] & 1u) : 0;
        const uint32_t p = tmem + (uint32_t)((MT == 1 ? buf : m) * kTile), dst = tmem + (uint32_t)(S::kColO + m * D);
        const uint32_t more = pn[m] > 0;
#pragma unroll
        for (int i = 0; i < kTile / 16; ++i)
          tc::mma_16_ta_warp(dst, p + 8 * i, vd + (uint64_t)(2048 * i >> 4), idesc_o, i > 0 ? 1u : more, lead);
        // one score buffer: the next scores, issued after this product, say as much
        if (last) tc::mma_commit_warp(o_last(m), lead);
        else if (S::kSBuf == 2) tc::mma_commit_warp(o_done(m), lead);
        ++pn[m];
      };
      // Step t issues P V of tile t - 1 and the scores of tile t.  The tensor
      // cores run the products in the order of issue, so scores may overwrite
      // probabilities that the product issued before them reads.  One block
      // with two score buffers issues the scores first: its softmax of tile t
      // runs during the products of tile t - 1.
      int kst = Ring::first(0), vst = Ring::first(1);
      uint32_t kph = 0, vph = 0;
      for (int t = t0; t <= t1; ++t) {
        if (t > t0) ok &= tc::mbar_wait_warp(full(vst), vph);
        if (t < t1) ok &= tc::mbar_wait_warp(full(kst), kph);
        if (!ok) break;
        tc::fence_after_sync();
        if (S::kSBuf == 2 && t < t1) {
          if (!have_q[0]) ok &= tc::mbar_wait_warp(q_full(0), 0), have_q[0] = true;
          if (!ok) break;
          scores(0, kst);
          tc::mma_commit_warp(empty(kst), lead);
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
        if (t > t0) tc::mma_commit_warp(empty(vst), lead);
        if (S::kSBuf == 1 && t < t1) tc::mma_commit_warp(empty(kst), lead);
        if (t > t0) Ring::on(1, vst, vph);
        Ring::on(0, kst, kph);
      }
      if (!ok && lane == 0) flag(g, TR_CACHE_ERR_WAIT);
    }
    __syncwarp();
  }
  } else {
    if (S::kMove) {
      if (PAIRED) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
      else asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    }
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
    float mx = -INFINITY, sum = 0.f;
    bool ok = true;
    const uint32_t lane_col = (uint32_t)(32 * quarter) << 16;
    const uint32_t o_col = tmem + lane_col + (uint32_t)(S::kColO + m * D);
    if (ta < tb) {
      // The warp's 32 rows of Q into the swizzled layout that TMA would
      // write; D / 8 neighbouring lanes take a row, so that a load reads
      // whole lines.
      const uint32_t dst = sbase + m * S::kTileBytes + 32 * quarter * 128;
      const uint32_t flip = g.negate ? 0x80008000u : 0u;
      constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
      const int c = lane % kLanes;
      const long long qoff = valid ? qrow - g.q : -1;
      constexpr int kLoads = 32 / kAtOnce, kBatch = kLoads < 8 ? kLoads : 8;  // all loads of a batch before its stores
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
          tc::st_shared_v4(dst + (c >> 3) * (kTile * 128) + r1 * 128 + (((c & 7) ^ (r1 & 7)) << 4), v[i].x ^ flip,
                           v[i].y ^ flip, v[i].z ^ flip, v[i].w ^ flip);
        }
      }
      tc::fence_async_shared();
      tc::mbar_arrive(q_full(m));

      for (int t = ta; t < tb; ++t) {
        const int n = t - ta;
        const int buf = S::kSBuf == 2 ? n & 1 : 0;
        const uint32_t s_par = S::kSBuf == 2 ? (uint32_t)(n >> 1) & 1u : (uint32_t)n & 1u;
        ok = __all_sync(0xffffffffu, tc::mbar_wait(s_full(m, buf), s_par));
        if (!ok) break;
        tc::fence_after_sync();
        if (live) {
          const uint32_t s_col = tmem + lane_col + (uint32_t)((MT == 1 ? buf : m) * kTile);
          uint32_t s[kTile];
#pragma unroll
          for (int i = 0; i < kTile; i += 32) tc::tmem_ld32_issue(s_col + i, s + i);
#pragma unroll
          for (int i = 0; i < kTile; i += 32) tc::tmem_ld32_wait(s + i);
          const int key0 = t * kTile;
          if (__any_sync(0xffffffffu, lo > key0 || hi < key0 + kTile)) {
            const int c0 = lo - key0, c1 = hi - key0;
#pragma unroll
            for (int i = 0; i < kTile; ++i)
              if (i < c0 || i >= c1) s[i] = 0xff800000u;  // -inf
          }
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < kTile; i += 8)
#pragma unroll
            for (int j = 0; j < 4; ++j) top[j] = max3(top[j], s[i + 2 * j], s[i + 2 * j + 1]);
          const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * g.scale;
          if (n == 0) {
            mx = now;
          } else if (__any_sync(0xffffffffu, now > mx + 8.f)) {
            // the sums so far (all products up to the last tile's are in) move to the new maximum
            const bool up = now > mx + 8.f;
            const float f = up ? exp2_fast(mx - now) : 1.f;
            if (S::kSBuf == 2) {  // (one buffer: these scores came after the last tile's product)
              ok = __all_sync(0xffffffffu, tc::mbar_wait(o_done(m), (uint32_t)(n - 1) & 1u));
              if (!ok) break;
              tc::fence_after_sync();
            }
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              uint32_t o[32];
              tc::tmem_ld32_issue(o_col + c, o);
              tc::tmem_ld32_wait(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tc::tmem_st32(o_col + c, o);
            }
            tc::tmem_st_wait();
            if (up) mx = now;
            sum *= f;
          }
          const float neg = mx == -INFINITY ? 0.f : -mx;  // a row that has seen nothing: exp2(-inf) = 0
          const pack::f2 sc2 = pack::make(g.scale, g.scale), neg2 = pack::make(neg, neg);
          pack::f2 acc[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
          for (int i = 0; i < kTile; i += 2) {
            const float2 e = pack::split(pack::fma(pack::make(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), sc2, neg2));
            const float p0 = exp2_fast(e.x), p1 = exp2_fast(e.y);
            acc[(i >> 1) & 3] = pack::add(acc[(i >> 1) & 3], pack::make(p0, p1));
            s[i >> 1] = Bits<T>::pack(p0, p1);
          }
          const float2 x = pack::split(pack::add(pack::add(acc[0], acc[1]), pack::add(acc[2], acc[3])));
          sum += x.x + x.y;
          tc::tmem_st32(s_col, s);
          tc::tmem_st32(s_col + 32, s + 32);
          tc::tmem_st_wait();
        }
        tc::fence_before_sync();
        tc::mbar_arrive(p_full(m, buf));
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
      const float inv = parts ? 1.f : sum > 0.f || sum != sum ? 1.f / sum : 0.f;
      bool finite = true;
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
            for (int j = 0; j < 8; ++j) {
              v[j] = __uint_as_float(o[i + j]) * inv;
              if (PAIRED) finite &= finite1(v[j]);
            }
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
        if (parts) g.part_ml[(long long)split * all_rows + out_row] = make_float2(mx, sum);
        else if (g.lse) g.lse[out_row] = sum > 0.f || sum != sum ? mx * 0.693147180559945309f + logf(sum) : -INFINITY;
      }
      // PAIRED: a check of the values would stand in the way of a CTA's one or
      // two tiles (16 prompts of 227 tokens 51 us against 49).  Instead a row
      // that came out not finite, and not because of what it sees, is taken
      // again by itself: the keys are few.  The lanes that do write over what
      // the row's own lane has just written, so its stores come first.
      if (PAIRED) {
        __syncwarp();
        unsigned bad = __ballot_sync(0xffffffffu, valid && !finite);
        while (bad) {
          const int src = __ffs(bad) - 1;
          bad &= bad - 1;
          const int rlo = max(__shfl_sync(0xffffffffu, lo, src), ta * kTile);
          const int rhi = min(__shfl_sync(0xffffffffu, hi, src), tb * kTile);
          const int end = min(tb * kTile, k.len);
          if (hidden_values_finite<T>(g, k.seq, hk, ta * kTile, min(rlo, end)) &&
              hidden_values_finite<T>(g, k.seq, hk, max(rhi, ta * kTile), end))
            continue;
          const unsigned long long qp = __shfl_sync(0xffffffffu, (unsigned long long)qrow, src);
          const unsigned long long op = __shfl_sync(0xffffffffu, (unsigned long long)orow, src);
          const long long orow_id = __shfl_sync(0xffffffffu, out_row, src);
          float m1, l1;
          float4 v = row_by_warp<T>(g, k.seq, hk, reinterpret_cast<const char *>(qp), rlo, rhi, m1, l1);
          const float f = l1 > 0.f || l1 != l1 ? 1.f / l1 : 0.f;
          if (4 * lane < g.c.d)
            reinterpret_cast<uint2 *>(op)[lane] = make_uint2(Bits<T>::pack(v.x * f, v.y * f), Bits<T>::pack(v.z * f, v.w * f));
          if (lane == 0 && g.lse) g.lse[orow_id] = l1 > 0.f || l1 != l1 ? m1 * 0.693147180559945309f + logf(l1) : -INFINITY;
        }
      }
    }
    if (opens) {
      named_sync(kTile * MT + 32);  // the check is over, and the rows' results are in
      if (bad_values && ok) put_back<T>(g, k.seq, k.tok0, k.base, k.len, k.rows, k.first, kRows, hk, split, warp, ta, tb);
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

// Joins the splits of each row: one warp per row, in the splits' order.
template <typename T>
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
      if (holds) {
        const float4 v = reinterpret_cast<const float4 *>(g.part + (s * rows + row) * g.c.d)[lane];
        acc.x += v.x * f, acc.y += v.y * f, acc.z += v.z * f, acc.w += v.w * f;
      }
    }
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  if (holds)
    reinterpret_cast<uint2 *>(orow)[lane] =
        make_uint2(Bits<T>::pack(acc.x * inv, acc.y * inv), Bits<T>::pack(acc.z * inv, acc.w * inv));
  if (g.lse && lane == 0) g.lse[row] = l > 0.f || l != l ? m * 0.693147180559945309f + logf(l) : -INFINITY;
}

// ---------------------------------------------------------------- host side
constexpr int kPairedTiles = 4;  // see Shape

struct Plan {
  bool few;               // tr_attend_few.cu's kernel
  int mt, slots;          // else k_attend's blocks of 128 mt rows
  bool paired;            // two CTAs an SM
  int splits, split_tiles;  // and the parts of the keys, in tiles
  size_t part_ml, total;  // workspace
};

Plan plan_of(const tr_cache *c, int q_heads, int window, int max_new, int max_len) {
  Plan p{};
  const int group = q_heads / c->heads;
  const long long most = (long long)(max_new < c->total_new ? max_new : c->total_new) * group;
  const int sms = sm_count() > 0 ? sm_count() : 1;
  // (its units, tiles of all blocks and key heads, are counted in 31 bits)
  const long long blocks16 = (long long)c->total_new * group / kFewRows + c->batch;
  const long long table_tiles = ((long long)c->max_pages * c->page + kTile - 1) / kTile + kFewItemCost;
  if (most <= kFewRows && c->batch <= kFewMaxBatch && blocks16 * c->heads <= INT_MAX / table_tiles) {
    p.few = true;
    p.total = few_workspace_bytes(c->head_dim, sms);
    return p;
  }
  const long long cap = (long long)c->max_pages * c->page;
  long long keys = max_len < cap ? max_len : cap;
  if (window > 0 && keys > (long long)window + max_new) keys = (long long)window + max_new;
  const int tiles = (int)((keys + kTile - 1) / kTile);
  p.paired = tiles <= kPairedTiles;
  p.mt = most <= kTile || p.paired ? 1 : 2;
  const int rows = kTile * p.mt;
  p.slots = (int)((long long)c->total_new * group / rows) + c->batch + 1;  // (tokens of no sequence: one more)
  if (p.paired) {
    p.splits = 1;
    p.split_tiles = tiles;
    return p;
  }
  // Parts of the keys: as many as finish earliest when `sms` CTAs run at a
  // time, one costing its tiles and about kCtaTiles more, and the join
  // writing and reading a row's fp32 sums once per part (kJoinRows rows in
  // the time of one tile).
  constexpr double kCtaTiles = 4.0, kJoinRows = 8192.0;
  const double blocks = (double)(p.slots - 1) * c->heads;
  double best = 0;
  for (int s = 1; s <= 64 && s <= (tiles > 1 ? tiles : 1); ++s) {
    const double waves = std::ceil(blocks * s / sms);
    const double t = waves * ((tiles + s - 1) / s + kCtaTiles) +
                     (s > 1 ? kCtaTiles + (double)c->total_new * q_heads * s / kJoinRows : 0.0);
    if (s == 1 || t < best) {
      best = t;
      p.splits = s;
    }
  }
  p.split_tiles = (tiles + p.splits - 1) / p.splits;
  if (p.splits > 1) {
    const size_t r = (size_t)c->total_new * q_heads * p.splits;
    p.part_ml = align_up(r * c->head_dim * sizeof(float), 256);
    p.total = p.part_ml + align_up(r * sizeof(float2), 256);
  }
  return p;
}

std::atomic<int> g_attend_smem_set[64];

template <typename T, int D, int MT, bool PAIRED>
cudaError_t launch_attend_t(const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &g, int slots,
                            cudaStream_t st) {
  using S = Shape<D, MT, PAIRED>;
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  const int bit = 1 << (Bits<T>::kBf16 * 6 + (D == 128) * 3 + (PAIRED ? 2 : MT - 1));
  if (!(g_attend_smem_set[dev & 63].load() & bit)) {
    err = cudaFuncSetAttribute(k_attend<T, D, MT, PAIRED>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
    if (err != cudaSuccess) return err;
    g_attend_smem_set[dev & 63].fetch_or(bit);
  }
  return launch_kernel(k_attend<T, D, MT, PAIRED>, dim3(slots, g.c.heads, g.splits), dim3(S::kThreads), S::kSmem, st,
                       false, mk, mv, g);
}

template <typename T, int D>
cudaError_t launch_attend_d(const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &g, const Plan &p,
                            cudaStream_t st) {
  return p.paired    ? launch_attend_t<T, D, 1, true>(mk, mv, g, p.slots, st)
         : p.mt == 1 ? launch_attend_t<T, D, 1, false>(mk, mv, g, p.slots, st)
                     : launch_attend_t<T, D, 2, false>(mk, mv, g, p.slots, st);
}

template <typename T>
cudaError_t launch_attend(const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &g, const Plan &p,
                          cudaStream_t st) {
  const cudaError_t err =
      g.c.d <= 64 ? launch_attend_d<T, 64>(mk, mv, g, p, st) : launch_attend_d<T, 128>(mk, mv, g, p, st);
  if (err != cudaSuccess || g.splits == 1) return err;
  const long long rows = (long long)g.c.total_new * g.q_heads;
  return launch_kernel(k_attend_join<T>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, true, g);
}

}  // namespace
}  // namespace tr

using namespace tr;

extern "C" {

size_t tr_cache_attend_workspace_bytes(const tr_cache *c, int32_t q_heads, int32_t window, int32_t max_new,
                                       int32_t max_len) {
  if (check_cache(c) != TR_OK || q_heads <= 0 || q_heads % c->heads || window < 0 || max_new < 0 || max_len < 0)
    return 0;
  return plan_of(c, q_heads, window, max_new, max_len).total;
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
  if ((long long)c->total_new * q->heads > INT_MAX - 65536) return TR_ERR_UNSUPPORTED;
  if (c->heads > 65535) return TR_ERR_UNSUPPORTED;
  if (c->total_new == 0) return TR_OK;
  const Plan p = plan_of(c, q->heads, window, max_new, max_len);
  if (p.total && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < p.total)) return TR_ERR_WORKSPACE;
  AttendArgs g{};
  g.c = cache_view(c);
  g.q = static_cast<const char *>(q->p);
  g.o = static_cast<char *>(o->p);
  g.q_tok = q->token_stride, g.q_head = q->head_stride;
  g.o_tok = o->token_stride, g.o_head = o->head_stride;
  g.q_heads = q->heads, g.group = q->heads / c->heads;
  g.lse = lse;
  // A zero scale becomes a factor too small to matter: -inf marks masked
  // scores, and -inf * 0 would be NaN.
  g.scale = fmaxf(fabsf(scale) * 1.44269504088896341f, 1e-30f);
  g.negate = scale < 0.f;
  g.causal = causal, g.window = window;
  g.splits = p.splits;
  g.split_tiles = p.split_tiles;
  while ((1 << g.page_log2) < c->page) ++g.page_log2;
  g.part = static_cast<float *>(ws);
  g.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(ws) + p.part_ml);
  g.err = d_error;
  CUtensorMap mk{}, mv{};
  const long long rows = (long long)c->pages * c->heads * c->page;
  const int box = c->page < kTile ? c->page : kTile;
  const CUtensorMapDataType type =
      c->dtype == TR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  // an empty cache keeps one row in the maps' extents: no page id is valid, so nothing reads it
  if (!make_map(&mk, c->k, rows > 0 ? rows : 1, c->head_dim, box, 64, CU_TENSOR_MAP_SWIZZLE_128B, type) ||
      !make_map(&mv, c->v, rows > 0 ? rows : 1, c->head_dim, box, 64, CU_TENSOR_MAP_SWIZZLE_128B, type))
    return TR_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (p.few) {
    g.ctas = sm_count() > 0 ? sm_count() : 1;
    return launch_few(mk, mv, g, c->dtype == TR_BF16, ws, st) == cudaSuccess ? TR_OK : TR_ERR_CUDA;
  }
  const cudaError_t err =
      c->dtype == TR_BF16 ? launch_attend<__nv_bfloat16>(mk, mv, g, p, st) : launch_attend<__half>(mk, mv, g, p, st);
  return err == cudaSuccess ? TR_OK : TR_ERR_CUDA;
}

}  // extern "C"
