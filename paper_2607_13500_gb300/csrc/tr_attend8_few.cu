// Attention of few rows per key head over the paged cache held in 8 bits:
// bound, like its 16-bit counterpart (tr_attend_few.cu, whose shares, walk and
// join it uses), by reading K and V once, and they are half as long.
//
// Codes become halves in registers, two at a time and exactly, on their way
// into warp-level products (m16n8k16), whose 16 keys are one block, so scales
// cost next to nothing:
//   K   one factor for the 16 keys' scores;
//   V   a factor of the block's probabilities: with m the row's maximum of the
//       scores s and L that of s + e, a probability enters the product as
//       2^(s - m) 2^(e + m - L), and 2^(L - m) enters the result.
// bf16 queries enter as halves as well, each row divided by a power of two.
// What enters the second product is taken times 2^6 (2^14 at most) and rounded
// to halves: it keeps its bits down to 2^-20 of what the row's greatest key
// adds, and what is lost below is 2^-31 of it.  (With V's scales relative to
// the largest of the tiles, keys that a row does not see would take its bits.)
//
// A consumer warp takes 32 keys of every second tile of 128, so that two tiles
// are under way and one's turning and exponentials stand beside the other's
// products (all eight warps on 16 keys each of every tile: one token of 64
// requests over 256 to 16384 keys 86 us, so 76).  A piece's queries and first
// scales come from a warp of their own, a piece ahead (62, so 59).
//
// 28 heads of 128 over 4, bf16: those 64 requests 60 us (4.1 TB/s: ragged
// lengths end in part tiles, and the join takes 3), with 16384 keys each 183 us
// (5.9 TB/s, 0.88 of a copy).  One token over 611 keys, 32 heads: 12.7 us of
// latencies in a row, and a second launch.
#include <atomic>

#include "tr_attend8.cuh"
#include "tr_attend_few.cuh"

namespace tr {
namespace {

using namespace attend8;
using namespace attend::few;

constexpr int kAllThreads = 32 * (kWarps + 4);  // consumers, the producers of K, of V and of queries, one more for whole warpgroups

// What a piece needs besides tiles, as the consumers' lanes take it.
template <int D>
struct Queries {
  uint4 q[D / 16][32];           // fragments of the first product, halves
  float scale[2][32];            // what a score of the lane's two rows is multiplied by, K's scale apart
  uint32_t blocks[kWarps][32];   // scales of each warp's two blocks of its first 16 tiles, in two lanes each
};

template <int D>
struct Few8 {
  static constexpr int kTileBytes = kTile * D;
  static constexpr int kQueryBytes = 2 * (int)sizeof(Queries<D>);  // the present piece's and the next one's
  // Rows joined at a time, each quarter of a row 4 floats on, so that a phase's stores lie in different banks.
  static constexpr int kRows = 8, kJoinRow = D + 16;
  static constexpr int kJoinBytes = kWarps * kRows * kJoinRow * 4;
  static constexpr int kFit = (227 * 1024 - 4096 - 1024 - kJoinBytes - kQueryBytes) / kTileBytes;
  static constexpr int kStages = kFit < 16 ? kFit : 16;
  static constexpr size_t kSmem = (size_t)kStages * kTileBytes + kJoinBytes + kQueryBytes + 1024 + 512;
};

constexpr int kLift = 6;  // what enters the second product is taken times 2^6 (and grows by 2^8 at most)
// A probability under 2^-126 becomes zero.  Times 2^100 at most, that is what the second product loses anyway (2^-31 of the
// greatest, which is 2^5 at least); where the factor is larger, what is more enters the exponential (and the sum, where
// such probabilities, 2^-86 at most, do not count).
constexpr float kMostLift = 100.f;

__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
  return v;
}

template <typename T, int D>
__global__ void __launch_bounds__(kAllThreads, 1)
    k_attend8_few(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ Attend8Args p) {
  using F = Few8<D>;
  using Ring = CodeRing<D, F::kStages>;
  const AttendArgs &g = p.a;
  extern __shared__ unsigned char smem_raw[];
  __shared__ int runs[kFewMaxBatch / 32];  // units of 32 sequences each
  __shared__ float tops[2][kWarps][kFewRows], tots[2][kWarps][kFewRows];  // (two: of a piece and the next one)
  __shared__ int bad, share0, share_units;  // bad: values were taken out of a tile
  const uint32_t base = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  float *join = reinterpret_cast<float *>(smem_raw + (base - tc::smem_u32(smem_raw)) + F::kStages * F::kTileBytes);
  Queries<D> *queries = reinterpret_cast<Queries<D> *>(reinterpret_cast<unsigned char *>(join) + F::kJoinBytes);
  const uint32_t bars = tc::smem_u32(join) + F::kJoinBytes + F::kQueryBytes;
  auto q_full = [&](int i) { return bars + 8u * (2 * F::kStages + i); };
  auto q_empty = [&](int i) { return bars + 8u * (2 * F::kStages + 2 + i); };
  // (the warp's index by shuffle: the compiler then knows it to be uniform)
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

  Ring ring;
  ring.base = base, ring.full0 = bars, ring.empty0 = bars + 8u * F::kStages;
  if (threadIdx.x == 0) {
    for (int s = 0; s < F::kStages; ++s) {
      tc::mbar_init(ring.full(s), 1);
      tc::mbar_init(ring.empty(s), kWarps / 2);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(q_full(i), 1);
      tc::mbar_init(q_empty(i), kWarps);
    }
    tc::mbar_fence_init();
    tc::tma_prefetch_map(&map_k);
    tc::tma_prefetch_map(&map_v);
    bad = 0;
  }
  pdl_wait();  // q and the cache come from the kernels before
  pdl_trigger();
  __syncthreads();  // the barriers are ready
  Walk<kItemCost> w;
  Seq run0;
  const Shares shares(count_units<kItemCost>(g, runs, kWarps + 4, run0), g.ctas);
  const int share = shares.start(blockIdx.x), share_end = shares.start(blockIdx.x + 1);
  if (share >= share_end) return;
  if (threadIdx.x == 0) share0 = share, share_units = share_end - share;  // for the consumers' second walk
  w.seek(g, runs, run0, share, share_end);

  // Of the share's tiles warps 0 to 3 take the even ones and 4 to 7 the odd
  // ones, a quarter each: 32 keys, two blocks.  The block of warp x's nth tile
  // (of a piece that `tiles` came before; nth and the 15 on) that the lane holds
  // the scales of:
  constexpr int kPieces = D / 64;          // 16-byte pieces of a key's row a lane takes
  constexpr int kTiles = D / 8;            // n-tiles of the second product
  const int gq = lane >> 2, c = lane & 3;  // quad (row or key of a fragment), lane of the quad
  auto key_of = [&](int x, int tiles, int tile, int count, int len, int nth) {
    const int n = ((tiles ^ (x >> 2)) & 1) + 2 * (nth + (lane >> 1));
    return n < count ? (tile + n) * kTile + 32 * (x & 3) + 16 * (lane & 1) : len;
  };
  if (warp >= kWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == kWarps + 2) {
      // ---------------------------------------------------------------- queries, and each piece's first scales
      // By a warp of its own, a piece ahead: what a piece needs takes two waits
      // for memory one after the other, and a row's largest magnitude.
      int n = 0, tiles = 0;
      while (w.next(g)) {
        const int hk = w.item % g.c.heads, block0 = w.item / g.c.heads * kFewRows;
        const int rows = min(kFewRows, w.s.rows - block0);
        int page[kWarps];
#pragma unroll
        for (int x = 0; x < kWarps; ++x) {
          const int j = key_of(x, tiles, w.tile, w.count, w.s.len, 0), i = j >> g.page_log2;
          page[x] = j < w.s.len && i < g.c.max_pages ? __ldg(g.c.table + (long long)w.seq() * g.c.max_pages + i) : -1;
        }
        uint32_t raw[2][kPieces * 8];  // the lane's channels of its two rows
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = gq + 8 * i, row = block0 + r;
          const bool valid = r < rows;
          const int tok = valid ? row / g.group : 0, head = hk * g.group + (valid ? row - tok * g.group : 0);
          const char *qrow = g.q + 2 * ((long long)(w.s.tok0 + tok) * g.q_tok + (long long)head * g.q_head);
#pragma unroll
          for (int s = 0; s < 2 * kPieces; ++s) {
            const int ch = kPieces * c * 16 + 8 * s;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (valid && ch < g.c.d) v = *reinterpret_cast<const uint4 *>(qrow + 2 * ch);
            raw[i][4 * s] = v.x, raw[i][4 * s + 1] = v.y, raw[i][4 * s + 2] = v.z, raw[i][4 * s + 3] = v.w;
          }
        }
        uint32_t blocks[kWarps];
#pragma unroll
        for (int x = 0; x < kWarps; ++x) {
          const int j = key_of(x, tiles, w.tile, w.count, w.s.len, 0);
          blocks[x] = (unsigned)page[x] < (unsigned)g.c.pages ? scales_at(p, scale_at(g.c, page[x], hk, j & (g.c.page - 1))) : kNoScales;
        }
        Queries<D> &out = queries[n & 1];
        if (!tc::mbar_wait_warp(q_empty(n & 1), (n >> 1 & 1) ^ 1)) {
          if (lane == 0) flag(g, TR_CACHE_ERR_WAIT);
          break;
        }
#pragma unroll
        for (int x = 0; x < kWarps; ++x) out.blocks[x][lane] = blocks[x];
        const uint32_t flip = g.negate ? 0x80008000u : 0u;
        float down[2] = {1.f, 1.f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float scale = g.scale;
          if (Bits<T>::kBf16) {
            uint32_t most = 0u;
#pragma unroll
            for (int k = 0; k < 8 * kPieces; ++k) most = max(most, top_of_pair(raw[i][k]));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const int e = query_exp(most);
            down[i] = pow2(-e);
            scale *= pow2(e);
          }
          out.scale[i][lane] = scale;
        }
#pragma unroll
        for (int m = 0; m < 4 * kPieces; ++m) {
          // a0, a2: the row g's first and second pair of channels 4 m .. 4 m + 3 of the lane's; a1, a3: row g + 8's
          uint32_t a[4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            a[i] = (Bits<T>::kBf16 ? query_pair(raw[i][2 * m], down[i]) : raw[i][2 * m]) ^ flip;
            a[2 + i] = (Bits<T>::kBf16 ? query_pair(raw[i][2 * m + 1], down[i]) : raw[i][2 * m + 1]) ^ flip;
          }
          out.q[m][lane] = make_uint4(a[0], a[1], a[2], a[3]);
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(q_full(n & 1));
        tiles += w.count;
        ++n;
      }
      return;
    }
    if (warp > kWarps + 2) return;
    ring.take(warp - kWarps);
    const CUtensorMap *map = warp == kWarps ? &map_k : &map_v;
    bool ok = true;
    while (ok && w.next(g)) {
      const int hk = w.item % g.c.heads, end = w.tile + w.count;
      ring.seen = keys_of_seq(g, w.s);
      int id = ring.page_id(g, w.seq(), w.s.len, w.tile);
      for (int t = w.tile; t < end && ok; ++t) {
        const int next = t + 1 < end ? ring.page_id(g, w.seq(), w.s.len, t + 1) : -1;
        ok = ring.load(g, map, id, w.s.len, hk, t);
        id = next;
      }
    }
    if (!ok && lane == 0) flag(g, TR_CACHE_ERR_WAIT);
    ring.drain();
    return;
  }

  // ------------------------------------------------------------------ consumers
  asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");  // (with 88 what 168 at launch give)
  const int odd = warp >> 2, quarter = warp & 3;
  int kst = Ring::first(0), vst = Ring::first(1);
  uint32_t kph = 0, vph = 0;
  int tiles = 0;   // of the share so far
  bool ok = true;  // once a wait has timed out the warp only keeps up with the others' barriers
  struct Piece {
    int hk, block0, rows, tok0, base, len, seq, tile, count;
    bool whole, starts;
  } now;
  auto next_piece = [&](Piece &x) {
    if (!w.next(g)) return false;
    x.hk = w.item % g.c.heads, x.block0 = w.item / g.c.heads * kFewRows;
    x.rows = min(kFewRows, w.s.rows - x.block0);
    x.tok0 = w.s.tok0, x.base = w.s.base, x.len = w.s.len, x.seq = w.seq();
    x.tile = w.tile, x.count = w.count, x.whole = w.whole, x.starts = w.starts;
    return true;
  };
  int nth_piece = 0;
  for (bool more = next_piece(now); more; ++nth_piece) {
    const int turn = nth_piece & 1;
    auto scales = [&](int nth) {
      return block_scales(p, now.seq, now.hk, now.len, key_of(warp, tiles, now.tile, now.count, now.len, nth));
    };
    // this lane's two rows of a fragment, and the keys they see
    int lo[2], hi[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = gq + 8 * i;
      const bool valid = r < now.rows;
      const int own = now.base + (valid ? (now.block0 + r) / g.group : 0);
      hi[i] = !valid ? INT_MAX : g.causal ? min(now.len, own + 1) : now.len;
      lo[i] = valid && g.window > 0 ? window_start(own, g.window) : 0;
    }
    if (ok) {
      ok = tc::mbar_wait_warp(q_full(turn), (uint32_t)(nth_piece >> 1) & 1u);
      if (!ok && lane == 0) flag(g, TR_CACHE_ERR_WAIT);
    }
    const Queries<D> &in = queries[turn];
    uint32_t q[kPieces * 4][4];
#pragma unroll
    for (int m = 0; m < 4 * kPieces; ++m) {
      const uint4 v = in.q[m][lane];
      q[m][0] = v.x, q[m][1] = v.y, q[m][2] = v.z, q[m][3] = v.w;
    }
    const float fr[2] = {in.scale[0][lane], in.scale[1][lane]};
    uint32_t ahead = in.blocks[warp][lane];
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(q_empty(turn));
    float held_k = 1.f;   // 2^e of keys
    int held_v = 0;       // e of values
    float o[kTiles][4];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
    // m and L, whole numbers (less than 8 too low: they follow in steps)
    float mx[2] = {-INFINITY, -INFINITY}, wx[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};

    int nth = 0;  // of this warp's tiles
    for (int n0 = 0; ok && n0 < now.count; ++n0) {
      if (((tiles + n0) & 1) != odd) {
        Ring::on(0, kst, kph);
        Ring::on(1, vst, vph);
        continue;
      }
      const int t = now.tile + n0;
      if ((nth & 15) == 0) {  // the next 16 tiles' scales, long before they are needed
        held_k = pow2((int)(ahead & 0xffu) - 127);
        held_v = ahead >> 8 < 255u ? (int)(ahead >> 8) - 127 : -127;
        ahead = scales(nth + 16);
      }
      float fk[2];
      int ev[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        fk[h] = __shfl_sync(0xffffffffu, held_k, 2 * (nth & 15) + h);
        ev[h] = __shfl_sync(0xffffffffu, held_v, 2 * (nth & 15) + h);
      }
      ++nth;
      // ---- scores of 32 keys: four products of 8 keys
      ok = __all_sync(0xffffffffu, tc::mbar_wait(ring.full(kst), kph));
      if (!ok) {
        if (lane == 0) flag(g, TR_CACHE_ERR_WAIT);
        break;
      }
      const uint32_t kt = base + kst * F::kTileBytes + 32 * quarter * D;
      float s[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = 0.f;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
          const uint4 v = lds128(kt + Ring::piece(8 * n + gq, kPieces * c + j));
          const uint32_t *word = &v.x;
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            uint32_t b0, b1;
            halves4(word[m], b0, b1);
            mma16816<__half>(s[n], q[4 * j + m][0], q[4 * j + m][1], q[4 * j + m][2], q[4 * j + m][3], b0, b1);
          }
        }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(ring.empty(kst));
      Ring::on(0, kst, kph);

      // ---- the values' codes: of keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9 of each block
      ok = __all_sync(0xffffffffu, tc::mbar_wait(ring.full(vst), vph));
      if (!ok) {
        if (lane == 0) flag(g, TR_CACHE_ERR_WAIT);
        break;
      }
      const uint32_t vt = base + vst * F::kTileBytes + 32 * quarter * D;
      uint32_t v[2][4][D / 32];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = 16 * h + 2 * c + (j & 1) + 8 * (j >> 1);
          if (D == 128) {
            const uint4 x = lds128(vt + Ring::piece(key, gq));
            v[h][j][0] = x.x, v[h][j][1] = x.y, v[h][j][D / 32 - 2] = x.z, v[h][j][D / 32 - 1] = x.w;
          } else {
            const uint2 x = lds64(vt + Ring::piece(key, gq >> 1) + 8 * (gq & 1));
            v[h][j][0] = x.x, v[h][j][1] = x.y;
          }
        }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(ring.empty(vst));
      Ring::on(1, vst, vph);

      // ---- softmax: s[n][0..1] row g, s[n][2..3] row g + 8, keys 8 n + 2 c and + 1
      const int key0 = t * kTile + 32 * quarter;
      const bool ends = key0 + 32 > now.len;
      const int most = min(key0 + 32, now.len);  // open: some row does not see some of the sequence's keys here
      const bool open = __any_sync(0xffffffffu, lo[0] > key0 || hi[0] < most || lo[1] > key0 || hi[1] < most);
      if (open || ends) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int key = key0 + 8 * n + 2 * c + (j & 1);
            if (key < lo[j >> 1] || key >= hi[j >> 1]) s[n][j] = -INFINITY;
          }
        bool found = false;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const bool behind = key0 + 16 * h + 2 * c + (j & 1) + 8 * (j >> 1) >= now.len;  // it may be NaN there
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
              if (behind) v[h][j][i] = 0u;
              if (open) found |= clean_codes(v[h][j][i]);
            }
          }
        if (found) bad = 1;  // (any thread's word will do)
      }
      float peak[2][2], fs[2][2];  // of the lane's two rows and the two blocks
      bool over = false;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          fs[i][h] = block_factor(fr[i], fk[h]);
          peak[i][h] = fmaxf(fmaxf(s[2 * h][2 * i], s[2 * h][2 * i + 1]), fmaxf(s[2 * h + 1][2 * i], s[2 * h + 1][2 * i + 1])) * fs[i][h];
          over |= peak[i][h] > mx[i] + 8.f || peak[i][h] + (float)ev[h] > wx[i] + 8.f;
        }
      if (__any_sync(0xffffffffu, over)) {
        float f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float m = fmaxf(peak[i][0], peak[i][1]), x = fmaxf(peak[i][0] + (float)ev[0], peak[i][1] + (float)ev[1]);
#pragma unroll
          for (int d = 1; d < 4; d <<= 1) {
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
          }
          m = ceilf(m), x = ceilf(x);
          if (m > mx[i]) sum[i] *= exp2_fast(mx[i] - m), mx[i] = m;
          f[i] = 1.f;
          if (x > wx[i]) f[i] = exp2_fast(wx[i] - x), wx[i] = x;
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          o[i][0] *= f[0], o[i][1] *= f[0];
          o[i][2] *= f[1], o[i][3] *= f[1];
        }
      }
      uint32_t pr[2][4];  // the A fragments of the second product
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float lift = (float)(ev[h] + kLift) + (mx[i] - wx[i]), f = fs[i][h];
          const float neg = (mx[i] == -INFINITY ? 0.f : -mx[i]) + fmaxf(lift - kMostLift, 0.f);
          const float by = pow2((int)fmaxf(fminf(lift, kMostLift), -126.f));  // (NaN where the row has seen nothing: times zeros)
          float p0[2], p1[2];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            p0[n] = exp2_fast(fmaf(s[2 * h + n][2 * i], f, neg)), p1[n] = exp2_fast(fmaf(s[2 * h + n][2 * i + 1], f, neg));
            pr[h][2 * n + i] = Bits<__half>::pack(p0[n] * by, p1[n] * by);
          }
          sum[i] += (p0[0] + p1[0]) + (p0[1] + p1[1]);
        }

      // ---- o += p V: n-tile i holds channels D / 8 g + i
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            // channels 4 i + 2 j and + 1 of a pair of keys: one after the other
            uint32_t a0, a1, b0, b1;
            halves4(__byte_perm(v[h][0][i], v[h][1][i], j ? 0x7362u : 0x5140u), a0, a1);
            halves4(__byte_perm(v[h][2][i], v[h][3][i], j ? 0x7362u : 0x5140u), b0, b1);
            mma16816<__half>(o[4 * i + 2 * j], pr[h][0], pr[h][1], pr[h][2], pr[h][3], a0, b0);
            mma16816<__half>(o[4 * i + 2 * j + 1], pr[h][0], pr[h][1], pr[h][2], pr[h][3], a1, b1);
          }
    }
    // ------------------------------------------------------------------ the piece's result
    const Piece done = now;
    tiles += done.count;
    more = next_piece(now);
    float(&top)[kWarps][kFewRows] = tops[turn], (&tot)[kWarps][kFewRows] = tots[turn];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
      if (c == 0) top[warp][gq + 8 * i] = mx[i], tot[warp][gq + 8 * i] = sum[i];
    }
    named_sync(32 * kWarps);  // (and the last piece's results are read)
    // The row's maximum and sum over the warps.  (A maximum passes over NaN
    // scores, so a warp that saw no other has the maximum of one that saw
    // nothing: its sum, 0 or NaN, enters as it is.)
    auto row_total = [&](int r, float &m, float &l) {
      m = -INFINITY, l = 0.f;
#pragma unroll
      for (int j = 0; j < kWarps; ++j) m = fmaxf(m, top[j][r]);
#pragma unroll
      for (int j = 0; j < kWarps; ++j) l += top[j][r] == -INFINITY ? tot[j][r] : tot[j][r] * exp2_fast(top[j][r] - m);
    };
    const int part = 2 * blockIdx.x + (done.starts ? 1 : 0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r0 = 8 * i;
      if (r0 >= done.rows) break;
      if (i) named_sync(32 * kWarps);
      // Sums are divided by the row's total before V's scale, up to 2^127, enters.
      float m, l;
      row_total(gq + r0, m, l);
      const float up = mx[i] == -INFINITY ? 0.f : exp2_fast(0.5f * (wx[i] - (float)kLift - m));  // in two steps: it may be 2^-140
      const float f = (l > 0.f || l != l ? 1.f / l : 0.f) * up;
      // accumulator column 2 c + (j & 1) of n-tile k is channel D / 8 (2 c + (j & 1)) + k
      float *dst = join + (warp * F::kRows + gq) * F::kJoinRow + (2 * kTiles + 4) * c;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int k = 0; k < kTiles; k += 4)
          *reinterpret_cast<float4 *>(dst + kTiles * b + k) =
              make_float4(o[k][2 * i + b] * f * up, o[k + 1][2 * i + b] * f * up, o[k + 2][2 * i + b] * f * up,
                          o[k + 3][2 * i + b] * f * up);
      named_sync(32 * kWarps);
      const int r = r0 + (int)threadIdx.x / (D / 4), ch = (int)threadIdx.x % (D / 4) * 4;
      if ((int)threadIdx.x < F::kRows * (D / 4) && r < done.rows && ch < g.c.d) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < kWarps; ++j) {
          const float4 x = *reinterpret_cast<const float4 *>(join + (j * F::kRows + r - r0) * F::kJoinRow + ch + ch / (D / 4) * 4);
          v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
        }
        row_total(r, m, l);
        put_row<T, true>(g, done.whole, done.tok0, part, done.block0, done.hk, r, ch, v, m, l);
      }
    }
  }

  // What was taken out of open tiles goes to the rows that see it, when the
  // share's tiles are all used up.
  named_sync(32 * kWarps);  // the rows written by other warps
  if (!ok || !bad) return;
  w.seek(g, runs, seq_of(g, lane), share0, share0 + share_units);
  while (w.next(g)) {
    const int hk = w.item % g.c.heads, block0 = w.item / g.c.heads * kFewRows;
    const int rows = min(kFewRows, w.s.rows - block0), part = 2 * blockIdx.x + (w.starts ? 1 : 0);
    for_bad_codes(g, edges_of_rows(g, w.s.base, w.s.len, block0, block0 + rows), w.seq(), hk, w.tile, w.tile + w.count,
                  [&](int j, const float4 &v) {
                    for (int r = warp; r < rows; r += kWarps) {
                      const int tok = (block0 + r) / g.group, head = hk * g.group + (block0 + r) % g.group;
                      const int own = w.s.base + tok;
                      if ((g.causal && j > own) || (g.window > 0 && j < window_start(own, g.window))) continue;
                      add_to_row<T>(g.o + 2 * ((long long)(w.s.tok0 + tok) * g.o_tok + (long long)head * g.o_head),
                                    w.whole ? nullptr : g.part + ((long long)part * kFewRows + r) * g.c.d, v);
                    }
                  });
  }
}

std::atomic<int> g_few8_smem_set[64];

template <typename T, int D>
cudaError_t launch_few8_t(const CUtensorMap &mk, const CUtensorMap &mv, const Attend8Args &p, int variant, cudaStream_t st) {
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  if (!(g_few8_smem_set[dev & 63].load() & (1 << variant))) {
    err = cudaFuncSetAttribute(k_attend8_few<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Few8<D>::kSmem);
    if (err != cudaSuccess) return err;
    g_few8_smem_set[dev & 63].fetch_or(1 << variant);
  }
  err = launch_kernel(k_attend8_few<T, D>, dim3(p.a.ctas), dim3(kAllThreads), Few8<D>::kSmem, st, false, mk, mv, p);
  if (err != cudaSuccess) return err;
  const long long rows = (long long)p.a.c.total_new * p.a.q_heads;
  return launch_kernel(k_few_join<T, true, kItemCost>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, true, p.a);
}

}  // namespace

namespace attend8 {

cudaError_t launch_few8(const CUtensorMap &mk, const CUtensorMap &mv, Attend8Args p, bool bf16, void *ws, cudaStream_t st) {
  p.a.part = static_cast<float *>(ws);
  p.a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(ws) + few::part_bytes(p.a.c.d, p.a.ctas));
  if (bf16)
    return p.a.c.d <= 64 ? launch_few8_t<__nv_bfloat16, 64>(mk, mv, p, 0, st)
                         : launch_few8_t<__nv_bfloat16, 128>(mk, mv, p, 1, st);
  return p.a.c.d <= 64 ? launch_few8_t<__half, 64>(mk, mv, p, 2, st) : launch_few8_t<__half, 128>(mk, mv, p, 3, st);
}

}  // namespace attend8
}  // namespace tr
