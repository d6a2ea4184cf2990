// Attention of few rows per key head (single tokens, short drafts) over the
// paged cache: bound by reading K and V once, so everything serves that.
//
// Work is counted in units of one 128-key tile of one key head (and block of
// 16 rows) and cut into equal shares, one per CTA and one CTA per SM,
// whatever the sequences' lengths: a share covers a run of tiles that may
// cross heads and sequences.  The lengths are read on the device, so a
// captured graph stays balanced as they grow.  An item (block, key head)
// that lies in one share is finished there; one that is cut leaves a partial
// (maximum, sum, weighted values) per share, joined by k_few_join.
//
// Two warps fill the tile ring by TMA; eight warps take 16 keys of each tile
// and run both products on warp-level tensor-core instructions (m16n8k16)
// from registers: at up to 16 rows the 128-row tcgen05 shapes would compute
// mostly padding and put a tensor-memory round trip between the products,
// while here the scores never leave the registers of the warp.  The order of
// channels inside a product is free, so each lane takes whole 16-byte chunks
// of K rows (chunk 2 c + s of lane (g, c): the 128-byte swizzle spreads them
// over all banks) and the queries are laid out to match; for V a lane takes
// 8 channels of four keys and pairs keys with byte permutes.
//
// Measured on GB300, bf16, heads of 128, both kernels: one token of 64 requests
// over 256 to 16384 keys, 28/4 heads, 88 us (480 MB: 5.5 TB/s of the measured
// 6.77 copy); one token of one request over 611 keys, 32 heads, 10.8 us in a
// graph (latency: launch, lengths, page ids, one tile, join).  With heads of 128
// the 168 registers of a thread spill 16 bytes.
#include <atomic>

#include "tr_attend.cuh"

namespace tr {
namespace {

using namespace attend;

constexpr int kWarps = 8;                     // consumer warps: 16 keys of a tile each
constexpr int kThreads = 32 * (kWarps + 2);   // and the producers of K and of V
constexpr int kPass = 4;                      // rows joined per pass at an item's end

template <int D>
struct Few {
  static constexpr int kHalves = D / 64;
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kJoinRow = D + 4;  // floats
  static constexpr int kJoinBytes = kWarps * kPass * kJoinRow * 4;
  static constexpr int kFit = (227 * 1024 - 4096 - 1024 - kJoinBytes) / kTileBytes;
  static constexpr int kStages = kFit < 12 ? kFit : 12;
  static constexpr size_t kSmem = (size_t)kStages * kTileBytes + kJoinBytes + 1024 + 4096;
};

// What a sequence brings: its rows and the tiles that some row of it sees.
struct Seq {
  int tok0, rows, len, base;
  int tile0, tiles;  // first tile, tiles
  int items;         // blocks of rows x key heads
};
__device__ __forceinline__ Range keys_of_seq(const AttendArgs &g, const Seq &s) {
  Block k;
  k.len = s.len;
  k.base = s.base;
  return keys_of_rows(g, k, 0, s.rows);
}
__device__ __forceinline__ Seq seq_of(const AttendArgs &g, int b) {
  Seq s{0, 0, 0, 0, 0, 0, 0};
  if (b >= g.c.batch) return s;
  const int t0 = __ldg(g.c.cu_new + b), t1 = min(__ldg(g.c.cu_new + b + 1), g.c.total_new);
  if (t0 < 0 || t1 <= t0) return s;
  s.tok0 = t0;
  s.rows = (t1 - t0) * g.group;
  s.len = cache_len(g.c, b);
  s.base = max(__ldg(g.c.lens + b), 0) - (t1 - t0);
  const Range r = keys_of_seq(g, s);
  s.tile0 = r.lo / kTile;
  s.tiles = (r.hi + kTile - 1) / kTile - s.tile0;
  s.items = (s.rows + kFewRows - 1) / kFewRows * g.c.heads;
  return s;
}
// An item counts kExtra units before its tiles', the time that taking it up
// and finishing it cost (about 3 us against 1.3 us a tile): without them the
// shares that hold many short items end last.
constexpr int kExtra = kFewItemCost;
__device__ __forceinline__ int units_of(const Seq &s) { return s.tiles > 0 ? s.items * (s.tiles + kExtra) : 0; }

// Share c of `all` units over `ctas` CTAs: the first all % ctas shares are
// one unit longer.
struct Shares {
  int size, longer;
  __device__ __forceinline__ Shares(int all, int ctas) : size(all / ctas), longer(all % ctas) {}
  __device__ __forceinline__ int start(int c) const { return c * size + min(c, longer); }
  __device__ __forceinline__ int of(int unit) const {
    const int head = longer * (size + 1);
    return unit < head ? unit / (size + 1) : longer + (unit - head) / max(size, 1);
  }
};

// The sequences 32 at a time, a lane each.
__device__ __forceinline__ Seq seq_from(const Seq &mine, int lane) {
  Seq s;
  s.tok0 = __shfl_sync(0xffffffffu, mine.tok0, lane);
  s.rows = __shfl_sync(0xffffffffu, mine.rows, lane);
  s.len = __shfl_sync(0xffffffffu, mine.len, lane);
  s.base = __shfl_sync(0xffffffffu, mine.base, lane);
  s.tile0 = __shfl_sync(0xffffffffu, mine.tile0, lane);
  s.tiles = __shfl_sync(0xffffffffu, mine.tiles, lane);
  s.items = __shfl_sync(0xffffffffu, mine.items, lane);
  return s;
}

// Total units, and `mine` = this lane's sequence of the first run.  With more
// than one run their units are left in shared memory by all warps together.
__device__ __forceinline__ int count_units(const AttendArgs &g, int *runs, int warps, Seq &mine) {
  const int lane = threadIdx.x & 31;
  const int n = (g.c.batch + 31) / 32;
  mine = seq_of(g, lane);
  if (n <= 1) return (int)__reduce_add_sync(0xffffffffu, (unsigned)units_of(mine));
  for (int i = threadIdx.x >> 5; i < n; i += warps) {
    const int u = (int)__reduce_add_sync(0xffffffffu, (unsigned)units_of(seq_of(g, 32 * i + lane)));
    if (lane == 0) runs[i] = u;
  }
  __syncthreads();
  int all = 0;
  for (int i = lane; i < n; i += 32) all += runs[i];
  return (int)__reduce_add_sync(0xffffffffu, (unsigned)all);
}

// A walk over the units of a share, item by item; the same in all lanes
// (but `mine`).
struct Walk {
  int u, end;  // next unit, end of the share
  int first;   // first unit of the sequence
  int run, at; // the sequence: its run of 32, its lane
  Seq mine;    // this lane's sequence of the run
  Seq s;       // the sequence
  // the current piece
  int item, tile, count;  // item of the sequence, first tile (absolute), tiles
  bool whole;             // the piece is the whole item
  bool starts;            // it holds the item's first tile

  __device__ __forceinline__ int seq() const { return 32 * run + at; }
  __device__ __forceinline__ void seek(const AttendArgs &g, const int *runs, const Seq &run0, int from, int to) {
    const int lane = threadIdx.x & 31, n = (g.c.batch + 31) / 32;
    u = from;
    end = to;
    first = 0;
    run = 0;
    mine = run0;
    if (n > 1) {
      while (run + 1 < n && u >= first + runs[run]) first += runs[run++];
      if (run) mine = seq_of(g, 32 * run + lane);
    }
    const int own = units_of(mine);
    int before = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += v;
    }
    at = max(__ffs(__ballot_sync(0xffffffffu, u < first + before)), 1) - 1;
    first += __shfl_sync(0xffffffffu, before - own, at);
    s = seq_from(mine, at);
  }
  // The next piece; false at the end of the share.
  __device__ __forceinline__ bool next(const AttendArgs &g) {
    while (u < end) {
      if (u >= first + units_of(s)) {  // on to the next sequence that has units
        first += units_of(s);
        unsigned any = __ballot_sync(0xffffffffu, units_of(mine) > 0) & ~(at == 31 ? 0xffffffffu : (2u << at) - 1u);
        while (!any && 32 * (run + 1) < g.c.batch) {
          mine = seq_of(g, 32 * ++run + (threadIdx.x & 31));
          any = __ballot_sync(0xffffffffu, units_of(mine) > 0);
        }
        if (!any) return false;
        at = __ffs(any) - 1;
        s = seq_from(mine, at);
      }
      if (s.tiles <= 0) return false;
      const int rel = u - first, each = s.tiles + kExtra;
      item = rel / each;
      const int t = rel - item * each, n = min(each - t, end - u);
      const int from = max(t - kExtra, 0);
      count = t + n - kExtra - from;
      tile = s.tile0 + from;
      whole = count == s.tiles;
      starts = from == 0;
      u += n;
      if (count > 0) return true;  // (else only the item's own units: its tiles are the next share's)
    }
    return false;
  }
};

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  if (Bits<T>::kBf16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ void named_sync(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }

// Four channels of row r of the piece: into the output, or into its share's
// partial result.
template <typename T>
__device__ __forceinline__ void put_row(const AttendArgs &g, const Walk &w, int part, int block0, int hk, int r, int ch,
                                        const float4 &v, float m, float l) {
  if (w.whole) {
    const int row = block0 + r, tok = row / g.group, head = hk * g.group + row - tok * g.group;
    const long long t = w.s.tok0 + tok;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    *reinterpret_cast<uint2 *>(g.o + 2 * (t * g.o_tok + (long long)head * g.o_head + ch)) =
        make_uint2(Bits<T>::pack(v.x * inv, v.y * inv), Bits<T>::pack(v.z * inv, v.w * inv));
    if (ch == 0 && g.lse) g.lse[t * g.q_heads + head] = l > 0.f || l != l ? m * 0.693147180559945309f + logf(l) : -INFINITY;
  } else {
    *reinterpret_cast<float4 *>(g.part + ((long long)part * kFewRows + r) * g.c.d + ch) = v;
    if (ch == 0) g.part_ml[part * kFewRows + r] = make_float2(m, l);
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
    k_attend_few(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const __grid_constant__ AttendArgs g) {
  using F = Few<D>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ int runs[kFewMaxBatch / 32];  // units of 32 sequences each
  __shared__ float top[kWarps][kFewRows], tot[kWarps][kFewRows];
  __shared__ int bad, share0, share_units;  // bad: values were taken out of a tile
  const uint32_t base = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  float *join = reinterpret_cast<float *>(smem_raw + (base - tc::smem_u32(smem_raw)) + F::kStages * F::kTileBytes);
  const uint32_t bars = tc::smem_u32(join) + F::kJoinBytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  TileRing<D, F::kStages, false> ring;
  ring.base = base, ring.full0 = bars, ring.empty0 = bars + 8u * F::kStages, ring.raw0 = 0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < F::kStages; ++s) {
      tc::mbar_init(ring.full(s), 1);
      tc::mbar_init(ring.empty(s), kWarps);
    }
    tc::mbar_fence_init();
    tc::tma_prefetch_map(&map_k);
    tc::tma_prefetch_map(&map_v);
    bad = 0;
  }
  pdl_wait();  // q and the cache come from the kernels before
  pdl_trigger();
  __syncthreads();  // the barriers are ready
  Walk w;
  Seq run0;
  const Shares shares(count_units(g, runs, kWarps + 2, run0), g.ctas);
  const int share = shares.start(blockIdx.x), share_end = shares.start(blockIdx.x + 1);
  if (share >= share_end) return;
  if (threadIdx.x == 0) share0 = share, share_units = share_end - share;  // for the consumers' second walk
  w.seek(g, runs, run0, share, share_end);

  if (warp >= kWarps) {
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
  const int gq = lane >> 2, c = lane & 3;  // quad (row or key of a fragment), lane of the quad
  using Ring = TileRing<D, F::kStages, false>;
  int kst = Ring::first(0), vst = Ring::first(1);
  uint32_t kph = 0, vph = 0;
  bool ok = true;  // once a wait has timed out the warp only keeps up with the others' barriers
  while (w.next(g)) {
    const int hk = w.item % g.c.heads, block0 = w.item / g.c.heads * kFewRows;
    const int rows = min(kFewRows, w.s.rows - block0);
    // this lane's two rows of a fragment, and the keys they see
    const char *qrow[2];
    int lo[2], hi[2];
    uint32_t q[F::kHalves * 2][8];  // [half, chunk parity][row g: 4 words, row g + 8: 4 words]
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = gq + 8 * i, row = block0 + r;
      const bool valid = r < rows;
      const int tok = valid ? row / g.group : 0, head = hk * g.group + (valid ? row - tok * g.group : 0);
      const int own = w.s.base + tok;
      hi[i] = !valid ? INT_MAX : g.causal ? min(w.s.len, own + 1) : w.s.len;
      lo[i] = valid && g.window > 0 ? window_start(own, g.window) : 0;
      qrow[i] = g.q + 2 * ((long long)(w.s.tok0 + tok) * g.q_tok + (long long)head * g.q_head);
      const uint32_t flip = g.negate ? 0x80008000u : 0u;
#pragma unroll
      for (int s = 0; s < F::kHalves * 2; ++s) {
        const int ch = (s >> 1) * 64 + (2 * c + (s & 1)) * 8;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (valid && ch < g.c.d) {
          v = *reinterpret_cast<const uint4 *>(qrow[i] + 2 * ch);
          v.x ^= flip, v.y ^= flip, v.z ^= flip, v.w ^= flip;
        }
        q[s][4 * i] = v.x, q[s][4 * i + 1] = v.y, q[s][4 * i + 2] = v.z, q[s][4 * i + 3] = v.w;
      }
    }
    float o[F::kHalves][8][4];
#pragma unroll
    for (int h = 0; h < F::kHalves; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[h][i][j] = 0.f;
    float mx[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};

    for (int t = w.tile; ok && t < w.tile + w.count; ++t) {
      // ---- scores of 16 keys: two products of 8 keys
      ok = __all_sync(0xffffffffu, tc::mbar_wait(ring.full(kst), kph));
      if (!ok) {
        if (lane == 0) flag(g, TR_CACHE_ERR_WAIT);
        break;
      }
      const uint32_t kt = base + kst * F::kTileBytes + (uint32_t)(16 * warp) * 128u;
      float s[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        // two chains of products, so that one's latency hides the other's
        float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < F::kHalves * 2; ++j) {
          const uint4 v = lds128(kt + (j >> 1) * (kTile * 128) + (8 * n + gq) * 128 + (((2 * c + (j & 1)) ^ gq) << 4));
          mma16816<T>(x, q[j][0], q[j][4], q[j][1], q[j][5], v.x, v.y);
          mma16816<T>(y, q[j][2], q[j][6], q[j][3], q[j][7], v.z, v.w);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = x[i] + y[i];
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(ring.empty(kst));
      Ring::on(0, kst, kph);

      // ---- softmax: s[n][0..1] row g, s[n][2..3] row g + 8, keys 8 n + 2 c and + 1
      const int key0 = t * kTile + 16 * warp;
      const bool ends = key0 + 16 > w.s.len;
      const int most = min(key0 + 16, w.s.len);  // open: some row does not see some of the sequence's keys here
      const bool open = __any_sync(0xffffffffu, lo[0] > key0 || hi[0] < most || lo[1] > key0 || hi[1] < most);
      if (open || ends) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int key = key0 + 8 * n + 2 * c + (j & 1);
            if (key < lo[j >> 1] || key >= hi[j >> 1]) s[n][j] = -INFINITY;
          }
      }
      float now[2], f[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        now[i] = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1])) * g.scale;
        now[i] = fmaxf(now[i], __shfl_xor_sync(0xffffffffu, now[i], 1));
        now[i] = fmaxf(now[i], __shfl_xor_sync(0xffffffffu, now[i], 2));
      }
      if (__any_sync(0xffffffffu, now[0] > mx[0] + 8.f || now[1] > mx[1] + 8.f)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bool up = now[i] > mx[i] + 8.f;
          f[i] = up ? exp2_fast(mx[i] - now[i]) : 1.f;
          if (up) mx[i] = now[i];
          sum[i] *= f[i];
        }
#pragma unroll
        for (int h = 0; h < F::kHalves; ++h)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[h][i][0] *= f[0], o[h][i][1] *= f[0];
            o[h][i][2] *= f[1], o[h][i][3] *= f[1];
          }
      }
      uint32_t p[4];  // the A fragment of the second product
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float neg = mx[i] == -INFINITY ? 0.f : -mx[i];
          const float p0 = exp2_fast(fmaf(s[n][2 * i], g.scale, neg)), p1 = exp2_fast(fmaf(s[n][2 * i + 1], g.scale, neg));
          sum[i] += p0 + p1;
          p[2 * n + i] = Bits<T>::pack(p0, p1);
        }

      // ---- o += p V: n-tile i of a half holds channels 8 g + i
      ok = __all_sync(0xffffffffu, tc::mbar_wait(ring.full(vst), vph));
      if (!ok) {
        if (lane == 0) flag(g, TR_CACHE_ERR_WAIT);
        break;
      }
      bool found = false;
      const uint32_t vt = base + vst * F::kTileBytes + (uint32_t)(16 * warp) * 128u;
#pragma unroll
      for (int h = 0; h < F::kHalves; ++h) {
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = 2 * c + (j & 1) + 8 * (j >> 1);
          v[j] = lds128(vt + h * (kTile * 128) + key * 128 + ((gq ^ (key & 7)) << 4));
        }
        if (ends) {  // the sequence ends among these keys: what lies behind may be NaN
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (key0 + 2 * c + (j & 1) + 8 * (j >> 1) >= w.s.len) v[j] = make_uint4(0u, 0u, 0u, 0u);
        }
        if (open) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            found |= clean_pair<T>(v[j].x) | clean_pair<T>(v[j].y) | clean_pair<T>(v[j].z) | clean_pair<T>(v[j].w);
          }
        }
        const uint32_t *v0 = &v[0].x, *v1 = &v[1].x, *v2 = &v[2].x, *v3 = &v[3].x;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t sel = i & 1 ? 0x7632u : 0x5410u;
          mma16816<T>(o[h][i], p[0], p[1], p[2], p[3], __byte_perm(v0[i >> 1], v1[i >> 1], sel),
                      __byte_perm(v2[i >> 1], v3[i >> 1], sel));
        }
      }
      if (found) bad = 1;  // (any thread's word will do)
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(ring.empty(vst));
      Ring::on(1, vst, vph);
    }

    // ------------------------------------------------------------------ the piece's result
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
      if (c == 0) top[warp][gq + 8 * i] = mx[i], tot[warp][gq + 8 * i] = sum[i];
    }
    named_sync(32 * kWarps);
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float m = -INFINITY;
#pragma unroll
      for (int j = 0; j < kWarps; ++j) m = fmaxf(m, top[j][gq + 8 * i]);
      f[i] = mx[i] == -INFINITY ? 0.f : exp2_fast(mx[i] - m);
    }
    const int part = 2 * blockIdx.x + (w.starts ? 1 : 0);
    for (int r0 = 0; r0 < rows; r0 += kPass) {
      // accumulator column 2 c + (j & 1) of n-tile i is channel 8 (2 c + (j & 1)) + i
      const int mine = gq - (r0 & 7);  // row of the pass that this quad holds (of its rows g or g + 8)
      if (mine >= 0 && mine < kPass) {
        float *dst = join + (warp * kPass + mine) * F::kJoinRow + 16 * c;
#pragma unroll
        for (int h = 0; h < F::kHalves; ++h)
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
              float4 v;
              if (r0 < 8)
                v = make_float4(o[h][i][b] * f[0], o[h][i + 1][b] * f[0], o[h][i + 2][b] * f[0], o[h][i + 3][b] * f[0]);
              else
                v = make_float4(o[h][i][2 + b] * f[1], o[h][i + 1][2 + b] * f[1], o[h][i + 2][2 + b] * f[1],
                                o[h][i + 3][2 + b] * f[1]);
              *reinterpret_cast<float4 *>(dst + 64 * h + 8 * b + i) = v;
            }
      }
      named_sync(32 * kWarps);
      const int r = r0 + (int)threadIdx.x / (D / 4), ch = (int)threadIdx.x % (D / 4) * 4;
      if ((int)threadIdx.x < kPass * (D / 4) && r < rows && ch < g.c.d) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int j = 0; j < kWarps; ++j) {
          const float4 x = *reinterpret_cast<const float4 *>(join + (j * kPass + r - r0) * F::kJoinRow + ch);
          v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
          m = fmaxf(m, top[j][r]);
        }
        // A maximum passes over NaN scores, so a warp that saw no other has the
        // maximum of one that saw nothing: its sum, 0 or NaN, enters as it is.
#pragma unroll
        for (int j = 0; j < kWarps; ++j) l += top[j][r] == -INFINITY ? tot[j][r] : tot[j][r] * exp2_fast(top[j][r] - m);
        put_row<T>(g, w, part, block0, hk, r, ch, v, m, l);
      }
      named_sync(32 * kWarps);
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
    for_bad_values<T>(g, edges_of_rows(g, w.s.base, w.s.len, block0, block0 + rows), w.seq(), hk, w.tile, w.tile + w.count,
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

// Joins the pieces of the items that several shares cover, one warp per row,
// in the shares' order; rows of sequences without a visible tile get zeros.
template <typename T>
__global__ void __launch_bounds__(256) k_few_join(const __grid_constant__ AttendArgs g) {
  __shared__ int runs[kFewMaxBatch / 32];
  const int lane = threadIdx.x & 31;
  Seq run0;
  const Shares shares(count_units(g, runs, 8, run0), g.ctas);  // reads nothing that k_attend_few writes
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= (long long)g.c.total_new * g.q_heads) {
    pdl_wait();
    return;
  }
  const int t = (int)(row / g.q_heads), h = (int)(row - (long long)t * g.q_heads);
  const int b = find_token(g.c, t).seq;
  float m = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  const bool holds = 4 * lane < g.c.d;
  const Seq mine = b < 32 ? run0 : seq_of(g, b / 32 * 32 + lane);
  Seq s = seq_from(mine, b & 31);
  if (b < 0) s.tiles = 0;
  if (s.tiles > 0) {
    unsigned x = lane < b % 32 ? units_of(mine) : 0;
    for (int i = lane; i < b / 32; i += 32) x += runs[i];
    const int local = (t - s.tok0) * g.group + h % g.group, r = local % kFewRows;
    const int u0 = (int)__reduce_add_sync(0xffffffffu, x) + (local / kFewRows * g.c.heads + h / g.group) * (s.tiles + kExtra) + kExtra;
    const int c0 = shares.of(u0), c1 = shares.of(u0 + s.tiles - 1);
    pdl_wait();
    if (c0 == c1) return;  // finished by its share
    // 32 shares at a time: a lane each for (maximum, sum), then the values,
    // several loads in flight
    for (int i0 = c0; i0 <= c1; i0 += 32) {
      const int c = i0 + lane;
      const int slot = 2 * c + (shares.start(c) <= u0 ? 1 : 0);
      float2 ml = make_float2(-INFINITY, 0.f);
      if (c <= c1) ml = g.part_ml[slot * kFewRows + r];
      const bool seen = ml.y != 0.f;  // NaN counts
      float now = seen ? ml.x : -INFINITY;
#pragma unroll
      for (int o = 16; o; o >>= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, o));
      const float before = m;
      m = fmaxf(m, now);
      const float f = before == -INFINITY ? 0.f : exp2_fast(before - m);
      const float e = seen ? exp2_fast(ml.x - m) : 0.f;
      float add = seen ? ml.y * e : 0.f;
#pragma unroll
      for (int o = 16; o; o >>= 1) add += __shfl_xor_sync(0xffffffffu, add, o);
      l = l * f + add;
      acc.x *= f, acc.y *= f, acc.z *= f, acc.w *= f;
      unsigned left = __ballot_sync(0xffffffffu, seen);
      while (left) {
        constexpr int kU = 4;
        float4 v[kU];
        float w[kU];
#pragma unroll
        for (int k = 0; k < kU; ++k) {
          const int src = left ? __ffs(left) - 1 : 0;
          const bool have = left != 0;
          left &= left - 1;
          const int from_slot = __shfl_sync(0xffffffffu, slot, src);
          w[k] = __shfl_sync(0xffffffffu, e, src);
          v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (have && holds)
            v[k] = reinterpret_cast<const float4 *>(g.part + ((long long)from_slot * kFewRows + r) * g.c.d)[lane];
        }
#pragma unroll
        for (int k = 0; k < kU; ++k) {
          acc.x += v[k].x * w[k];
          acc.y += v[k].y * w[k];
          acc.z += v[k].z * w[k];
          acc.w += v[k].w * w[k];
        }
      }
    }
  }
  if (s.tiles <= 0) pdl_wait();  // o may still be read by the kernel before last
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  if (holds)
    reinterpret_cast<uint2 *>(g.o + 2 * ((long long)t * g.o_tok + (long long)h * g.o_head))[lane] =
        make_uint2(Bits<T>::pack(acc.x * inv, acc.y * inv), Bits<T>::pack(acc.z * inv, acc.w * inv));
  if (g.lse && lane == 0) g.lse[row] = l > 0.f || l != l ? m * 0.693147180559945309f + logf(l) : -INFINITY;
}

std::atomic<int> g_few_smem_set[64];

template <typename T, int D>
cudaError_t launch_few_t(const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &g, int variant,
                         cudaStream_t st) {
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  if (!(g_few_smem_set[dev & 63].load() & (1 << variant))) {
    err = cudaFuncSetAttribute(k_attend_few<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Few<D>::kSmem);
    if (err != cudaSuccess) return err;
    g_few_smem_set[dev & 63].fetch_or(1 << variant);
  }
  err = launch_kernel(k_attend_few<T, D>, dim3(g.ctas), dim3(kThreads), Few<D>::kSmem, st, false, mk, mv, g);
  if (err != cudaSuccess) return err;
  const long long rows = (long long)g.c.total_new * g.q_heads;
  return launch_kernel(k_few_join<T>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, true, g);
}

size_t few_part_bytes(int d, int ctas) { return align_up((size_t)2 * ctas * kFewRows * d * sizeof(float), 256); }

}  // namespace

namespace attend {

size_t few_workspace_bytes(int d, int ctas) {
  return few_part_bytes(d, ctas) + align_up((size_t)2 * ctas * kFewRows * sizeof(float2), 256);
}

cudaError_t launch_few(const CUtensorMap &mk, const CUtensorMap &mv, AttendArgs g, bool bf16, void *ws, cudaStream_t st) {
  g.part = static_cast<float *>(ws);
  g.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(ws) + few_part_bytes(g.c.d, g.ctas));
  if (bf16)
    return g.c.d <= 64 ? launch_few_t<__nv_bfloat16, 64>(mk, mv, g, 0, st)
                       : launch_few_t<__nv_bfloat16, 128>(mk, mv, g, 1, st);
  return g.c.d <= 64 ? launch_few_t<__half, 64>(mk, mv, g, 2, st) : launch_few_t<__half, 128>(mk, mv, g, 3, st);
}

}  // namespace attend
}  // namespace tr
