// What the kernels of few rows per key head share (tr_attend_few.cu, tr_attend8_few.cu):
// the work in units of 128-key tiles, its equal shares and the walk over
// them, warp-level products, and the join of items that several shares cover.
#pragma once

#include "tr_attend.cuh"

namespace tr {
namespace attend {
namespace few {

constexpr int kWarps = 8;                     // consumer warps: 16 keys of a tile each
constexpr int kThreads = 32 * (kWarps + 2);   // and the producers of K and of V
constexpr int kPass = 4;                      // rows joined per pass at an item's end

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
// and finishing it cost (in 16 bits about 3 us against 1.3 us a tile): without
// them the shares that hold many short items end last.
template <int kExtra>
__device__ __forceinline__ int units_of(const Seq &s) {
  return s.tiles > 0 ? s.items * (s.tiles + kExtra) : 0;
}

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
template <int kExtra>
__device__ __forceinline__ int count_units(const AttendArgs &g, int *runs, int warps, Seq &mine) {
  const int lane = threadIdx.x & 31;
  const int n = (g.c.batch + 31) / 32;
  mine = seq_of(g, lane);
  if (n <= 1) return (int)__reduce_add_sync(0xffffffffu, (unsigned)units_of<kExtra>(mine));
  for (int i = threadIdx.x >> 5; i < n; i += warps) {
    const int u = (int)__reduce_add_sync(0xffffffffu, (unsigned)units_of<kExtra>(seq_of(g, 32 * i + lane)));
    if (lane == 0) runs[i] = u;
  }
  __syncthreads();
  int all = 0;
  for (int i = lane; i < n; i += 32) all += runs[i];
  return (int)__reduce_add_sync(0xffffffffu, (unsigned)all);
}

// A walk over the units of a share, item by item; the same in all lanes
// (but `mine`).
template <int kExtra>
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
    const int own = units_of<kExtra>(mine);
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
      if (u >= first + units_of<kExtra>(s)) {  // on to the next sequence that has units
        first += units_of<kExtra>(s);
        unsigned any = __ballot_sync(0xffffffffu, units_of<kExtra>(mine) > 0) & ~(at == 31 ? 0xffffffffu : (2u << at) - 1u);
        while (!any && 32 * (run + 1) < g.c.batch) {
          mine = seq_of(g, 32 * ++run + (threadIdx.x & 31));
          any = __ballot_sync(0xffffffffu, units_of<kExtra>(mine) > 0);
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
// partial result.  NORMED: v is divided by l already.
template <typename T, bool NORMED = false>
__device__ __forceinline__ void put_row(const AttendArgs &g, bool whole, int tok0, int part, int block0, int hk, int r, int ch,
                                        const float4 &v, float m, float l) {
  if (whole) {
    const int row = block0 + r, tok = row / g.group, head = hk * g.group + row - tok * g.group;
    const long long t = tok0 + tok;
    const float inv = NORMED ? 1.f : l > 0.f || l != l ? 1.f / l : 0.f;
    *reinterpret_cast<uint2 *>(g.o + 2 * (t * g.o_tok + (long long)head * g.o_head + ch)) =
        make_uint2(Bits<T>::pack(v.x * inv, v.y * inv), Bits<T>::pack(v.z * inv, v.w * inv));
    if (ch == 0 && g.lse) g.lse[t * g.q_heads + head] = l > 0.f || l != l ? m * 0.693147180559945309f + logf(l) : -INFINITY;
  } else {
    *reinterpret_cast<float4 *>(g.part + ((long long)part * kFewRows + r) * g.c.d + ch) = v;
    if (ch == 0) g.part_ml[part * kFewRows + r] = make_float2(m, l);
  }
}

// Joins the pieces of the items that several shares cover, one warp per row,
// in the shares' order; rows of sequences without a visible tile get zeros.
// NORMED: the pieces' values are divided by their sums.
template <typename T, bool NORMED, int kExtra>
__global__ void __launch_bounds__(256) k_few_join(const __grid_constant__ AttendArgs g) {
  __shared__ int runs[kFewMaxBatch / 32];
  const int lane = threadIdx.x & 31;
  Seq run0;
  const Shares shares(count_units<kExtra>(g, runs, 8, run0), g.ctas);  // reads nothing that k_attend_few writes
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
    unsigned x = lane < b % 32 ? units_of<kExtra>(mine) : 0;
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
      const float add1 = seen ? ml.y * e : 0.f;
      float add = add1;
#pragma unroll
      for (int o = 16; o; o >>= 1) add += __shfl_xor_sync(0xffffffffu, add, o);
      const float was = l, kept = l * f;
      l = kept + add;
      // NORMED: shares of the sum so far, 1 at most, so that values near the end of fp32 stay below it; those under
      // 2^-126 in two factors, of which kFar is one: a value may outweigh its small probability
      const float inv = NORMED && (l > 0.f || l != l) ? 1.f / l : 0.f;
      float keep = NORMED ? kept * inv : f, mine = NORMED ? add1 * inv : e;
      unsigned far = 0u;
      if (NORMED) {
        far = __ballot_sync(0xffffffffu, seen && ml.x - m < -126.f);
        if (far >> lane & 1u) mine = ml.y * exp2_fast(ml.x - m + 126.f) * inv;
        if (before - m < -126.f && before > -INFINITY) {
          keep = was * exp2_fast(before - m + 126.f) * inv;
          acc.x *= kFar, acc.y *= kFar, acc.z *= kFar, acc.w *= kFar;
        }
      }
      acc.x *= keep, acc.y *= keep, acc.z *= keep, acc.w *= keep;
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
          w[k] = __shfl_sync(0xffffffffu, mine, src);
          v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (have && holds)
            v[k] = reinterpret_cast<const float4 *>(g.part + ((long long)from_slot * kFewRows + r) * g.c.d)[lane];
          if (NORMED && (far >> src & 1u)) v[k].x *= kFar, v[k].y *= kFar, v[k].z *= kFar, v[k].w *= kFar;
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
  const float inv = NORMED ? 1.f : l > 0.f || l != l ? 1.f / l : 0.f;
  if (holds)
    reinterpret_cast<uint2 *>(g.o + 2 * ((long long)t * g.o_tok + (long long)h * g.o_head))[lane] =
        make_uint2(Bits<T>::pack(acc.x * inv, acc.y * inv), Bits<T>::pack(acc.z * inv, acc.w * inv));
  if (g.lse && lane == 0) g.lse[row] = l > 0.f || l != l ? m * 0.693147180559945309f + logf(l) : -INFINITY;
}

inline size_t part_bytes(int d, int ctas) { return align_up((size_t)2 * ctas * kFewRows * d * sizeof(float), 256); }

}  // namespace few
}  // namespace attend
}  // namespace tr
