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

#include "tr_attend_few.cuh"

namespace tr {
namespace {

using namespace attend;
using namespace attend::few;

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
  Walk<kFewItemCost> w;
  Seq run0;
  const Shares shares(count_units<kFewItemCost>(g, runs, kWarps + 2, run0), g.ctas);
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
        put_row<T>(g, w.whole, w.s.tok0, part, block0, hk, r, ch, v, m, l);
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
  return launch_kernel(k_few_join<T, false, kFewItemCost>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, true, g);
}

}  // namespace

namespace attend {

size_t few_workspace_bytes(int d, int ctas) {
  return few::part_bytes(d, ctas) + align_up((size_t)2 * ctas * kFewRows * sizeof(float2), 256);
}

cudaError_t launch_few(const CUtensorMap &mk, const CUtensorMap &mv, AttendArgs g, bool bf16, void *ws, cudaStream_t st) {
  g.part = static_cast<float *>(ws);
  g.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(ws) + few::part_bytes(g.c.d, g.ctas));
  if (bf16)
    return g.c.d <= 64 ? launch_few_t<__nv_bfloat16, 64>(mk, mv, g, 0, st)
                       : launch_few_t<__nv_bfloat16, 128>(mk, mv, g, 1, st);
  return g.c.d <= 64 ? launch_few_t<__half, 64>(mk, mv, g, 2, st) : launch_few_t<__half, 128>(mk, mv, g, 3, st);
}

}  // namespace attend
}  // namespace tr
