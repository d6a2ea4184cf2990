// The append of keys and values to the paged cache held in 8 bits
// (tr_cache8_append), norm and rotation applied on the way as in
// tr_cache_append.
//
// A block is 16 keys of a head; its values are c 2^e with e4m3 codes c.  With
// a = the largest finite magnitude among the block's new rows x,
//   e = the least e with a <= 448 2^e (at least the old one, if the block has older keys),
//   c = round(x 2^-e),   older keys: c <- round(c 2^(e_old - e)).
// The scale is a power of two so that moving a block to a larger one rounds
// nothing but what falls under the codes' smallest step.
//
// A CTA takes the new rows of one block of a sequence, of all heads: its
// tokens share their angles and the block its page.  A warp takes one head's
// keys or values at a time, all 16 rows in its registers from the load to the
// codes, because the scale has to be known before the first code.
//
// 29.6k tokens into an empty cache, normed and rotated, 28 heads of 128 over 4,
// bf16: 108 us with the queries (4.6 TB/s), 39 without; one token of 64
// sequences 5.0 us.
#include "tr_cache8.cuh"
#include "tr_rotary.cuh"

namespace tr {
namespace {

using namespace rotary;
using namespace cache8;

struct Append8Args {
  RotArgs g;      // seg[0]: queries; seg[1], seg[2]: the rows of keys and values
  Scales scale;
  int blocks;     // slots of blocks
  int parts;      // CTAs of one: its heads' keys and values in turn
  int every;      // one CTA in so many is a block's, while there are any; the others take the queries
};

// Sequence b's blocks have the slots from cu_new[b] / 16 + 2 b on: n new keys
// lie in n / 16 + 2 blocks at most.
struct NewBlock {
  int seq;         // -1: an empty slot
  int tok0;        // token of row 0 of the block (it may lie before the sequence's first)
  int r0, r1;      // its new rows
  int key;         // key of row 0
  bool lost;       // some of the sequence's tokens have no key: lens and cu_new disagree (in its first slot)
};
__device__ __forceinline__ NewBlock find_new_block(const CacheView &c, int slot) {
  const int lane = threadIdx.x & 31;
  int b = -1, t0 = 0, end = 0, len = 0;  // of the last sequence whose slots start at or before this one
  for (int i0 = 0; i0 < c.batch; i0 += 32) {
    const int i = i0 + lane;
    int from = 0, to = 0, n = 0;
    if (i < c.batch) from = __ldg(c.cu_new + i), to = __ldg(c.cu_new + i + 1), n = __ldg(c.lens + i);
    const unsigned m = __ballot_sync(0xffffffffu, i < c.batch && (long long)(from / kBlock) + 2ll * i <= slot);
    if (m) {
      const int src = __popc(m) - 1;
      b = i0 + src;
      t0 = __shfl_sync(0xffffffffu, from, src), end = __shfl_sync(0xffffffffu, to, src), len = __shfl_sync(0xffffffffu, n, src);
    }
    if (m != 0xffffffffu) break;
  }
  NewBlock k{-1, 0, 0, 0, 0, false};
  if (b < 0) return k;
  const int t1 = min(end, c.total_new);
  const long long base = (long long)max(len, 0) - end + t0;  // key of token t0
  const long long nth = slot - (t0 / kBlock + 2ll * b);
  if (t0 < 0 || t1 <= t0 || nth < 0) return k;
  k.lost = base < 0 && nth == 0;
  const long long first = base < 0 ? 0 : base;  // keys before the sequence's first do not exist
  const long long key = (first / kBlock + nth) * kBlock, last = base + (t1 - t0);  // one past the last new key
  if (key >= last) return k;
  k.seq = b;
  k.key = (int)key;
  k.r0 = (int)(first > key ? first - key : 0);
  k.r1 = (int)(last - key < kBlock ? last - key : kBlock);
  k.tok0 = (int)(t0 + key - base);
  return k;
}

__device__ __forceinline__ bool finite1(float v) { return fabsf(v) <= 3.402823466e38f; }

// One head's new rows of a block, by a warp: d / (2 V) <= 8 or 16 lanes a row.
// They stay in registers as they came, from the load to the codes; the norm's
// factors are kept and the rotation is done twice, for the scale and for the
// codes (held in fp32 instead, rows took 128 registers and two CTAs filled an
// SM: 29.6k tokens with their queries 126 us against 114).
template <typename T, int V, bool PAIRS>
struct BlockRows {
  static constexpr int kPasses = V == 8 ? 4 : 8;
  Chunk<T, V> ra[kPasses], rb[kPasses];
  int slot, at_once, row0;
  bool holds;
  SlotPlace at;

  __device__ __forceinline__ BlockRows(const RotArgs &g) {
    const int lane = threadIdx.x & 31;
    slot = lane & ((1 << g.lanes_log2) - 1);
    at_once = 32 >> g.lanes_log2, row0 = lane >> g.lanes_log2;
    holds = slot < g.slots;
    at = slot_place<V, PAIRS>(slot, g.half);
  }
  __device__ __forceinline__ bool live(const NewBlock &k, int p) const {
    const int r = p * at_once + row0;
    return holds && r >= k.r0 && r < k.r1;
  }
  __device__ __forceinline__ void load(const Rows &s, const NewBlock &k, int head) {
#pragma unroll
    for (int p = 0; p < kPasses; ++p)
      if (live(k, p)) {
        const char *src = s.in + row_bytes<T>(k.tok0 + p * at_once + row0, s.in_tok, head, s.in_head);
        ra[p].load(src + sizeof(T) * at.a);
        rb[p].load(src + sizeof(T) * at.b);
      }
  }
  // Row of pass p as it enters the cache; f: its norm's factor.
  __device__ __forceinline__ void values(const RotArgs &g, const Rows &s, const NewBlock &k, int p, float f, const float *cs,
                                         const float *sn, f2 (&x)[V / 2], f2 (&y)[V / 2]) const {
    ra[p].get(x);
    rb[p].get(y);
    if (s.w) {
      const f2 ff = pack::make(f, f);
      f2 wa[V / 2], wb[V / 2];
      get_weights<V>(s.w, at.a, at.b, wa, wb);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) x[i] = pack::mul(x[i], pack::mul(ff, wa[i])), y[i] = pack::mul(y[i], pack::mul(ff, wb[i]));
    }
    if (s.turn && at.turns) {
      const int t = (p * at_once + row0 - k.r0) * g.half + slot * V;
      turn<V, PAIRS>(x, y, cs + t, sn + t);
    }
  }

  // Codes and scale of one head's keys or values.
  __device__ __forceinline__ void put(const RotArgs &g, const Rows &s, const NewBlock &k, int page, int head, uint8_t *codes,
                                      uint8_t *scales, const float *cs, const float *sn) const {
    const int lane = threadIdx.x & 31;
    const long long sc = scale_at(g.cache, page, head, k.key & (g.cache.page - 1));
    const int before = exp_of(scales[sc]);
    float norm[kPasses];
    uint32_t most = 0u;  // largest magnitude, as fp32 bits
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      f2 x[V / 2], y[V / 2];
      norm[p] = 1.f;
      if (s.w) {
        ra[p].get(x);
        rb[p].get(y);
        f2 s2 = 0ull;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) s2 = pack::fma(x[i], x[i], pack::fma(y[i], y[i], s2));
        const float2 t = pack::split(s2);
        norm[p] = rsqrtf(group_sum(live(k, p) ? t.x + t.y : 0.f, g.lanes_log2) * g.inv_d + g.eps);
      }
      if (live(k, p)) {
        values(g, s, k, p, norm[p], cs, sn, x, y);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          const float2 u = pack::split(x[i]), w = pack::split(y[i]);
          most = max(max(most, __float_as_uint(u.x) & 0x7fffffffu), __float_as_uint(u.y) & 0x7fffffffu);
          most = max(max(most, __float_as_uint(w.x) & 0x7fffffffu), __float_as_uint(w.y) & 0x7fffffffu);
        }
      }
    }
    // a <= 448 2^e = 1.75 2^(8 + e)
    uint32_t top = __reduce_max_sync(0xffffffffu, most);
    const bool bad = top >= 0x7f800000u;  // some are not finite: of the others then
    if (bad) {
      most = 0u;
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        f2 x[V / 2], y[V / 2];
        if (!live(k, p)) continue;
        values(g, s, k, p, norm[p], cs, sn, x, y);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          const float2 u = pack::split(x[i]), w = pack::split(y[i]);
          const float v[4] = {u.x, u.y, w.x, w.y};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (finite1(v[j])) most = max(most, __float_as_uint(v[j]) & 0x7fffffffu);
        }
      }
      top = __reduce_max_sync(0xffffffffu, most);
    }
    const bool older = k.r0 > 0;
    int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = min(max(e, kMinExp), kMaxExp);
    if (older) e = max(e, before);
    uint8_t *rows =
        codes + (((long long)page * g.cache.heads + head) * g.cache.page + (k.key & (g.cache.page - 1))) * g.d;
    if (older && e > before) {  // the older keys' codes, by 2^(before - e)
      const int down = min(e - before, 24);  // (beyond, all codes become zero)
      const uint32_t f = down <= 14 ? (uint32_t)(15 - down) << 10 : 1u << (24 - down);  // in half precision
      const uint32_t f2x = down == 24 ? 0u : f | f << 16;
      for (int i = lane; i < k.r0 * g.d / 16; i += 32) {
        uint4 *at16 = reinterpret_cast<uint4 *>(rows) + i;
        uint4 v = *at16;
        uint32_t *w = &v.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t lo, hi;
          halves4(w[j], lo, hi);
          asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(lo) : "r"(f2x));
          asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(hi) : "r"(f2x));
          w[j] = (uint32_t)codes_of_halves(lo) | (uint32_t)codes_of_halves(hi) << 16;
        }
        *at16 = v;
      }
    }
    if (lane == 0) scales[sc] = (uint8_t)(e + 127);
    const float f = pow2(-e);
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      if (!live(k, p)) continue;
      f2 x[V / 2], y[V / 2];
      values(g, s, k, p, norm[p], cs, sn, x, y);
      uint32_t ca[V / 4], cb[V / 4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f2 *z = h ? y : x;
        uint32_t *out = h ? cb : ca;
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
          const float2 u = pack::split(pack::mul(z[2 * i], pack::make(f, f))), w = pack::split(pack::mul(z[2 * i + 1], pack::make(f, f)));
          out[i] = (uint32_t)codes_of(u.x, u.y) | (uint32_t)codes_of(w.x, w.y) << 16;
          if (bad) {  // held as NaN (an infinite one would be the largest code)
            const float nan = __int_as_float(0x7fc00000);
            out[i] = (uint32_t)codes_of(finite1(u.x) ? u.x : nan, finite1(u.y) ? u.y : nan) |
                     (uint32_t)codes_of(finite1(w.x) ? w.x : nan, finite1(w.y) ? w.y : nan) << 16;
          }
        }
      }
      uint8_t *dst = rows + (p * at_once + row0) * g.d;
      if constexpr (V == 8) {
        *reinterpret_cast<uint2 *>(dst + at.a) = make_uint2(ca[0], ca[1]);
        *reinterpret_cast<uint2 *>(dst + at.b) = make_uint2(cb[0], cb[1]);
      } else {
        *reinterpret_cast<uint32_t *>(dst + at.a) = ca[0];
        *reinterpret_cast<uint32_t *>(dst + at.b) = cb[0];
      }
    }
  }
};

// PACK: a CTA takes two blocks, each with half of its warps.  A block's
// CTA waits for one load after the other (its sequence, rows, page), and its
// keys' warps take longer than its values'; with two blocks, and each warp
// keys and then values, that is once for both (29.6k tokens 113 us, so 108).
// Single tokens gain as well, although every second slot of theirs stays empty
// (448 sequences 12.0 us, so 11.3; 512 13.9, so 14.3; 1024 28.3, so 24.1; 4096
// 233, so 143: there every CTA's search for its sequence tells).  It costs
// registers, so few blocks go without.
template <typename T, int V, bool PAIRS, bool NORM, bool PACK>
__global__ void __launch_bounds__(kRotThreads, 3) k_append8(const __grid_constant__ Append8Args a) {
  __shared__ __align__(16) float cs[(1 + PACK) * kMaxTrig], sn[(1 + PACK) * kMaxTrig];
  __shared__ long long home[kMaxTokens];
  const RotArgs &g = a.g;
  pdl_wait();  // q, k, v come from the kernel before
  const int nth = blockIdx.x / a.every, all = PACK ? (a.blocks + 1) / 2 : a.blocks * a.parts;
  if (nth >= all || nth * a.every != (int)blockIdx.x) {
    rotate_rows<T, V, PAIRS, NORM>(g, blockIdx.x - min(nth + 1, all), cs, sn, home);
    return;
  }
  const CacheView &c = g.cache;
  constexpr int kWarps = kRotThreads / 32;
  const int half = PACK ? threadIdx.x / (kRotThreads / 2) : 0, threads = PACK ? kRotThreads / 2 : kRotThreads;
  const NewBlock k = find_new_block(c, PACK ? 2 * nth + half : nth / a.parts);
  // the first head's rows asked for before the page and the angles
  const int warp = (threadIdx.x & (threads - 1)) >> 5, step = PACK ? kWarps / 2 : a.parts * kWarps;
  int u = PACK ? warp : nth % a.parts * kWarps + warp;
  const int at = kBlock * g.half;  // the second half's angles
  BlockRows<T, V, PAIRS> rows(g);
  auto load = [&]() {
    const bool val = u >= c.heads;
    if (u < 2 * c.heads) rows.load(val ? g.seg[2] : g.seg[1], k, val ? u - c.heads : u);
  };
  if (k.seq >= 0) load();
  const int page = k.seq >= 0 ? page_of(c, k.seq, k.key) : -1;
  if (g.err && (threadIdx.x & (threads - 1)) == 0 && (k.lost || (k.seq >= 0 && page < 0))) atomicOr(g.err, TR_CACHE_ERR_PAGE);
  if (page < 0) return;
  if (g.seg[1].turn) {
    fill_trig(g, k.tok0 + k.r0, k.r1 - k.r0, cs + half * at, sn + half * at, threads);
    if (PACK) asm volatile("bar.sync %0, %1;" ::"r"(1 + half), "r"(threads) : "memory");
    else __syncthreads();
  }
  while (u < 2 * c.heads) {
    const bool val = u >= c.heads;
    rows.put(g, val ? g.seg[2] : g.seg[1], k, page, val ? u - c.heads : u, static_cast<uint8_t *>(val ? c.v : c.k),
             val ? a.scale.v : a.scale.k, cs + half * at, sn + half * at);
    u += step;
    load();
  }
}

template <typename T, int V, bool PAIRS>
cudaError_t launch_append8_t(Append8Args &a, cudaStream_t st) {
  Append8Args q = a;
  q.g.seg[1] = q.g.seg[2] = Rows{};
  // a block's heads over several CTAs while the SMs (three CTAs each) would not all get some
  const int sms = sm_count() > 0 ? sm_count() : 1, rounds = (2 * a.g.cache.heads + kRotThreads / 32 - 1) / (kRotThreads / 32);
  a.parts = a.blocks ? 3 * sms / a.blocks : 1;
  a.parts = a.parts < 1 ? 1 : a.parts > rounds ? rounds : a.parts;
  const bool pack = a.blocks >= 6 * sms;  // every SM gets as many CTAs as it holds all the same
  const int all = pack ? (a.blocks + 1) / 2 : a.blocks * a.parts, ctas = all + (a.g.seg[0].in ? cut_segments(q.g) : 0);
  a.every = all ? ctas / all : 1;
  if (ctas == 0) return cudaSuccess;  // no sequence, fewer rows than a block's, no queries
  a.g.seg[0] = q.g.seg[0];
  a.g.seg[1].cta0 = a.g.seg[2].cta0 = INT_MAX;  // (of the queries' CTAs: none is for keys or values)
  auto kernel = pack ? a.g.seg[0].w ? k_append8<T, V, PAIRS, true, true> : k_append8<T, V, PAIRS, false, true>
                : a.g.seg[0].w ? k_append8<T, V, PAIRS, true, false> : k_append8<T, V, PAIRS, false, false>;
  return launch_kernel(kernel, dim3(ctas), dim3(kRotThreads), 0, st, false, a);
}

template <typename T>
cudaError_t launch_append8(Append8Args &a, int dtype, int rot, int layout, cudaStream_t st) {
  const bool pairs = layout == TR_ROTARY_PAIRS;
  if (pairs_per_lane(dtype, a.g.d, rot) == 8)
    return pairs ? launch_append8_t<T, 8, true>(a, st) : launch_append8_t<T, 8, false>(a, st);
  return pairs ? launch_append8_t<T, 4, true>(a, st) : launch_append8_t<T, 4, false>(a, st);
}

}  // namespace
}  // namespace tr

using namespace tr;

extern "C" {

tr_status tr_cache8_append(const tr_cache8 *c8, const tr_heads *k, const tr_heads *v, const tr_rotary *r,
                           const int32_t *pos, const float *k_weight, const tr_heads *q, const float *q_weight,
                           const tr_heads *q_out, float eps, int32_t *d_error, void *stream) {
  tr_status rc = check_cache8(c8);
  if (rc != TR_OK) return rc;
  const tr_cache *c = &c8->c;
  if (r) {
    if ((rc = check_rotary(r)) != TR_OK) return rc;
    if (r->head_dim != c->head_dim || (r->rot_dim && !pos)) return TR_ERR_ARG;
  }
  if (!k || !k->p || !v || !v->p || k->heads != c->heads || v->heads != c->heads) return TR_ERR_ARG;
  if ((rc = check_heads(k, 2)) != TR_OK || (rc = check_heads(v, 2)) != TR_OK) return rc;
  if (misaligned16(k_weight) || (reinterpret_cast<uintptr_t>(pos) & 3u)) return TR_ERR_ALIGN;
  if ((rc = check_pair(q, q_out, q_weight, 2, false)) != TR_OK) return rc;
  // (slots of blocks and the queries' CTAs make up one grid)
  if ((long long)c->total_new / kBlock + 2ll * c->batch + 1 > INT_MAX / 2) return TR_ERR_UNSUPPORTED;
  if (c->total_new == 0) return TR_OK;
  const int rot = r ? r->rot_dim : 0;
  Append8Args a{};
  RotArgs &g = a.g;
  shape(g, c->dtype, c->head_dim, rot, c->total_new);
  if (rot) {
    g.turns = reinterpret_cast<const unsigned long long *>(r->turns);
    g.axis = r->axis;
    g.axes = r->axes;
    g.pos = pos;
  }
  g.sign = 1.f;
  g.eps = eps;
  g.seg[0] = rows_of(q, q_out, q_weight, rot > 0, 0);
  g.seg[1] = rows_of(k, nullptr, k_weight, rot > 0, 1);
  g.seg[2] = rows_of(v, nullptr, nullptr, 0, 2);
  g.cache = cache_view(c);
  g.err = d_error;
  a.scale = Scales{c8->k_scale, c8->v_scale};
  a.blocks = c->total_new / kBlock + 2 * c->batch;
  const int layout = r ? r->layout : TR_ROTARY_HALF;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t err = c->dtype == TR_BF16 ? launch_append8<__nv_bfloat16>(a, c->dtype, rot, layout, st)
                                              : launch_append8<__half>(a, c->dtype, rot, layout, st);
  return err == cudaSuccess ? TR_OK : TR_ERR_CUDA;
}

}  // extern "C"
