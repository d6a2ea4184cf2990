// The block tables of the paged caches, kept on the device: pages taken from
// a stack of free ones as sequences grow (tr_pages_extend) and given back as
// they shrink (tr_pages_truncate).
//
// With len and new of each sequence b, p the page size and F = free_count:
//   cu_new = prefix sums of new,  need_b = ceil((len + new) / p) - ceil(len / p),
//   the i-th page needed (sequence by sequence, in each in order) = free[F - 1 - i];
//   the i-th page given back goes to free[F + G - 1 - i], G of them in all,
// so that giving back undoes taking, bit for bit.
//
// Tens of kilobytes at most: the time is a launch, a scan of the sequences and
// a few loads that depend on one another.  So it is one launch: every CTA sums
// and scans all sequences for itself (a few integers each, from L2) and writes
// its part of the pages and rows; what the scans read is changed by the CTA
// that finishes last.
//
// In a graph of calls, back and on again (two launches; one that does nothing
// takes 2 us): one sequence by a token 4.6 us, 256 by up to five tokens 9.5, 2000
// by 131000 tokens in all 19.5.
#include <climits>
#include <initializer_list>

#include "tr_internal.cuh"

namespace tr {
namespace {

constexpr int kThreads = 1024;  // at most (a few sequences and rows: fewer, for cheaper barriers)
constexpr int kPerCta = 1024;  // pages or rows that are worth a CTA of their own

struct PagesArgs {
  int32_t *table, *lens, *free, *free_count, *ticket;
  int batch, max_pages, pages, page_log2;
  const int32_t *in;   // extend: new tokens; truncate: lengths to keep
  int total_new;
  int32_t *cu_new, *slots, *pos, *seq;
  int32_t *err;
};

// What a sequence does: tokens [len, to), pages [first, first + pages).
struct Change {
  long long len, to;
  int first, pages;
  bool bad;  // the state is not one that these calls leave
};
template <bool EXTEND>
__device__ __forceinline__ Change change_of(const PagesArgs &g, int b) {
  Change c{0, 0, 0, 0, false};
  if (b >= g.batch) return c;
  const long long most = (long long)g.max_pages << g.page_log2, up = (1ll << g.page_log2) - 1;
  c.len = max(g.lens[b], 0);
  const long long n = max(__ldg(g.in + b), 0);
  c.bad = c.len > most;
  if (c.bad) c.len = most;
  c.to = EXTEND ? c.len + n : min(c.len, n);
  const long long p0 = (c.len + up) >> g.page_log2, p1 = (c.to + up) >> g.page_log2;
  c.first = (int)min(p0, p1);
  c.pages = (int)min(EXTEND ? p1 - p0 : p0 - p1, (long long)INT_MAX);
  return c;
}

// Sums over the CTA of two numbers, and the OR of a third.
struct Sums {
  long long a, b;
  int bits;
};
__device__ __forceinline__ Sums warp_sums(Sums s) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    s.a += __shfl_xor_sync(0xffffffffu, s.a, o);
    s.b += __shfl_xor_sync(0xffffffffu, s.b, o);
  }
  s.bits = (int)__reduce_or_sync(0xffffffffu, (unsigned)s.bits);
  return s;
}
__device__ __forceinline__ Sums cta_sums(Sums s, Sums *part) {
  const int lane = threadIdx.x & 31;
  s = warp_sums(s);
  if (lane == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  s = lane < (int)blockDim.x >> 5 ? part[lane] : Sums{0, 0, 0};
  return warp_sums(s);
}
// Exclusive prefix sums over the CTA of two numbers, and their totals.
__device__ __forceinline__ int2 cta_scan(int2 v, int2 *part, int2 &all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int2 x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int a = __shfl_up_sync(0xffffffffu, x.x, o), b = __shfl_up_sync(0xffffffffu, x.y, o);
    if (lane >= o) x.x += a, x.y += b;
  }
  if (lane == 31) part[warp] = x;
  __syncthreads();
  const int2 w = lane < (int)blockDim.x >> 5 ? part[lane] : make_int2(0, 0);
  int2 s = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int a = __shfl_up_sync(0xffffffffu, s.x, o), b = __shfl_up_sync(0xffffffffu, s.y, o);
    if (lane >= o) s.x += a, s.y += b;
  }
  all = make_int2(__shfl_sync(0xffffffffu, s.x, 31), __shfl_sync(0xffffffffu, s.y, 31));
  const int bx = __shfl_sync(0xffffffffu, s.x - w.x, warp), by = __shfl_sync(0xffffffffu, s.y - w.y, warp);
  return make_int2(bx + x.x - v.x, by + x.y - v.y);
}
// The last i of [0, n) with at[i] <= u (at[0] <= u).
__device__ __forceinline__ int last_at(const int *at, int n, int u) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= u) lo = mid; else hi = mid;
  }
  return lo;
}

template <bool EXTEND>
__global__ void __launch_bounds__(kThreads) k_pages(const __grid_constant__ PagesArgs g) {
  __shared__ Sums sums[32];
  __shared__ int2 part[32];
  __shared__ int rows_at[kThreads], pages_at[kThreads];  // of a run of sequences: first row, first page moved
  __shared__ int len_at[kThreads], first_at[kThreads];
  __shared__ bool last;
  pdl_trigger();
  pdl_wait();  // the counts and the tables come from the kernels before
  const int threads = blockDim.x, tid = threadIdx.x, stride = threads * gridDim.x, me = blockIdx.x * threads + tid;
  const int runs = (g.batch + threads - 1) / threads;
  const int have = *g.free_count;
  // ---- whether the step can be taken
  Change mine = change_of<EXTEND>(g, tid);
  Sums s{0, 0, (unsigned)have > (unsigned)g.pages ? TR_PAGES_ERR_STATE : 0};
  for (int r = 0; r < runs; ++r) {
    const Change c = r ? change_of<EXTEND>(g, r * threads + tid) : mine;
    s.a += c.to - c.len;
    s.b += c.pages;
    if (c.bad) s.bits |= TR_PAGES_ERR_STATE;
    if (EXTEND && c.to > (long long)g.max_pages << g.page_log2) s.bits |= TR_PAGES_ERR_LONG;
  }
  s = cta_sums(s, sums);
  const long long rows = s.a, moved = s.b;
  int bits = s.bits;
  if (EXTEND) {
    if (moved > have) bits |= TR_PAGES_ERR_FULL;
    if (rows > g.total_new) bits |= TR_PAGES_ERR_ROWS;
  } else if (have + moved > g.pages) {
    bits |= TR_PAGES_ERR_STATE;
  }
  const bool take = bits == 0;

  // ---- pages and rows, a run of sequences at a time
  int2 before = make_int2(0, 0);
  for (int r = 0; take && r < runs; ++r) {
    const int b0 = r * threads, n = min(g.batch - b0, threads);
    if (r) mine = change_of<EXTEND>(g, b0 + tid);
    int2 all;
    const int2 at = cta_scan(make_int2(EXTEND ? (int)(mine.to - mine.len) : 0, mine.pages), part, all);
    if (r) __syncthreads();  // the last sequences' are used up
    rows_at[tid] = before.x + at.x;
    pages_at[tid] = before.y + at.y;
    len_at[tid] = (int)mine.len;
    first_at[tid] = mine.first;
    __syncthreads();
    if (EXTEND && blockIdx.x == 0 && tid < n) g.cu_new[b0 + tid] = before.x + at.x;
    const int p1 = before.y + all.y, r1 = before.x + all.x;
    for (int u = before.y + me; u < p1; u += stride) {
      const int i = last_at(pages_at, n, u);
      int32_t *entry = g.table + (long long)(b0 + i) * g.max_pages + first_at[i] + (u - pages_at[i]);
      if (EXTEND) {
        *entry = g.free[have - 1 - u];
      } else {
        g.free[have + (int)moved - 1 - u] = *entry;
        *entry = -1;
      }
    }
    if (EXTEND) {
      for (int t = before.x + me; t < r1; t += stride) {
        const int i = last_at(rows_at, n, t), key = len_at[i] + (t - rows_at[i]);
        const int j = key >> g.page_log2;
        const int id = j >= first_at[i] ? g.free[have - 1 - (pages_at[i] + j - first_at[i])]
                                        : g.table[(long long)(b0 + i) * g.max_pages + j];
        g.slots[t] = (unsigned)id < (unsigned)g.pages ? (id << g.page_log2) + (key & ((1 << g.page_log2) - 1)) : -1;
        g.pos[t] = key;
        g.seq[t] = b0 + i;
      }
    }
    before = make_int2(r1, p1);
  }
  if (EXTEND) {  // rows of no sequence
    for (int t = (take ? (int)rows : 0) + me; t < g.total_new; t += stride) g.slots[t] = g.pos[t] = g.seq[t] = -1;
    if (blockIdx.x == 0) {
      if (!take)
        for (int b = tid; b < g.batch; b += threads) g.cu_new[b] = 0;
      if (tid == 0) g.cu_new[g.batch] = take ? (int)rows : 0;
    }
  }
  // ---- the lengths and the stack's height, once every CTA has read them
  if (gridDim.x > 1) {
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(g.ticket, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
  } else {
    __syncthreads();
  }
  if (take) {
    for (int r = 0; r < runs; ++r) {
      const int b = r * threads + tid;
      if (b >= g.batch) break;
      if (runs > 1) mine = change_of<EXTEND>(g, b);
      g.lens[b] = (int)mine.to;
    }
  }
  if (tid == 0 && bits && g.err) atomicOr(g.err, bits);
  if (tid == 0) {
    if (take) *g.free_count = have + (EXTEND ? -(int)moved : (int)moved);
    if (gridDim.x > 1) *g.ticket = 0;
  }
}

tr_status check_pages(const tr_pages *p) {
  if (!p || !p->free_count || !p->ticket || p->batch < 0 || p->max_pages < 0 || p->pages < 0) return TR_ERR_ARG;
  if ((p->batch && (!p->lens || (p->max_pages && !p->table))) || (p->pages && !p->free)) return TR_ERR_ARG;
  if (p->page < 16 || p->page > 256 || (p->page & (p->page - 1))) return TR_ERR_UNSUPPORTED;
  // slots and keys of a sequence are int32
  if ((long long)p->pages * p->page > INT32_MAX || (long long)p->max_pages * p->page > INT32_MAX - 65536)
    return TR_ERR_UNSUPPORTED;
  if (p->batch > INT_MAX - kThreads) return TR_ERR_UNSUPPORTED;
  for (const void *a : {(const void *)p->table, (const void *)p->lens, (const void *)p->free, (const void *)p->free_count,
                        (const void *)p->ticket})
    if (reinterpret_cast<uintptr_t>(a) & 3u) return TR_ERR_ALIGN;
  return TR_OK;
}

PagesArgs pages_args(const tr_pages *p, const int32_t *in, int32_t *err) {
  PagesArgs g{};
  g.table = p->table, g.lens = p->lens, g.free = p->free, g.free_count = p->free_count, g.ticket = p->ticket;
  g.batch = p->batch, g.max_pages = p->max_pages, g.pages = p->pages;
  while ((1 << g.page_log2) < p->page) ++g.page_log2;
  g.in = in;
  g.err = err;
  return g;
}

// work: pages or rows at most.
template <bool EXTEND>
cudaError_t launch_pages(const PagesArgs &g, long long work, cudaStream_t st) {
  const long long sms = sm_count() > 0 ? sm_count() : 1, want = (work + kPerCta - 1) / kPerCta;
  const int ctas = (int)(want < 1 ? 1 : want > sms ? sms : want);
  int threads = 128;
  while (threads < kThreads && (threads < g.batch || 4ll * threads < work)) threads *= 2;
  return launch_kernel(k_pages<EXTEND>, dim3(ctas), dim3(threads), 0, st, true, g);
}

}  // namespace
}  // namespace tr

using namespace tr;

extern "C" {

tr_status tr_pages_extend(const tr_pages *p, const int32_t *d_new, int32_t total_new, int32_t *cu_new, int32_t *slots,
                          int32_t *pos, int32_t *seq, int32_t *d_error, void *stream) {
  const tr_status rc = check_pages(p);
  if (rc != TR_OK) return rc;
  if (total_new < 0 || !cu_new || (p->batch && !d_new) || (total_new && (!slots || !pos || !seq))) return TR_ERR_ARG;
  for (const void *a : {(const void *)d_new, (const void *)cu_new, (const void *)slots, (const void *)pos, (const void *)seq})
    if (reinterpret_cast<uintptr_t>(a) & 3u) return TR_ERR_ALIGN;
  if (total_new > INT_MAX - kThreads * 1024) return TR_ERR_UNSUPPORTED;
  PagesArgs g = pages_args(p, d_new, d_error);
  g.total_new = total_new;
  g.cu_new = cu_new, g.slots = slots, g.pos = pos, g.seq = seq;
  return launch_pages<true>(g, total_new, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TR_OK : TR_ERR_CUDA;
}

tr_status tr_pages_truncate(const tr_pages *p, const int32_t *d_keep, int32_t *d_error, void *stream) {
  const tr_status rc = check_pages(p);
  if (rc != TR_OK) return rc;
  if (p->batch && !d_keep) return TR_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(d_keep) & 3u) return TR_ERR_ALIGN;
  if (p->batch == 0) return TR_OK;
  const PagesArgs g = pages_args(p, d_keep, d_error);
  const long long most = (long long)p->batch * p->max_pages;
  // few of the pages that could come back do as a rule: the last steps' of each sequence, or some sequences whole
  const long long work = 4ll * p->batch + (most < p->pages ? most : p->pages) / 16;
  return launch_pages<false>(g, work, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TR_OK : TR_ERR_CUDA;
}

}  // extern "C"
