// kvr_paged.cu -- the paged full-context cache (include/kvr.h, kvr_paged_*): its
// handle, the plan of pages and slots, and the append.
#include "kvr_paged.cuh"

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <new>

#include "../../include/kvr.h"
#include "kvr_internal.h"
#include "kvr_ptx.cuh"

namespace kvr {
namespace paged {
namespace {

// ---- plan -------------------------------------------------------------------

constexpr int kPlan = 512;        // threads of a CTA of the plan
constexpr int kPlanFew = 256;     // the same for as many sequences or fewer
constexpr int kCluster = 8;       // CTAs of the plan
constexpr int kInPlan = 2048;     // slots that the plan's cluster writes itself
constexpr int kFill = 256, kFillTokens = 2048;  // of a CTA that writes slots alone

__global__ void __launch_bounds__(256) init_kernel(const __grid_constant__ View c) {
  kvr::pdl_begin();
  const long long i0 = (long long)blockIdx.x * 256 + threadIdx.x, step = (long long)gridDim.x * 256;
  for (long long i = i0; i < (long long)c.S * c.tstride; i += step) c.table[i] = -1;
  for (long long i = i0; i < c.n_pages; i += step) c.stack[i] = c.n_pages - 1 - (int)i;
  for (long long i = i0; i < c.S; i += step) c.len[i] = c.from[i] = c.first[i] = 0;
  for (long long i = i0; i <= c.S; i += step) c.tiles[i] = 0;
  if (i0 == 0) c.free[0] = c.n_pages, c.free[1] = 1;
}

// What a sequence's new length takes and gives back.
struct Change {
  int old, want, have, need;  // rows and pages, before and after
  bool bad;
  __device__ int back() const { return max(have - need, 0); }
  __device__ int take() const { return max(need - have, 0); }
};
__device__ __forceinline__ Change change_of(const View &c, const int32_t *want, int s, int n_new) {
  Change x{};
  if (s >= c.S) return x;
  const long long most = (long long)c.tstride << c.psh;
  x.old = (int)min((long long)max(c.len[s], 0), most);
  x.want = want[s];
  x.bad = x.want < 0 || x.want > most || (long long)x.want - x.old > n_new;
  if (x.bad) x.want = x.old;
  x.have = (int)(((long long)x.old + c.P - 1) >> c.psh);
  x.need = (int)(((long long)x.want + c.P - 1) >> c.psh);
  return x;
}

// What sequences ask for, summed: pages taken (any number may be asked for), given
// back, and tiles (which only matter where the plan is carried out).
struct Sums {
  long long take;
  int back, tiles;
};
__device__ __forceinline__ Sums operator+(Sums a, const Sums &b) {
  a.take += b.take, a.back += b.back, a.tiles += b.tiles;
  return a;
}
__device__ __forceinline__ Sums operator-(Sums a, const Sums &b) {
  a.take -= b.take, a.back -= b.back, a.tiles -= b.tiles;
  return a;
}

// Sum over the CTA of the values before this thread's, and of all of them.
template <int N>
__device__ Sums scan(const Sums &x, Sums *s_warp, Sums *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sums y = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    Sums z;
    z.take = __shfl_up_sync(0xffffffffu, y.take, o);
    z.back = __shfl_up_sync(0xffffffffu, y.back, o);
    z.tiles = __shfl_up_sync(0xffffffffu, y.tiles, o);
    if (lane >= o) y = y + z;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = y;
  __syncthreads();
  Sums before{}, all{};
#pragma unroll
  for (int w = 0; w < N / 32; ++w) {
    if (w == warp) before = all;
    all = all + s_warp[w];
  }
  *total = all;
  return before + y - x;
}

// Sequence whose entries hold entry e: the last one that starts at or before it.
template <int N>
__device__ __forceinline__ int find(const int *start, int e) {
  int lo = 0;
#pragma unroll
  for (int step = N / 2; step > 0; step >>= 1)
    if (start[lo + step] <= e) lo += step;
  return lo;
}

// Token t of a sequence's growth: its slot, and its page's entry in the table where
// the page is new.  Pages behind the first `have` are the stack's, from `top` down.
__device__ __forceinline__ int place(const View &c, int s, int t, int from, int len, int top) {
  if (t >= len - from) return -1;
  const int pos = from + t;
  const int at = pos >> c.psh, have = (from + c.P - 1) >> c.psh;
  int32_t *entry = c.table + (long long)s * c.tstride + at;
  const int page = at < have ? *entry : c.stack[top - (at - have)];
  if (at >= have && (pos & (c.P - 1)) == 0) *entry = page;
  return (page << c.psh) + (pos & (c.P - 1));
}

// One cluster.  S lengths are little work, and what they ask of the stack is a sum
// over all of them, which every CTA forms for itself, a thread the same number of
// neighbours; pages that go back (an ended sequence has hundreds), and the new tokens'
// slots with the pages they need, are dealt out to all threads of the cluster.  Many
// slots are left to the launch that follows.  Latency binds.  us a pass of two plans:
// 64 sequences that drop five tokens and take five 5.7 in a graph (512 threads a CTA
// 6.9, 1,024 22); 64 x 64 slots 6.2 in the cluster and 5.8 in a launch of their own, 64
// x 255 9.5 and 6.0; 256 prompts of up to 8,191 tokens given up and taken, 29 thousand
// pages and two million slots, 641 in one CTA, 59 with slots in a launch of their own,
// 15 with the cluster.  Above 512 sequences a thread returns the pages of its own one
// after the other: of 512 sequences half end and come again, 40 pages each, in 8.6, of
// 1,024 in 47, and one that ends with 7,900 pages takes 471 (of 512 sequences 12).
template <int N>
__global__ void __launch_bounds__(N) plan_kernel(const __grid_constant__ View c,
                                                 const int32_t *want, int n_new, int32_t *slots) {
  kvr::pdl_begin();
  __shared__ Sums s_warp[N / 32];
  __shared__ int s_start[N], s_page[N];
  const int tid = threadIdx.x, rank = (int)ptx::cluster_rank();
  const int each = (c.S + N - 1) / N, first = tid * each;  // sequences of a thread
  const int had = c.free[0];
  auto sums_of = [](const Change &x) {
    return Sums{x.take(), x.back(), (x.want + kTile - 1) / kTile};
  };
  Change x{};
  Sums mine{}, total{};
  bool bad = false;
#pragma unroll 4
  for (int j = 0; j < each; ++j) {
    x = change_of(c, want, first + j, n_new);
    mine = mine + sums_of(x);
    bad |= x.bad;
  }
  const Sums at = scan<N>(mine, s_warp, &total);
  bad = __syncthreads_or(bad);
  ptx::cluster_sync();  // every CTA has read the state
  const long long top = (long long)had + total.back;
  const long long many = slots ? (long long)c.S * n_new : 0;
  if (bad || total.take > top || top > c.n_pages) {
    if (tid == 0 && rank == 0) {
      atomicOr(c.err, bad ? (unsigned)kvr::ERR_LENGTH : (unsigned)kvr::ERR_CAPACITY);
      c.free[1] = 0;
    }
    if (many <= kInPlan)
      for (int i = rank * N + tid; i < many; i += kCluster * N) slots[i] = -1;
    return;
  }
  // Page `page` of sequence s goes back, the e-th of the call.
  auto give = [&](int s, int page, long long e) {
    int32_t *entry = c.table + (long long)s * c.tstride + page;
    const long long to = top - 1 - e;
    if (to >= 0 && to < c.n_pages) c.stack[to] = *entry;
    *entry = -1;
  };
  if (each == 1) {
    if (total.back > 0) {
      s_start[tid] = at.back;
      s_page[tid] = x.need;
      __syncthreads();
#pragma unroll 4
      for (int e = rank * N + tid; e < total.back; e += kCluster * N) {
        const int i = find<N>(s_start, e);
        give(i, s_page[i] + e - s_start[i], e);
      }
    }
  } else {
    Sums before = at;
    for (int j = 0; j < each && total.back > 0; ++j) {
      const Change y = change_of(c, want, first + j, n_new);
      if (j % kCluster == rank)
        for (int e = 0; e < y.back(); ++e) give(first + j, y.need + e, (long long)before.back + e);
      before = before + sums_of(y);
    }
    ptx::cluster_sync();  // every CTA has read the lengths again
  }
  if (rank == 0) {
    Sums before = at;
#pragma unroll 4
    for (int j = 0; j < each; ++j) {
      const int s = first + j;
      if (s >= c.S) break;
      if (each > 1) x = change_of(c, want, s, n_new);
      c.len[s] = x.want;
      c.from[s] = min(x.old, x.want);
      c.first[s] = (int)(top - 1 - before.take);
      c.tiles[s] = before.tiles;
      before = before + sums_of(x);
    }
    if (tid == 0) {
      c.tiles[c.S] = total.tiles;
      c.free[0] = (int)(top - total.take), c.free[1] = 1;
    }
  }
  if (many == 0 || many > kInPlan) return;
  ptx::cluster_sync();  // pages are back, the state is written
  for (int i = rank * N + tid; i < many; i += kCluster * N) {
    const int s = i / n_new;
    slots[i] = place(c, s, i - s * n_new, c.from[s], c.len[s], c.first[s]);
  }
}

__global__ void __launch_bounds__(kFill) fill_kernel(const __grid_constant__ View c, int n_new,
                                                     int32_t *slots) {
  kvr::pdl_begin();
  const bool done = c.free[1] != 0;
  for (int s = blockIdx.y; s < c.S; s += gridDim.y) {
    const int from = c.from[s], len = c.len[s], first = c.first[s];
    int32_t *to = slots + (long long)s * n_new;
    const int t0 = blockIdx.x * kFillTokens;
#pragma unroll
    for (int i = 0; i < kFillTokens / kFill; ++i) {
      const int t = t0 + i * kFill + threadIdx.x;
      if (t < n_new) to[t] = done ? place(c, s, t, from, len, first) : -1;
    }
  }
}

template <int N>
cudaError_t launch_plan(const View &c, const int32_t *lens, int n_new, int32_t *slots,
                        cudaStream_t st) {
  return kvr::launch_pdl_cluster(plan_kernel<N>, dim3(kCluster), dim3(N), kCluster, 0, st, c, lens,
                                 n_new, slots);
}

// ---- append -----------------------------------------------------------------

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b, __nv_bfloat16) {
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b, __nv_bfloat16) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b, float) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
  return __float_as_uint(r);
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b, float) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
  return __float_as_uint(r);
}
template <typename T>
__device__ __forceinline__ void widen(const uint4 &x, uint4 &lo, uint4 &hi) {
  lo.x = min2(lo.x, x.x, T{}), hi.x = max2(hi.x, x.x, T{});
  lo.y = min2(lo.y, x.y, T{}), hi.y = max2(hi.y, x.y, T{});
  lo.z = min2(lo.z, x.z, T{}), hi.z = max2(hi.z, x.z, T{});
  lo.w = min2(lo.w, x.w, T{}), hi.w = max2(hi.w, x.w, T{});
}

struct AppendParams {
  View c;
  int lb, nl, n, n_new, runs;
  const int32_t *slots;  // [n][n_new]
  const uint8_t *k, *v;  // [n][nl][n_new][H][d]
};

// A warp takes the tokens of a call that fall into one page, for one layer and
// head.  It alone writes that page's part, so it also knows when the page is full
// and can say what its keys lie between: the bounds cost no pass of their own, and
// what is dropped from the middle of a page cannot leave any that are too wide.  Bound
// by bytes: 2 x 8,191 tokens (1.5B geometry) 150 us, 6.3 TB/s read and written.
template <typename T, int D>
__global__ void __launch_bounds__(256) append_kernel(const __grid_constant__ AppendParams p) {
  kvr::pdl_begin();
  constexpr int kRow = D * (int)sizeof(T), kVec = kRow / 16, kPer = 32 / kVec;
  const View &c = p.c;
  const int lane = threadIdx.x & 31, vec = lane % kVec, sub = lane / kVec;
  const long long items = (long long)p.n * p.nl * c.H * p.runs;
  for (long long it = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); it < items;
       it += (long long)gridDim.x * 8) {
    const int h = (int)(it % c.H);
    const int run = (int)(it / c.H % p.runs);
    const int lr = (int)(it / ((long long)c.H * p.runs) % p.nl);
    const int n = (int)(it / ((long long)c.H * p.runs * p.nl));
    const int32_t *slots = p.slots + (long long)n * p.n_new;
    const int first = slots[0];
    if (first < 0) continue;
    const int r0 = first & (c.P - 1);
    const int t0 = run == 0 ? 0 : (run << c.psh) - r0;  // the run's first token
    if (t0 >= p.n_new) continue;
    const int most = min(p.n_new - t0, c.P - (run == 0 ? r0 : 0));
    const int slot = slots[t0];
    if (slot < 0) continue;
    const int row0 = slot & (c.P - 1), page = slot >> c.psh;
    // slots follow one another, up to the page's end or the sequence's
    int count = 0;
    bool wrong = page >= c.n_pages || (run > 0 && row0 != 0);
    for (int i = 0; i < most && !wrong; i += 32) {
      const int x = i + lane < most ? slots[t0 + i + lane] : -1;
      const unsigned fits = __ballot_sync(0xffffffffu, x == slot + i + lane);
      wrong = __any_sync(0xffffffffu, x >= 0 && x != slot + i + lane);
      const int good = fits == 0xffffffffu ? 32 : __ffs(~fits) - 1;
      count += good;
      if (good < 32) break;
    }
    if (wrong) {
      if (lane == 0) atomicOr(c.err, (unsigned)kvr::ERR_LENGTH);
      continue;
    }
    const long long in = ((((long long)n * p.nl + lr) * p.n_new + t0) * c.H + h) * kRow;
    const long long in_step = (long long)c.H * kRow;
    uint8_t *kp = c.K + pool_row(c, p.lb + lr, page, h) * kRow;
    uint8_t *vp = c.V + pool_row(c, p.lb + lr, page, h) * kRow;
    const bool full = row0 + count == c.P;
    uint4 lo, hi;
    bool any = false;
    for (int i = sub; i < count; i += kPer) {
      const uint4 k = __ldg(reinterpret_cast<const uint4 *>(p.k + in + i * in_step) + vec);
      const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p.v + in + i * in_step) + vec);
      reinterpret_cast<uint4 *>(kp + (long long)(row0 + i) * kRow)[vec] = k;
      reinterpret_cast<uint4 *>(vp + (long long)(row0 + i) * kRow)[vec] = v;
      if (!any) lo = hi = k, any = true;
      widen<T>(k, lo, hi);
    }
    if (!full) continue;
    for (int i = sub; i < row0; i += kPer) {  // rows of earlier calls
      const uint4 k = reinterpret_cast<const uint4 *>(kp + (long long)i * kRow)[vec];
      if (!any) lo = hi = k, any = true;
      widen<T>(k, lo, hi);
    }
    // (a page has 16 rows at least: every part of the warp has seen some)
#pragma unroll
    for (int o = kVec; o < 32; o <<= 1) {
      uint4 a, b;
      a.x = __shfl_xor_sync(0xffffffffu, lo.x, o), b.x = __shfl_xor_sync(0xffffffffu, hi.x, o);
      a.y = __shfl_xor_sync(0xffffffffu, lo.y, o), b.y = __shfl_xor_sync(0xffffffffu, hi.y, o);
      a.z = __shfl_xor_sync(0xffffffffu, lo.z, o), b.z = __shfl_xor_sync(0xffffffffu, hi.z, o);
      a.w = __shfl_xor_sync(0xffffffffu, lo.w, o), b.w = __shfl_xor_sync(0xffffffffu, hi.w, o);
      widen<T>(a, lo, hi);
      widen<T>(b, lo, hi);
    }
    if (sub == 0) {
      uint4 *bp = reinterpret_cast<uint4 *>(
          c.bounds + (((long long)(p.lb + lr) * c.n_pages + page) * c.H + h) * 2 * kRow);
      bp[vec] = lo;
      bp[kVec + vec] = hi;
    }
  }
}

template <typename T, int D>
cudaError_t launch_append(const AppendParams &p, int sms, cudaStream_t st) {
  const long long items = (long long)p.n * p.nl * p.c.H * p.runs;
  const long long grid = std::min<long long>((items + 7) / 8, 8ll * sms);
  return kvr::launch_pdl(append_kernel<T, D>, dim3((unsigned)grid), dim3(256), 0, st, p);
}

}  // namespace
}  // namespace paged
}  // namespace kvr

using kvr::report_error;
using kvr::paged::View;

struct kvr_paged {
  kvr_paged_desc desc;
  View view;
  kvr::paged::Device device;
  uint64_t launches = 0;
};

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

template <typename... A>
kvr_status fail(kvr_status st, const char *fmt, A... a) {
  char buf[256];
  snprintf(buf, sizeof buf, fmt, a...);
  return static_cast<kvr_status>(report_error(st, buf));
}
kvr_status fail(kvr_status st, const char *msg) {
  return static_cast<kvr_status>(report_error(st, msg));
}
kvr_status cuda_fail(const char *where, cudaError_t e) {
  return static_cast<kvr_status>(kvr::report_cuda_error(where, e));
}
cudaStream_t as_stream(void *s) { return static_cast<cudaStream_t>(s); }
bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool aligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

struct Layout {
  size_t K, V, bounds, table, len, from, first, tiles, stack, free, ticket, err, total;
};

bool layout_of(const kvr_paged_desc *d, Layout *l) {
  if (!d || d->n_seq < 1 || d->n_seq > 65535 || d->n_layers < 1 || d->n_kv_heads < 1 ||
      d->group < 1 || d->group > kvr::paged::kHeads ||
      (d->head_dim != 64 && d->head_dim != 128) || d->n_pages < 1 || d->table_pages < 1 ||
      (d->page_rows != 16 && d->page_rows != 32 && d->page_rows != 64 && d->page_rows != 128) ||
      (long long)d->n_pages * d->page_rows > INT_MAX ||
      (long long)d->table_pages * d->page_rows > INT_MAX ||
      (long long)d->n_layers * d->n_kv_heads > 65535 ||
      (long long)d->n_layers * d->n_kv_heads * d->n_seq >= INT_MAX ||
      // tiles are counted in 32 bits (2^31 of them are 8 TB of keys and values)
      (long long)d->n_layers * d->n_kv_heads * d->n_pages >
          INT_MAX / (d->page_rows / kvr::paged::kTile) ||
      (d->kv_dtype != KVR_BF16 && d->kv_dtype != KVR_F32) ||
      (d->out_dtype != KVR_BF16 && d->out_dtype != KVR_F32) ||
      !(d->softmax_scale >= 0.f && std::isfinite(d->softmax_scale)))
    return false;
  const size_t es = d->kv_dtype == KVR_BF16 ? 2 : 4;
  const size_t units = (size_t)d->n_layers * d->n_pages * d->n_kv_heads, row = d->head_dim * es;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes);
    return at;
  };
  l->K = take(units * d->page_rows * row);
  l->V = take(units * d->page_rows * row);
  l->bounds = take(units * 2 * row);
  l->table = take((size_t)d->n_seq * d->table_pages * 4);
  l->len = take((size_t)d->n_seq * 4);
  l->from = take((size_t)d->n_seq * 4);
  l->first = take((size_t)d->n_seq * 4);
  l->tiles = take(((size_t)d->n_seq + 1) * 4);
  l->stack = take((size_t)d->n_pages * 4);
  l->free = take(2 * 4);
  l->ticket = take(kvr::paged::kMostCtas * 4);
  l->err = take(16);
  l->total = off;
  return true;
}

kvr_status check_layers(const kvr_paged *c, int lb, int le) {
  if (!c) return fail(KVR_EINVAL, "null cache");
  if (lb < 0 || le > c->desc.n_layers || lb >= le)
    return fail(KVR_EINVAL, "layer range [%d, %d) outside [0, %d)", lb, le, c->desc.n_layers);
  return KVR_OK;
}

bool choice_ok(int budget, int window) {
  return budget >= 0 && window >= 1 && (long long)budget + window <= (1 << 24);
}

// Tiles of an attention over nl layers at most: of a pool that is full, or of `keep`
// pages of every unit; and of one unit.
void set_most(const kvr_paged *c, int keep, kvr::paged::AttendParams *p) {
  const kvr_paged_desc &d = c->desc;
  const long long a_page = d.page_rows / kvr::paged::kTile, units = (long long)p->nl * d.n_kv_heads;
  const long long of_one = keep ? std::min(keep, d.table_pages) : d.table_pages;
  p->most = std::min<long long>(d.n_pages, d.n_seq * of_one) * a_page * units;
  p->longest = std::min<long long>(d.n_pages, of_one) * a_page;
}

size_t score_stride(const kvr_paged *c) { return ((size_t)c->desc.table_pages + 1) / 2 * 2; }

// Parts of a workspace of either attention; `pages` of a choice, or none.
struct Work {
  size_t parts, score, list, rows, tiles, total;
  int keep;
};
Work work_of(const kvr_paged *c, int nl, int budget, int window) {
  const kvr_paged_desc &d = c->desc;
  Work w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 15) / 16 * 16;
    return at;
  };
  if (window > 0) w.keep = (int)std::min<long long>((long long)budget + window, d.table_pages);
  w.parts = take((size_t)2 * kvr::paged::attend_ctas(c->view, c->device) *
                 kvr::paged::part_floats(d.head_dim) * sizeof(float));
  if (window > 0) {
    const size_t units = (size_t)d.n_seq * nl * d.n_kv_heads;
    w.score = take(units * score_stride(c) * sizeof(float2));
    w.list = take(units * w.keep * sizeof(int32_t));
    w.rows = take((size_t)d.n_seq * sizeof(int32_t));
    w.tiles = take(((size_t)d.n_seq + 1) * sizeof(int32_t));
  }
  w.total = off;
  return w;
}

}  // namespace

extern "C" {

size_t kvr_paged_required_bytes(const kvr_paged_desc *desc) {
  Layout l;
  return layout_of(desc, &l) ? l.total : 0;
}

kvr_status kvr_paged_create(const kvr_paged_desc *desc, void *dev_buf, size_t bytes,
                            void *stream, kvr_paged **out) {
  if (!out) return fail(KVR_EINVAL, "null output handle");
  *out = nullptr;
  Layout l;
  if (!layout_of(desc, &l)) return fail(KVR_EINVAL, "invalid paged cache descriptor");
  if (!dev_buf) return fail(KVR_EINVAL, "null device buffer");
  if (reinterpret_cast<uintptr_t>(dev_buf) % kAlign)
    return fail(KVR_EINVAL, "device buffer not %zu-byte aligned", kAlign);
  if (bytes < l.total)
    return fail(KVR_ENOMEM, "buffer of %zu bytes < required %zu", bytes, l.total);
  kvr_paged *c = new (std::nothrow) kvr_paged();
  if (!c) return fail(KVR_ENOMEM, "host allocation failed");
  c->desc = *desc;
  uint8_t *b = static_cast<uint8_t *>(dev_buf);
  auto i32 = [&](size_t at) { return reinterpret_cast<int32_t *>(b + at); };
  View &v = c->view;
  v.K = b + l.K;
  v.V = b + l.V;
  v.bounds = b + l.bounds;
  v.table = i32(l.table);
  v.len = i32(l.len);
  v.from = i32(l.from);
  v.first = i32(l.first);
  v.tiles = i32(l.tiles);
  v.stack = i32(l.stack);
  v.free = i32(l.free);
  v.ticket = reinterpret_cast<unsigned *>(b + l.ticket);
  v.err = reinterpret_cast<unsigned *>(b + l.err);
  v.S = desc->n_seq;
  v.L = desc->n_layers;
  v.H = desc->n_kv_heads;
  v.G = desc->group;
  v.d = desc->head_dim;
  v.P = desc->page_rows;
  v.n_pages = desc->n_pages;
  v.tstride = desc->table_pages;
  v.psh = 31 - __builtin_clz((unsigned)desc->page_rows);
  v.scale = desc->softmax_scale > 0.f ? desc->softmax_scale
                                      : 1.0f / std::sqrt((float)desc->head_dim);
  v.io_bf16 = desc->kv_dtype == KVR_BF16;
  v.out_bf16 = desc->out_dtype == KVR_BF16;
  cudaError_t e = kvr::paged::prepare_attend(v, &c->device);
  if (e == cudaSuccess) e = kvr::paged::prepare_select(v);
  // tickets and the error word lie side by side
  if (e == cudaSuccess)
    e = cudaMemsetAsync(b + l.ticket, 0, l.total - l.ticket, as_stream(stream));
  if (e == cudaSuccess) {
    const long long most = std::max<long long>((long long)v.S * v.tstride, v.n_pages);
    const int grid = (int)std::min<long long>((most + 255) / 256, 4ll * c->device.sms);
    e = kvr::launch_pdl(kvr::paged::init_kernel, dim3(grid), dim3(256), 0, as_stream(stream), v);
  }
  if (e != cudaSuccess) {
    delete c;
    return cuda_fail("kvr_paged_create", e);
  }
  c->launches = 1;
  *out = c;
  return KVR_OK;
}

void kvr_paged_destroy(kvr_paged *cache) { delete cache; }

kvr_status kvr_paged_plan(kvr_paged *c, const int32_t *lens, int n_new, int32_t *slots,
                          void *stream) {
  if (!c || !lens) return fail(KVR_EINVAL, "null cache or lengths");
  if (n_new < 0 || n_new > (1 << 24)) return fail(KVR_EINVAL, "%d new tokens", n_new);
  if ((n_new > 0) != (slots != nullptr))
    return fail(KVR_EINVAL, "slots go with new tokens: %d of them", n_new);
  if (!aligned4(lens) || !aligned4(slots))
    return fail(KVR_EINVAL, "lengths and slots must be 4-byte aligned");
  const View &w = c->view;
  const cudaStream_t cs = as_stream(stream);
  const long long many = (long long)w.S * n_new;
  cudaError_t e = w.S <= kvr::paged::kPlanFew
                      ? kvr::paged::launch_plan<kvr::paged::kPlanFew>(w, lens, n_new, slots, cs)
                      : kvr::paged::launch_plan<kvr::paged::kPlan>(w, lens, n_new, slots, cs);
  if (e != cudaSuccess) return cuda_fail("kvr_paged_plan", e);
  c->launches += 1;
  if (many > kvr::paged::kInPlan) {
    const dim3 grid((n_new + kvr::paged::kFillTokens - 1) / kvr::paged::kFillTokens,
                    std::min(w.S, 65535));
    e = kvr::launch_pdl(kvr::paged::fill_kernel, grid, dim3(kvr::paged::kFill), 0, cs, w, n_new,
                        slots);
    if (e != cudaSuccess) return cuda_fail("kvr_paged_plan: slots", e);
    c->launches += 1;
  }
  return KVR_OK;
}

kvr_status kvr_paged_append(kvr_paged *c, int lb, int le, int n, int n_new,
                            const int32_t *slots, const void *k, const void *v, void *stream) {
  kvr_status st = check_layers(c, lb, le);
  if (st != KVR_OK) return st;
  if (n < 1 || n_new < 1 || n_new > (1 << 24))
    return fail(KVR_EINVAL, "%d sequences of %d tokens", n, n_new);
  if (!slots || !k || !v) return fail(KVR_EINVAL, "null slots, k or v");
  if (!aligned16(k) || !aligned16(v))
    return fail(KVR_EINVAL, "k and v must be 16-byte aligned");
  if (!aligned4(slots)) return fail(KVR_EINVAL, "slots must be 4-byte aligned");
  kvr::paged::AppendParams p{};
  p.c = c->view;
  p.lb = lb;
  p.nl = le - lb;
  p.n = n;
  p.n_new = n_new;
  // pages that n_new rows in a row can touch
  p.runs = (n_new + c->view.P - 2) / c->view.P + 1;
  p.slots = slots;
  p.k = static_cast<const uint8_t *>(k);
  p.v = static_cast<const uint8_t *>(v);
  const cudaStream_t cs = as_stream(stream);
  cudaError_t e;
  if (c->view.io_bf16)
    e = c->view.d == 128 ? kvr::paged::launch_append<__nv_bfloat16, 128>(p, c->device.sms, cs)
                         : kvr::paged::launch_append<__nv_bfloat16, 64>(p, c->device.sms, cs);
  else
    e = c->view.d == 128 ? kvr::paged::launch_append<float, 128>(p, c->device.sms, cs)
                         : kvr::paged::launch_append<float, 64>(p, c->device.sms, cs);
  if (e != cudaSuccess) return cuda_fail("kvr_paged_append", e);
  c->launches += 1;
  return KVR_OK;
}

size_t kvr_paged_attend_workspace_bytes(const kvr_paged *c, int lb, int le) {
  if (!c || lb < 0 || le > c->desc.n_layers || lb >= le) return 0;
  return work_of(c, le - lb, 0, 0).total;
}

size_t kvr_paged_attend_pages_workspace_bytes(const kvr_paged *c, int lb, int le, int budget,
                                              int window) {
  if (!c || lb < 0 || le > c->desc.n_layers || lb >= le || !choice_ok(budget, window)) return 0;
  return work_of(c, le - lb, budget, window).total;
}

kvr_status kvr_paged_attend(kvr_paged *c, int lb, int le, const void *q, void *out,
                            void *workspace, size_t workspace_bytes, void *stream) {
  kvr_status st = check_layers(c, lb, le);
  if (st != KVR_OK) return st;
  if (!q || !out || !workspace) return fail(KVR_EINVAL, "null q, out or workspace");
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace))
    return fail(KVR_EINVAL, "q, out and workspace must be 16-byte aligned");
  const Work w = work_of(c, le - lb, 0, 0);
  if (workspace_bytes < w.total)
    return fail(KVR_ENOMEM, "workspace of %zu bytes < required %zu", workspace_bytes, w.total);
  const View &v = c->view;
  kvr::paged::AttendParams p{};
  p.c = v;
  p.src = {v.table, v.tstride, 0, v.len, v.tiles};
  p.lb = lb;
  p.nl = le - lb;
  p.q = q;
  p.out = out;
  set_most(c, 0, &p);
  p.parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + w.parts);
  const cudaError_t e = kvr::paged::launch_attend(p, c->device, as_stream(stream));
  if (e != cudaSuccess) return cuda_fail("kvr_paged_attend", e);
  c->launches += 1;
  return KVR_OK;
}

kvr_status kvr_paged_attend_pages(kvr_paged *c, int lb, int le, const void *q, int budget,
                                  int window, void *out, int32_t *pages, void *workspace,
                                  size_t workspace_bytes, void *stream) {
  kvr_status st = check_layers(c, lb, le);
  if (st != KVR_OK) return st;
  if (!choice_ok(budget, window))
    return fail(KVR_EINVAL, "bad budget %d / window %d", budget, window);
  if (!q || !out || !workspace) return fail(KVR_EINVAL, "null q, out or workspace");
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace))
    return fail(KVR_EINVAL, "q, out and workspace must be 16-byte aligned");
  if (!aligned4(pages)) return fail(KVR_EINVAL, "pages must be 4-byte aligned");
  const Work w = work_of(c, le - lb, budget, window);
  if (workspace_bytes < w.total)
    return fail(KVR_ENOMEM, "workspace of %zu bytes < required %zu", workspace_bytes, w.total);
  const View &v = c->view;
  char *ws = static_cast<char *>(workspace);
  kvr::paged::SelectParams s{};
  s.c = v;
  s.lb = lb;
  s.nl = le - lb;
  s.q = q;
  s.budget = budget;
  s.window = window;
  s.keep = w.keep;
  s.score = reinterpret_cast<float2 *>(ws + w.score);
  s.sstride = (int)score_stride(c);
  s.list = reinterpret_cast<int32_t *>(ws + w.list);
  s.rows = reinterpret_cast<int32_t *>(ws + w.rows);
  s.tiles = reinterpret_cast<int32_t *>(ws + w.tiles);
  s.chosen = pages;
  int n = 0;
  cudaError_t e = kvr::paged::launch_select(s, c->device.sms, as_stream(stream), &n);
  c->launches += n;
  if (e != cudaSuccess) return cuda_fail("kvr_paged_attend_pages: choice", e);
  const long long units = (long long)(le - lb) * v.H;
  kvr::paged::AttendParams p{};
  p.c = v;
  p.src = {s.list, units * w.keep, w.keep, s.rows, s.tiles};
  p.lb = lb;
  p.nl = le - lb;
  p.q = q;
  p.out = out;
  set_most(c, w.keep, &p);
  p.parts = reinterpret_cast<float *>(ws + w.parts);
  e = kvr::paged::launch_attend(p, c->device, as_stream(stream));
  if (e != cudaSuccess) return cuda_fail("kvr_paged_attend_pages", e);
  c->launches += 1;
  return KVR_OK;
}

kvr_status kvr_paged_tables(const kvr_paged *c, const int32_t **table, int64_t *row_stride,
                            const int32_t **lens, const int32_t **n_free) {
  if (!c) return fail(KVR_EINVAL, "null cache");
  if (table) *table = c->view.table;
  if (row_stride) *row_stride = c->view.tstride;
  if (lens) *lens = c->view.len;
  if (n_free) *n_free = c->view.free;
  return KVR_OK;
}

kvr_status kvr_paged_rows(const kvr_paged *c, void **k, void **v, void **bounds) {
  if (!c) return fail(KVR_EINVAL, "null cache");
  if (k) *k = c->view.K;
  if (v) *v = c->view.V;
  if (bounds) *bounds = c->view.bounds;
  return KVR_OK;
}

kvr_status kvr_paged_launch_count(const kvr_paged *c, uint64_t *count) {
  if (!c || !count) return fail(KVR_EINVAL, "null argument");
  *count = c->launches;
  return KVR_OK;
}

kvr_status kvr_paged_sync_status(kvr_paged *c, void *stream) {
  if (!c) return fail(KVR_EINVAL, "null cache");
  // all on the caller's stream, as for the 4-bit cache
  const cudaStream_t cs = as_stream(stream);
  unsigned word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, c->view.err, sizeof word, cudaMemcpyDeviceToHost, cs);
  if (e == cudaSuccess) e = cudaStreamSynchronize(cs);
  if (e != cudaSuccess) return cuda_fail("kvr_paged_sync_status: read", e);
  if (!word) return KVR_OK;
  e = cudaMemsetAsync(c->view.err, 0, sizeof word, cs);
  if (e == cudaSuccess) e = cudaStreamSynchronize(cs);
  if (e != cudaSuccess) return cuda_fail("kvr_paged_sync_status: clear", e);
  return fail(KVR_EDEVICE, "device error word 0x%x (%s%s%s)", word,
              word & kvr::ERR_CAPACITY ? "capacity " : "",
              word & kvr::ERR_NONFINITE ? "non-finite " : "",
              word & kvr::ERR_LENGTH ? "length" : "");
}

}  // extern "C"
