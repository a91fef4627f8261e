// kvr_verify.cu -- verification of drafted tokens (include/kvr.h,
// kvr_verify_drafts): rejection sampling of a draft against the target, with
// given random numbers.  Two launches:
//
//   stats_kernel   every row's softmax statistics (max, sum of exponentials): one
//                  read of every logit, which is what the call costs.  A row is
//                  cut into items of 256 groups of 16 bytes' worth of logits, a
//                  warp each, all loads of an item in flight; an item's result is
//                  the same wherever the row lies, so equal rows have equal
//                  statistics and the same logits are never rejected.
//   decide_kernel  every CTA of a sequence joins its rows' items and takes the
//                  same decisions; together they run the race over the one row
//                  that the next token comes from.  Keys (weight / race, lower
//                  token) are whole numbers, so the order in which CTAs offer
//                  theirs does not matter.
//
// Bound by the logits' bytes: four tokens of 64 sequences over 152,064 (bf16) 49 us,
// 33 of them the statistics (5.4 TB/s); three of one over 32,000 (fp32) 7.6 us of
// latency.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "../../include/kvr.h"
#include "kvr_device.cuh"
#include "kvr_internal.h"
#include "kvr_ptx.cuh"

namespace {

using kvr::dev::to_f;
using namespace kvr::ptx;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kLoads = 8;                  // groups of a lane
constexpr int kItem = 32 * kLoads;         // groups of an item
constexpr float kLog2e = 1.4426950408889634f;

struct Params {
  int S, T, V;
  float c;  // log2(e) / temperature
  const void *target, *draft;
  long long ts, ds;
  const int32_t *tokens;
  const float *u, *race;
  const int32_t *counts;
  int32_t *accepted, *out;
  // workspace
  float2 *part;               // [S][2 T + 1][items]: (max, sum)
  unsigned long long *best;   // [S] greatest key
  unsigned *ticket;           // [S] CTAs that have offered theirs
  int items;                  // of a row
};

__device__ __forceinline__ int drafts_of(const Params &p, int s) {
  return p.counts ? max(0, min(p.counts[s], p.T)) : p.T;
}
// Row i of sequence s: the target's T + 1 rows, then the draft's T.
template <typename T>
__device__ __forceinline__ const T *row_of(const Params &p, int s, int i) {
  return i <= p.T ? static_cast<const T *>(p.target) + ((long long)s * (p.T + 1) + i) * p.ts
                  : static_cast<const T *>(p.draft) + ((long long)s * p.T + i - p.T - 1) * p.ds;
}

// A row in groups of N elements from its start.  Where the row does not start on
// 16 bytes a group is cut out of the two vectors that hold it, or read element by
// element where those reach beyond the row.
template <typename T>
struct Row {
  static constexpr int N = 16 / (int)sizeof(T);
  const T *p;
  int V, shift;  // shift: elements between the vector's start and the group's
  __device__ Row(const T *p, int V)
      : p(p), V(V), shift((int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T))) {}
  // Group v; elements beyond the row are -inf.
  __device__ __forceinline__ uint4 load(int v) const {
    const int e0 = v * N;
    if (shift == 0 && e0 + N <= V) return __ldg(reinterpret_cast<const uint4 *>(p + e0));
    if (shift != 0 && e0 >= shift && e0 - shift + 2 * N <= V) {
      const uint4 *at = reinterpret_cast<const uint4 *>(p + e0 - shift);
      const uint4 a = __ldg(at), b = __ldg(at + 1);
      const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      const int bytes = shift * (int)sizeof(T), bits = 8 * (bytes & 3);
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t lo = w[i], hi = w[i + 1];
#pragma unroll
        for (int k = 1; k < 4; ++k)
          if ((bytes >> 2) == k) lo = w[i + k], hi = i + k + 1 < 8 ? w[(i + k + 1) & 7] : 0u;
        o[i] = __funnelshift_r(lo, hi, bits);
      }
      return make_uint4(o[0], o[1], o[2], o[3]);
    }
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = N == 8 ? 0xFF80FF80u : 0xFF800000u;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e0 + i < V) {
        if (N == 8) {
          const uint32_t x = reinterpret_cast<const uint16_t *>(p)[e0 + i];
          const uint32_t keep = i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
          o[(i >> 1) & 3] = (o[(i >> 1) & 3] & keep) | (x << (16 * (i & 1)));
        } else {
          o[i & 3] = reinterpret_cast<const uint32_t *>(p)[e0 + i];
        }
      }
    return make_uint4(o[0], o[1], o[2], o[3]);
  }
  static __device__ __forceinline__ void widen(const uint4 &w, float (&x)[N]) {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (N == 8) {
        x[2 * i] = __uint_as_float(a[i] << 16);
        x[(2 * i + 1) % N] = __uint_as_float(a[i] & 0xFFFF0000u);
      } else {
        x[i] = __uint_as_float(a[i]);
      }
    }
  }
};

// The greatest element of a lane's groups; NaN does not count.
template <typename T>
__device__ __forceinline__ float greatest(const uint4 (&w)[kLoads]);
template <>
__device__ __forceinline__ float greatest<float>(const uint4 (&w)[kLoads]) {
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < kLoads; ++k)
    m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(w[k].x), __uint_as_float(w[k].y)),
                       fmaxf(__uint_as_float(w[k].z), __uint_as_float(w[k].w))));
  return m;
}
template <>
__device__ __forceinline__ float greatest<__nv_bfloat16>(const uint4 (&w)[kLoads]) {
  auto two = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162 *>(&x); };
  __nv_bfloat162 m = two(0xFF80FF80u);
#pragma unroll
  for (int k = 0; k < kLoads; ++k)
    m = __hmax2(m, __hmax2(__hmax2(two(w[k].x), two(w[k].y)), __hmax2(two(w[k].z), two(w[k].w))));
  return fmaxf(__low2float(m), __high2float(m));
}

// What logits are taken relative to: the maximum.  A NaN, or +inf less itself, makes
// the sum NaN.
__device__ __forceinline__ float above(float m) { return m == -INFINITY ? 0.f : m; }

template <typename T>
__global__ void __launch_bounds__(kThreads) stats_kernel(const __grid_constant__ Params p) {
  kvr::pdl_begin();
  constexpr int N = Row<T>::N;
  const int lane = threadIdx.x & 31, rows = 2 * p.T + 1;
  const long long all = (long long)gridDim.x * kWarps;
  // what decide_kernel counts in
  for (long long s = (long long)blockIdx.x * kThreads + threadIdx.x; s < p.S;
       s += (long long)gridDim.x * kThreads) {
    p.best[s] = 0;
    p.ticket[s] = 0;
  }
  const long long total = (long long)p.S * rows * p.items;
  for (long long at = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); at < total;
       at += all) {
    const unsigned row = (unsigned)(at / p.items);
    const int item = (int)(at - (long long)row * p.items);
    const int s = row / rows, i = row % rows;
    // a row behind the sequence's drafts takes no part
    const int n = drafts_of(p, s);
    if (i <= p.T ? i > n : i - p.T - 1 >= n) continue;
    const Row<T> r(row_of<T>(p, s, i), p.V);
    const int nv = (p.V + N - 1) / N;
    uint4 w[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int v = item * kItem + k * 32 + lane;
      const uint32_t none = N == 8 ? 0xFF80FF80u : 0xFF800000u;
      w[k] = v < nv ? r.load(v) : make_uint4(none, none, none, none);
    }
    const float m = kvr::dev::warp_max(greatest<T>(w));
    // Subtracted first, then scaled, as everywhere below: exact at the maximum.  (The
    // product c m rounds by 0.1 and more where m is 20 and the temperature 1e-5.)
    const uint64_t c2 = pk2(p.c, p.c), ref2 = pk2(-above(m), -above(m));
    uint64_t z2[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      float x[N];
      r.widen(w[k], x);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        float a, b;
        upk2(mul2(add2(pk2(x[e], x[e + 1]), ref2), c2), a, b);
        z2[(e >> 1) & 1] = add2(z2[(e >> 1) & 1], pk2(ex2(a), ex2(b)));
      }
    }
    float z, zb;
    upk2(add2(z2[0], z2[1]), z, zb);
    z += zb;
    z = kvr::dev::warp_sum(z);
    if (lane == 0) p.part[at] = make_float2(m, z);
  }
}

// One warp: row i of sequence s, joined: (max, 1 / sum), or (., NaN) without a
// softmax.
__device__ __forceinline__ float2 stats_of(const Params &p, int s, int i) {
  const float2 *part = p.part + ((long long)s * (2 * p.T + 1) + i) * p.items;
  const int lane = threadIdx.x & 31;
  float m = -INFINITY;
  for (int k = lane; k < p.items; k += 32) m = fmaxf(m, __ldcg(&part[k].x));
  m = kvr::dev::warp_max(m);
  float z = 0.f;
  for (int k = lane; k < p.items; k += 32) {
    const float2 x = __ldcg(part + k);
    z = fmaf(x.y, ex2((above(x.x) - above(m)) * p.c), z);
  }
  z = kvr::dev::warp_sum(z);
  return make_float2(m, z == z && z > 0.f && fabsf(m) < INFINITY ? 1.f / z : NAN);
}

// The greatest key of every step-th group of the vocabulary from `first`; every
// thread gets it.
template <typename T>
__device__ unsigned long long race_best(const Params &p, const T *tr, const T *dr, float2 tp,
                                        float2 tq, const float *race, int first, int step,
                                        unsigned long long *red) {
  constexpr int N = Row<T>::N;
  const Row<T> t(tr, p.V), d(dr ? dr : tr, p.V);
  const bool even = (reinterpret_cast<uintptr_t>(race) & 15) == 0;
  const int groups = (p.V + N - 1) / N;
  float most = 0.f;  // a thread's tokens ascend, so the first of equals stays
  int at = -1;
  constexpr int kAhead = 2;  // groups of a thread in flight
  for (int v0 = first + threadIdx.x; v0 < groups; v0 += kAhead * step) {
    uint4 tw[kAhead], dw[kAhead];
    float e[kAhead][N];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int v = v0 + k * step;
      const uint32_t none = N == 8 ? 0xFF80FF80u : 0xFF800000u;
      tw[k] = make_uint4(none, none, none, none);
      if (v < groups) {
        tw[k] = t.load(v);
        dw[k] = dr ? d.load(v) : make_uint4(0, 0, 0, 0);
        if (even && v * N + N <= p.V) {
#pragma unroll
          for (int i = 0; i < N / 4; ++i) {
            const float4 f = __ldg(reinterpret_cast<const float4 *>(race + v * N) + i);
            e[k][4 * i] = f.x, e[k][4 * i + 1] = f.y, e[k][4 * i + 2] = f.z,
                    e[k][4 * i + 3] = f.w;
          }
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) e[k][i] = v * N + i < p.V ? __ldg(race + v * N + i) : 1.f;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int v = v0 + k * step;
      if (v >= groups) break;
      float x[N], y[N];
      t.widen(tw[k], x);
      d.widen(dw[k], y);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float w = ex2((x[i] - tp.x) * p.c) * tp.y;
        if (dr) w -= ex2((y[i] - tq.x) * p.c) * tq.y;
        w *= rcp(e[k][i]);
        if (w > most) {  // not beyond the row, where x is -inf
          most = w;
          at = v * N + i;
        }
      }
    }
  }
  unsigned long long best =
      at < 0 ? 0
             : ((unsigned long long)__float_as_uint(most) << 32) | (0xFFFFFFFFu - (unsigned)at);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned long long k = __shfl_xor_sync(0xffffffffu, best, o);
    if (k > best) best = k;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w)
    if (red[w] > best) best = red[w];
  return best;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) decide_kernel(const __grid_constant__ Params p) {
  kvr::pdl_begin();
  __shared__ unsigned long long s_red[kWarps];
  __shared__ float2 s_stat[2 * 64 + 1];
  __shared__ float s_p[64], s_q[64];
  __shared__ int s_last;
  const int s = blockIdx.y, n = drafts_of(p, s);
  const int32_t *tok = p.tokens + (size_t)s * p.T;
  for (int i = threadIdx.x >> 5; i < 2 * p.T + 1; i += kWarps)
    if (i <= p.T ? i <= n : i - p.T - 1 < n) {
      const float2 x = stats_of(p, s, i);
      if ((threadIdx.x & 31) == 0) s_stat[i] = x;
    }
  __syncthreads();
  for (int t = threadIdx.x; t < n; t += kThreads) {
    const int x = tok[t];
    const float2 tp = s_stat[t], tq = s_stat[p.T + 1 + t];
    const bool fine = x >= 0 && x < p.V;  // NaN: the sequence ends there
    s_p[t] = fine ? ex2((to_f(row_of<T>(p, s, t)[x]) - tp.x) * p.c) * tp.y : NAN;
    s_q[t] = fine ? ex2((to_f(row_of<T>(p, s, p.T + 1 + t)[x]) - tq.x) * p.c) * tq.y : NAN;
  }
  __syncthreads();
  int a = 0;
  while (a < n && p.u[(size_t)s * p.T + a] * s_q[a] < s_p[a]) ++a;
  const float2 tp = s_stat[a], tq = a < n ? s_stat[p.T + 1 + a] : make_float2(0.f, 0.f);
  const bool bad = a < n ? !(s_p[a] == s_p[a] && s_q[a] == s_q[a]) : tp.y != tp.y;
  const T *tr = row_of<T>(p, s, a);
  const T *dr = a < n ? row_of<T>(p, s, p.T + 1 + a) : nullptr;
  const float *race = p.race + (size_t)s * p.V;
  if (!bad) {
    const unsigned long long best = race_best<T>(p, tr, dr, tp, tq, race, blockIdx.x * kThreads,
                                                 gridDim.x * kThreads, s_red);
    if (threadIdx.x == 0 && best) atomicMax(p.best + s, best);
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) s_last = atomicAdd(p.ticket + s, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  unsigned long long best = bad ? 0 : __ldcg(p.best + s);
  if (!bad && !best)  // nothing is left of p - q: the target's own row
    best = race_best<T>(p, tr, nullptr, tp, tq, race, 0, kThreads, s_red);
  const int next = bad || !best ? -1 : (int)(0xFFFFFFFFu - (unsigned)best);
  if (threadIdx.x == 0) p.accepted[s] = a;
  for (int t = threadIdx.x; t <= p.T; t += kThreads)
    p.out[(size_t)s * (p.T + 1) + t] = t < a ? tok[t] : t == a ? next : -1;
}

template <typename... A>
kvr_status fail(kvr_status st, const char *fmt, A... a) {
  char buf[256];
  snprintf(buf, sizeof buf, fmt, a...);
  return static_cast<kvr_status>(kvr::report_error(st, buf));
}
kvr_status fail(kvr_status st, const char *msg) {
  return static_cast<kvr_status>(kvr::report_error(st, msg));
}

// log2(e) / temperature; infinite or NaN where the temperature cannot be used.
float scale_of(float temperature) {
  return temperature > 0.f && std::isfinite(temperature) ? kLog2e / temperature : NAN;
}

bool desc_ok(const kvr_verify_desc *d) {
  return d && d->n_seq >= 1 && d->n_seq <= 65535 && d->n_draft >= 0 && d->n_draft <= 64 &&
         d->vocab >= 1 && std::isfinite(scale_of(d->temperature)) &&
         (d->logits_dtype == KVR_BF16 || d->logits_dtype == KVR_F32);
}

int items_of(int vocab, int es) {
  const int groups = (int)(((long long)vocab * es + 15) / 16);
  return (groups + kItem - 1) / kItem;
}

template <typename T>
cudaError_t launch(Params &p, cudaStream_t st) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  constexpr int N = Row<T>::N;
  p.items = items_of(p.V, (int)sizeof(T));
  const long long total = (long long)p.S * (2 * p.T + 1) * p.items;
  const long long grid = std::min<long long>((total + kWarps - 1) / kWarps, 4 * sms);
  e = kvr::launch_pdl(stats_kernel<T>, dim3((unsigned)grid), dim3(kThreads), 0, st, p);
  if (e != cudaSuccess) return e;
  // CTAs of a sequence: at most four an SM over all sequences, which run at once, a
  // group a thread at least (64 sequences of 152,064: 9 a sequence)
  const int ctas = (int)std::max<long long>(
      1, std::min<long long>(4 * sms / p.S, p.V / (N * kThreads)));
  return kvr::launch_pdl(decide_kernel<T>, dim3(ctas, p.S), dim3(kThreads), 0, st, p);
}

// Offsets of the workspace's parts.
struct Work {
  size_t part, best, ticket, total;
};
Work work_of(const kvr_verify_desc *d) {
  Work w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 15) / 16 * 16;
    return at;
  };
  // (the workspace serves either type of logits)
  w.part = take((size_t)d->n_seq * (2 * d->n_draft + 1) * items_of(d->vocab, 4) * sizeof(float2));
  w.best = take((size_t)d->n_seq * sizeof(unsigned long long));
  w.ticket = take((size_t)d->n_seq * sizeof(unsigned));
  w.total = off;
  return w;
}

}  // namespace

extern "C" {

size_t kvr_verify_workspace_bytes(const kvr_verify_desc *d) {
  if (!desc_ok(d)) return 0;
  return work_of(d).total;
}

kvr_status kvr_verify_drafts(const kvr_verify_desc *d, const void *target,
                             int64_t target_stride, const void *draft, int64_t draft_stride,
                             const int32_t *tokens, const float *u, const float *race,
                             const int32_t *counts, int32_t *accepted, int32_t *out_tokens,
                             void *workspace, size_t workspace_bytes, void *stream) {
  if (!desc_ok(d)) return fail(KVR_EINVAL, "invalid verification descriptor");
  if (!target || !race || !accepted || !out_tokens || !workspace)
    return fail(KVR_EINVAL, "null target, race, accepted, out_tokens or workspace");
  if (d->n_draft > 0 && (!draft || !tokens || !u))
    return fail(KVR_EINVAL, "null draft, tokens or u");
  if (target_stride < d->vocab || (d->n_draft > 0 && draft_stride < d->vocab))
    return fail(KVR_EINVAL, "row stride < vocab %d", d->vocab);
  if (reinterpret_cast<uintptr_t>(workspace) % 16)
    return fail(KVR_EINVAL, "workspace must be 16-byte aligned");
  const size_t need = kvr_verify_workspace_bytes(d);
  if (workspace_bytes < need)
    return fail(KVR_ENOMEM, "workspace of %zu bytes < required %zu", workspace_bytes, need);
  Params p{};
  p.S = d->n_seq;
  p.T = d->n_draft;
  p.V = d->vocab;
  p.c = scale_of(d->temperature);
  p.target = target;
  p.draft = draft;
  p.ts = target_stride;
  p.ds = draft_stride;
  p.tokens = tokens;
  p.u = u;
  p.race = race;
  p.counts = counts;
  p.accepted = accepted;
  p.out = out_tokens;
  char *ws = static_cast<char *>(workspace);
  const Work w = work_of(d);
  p.part = reinterpret_cast<float2 *>(ws + w.part);
  p.best = reinterpret_cast<unsigned long long *>(ws + w.best);
  p.ticket = reinterpret_cast<unsigned *>(ws + w.ticket);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = d->logits_dtype == KVR_BF16 ? launch<__nv_bfloat16>(p, st)
                                                    : launch<float>(p, st);
  return e == cudaSuccess ? KVR_OK
                          : static_cast<kvr_status>(kvr::report_cuda_error("kvr_verify_drafts", e));
}

}  // extern "C"
