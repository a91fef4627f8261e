// kvr_verify.cu -- verification of drafted tokens (include/kvr.h,
// kvr_verify_drafts): rejection sampling of a draft against the target, with
// given random numbers.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdio>

#include "../../include/kvr.h"
#include "kvr_device.cuh"
#include "kvr_internal.h"

namespace {

using kvr::dev::to_f;

constexpr int kThreads = 256;

struct Params {
  int S, T, V;
  float c;  // 1 / temperature
  const void *target, *draft;
  long long ts, ds;
  const int32_t *tokens;
  const float *u, *race;
  const int32_t *counts;
  int32_t *accepted, *out;
  float2 *stats;  // [S][2 T + 1]: target rows, then draft rows: (max, 1 / sum)
};

__device__ __forceinline__ float block_max(float x, float *red) {
  x = kvr::dev::warp_max(x);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = red[0];
  for (int w = 1; w < kThreads / 32; ++w) x = fmaxf(x, red[w]);
  __syncthreads();
  return x;
}
__device__ __forceinline__ float block_sum(float x, float *red) {
  x = kvr::dev::warp_sum(x);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.f;
  for (int w = 0; w < kThreads / 32; ++w) x += red[w];
  __syncthreads();
  return x;
}

__device__ __forceinline__ int drafts_of(const Params &p, int s) {
  return p.counts ? max(0, min(p.counts[s], p.T)) : p.T;
}
// Row i of sequence s: the target's T + 1 rows, then the draft's T.
template <typename T>
__device__ __forceinline__ const T *row_of(const Params &p, int s, int i) {
  return i <= p.T ? static_cast<const T *>(p.target) + ((long long)s * (p.T + 1) + i) * p.ts
                  : static_cast<const T *>(p.draft) + ((long long)s * p.T + i - p.T - 1) * p.ds;
}

// The softmax statistics of every row: one CTA a row.
template <typename T>
__global__ void __launch_bounds__(kThreads) stats_kernel(const Params p) {
  kvr::pdl_begin();
  __shared__ float red[kThreads / 32];
  const int i = blockIdx.x, s = blockIdx.y;
  const T *x = row_of<T>(p, s, i);
  float m = -INFINITY;
  bool nan = false;
  for (int v = threadIdx.x; v < p.V; v += kThreads) {
    const float y = to_f(x[v]) * p.c;
    nan |= y != y;
    m = fmaxf(m, y);
  }
  m = block_max(nan ? INFINITY : m, red);
  float z = 0.f;
  if (isfinite(m))
    for (int v = threadIdx.x; v < p.V; v += kThreads) z += expf(to_f(x[v]) * p.c - m);
  z = block_sum(z, red);
  if (threadIdx.x == 0)
    p.stats[(size_t)s * (2 * p.T + 1) + i] = make_float2(m, isfinite(m) ? 1.f / z : NAN);
}

// The decisions of a sequence and its next token: one CTA a sequence.
template <typename T>
__global__ void __launch_bounds__(kThreads) decide_kernel(const Params p) {
  kvr::pdl_begin();
  __shared__ unsigned long long s_best[kThreads / 32];
  __shared__ int s_any;
  const int s = blockIdx.x, n = drafts_of(p, s);
  const float2 *st = p.stats + (size_t)s * (2 * p.T + 1);
  const int32_t *tok = p.tokens + (size_t)s * p.T;
  int a = 0;
  bool bad = false;
  for (; a < n; ++a) {
    const float2 tp = st[a], tq = st[p.T + 1 + a];
    const int x = tok[a];
    if (!isfinite(tp.y) || !isfinite(tq.y) || x < 0 || x >= p.V) {
      bad = true;
      break;
    }
    const float pp = expf(to_f(row_of<T>(p, s, a)[x]) * p.c - tp.x) * tp.y;
    const float qq = expf(to_f(row_of<T>(p, s, p.T + 1 + a)[x]) * p.c - tq.x) * tq.y;
    if (!(p.u[(size_t)s * p.T + a] * qq < pp)) break;
  }
  if (a == n) bad = !isfinite(st[a].y);
  int next = -1;
  if (!bad) {
    const T *tr = row_of<T>(p, s, a);
    const T *dr = a < n ? row_of<T>(p, s, p.T + 1 + a) : nullptr;
    const float2 tp = st[a], tq = a < n ? st[p.T + 1 + a] : make_float2(0.f, 0.f);
    const float *race = p.race + (size_t)s * p.V;
    for (int pass = 0; pass < 2; ++pass) {  // the second: an empty residual
      unsigned long long best = 0;
      for (int v = threadIdx.x; v < p.V; v += kThreads) {
        float w = expf(to_f(tr[v]) * p.c - tp.x) * tp.y;
        if (dr) w -= expf(to_f(dr[v]) * p.c - tq.x) * tq.y;
        if (w > 0.f) {
          const unsigned long long k =
              ((unsigned long long)__float_as_uint(w / race[v]) << 32) | (0xFFFFFFFFu - v);
          if (k > best) best = k;
        }
      }
      for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long k = __shfl_xor_sync(0xffffffffu, best, o);
        if (k > best) best = k;
      }
      if ((threadIdx.x & 31) == 0) s_best[threadIdx.x >> 5] = best;
      __syncthreads();
      for (int w = 0; w < kThreads / 32; ++w)
        if (s_best[w] > best) best = s_best[w];
      __syncthreads();
      if (best) {
        next = (int)(0xFFFFFFFFu - (unsigned)(best & 0xFFFFFFFFu));
        break;
      }
      dr = nullptr;
    }
  }
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

bool desc_ok(const kvr_verify_desc *d) {
  return d && d->n_seq >= 1 && d->n_seq <= 65535 && d->n_draft >= 0 && d->n_draft <= 64 &&
         d->vocab >= 1 && d->temperature >= 0.f && std::isfinite(d->temperature) &&
         (d->logits_dtype == KVR_BF16 || d->logits_dtype == KVR_F32);
}

template <typename T>
cudaError_t launch(const Params &p, cudaStream_t st) {
  cudaError_t e = kvr::launch_pdl(stats_kernel<T>, dim3(2 * p.T + 1, p.S), dim3(kThreads), 0, st, p);
  if (e != cudaSuccess) return e;
  return kvr::launch_pdl(decide_kernel<T>, dim3(p.S), dim3(kThreads), 0, st, p);
}

}  // namespace

extern "C" {

size_t kvr_verify_workspace_bytes(const kvr_verify_desc *d) {
  if (!desc_ok(d)) return 0;
  return (size_t)d->n_seq * (2 * d->n_draft + 1) * sizeof(float2);
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
  p.c = d->temperature > 0.f ? 1.f / d->temperature : 1.f;
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
  p.stats = static_cast<float2 *>(workspace);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = d->logits_dtype == KVR_BF16 ? launch<__nv_bfloat16>(p, st)
                                                    : launch<float>(p, st);
  return e == cudaSuccess ? KVR_OK
                          : static_cast<kvr_status>(kvr::report_cuda_error("kvr_verify_drafts", e));
}

}  // extern "C"
