// kvr_kv4_attend.cu -- attention over the 4-bit cache (kvr_kv4.cuh).
#include <cuda_runtime.h>

#include "kvr_device.cuh"
#include "kvr_internal.h"
#include "kvr_kv4.cuh"

namespace kvr {
namespace kv4 {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;

// One CTA a (unit, token): its warps take every fourth row with an online
// softmax for the G heads, and are merged at the end.
template <typename T, typename O, int D>
__global__ void __launch_bounds__(kThreads)
    attend_kernel(const AttendParams p, const __grid_constant__ Seqs sq) {
  pdl_begin();
  const View &c = p.k.c;
  constexpr int E = D / 32;
  __shared__ float s_m[kWarps][8], s_z[kWarps][8], s_o[kWarps][8][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = blockIdx.x, h = blockIdx.y % c.H, lr = blockIdx.y / c.H, s = blockIdx.z;
  const size_t row = (((size_t)(p.k.s0 + s) * p.k.nl + lr) * p.n_q + t) * c.H + h;
  const T *q = static_cast<const T *>(p.q) + row * c.G * D;
  O *out = static_cast<O *>(p.out) + row * c.G * D;
  const int count = sq.count[s], n = t < count ? sq.len[s] - count + t + 1 : 0;
  const size_t u = unit_at(c, p.k.s0 + s, p.k.lb, lr, h);
  float qv[8][E], o[8][E], m[8], z[8];
  for (int g = 0; g < 8; ++g) {
    m[g] = -1e30f;
    z[g] = 0.f;
    for (int e = 0; e < E; ++e) {
      qv[g][e] = g < c.G ? dev::to_f(q[g * D + lane + 32 * e]) * c.scale : 0.f;
      o[g][e] = 0.f;
    }
  }
  for (int r = warp; r < n; r += kWarps) {
    const uint8_t *block = block_at(c, u, r);
    float k[E], v[E];
    for (int e = 0; e < E; ++e) {
      k[e] = k_value<D>(block, r % kBlock, lane + 32 * e);
      v[e] = v_value<D>(block, r % kBlock, lane + 32 * e);
    }
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      if (g >= c.G) break;
      float x = 0.f;
      for (int e = 0; e < E; ++e) x = fmaf(qv[g][e], k[e], x);
      x = dev::warp_sum(x);
      const float top = fmaxf(m[g], x), f = expf(m[g] - top), w = expf(x - top);
      m[g] = top;
      z[g] = fmaf(z[g], f, w);
      for (int e = 0; e < E; ++e) o[g][e] = fmaf(w, v[e], o[g][e] * f);
    }
  }
  for (int g = 0; g < 8; ++g) {
    if (lane == 0) {
      s_m[warp][g] = m[g];
      s_z[warp][g] = z[g];
    }
    for (int e = 0; e < E; ++e) s_o[warp][g][lane + 32 * e] = o[g][e];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < c.G * D; i += kThreads) {
    const int g = i / D, x = i % D;
    float top = -1e30f, zz = 0.f, a = 0.f;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w][g]);
    for (int w = 0; w < kWarps; ++w) {
      const float f = expf(s_m[w][g] - top);
      zz = fmaf(s_z[w][g], f, zz);
      a = fmaf(s_o[w][g][x], f, a);
    }
    dev::st1(&out[i], n > 0 ? a / zz : 0.f);
    if (x == 0) {
      if (n > 0 && !isfinite(zz)) atomicOr(c.err, ERR_NONFINITE);
      if (p.stats) {
        const size_t unit = ((size_t)(p.k.s0 + s) * p.k.nl + lr) * c.H + h;
        float *st = p.stats + (unit * p.n_q * c.G + t * c.G + g) * 2;
        st[0] = top;
        st[1] = 1.f / (zz * c.G);
      }
    }
  }
}

// Adds every row's probabilities: a warp a row.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
    score_kernel(const AttendParams p, const __grid_constant__ Seqs sq) {
  pdl_begin();
  const View &c = p.k.c;
  constexpr int E = D / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = blockIdx.x * kWarps + warp;
  const int h = blockIdx.y % c.H, lr = blockIdx.y / c.H, s = blockIdx.z;
  const int count = sq.count[s], n = sq.len[s];
  if (r >= n) return;
  const size_t u = unit_at(c, p.k.s0 + s, p.k.lb, lr, h);
  const uint8_t *block = block_at(c, u, r);
  float k[E], sum = 0.f;
  for (int e = 0; e < E; ++e) k[e] = k_value<D>(block, r % kBlock, lane + 32 * e);
  const size_t unit = ((size_t)(p.k.s0 + s) * p.k.nl + lr) * c.H + h;
  for (int t = max(0, r - (n - count)); t < count; ++t) {
    const size_t row = (((size_t)(p.k.s0 + s) * p.k.nl + lr) * p.n_q + t) * c.H + h;
    const T *q = static_cast<const T *>(p.q) + row * c.G * D;
    for (int g = 0; g < c.G; ++g) {
      float x = 0.f;
      for (int e = 0; e < E; ++e)
        x = fmaf(dev::to_f(q[g * D + lane + 32 * e]) * c.scale, k[e], x);
      x = dev::warp_sum(x);
      const float *st = p.stats + (unit * p.n_q * c.G + t * c.G + g) * 2;
      sum += expf(x - st[0]) * st[1];
    }
  }
  if (lane == 0) c.score[u * c.sstride + r] += sum;
}

template <typename T, typename O, int D>
cudaError_t launch_as(const AttendParams &p, const Seqs &q, cudaStream_t stream, int *launches) {
  const View &c = p.k.c;
  cudaError_t e = launch_pdl(attend_kernel<T, O, D>, dim3(p.n_q, p.k.nl * c.H, p.k.n),
                             dim3(kThreads), 0, stream, p, q);
  *launches = 1;
  if (e != cudaSuccess || !p.stats) return e;
  int most = 1;
  for (int i = 0; i < p.k.n; ++i) most = q.len[i] > most ? q.len[i] : most;
  *launches = 2;
  return launch_pdl(score_kernel<T, D>, dim3((most + kWarps - 1) / kWarps, p.k.nl * c.H, p.k.n),
                    dim3(kThreads), 0, stream, p, q);
}
template <typename T, typename O>
cudaError_t launch_io(const AttendParams &p, const Seqs &q, cudaStream_t stream, int *launches) {
  return p.k.c.d == 128 ? launch_as<T, O, 128>(p, q, stream, launches)
                        : launch_as<T, O, 64>(p, q, stream, launches);
}

}  // namespace

size_t attend_stat_floats(const View &c, int nl, int n_q) {
  return ((size_t)c.S * nl * c.H * n_q * c.G * 2 + 3) / 4 * 4;
}
size_t attend_part_floats(const View &, int, int) { return 0; }

cudaError_t launch_attend(const AttendParams &p, const Seqs &q, cudaStream_t stream,
                          int *launches) {
  const bool ob = p.k.c.out_bf16;
  if (p.k.c.io_bf16)
    return ob ? launch_io<__nv_bfloat16, __nv_bfloat16>(p, q, stream, launches)
              : launch_io<__nv_bfloat16, float>(p, q, stream, launches);
  return ob ? launch_io<float, __nv_bfloat16>(p, q, stream, launches)
            : launch_io<float, float>(p, q, stream, launches);
}

}  // namespace kv4
}  // namespace kvr
