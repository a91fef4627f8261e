// kvr_paged_select.cu -- the choice of pages for kvr_paged_attend_pages
// (include/kvr.h).  A page's score for the G query heads that share its KV head is
//   max_g sum_c q_gc (q_gc > 0 ? hi_c : lo_c),
// lo and hi the least and greatest key of each channel: no logit of its rows is above
// it.  The window newest pages stay, and the budget others of the greatest score.
//
//   score_kernel   every page's score in fp32 and a bound of its rounding error
//   select_kernel  a CTA a unit: the budget-th greatest score by radix passes.  Pages
//                  nearer to it than both their errors are scored again in 64 bits
//                  if not all of them stay, so that the choice is the definition's;
//                  equal scores keep the lower page, and a NaN ranks above every
//                  number.
#include "kvr_paged.cuh"

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "kvr_device.cuh"
#include "kvr_internal.h"

namespace kvr {
namespace paged {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kChunk = 64;  // pages of an item of the scores

using kvr::dev::to_f;

__device__ __forceinline__ int pages_of(const View &c, int s) {
  return min((c.len[s] + c.P - 1) >> c.psh, c.tstride);
}
// Bounds of the page at position `at` of sequence s, or null for a bad page.
template <typename T>
__device__ __forceinline__ const T *bounds_of(const View &c, int l, int s, int h, int at) {
  const int page = c.table[(long long)s * c.tstride + at];
  if ((unsigned)page >= (unsigned)c.n_pages) return nullptr;
  return reinterpret_cast<const T *>(c.bounds) +
         (((long long)l * c.n_pages + page) * c.H + h) * 2 * c.d;
}
__device__ __forceinline__ float nan_max(float a, float b) {
  return a != a ? a : b != b ? b : fmaxf(a, b);
}

// A warp a page: a lane sums D / 32 channels' products a head in a chain, then
// five steps between lanes.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) score_kernel(const __grid_constant__ SelectParams p) {
  kvr::pdl_begin();
  constexpr int kPer = D / 32;
  const View &c = p.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int chunks = (c.tstride + kChunk - 1) / kChunk;
  const long long items = (long long)c.S * p.nl * c.H * chunks;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const long long unit = it / chunks;
    const int first = (int)(it - unit * chunks) * kChunk;
    const int h = (int)(unit % c.H), lr = (int)(unit / c.H % p.nl);
    const int s = (int)(unit / c.H / p.nl);
    const int have = pages_of(c, s);
    if (have <= p.budget + p.window) continue;  // all of them stay
    const int end = min(first + kChunk, have - p.window);
    if (first >= end) continue;
    float q[kHeads][kPer];
    float most = 0.f;  // the greatest sum of |q| of a head
    const T *qs = static_cast<const T *>(p.q) + unit * c.G * D;
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        q[g][e] = g < c.G ? to_f(qs[g * D + lane * kPer + e]) : 0.f;
        sum += fabsf(q[g][e]);
      }
      most = nan_max(most, kvr::dev::warp_sum(sum));
    }
    for (int at = first + warp; at < end; at += kWarps) {
      const T *b = bounds_of<T>(c, p.lb + lr, s, h, at);
      float score = -INFINITY, big = 0.f;
      if (b) {
        float lo[kPer], hi[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          lo[e] = to_f(b[lane * kPer + e]);
          hi[e] = to_f(b[D + lane * kPer + e]);
          big = nan_max(big, nan_max(fabsf(lo[e]), fabsf(hi[e])));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) big = nan_max(big, __shfl_xor_sync(0xffffffffu, big, o));
#pragma unroll
        for (int g = 0; g < kHeads; ++g) {
          float x = 0.f;
#pragma unroll
          for (int e = 0; e < kPer; ++e)
            x = fmaf(q[g][e], q[g][e] > 0.f ? hi[e] : lo[e], x);
          x = kvr::dev::warp_sum(x);
          if (g < c.G) score = nan_max(score, x);
        }
      } else if (lane == 0) {
        atomicOr(c.err, (unsigned)kvr::ERR_LENGTH);
      }
      // Each of the D / 32 + 5 additions rounds by 2^-24 of a sum that is at most
      // sum |q| max |k|; products that underflow add 2^-149 each at most.
      if (lane == 0)
        p.score[unit * c.tstride + at] = make_float2(score, fmaf(most * big, 0x1p-20f, 1e-40f));
    }
  }
}

__device__ __forceinline__ unsigned key32(float x) {
  return x != x ? 0xFFFFFFFFu : kvr::dev::ord_bits(x + 0.f);
}
__device__ __forceinline__ unsigned long long key64(double x) {
  if (x != x) return ~0ull - 1;
  const unsigned long long b = (unsigned long long)__double_as_longlong(x + 0.0);
  return (b >> 63) ? ~b : b | (1ull << 63);
}

// The need-th greatest of key(0 .. n - 1), bits * 8 wide; *left: how many equal to it
// belong to the first `need`.
template <typename K, typename F>
__device__ K nth(int n, int need, F key, unsigned *hist, K *s_prefix, int *s_need) {
  K prefix = 0, mask = 0;
  for (int shift = (int)sizeof(K) * 8 - 8; shift >= 0; shift -= 8) {
    hist[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const K k = key(i);
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1u);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int seen = 0, d = 255;
      for (; d > 0 && seen + (int)hist[d] < need; --d) seen += (int)hist[d];
      *s_prefix = prefix | ((K)d << shift);
      *s_need = need - seen;
    }
    __syncthreads();
    prefix = *s_prefix;
    need = *s_need;
    mask |= (K)0xFF << shift;
    __syncthreads();
  }
  return prefix;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) select_kernel(const __grid_constant__ SelectParams p) {
  kvr::pdl_begin();
  static_assert(kThreads == 256, "a thread a digit");
  __shared__ unsigned hist[256];
  __shared__ unsigned s_key;
  __shared__ unsigned long long s_key64;
  __shared__ int s_need, s_base, s_warp[kWarps], s_count[2];
  __shared__ float s_err[kWarps];
  const View &c = p.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int U = p.nl * c.H;
  const long long unit = blockIdx.x;
  if (unit == (long long)c.S * U) {
    // what the attention reads of each sequence
    int before = 0;
    if (tid == 0) s_base = 0;
    for (int s0 = 0; s0 < c.S; s0 += kThreads) {
      const int s = s0 + tid;
      int rows = 0;
      if (s < c.S) {
        const int have = pages_of(c, s), kept = min(have, p.keep);
        rows = c.len[s] - ((have - kept) << c.psh);
        p.rows[s] = rows;
      }
      const int mine = (rows + kTile - 1) / kTile;
      int x = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      __syncthreads();
      if (lane == 31) s_warp[warp] = x;
      __syncthreads();
      int all = 0;
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) x += s_warp[w];
        all += s_warp[w];
      }
      if (s < c.S) p.tiles[s] = before + x - mine;
      before += all;
    }
    if (tid == 0) p.tiles[c.S] = before;
    return;
  }
  const int s = (int)(unit / U), u = (int)(unit - (long long)s * U);
  const int lr = u / c.H, h = u - lr * c.H;
  const int have = pages_of(c, s);
  const int32_t *table = c.table + (long long)s * c.tstride;
  int32_t *list = p.list + unit * p.keep;
  int32_t *chosen = p.chosen ? p.chosen + unit * ((long long)p.budget + p.window) : nullptr;
  const int kept = (int)min((long long)have, (long long)p.budget + p.window);
  if (chosen)
    for (int i = kept + tid; i < p.budget + p.window; i += kThreads) chosen[i] = -1;
  if (have <= p.budget + p.window) {
    for (int i = tid; i < kept; i += kThreads) {
      list[i] = table[i];
      if (chosen) chosen[i] = i;
    }
    return;
  }
  const int old = have - p.window, B = p.budget;
  float2 *sc = p.score + unit * c.tstride;
  // pages from `top` up stay; of those between `top` and `low` the settled ones do
  float top = INFINITY, low = INFINITY;
  bool settle = false;
  unsigned long long cut = 0;  // settled: the last key that stays
  int equal = 0;               // and how many with that key do
  if (B > 0) {
    float err = 0.f;
    for (int i = tid; i < old; i += kThreads) err = nan_max(err, sc[i].y);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) err = nan_max(err, __shfl_xor_sync(0xffffffffu, err, o));
    if (lane == 0) s_err[warp] = err;
    if (tid < 2) s_count[tid] = 0;
    const unsigned k = nth<unsigned>(old, B, [&](int i) { return key32(sc[i].x); }, hist, &s_key,
                                     &s_need);
    for (int w = 0; w < kWarps; ++w) err = nan_max(err, s_err[w]);
    const float t = __uint_as_float((k >> 31) ? k & 0x7FFFFFFFu : ~k);
    // twice the error on either side, rounded away from t
    top = __fadd_ru(t, 2.f * err);
    low = __fadd_rd(t, -2.f * err);
    if (!(fabsf(t) < INFINITY && err < INFINITY)) top = INFINITY, low = -INFINITY;
    const bool all = low == -INFINITY;
    auto sure = [&](float x) { return !all && x > top; };
    auto near = [&](float x) { return all || (x >= low && x <= top); };
    int n_sure = 0, n_near = 0;
    for (int i = tid; i < old; i += kThreads) {
      n_sure += sure(sc[i].x);
      n_near += near(sc[i].x);
    }
    atomicAdd(&s_count[0], n_sure);
    atomicAdd(&s_count[1], n_near);
    __syncthreads();
    settle = s_count[0] + s_count[1] != B;
    if (settle) {
      const T *q = static_cast<const T *>(p.q) + unit * c.G * D;
      for (int i0 = warp * 32; i0 < old; i0 += kThreads) {
        const int i = i0 + lane;
        const float x = i < old ? sc[i].x : 0.f;
        unsigned ask = __ballot_sync(0xffffffffu, i < old && near(x));
        unsigned long long key = i < old && sure(x) ? ~0ull : 0ull;
        while (ask) {
          const int at = __ffs(ask) - 1;
          ask &= ask - 1;
          const T *b = bounds_of<T>(c, p.lb + lr, s, h, i0 + at);
          unsigned long long best = 0;
          for (int g = 0; b && g < c.G; ++g) {
            double z = 0.0;
            for (int e = lane; e < D; e += 32) {
              const double w = (double)to_f(q[g * D + e]);
              z += w * (double)to_f(w > 0.0 ? b[D + e] : b[e]);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
            const unsigned long long y = key64(z);
            best = y > best ? y : best;
          }
          if (lane == at) key = best;
        }
        if (i < old) reinterpret_cast<unsigned long long *>(sc)[i] = key;
      }
      __syncthreads();
      const unsigned long long *keys = reinterpret_cast<const unsigned long long *>(sc);
      cut = nth<unsigned long long>(old, B, [&](int i) { return keys[i]; }, hist, &s_key64,
                                    &s_need);
      equal = s_need;
    }
  }
  // the pages that stay, in order
  if (tid == 0) s_base = 0, s_count[0] = 0;
  __syncthreads();
  for (int i0 = 0; i0 < have; i0 += kThreads) {
    const int i = i0 + tid;
    bool keep = false, tie = false;
    if (i >= old) {
      keep = i < have;
    } else if (settle) {
      const unsigned long long k = reinterpret_cast<const unsigned long long *>(sc)[i];
      keep = k > cut;
      tie = k == cut;
    } else if (B > 0) {
      keep = sc[i].x >= low;
    }
    // ties stay in order of position while there are some to stay
    const unsigned ties = __ballot_sync(0xffffffffu, tie);
    if (lane == 0) s_warp[warp] = __popc(ties);
    __syncthreads();
    int rank = s_count[0] + __popc(ties & ((1u << lane) - 1u)), all = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) rank += s_warp[w];
      all += s_warp[w];
    }
    keep |= tie && rank < equal;
    __syncthreads();
    const unsigned in = __ballot_sync(0xffffffffu, keep);
    if (lane == 0) s_warp[warp] = __popc(in);
    __syncthreads();
    int at = s_base + __popc(in & ((1u << lane) - 1u)), count = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) at += s_warp[w];
      count += s_warp[w];
    }
    if (keep && at < kept) {
      list[at] = table[i];
      if (chosen) chosen[at] = i;
    }
    __syncthreads();
    if (tid == 0) s_base += count, s_count[0] += all;
    __syncthreads();
  }
}

template <typename T, int D>
cudaError_t launch(const SelectParams &p, int sms, cudaStream_t st, int *launches) {
  const long long units = (long long)p.c.S * p.nl * p.c.H;
  const long long items = units * ((p.c.tstride + kChunk - 1) / kChunk);
  if (p.budget > 0) {
    const cudaError_t e =
        kvr::launch_pdl(score_kernel<T, D>, dim3((unsigned)std::min<long long>(items, 8ll * sms)),
                        dim3(kThreads), 0, st, p);
    if (e != cudaSuccess) return e;
    *launches += 1;
  }
  const cudaError_t e = kvr::launch_pdl(select_kernel<T, D>, dim3((unsigned)(units + 1)),
                                        dim3(kThreads), 0, st, p);
  if (e == cudaSuccess) *launches += 1;
  return e;
}

}  // namespace

cudaError_t launch_select(const SelectParams &p, int sms, cudaStream_t st, int *launches) {
  if (p.c.io_bf16)
    return p.c.d == 128 ? launch<__nv_bfloat16, 128>(p, sms, st, launches)
                        : launch<__nv_bfloat16, 64>(p, sms, st, launches);
  return p.c.d == 128 ? launch<float, 128>(p, sms, st, launches)
                      : launch<float, 64>(p, sms, st, launches);
}

}  // namespace paged
}  // namespace kvr
