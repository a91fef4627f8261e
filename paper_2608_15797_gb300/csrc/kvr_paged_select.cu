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
#include "kvr_ptx.cuh"

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

// 32 bytes of a lane, so that the four lanes of a row ask for whole lines.
struct Words {
  uint32_t w[8];
};
__device__ __forceinline__ Words ld32(const void *p) {
  Words r;
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]),
                 "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
               : "l"(p));
  return r;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// bf16 on tensor cores: 16 pages a warp against the 8 query heads, the positive part
// of q with the greatest keys and the negative part with the least.  A third product,
// |q| with max(|least|, |greatest|), says how large the terms of the sums are.
template <int D>
__global__ void __launch_bounds__(kThreads) score_mma_kernel(const __grid_constant__ SelectParams p) {
  kvr::pdl_begin();
  constexpr int kX = D / 64;  // 32-byte pieces of a lane in a row
  const View &c = p.c;
  const int lane = threadIdx.x & 31, row = lane >> 2, j = lane & 3;
  const int groups = (c.tstride + 15) / 16;
  const long long items = (long long)c.S * p.nl * c.H * groups;
  const uint8_t *qs = static_cast<const uint8_t *>(p.q);
  // An item: 16 pages of a unit.  The pages of the next one are looked up while the
  // bounds of this one come.
  struct Item {
    long long unit;
    int first, end, l, h, page[2];
  };
  const long long step = (long long)gridDim.x * kWarps;
  long long it = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  auto next = [&](Item &x) {  // the next item that has pages to score, from `it` on
    for (; it < items; it += step) {
      x.unit = it / groups;
      x.first = (int)(it - x.unit * groups) * 16;
      const int s = (int)(x.unit / ((long long)p.nl * c.H));
      const int u = (int)(x.unit - (long long)s * p.nl * c.H);
      const int have = pages_of(c, s);
      x.end = have - p.window;
      if (have <= p.budget + p.window || x.first >= x.end) continue;
      const int lr = u / c.H;
      x.h = u - lr * c.H;
      x.l = p.lb + lr;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int at = x.first + row + 8 * r;
        x.page[r] = c.table[(long long)s * c.tstride + (at < x.end ? at : x.first)];
      }
      it += step;
      return true;
    }
    return false;
  };
  Item x;
  bool more = next(x);
  while (more) {
    const long long unit = x.unit;
    const int first = x.first, end = x.end;
    Words lo[2][kX], hi[2][kX];
    bool there[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      there[r] = (unsigned)x.page[r] < (unsigned)c.n_pages;
      const uint8_t *b =
          c.bounds +
          (((long long)x.l * c.n_pages + (there[r] ? x.page[r] : 0)) * c.H + x.h) * (4 * D) + j * 32;
#pragma unroll
      for (int y = 0; y < kX; ++y) {
        lo[r][y] = ld32(b + y * 128);
        hi[r][y] = ld32(b + 2 * D + y * 128);
      }
    }
    more = next(x);
    float up[4] = {0.f, 0.f, 0.f, 0.f}, down[4] = {0.f, 0.f, 0.f, 0.f}, size[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < kX; ++x) {
      Words q{};
      if (row < c.G) {  // (16-byte aligned, no more)
        const uint4 *at = reinterpret_cast<const uint4 *>(qs + ((unit * c.G + row) * D) * 2 +
                                                          j * 32 + x * 128);
        const uint4 a = __ldg(at), b = __ldg(at + 1);
        q = Words{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t pos[2], neg[2], mag[2], big[2][2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t w = q.w[2 * i + y];
          const uint32_t below = ((w & 0x8000u) ? 0xFFFFu : 0u) | ((w >> 31) ? 0xFFFF0000u : 0u);
          pos[y] = w & ~below;
          neg[y] = w & below;
          mag[y] = w & 0x7FFF7FFFu;
#pragma unroll
          for (int r = 0; r < 2; ++r)
            big[r][y] = max2(lo[r][x].w[2 * i + y] & 0x7FFF7FFFu, hi[r][x].w[2 * i + y] & 0x7FFF7FFFu);
        }
        kvr::ptx::mma_bf16(up, hi[0][x].w[2 * i], hi[1][x].w[2 * i], hi[0][x].w[2 * i + 1],
                           hi[1][x].w[2 * i + 1], pos[0], pos[1]);
        kvr::ptx::mma_bf16(down, lo[0][x].w[2 * i], lo[1][x].w[2 * i], lo[0][x].w[2 * i + 1],
                           lo[1][x].w[2 * i + 1], neg[0], neg[1]);
        kvr::ptx::mma_bf16(size, big[0][0], big[1][0], big[0][1], big[1][1], mag[0], mag[1]);
      }
    }
    // pages row and row + 8, heads 2 j and 2 j + 1
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float score = -INFINITY, err = 0.f;
#pragma unroll
      for (int y = 0; y < 2; ++y)
        if (2 * j + y < c.G) {
          score = nan_max(score, up[2 * r + y] + down[2 * r + y]);
          err = nan_max(err, size[2 * r + y]);
        }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        score = nan_max(score, __shfl_xor_sync(0xffffffffu, score, o));
        err = nan_max(err, __shfl_xor_sync(0xffffffffu, err, o));
      }
      const int at = first + row + 8 * r;
      if (j == 0 && at < end) {
        if (!there[r]) {
          score = -INFINITY;
          err = 0.f;
          atomicOr(c.err, (unsigned)kvr::ERR_LENGTH);
        }
        // Of each of the D / 16 products of a chain, 17 terms may be cut at 2^-23 of
        // the sum of magnitudes: 136 x 2^-23 of it for d = 128, the same again for
        // the other chain and for the sum of magnitudes itself.
        p.score[unit * c.tstride + at] = make_float2(score, fmaf(err, 0x1p-14f, 1e-37f));
      }
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

// One warp: the digit (of 256, from the greatest) in which the need-th falls, and how
// many of that digit are needed.
__device__ __forceinline__ void digit_of(const unsigned *hist, int need, int lane, int *digit,
                                         int *left) {
  unsigned mine[8], sum = 0;  // lane 0 has the greatest digits
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    mine[i] = hist[255 - 8 * lane - i];
    sum += mine[i];
  }
  unsigned upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  unsigned before = upto - sum;
  if (before < (unsigned)need && upto >= (unsigned)need) {
    int i = 0;
    for (; i < 7 && before + mine[i] < (unsigned)need; ++i) before += mine[i];
    *digit = 255 - 8 * lane - i;
    *left = need - (int)before;
  }
}

// The need-th greatest of key(0 .. n - 1), by digits of 8 bits from bit `top` down
// (above it all keys are alike); *left: how many equal to it belong to the first
// `need`.
template <typename K, typename F>
__device__ K nth(int n, int need, int top, F key, unsigned *hist, int *s_digit, int *s_left,
                 int *left) {
  const int lane = threadIdx.x & 31;
  K prefix = 0, mask = 0;
  bool first = true;
  for (int shift = top - 7; ; shift -= 8) {
    const int low = max(shift, 0), width = shift + 8 - low;
    hist[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const K k = key(i);
      if (first || ((k ^ prefix) & mask) == 0)
        atomicAdd(&hist[(unsigned)(k >> low) & ((1u << width) - 1u)], 1u);
    }
    __syncthreads();
    if (threadIdx.x < 32) digit_of(hist, need, lane, s_digit, s_left);
    __syncthreads();
    prefix |= (K)*s_digit << low;
    mask |= ((K)((1u << width) - 1u)) << low;
    need = *s_left;
    first = false;
    if (low == 0) break;
  }
  *left = need;
  return prefix;
}

// One warp: a page's score in 64 bits, as a key.  (All heads at once: a chain of
// them costs the latency of as many sums.)  No bounds: 0, below every score's.
template <typename T, int D>
__device__ __forceinline__ unsigned long long exact_key(const T *q, const T *b, int G, int lane) {
  if (!b) return 0;
  constexpr int kPer = D / 32;
  double lo[kPer], hi[kPer], z[kHeads];
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    lo[e] = (double)to_f(b[e * 32 + lane]);
    hi[e] = (double)to_f(b[D + e * 32 + lane]);
  }
#pragma unroll
  for (int g = 0; g < kHeads; ++g) {
    z[g] = 0.0;
    if (g < G)
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const float w = to_f(q[g * D + e * 32 + lane]);
        z[g] += (double)w * (w > 0.f ? hi[e] : lo[e]);
      }
  }
  unsigned long long best = 0;
#pragma unroll
  for (int g = 0; g < kHeads; ++g) {
    if (g >= G) continue;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z[g] += __shfl_xor_sync(0xffffffffu, z[g], o);
    const unsigned long long y = key64(z[g]);
    best = y > best ? y : best;
  }
  return best;
}

constexpr int kHeld = 8192;  // scores of a unit that are held on chip

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) select_kernel(const __grid_constant__ SelectParams p) {
  kvr::pdl_begin();
  static_assert(kThreads == 256, "a thread a digit");
  __shared__ unsigned hist[256];
  __shared__ int s_digit, s_left, s_warp[kWarps], s_ties[kWarps], s_count[2];
  __shared__ float s_err[kWarps];
  __shared__ unsigned s_and[kWarps], s_or[kWarps], s_held[kHeld];
  __shared__ int s_near[kThreads];  // pages to be scored again, if they are few
  __shared__ unsigned long long s_key[kThreads];
  const View &c = p.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int U = p.nl * c.H;
  const long long unit = blockIdx.x;
  if (unit == (long long)c.S * U) {
    // what the attention reads of each sequence
    int before = 0;
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
  auto held = [&](int i) { return i < kHeld ? s_held[i] : key32(sc[i].x); };
  // Keys above `top` stay, those from `low` to it do if there is room for all of
  // them; else their scores in 64 bits say which.
  unsigned low = ~0u, top = ~0u;
  bool settle = false;
  unsigned long long cut = 0;  // settled: the last key that stays
  int equal = 0;               // and how many with that key do
  unsigned long long *keys = reinterpret_cast<unsigned long long *>(sc);
  if (B > 0) {
    float err = 0.f;
    unsigned both = ~0u, any = 0;
    for (int i = tid; i < old; i += kThreads) {
      const float2 x = sc[i];
      const unsigned k = key32(x.x);
      if (i < kHeld) s_held[i] = k;
      err = nan_max(err, x.y);
      both &= k, any |= k;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) err = nan_max(err, __shfl_xor_sync(0xffffffffu, err, o));
    both = __reduce_and_sync(0xffffffffu, both);
    any = __reduce_or_sync(0xffffffffu, any);
    if (lane == 0) s_err[warp] = err, s_and[warp] = both, s_or[warp] = any;
    if (tid < 2) s_count[tid] = 0;
    __syncthreads();
    err = s_err[0], both = s_and[0], any = s_or[0];
    for (int w = 1; w < kWarps; ++w) {
      err = nan_max(err, s_err[w]);
      both &= s_and[w], any |= s_or[w];
    }
    // bits above the first that differs are alike in all keys
    const unsigned differ = both ^ any;
    unsigned k = both;
    if (differ) {
      const int bit = 31 - __clz(differ);
      int left;
      const unsigned rest = bit == 31 ? ~0u : (1u << (bit + 1)) - 1u;
      k = (both & ~rest) | nth<unsigned>(old, B, bit, [&](int i) { return held(i) & rest; }, hist,
                                         &s_digit, &s_left, &left);
    }
    const float t = __uint_as_float((k >> 31) ? k & 0x7FFFFFFFu : ~k);
    const bool all = !(fabsf(t) < INFINITY && err < INFINITY);
    // twice the error on either side, rounded away from t
    top = all ? ~0u : key32(__fadd_ru(t, 2.f * err));
    low = all ? 0u : key32(__fadd_rd(t, -2.f * err));
    auto is_near = [&](unsigned x) { return all || (x >= low && x <= top); };
    int n_sure = 0;
    for (int i = tid; i < old; i += kThreads) {
      const unsigned x = held(i);
      n_sure += !all && x > top;
      if (is_near(x)) {
        const int at = atomicAdd(&s_count[1], 1);
        if (at < kThreads) s_near[at] = i;
      }
    }
    n_sure = __reduce_add_sync(0xffffffffu, n_sure);
    if (lane == 0) atomicAdd(&s_count[0], n_sure);
    __syncthreads();
    const int near = s_count[1], need = B - s_count[0];
    const T *q = static_cast<const T *>(p.q) + unit * c.G * D;
    if (near == need) {
      // all of them stay
    } else if (near <= kThreads && old <= kHeld) {
      // few: each counts those that go before it, and its key on chip says the rest
      for (int k = warp; k < near; k += kWarps) {
        const unsigned long long y =
            exact_key<T, D>(q, bounds_of<T>(c, p.lb + lr, s, h, s_near[k]), c.G, lane);
        if (lane == 0) s_key[k] = y;
      }
      __syncthreads();
      if (tid < near) {
        const unsigned long long y = s_key[tid];
        const int i = s_near[tid];
        int above = 0;
        for (int k = 0; k < near; ++k)
          above += s_key[k] > y || (s_key[k] == y && s_near[k] < i);
        s_held[i] = above < need ? ~0u : 0u;
      }
      low = all ? ~0u : low > 0 ? low : 1u;
      __syncthreads();
    } else {
      settle = true;
      for (int i0 = warp * 32; i0 < old; i0 += kThreads) {
        const int i = i0 + lane;
        const unsigned x = i < old ? held(i) : 0u;
        unsigned ask = __ballot_sync(0xffffffffu, i < old && is_near(x));
        unsigned long long key = i < old && !all && x > top ? ~0ull : 0ull;
        while (ask) {
          const int at = __ffs(ask) - 1;
          ask &= ask - 1;
          const unsigned long long y =
              exact_key<T, D>(q, bounds_of<T>(c, p.lb + lr, s, h, i0 + at), c.G, lane);
          if (lane == at) key = y;
        }
        if (i < old) keys[i] = key;
      }
      __syncthreads();
      cut = nth<unsigned long long>(old, B, 63, [&](int i) { return keys[i]; }, hist, &s_digit,
                                    &s_left, &equal);
    }
  }
  // The pages that stay, in order: a warp goes through an equal part of them, once to
  // count and once to write.
  const int part = ((have + kWarps - 1) / kWarps + 31) / 32 * 32;
  const int from = min(warp * part, have), upto = min(from + part, have);
  auto state = [&](int i, bool &tie) {  // does page i stay, or is it a tie
    tie = false;
    if (i >= old) return i < have;
    if (settle) {
      const unsigned long long k = keys[i];
      tie = k == cut;
      return k > cut;
    }
    return B > 0 && held(i) >= low;
  };
  int stay = 0, ties = 0;
  for (int i0 = from; i0 < upto; i0 += 32) {
    bool tie;
    const bool in = state(i0 + lane, tie) && i0 + lane < upto;
    stay += __popc(__ballot_sync(0xffffffffu, in));
    ties += __popc(__ballot_sync(0xffffffffu, tie && i0 + lane < upto));
  }
  if (lane == 0) s_warp[warp] = stay, s_ties[warp] = ties;
  __syncthreads();
  int at = 0, rank = 0;  // of the warp's first page that stays, of its first tie
  for (int w = 0; w < warp; ++w) {
    at += s_warp[w] + min(max(equal - rank, 0), s_ties[w]);
    rank += s_ties[w];
  }
  for (int i0 = from; i0 < upto; i0 += 32) {
    const int i = i0 + lane;
    bool tie;
    bool in = state(i, tie) && i < upto;
    // ties stay in order of position while there is room
    const unsigned tied = __ballot_sync(0xffffffffu, tie && i < upto);
    in |= tie && i < upto && rank + __popc(tied & ((1u << lane) - 1u)) < equal;
    const unsigned kept_here = __ballot_sync(0xffffffffu, in);
    const int to = at + __popc(kept_here & ((1u << lane) - 1u));
    if (in && to < kept) {
      list[to] = table[i];
      if (chosen) chosen[to] = i;
    }
    at += __popc(kept_here);
    rank += __popc(tied);
  }
}

template <typename T, int D>
cudaError_t launch(const SelectParams &p, int sms, cudaStream_t st, int *launches) {
  const long long units = (long long)p.c.S * p.nl * p.c.H;
  if (p.budget > 0) {
    cudaError_t e;
    if constexpr (sizeof(T) == 2) {
      const long long ctas = (units * ((p.c.tstride + 15) / 16) + kWarps - 1) / kWarps;
      e = kvr::launch_pdl(score_mma_kernel<D>, dim3((unsigned)std::min<long long>(ctas, 8ll * sms)),
                          dim3(kThreads), 0, st, p);
    } else {
      const long long ctas = units * ((p.c.tstride + kChunk - 1) / kChunk);
      e = kvr::launch_pdl(score_kernel<T, D>, dim3((unsigned)std::min<long long>(ctas, 8ll * sms)),
                          dim3(kThreads), 0, st, p);
    }
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
