// kvr_paged_select.cu -- the choice of pages for kvr_paged_attend_pages
// (include/kvr.h).  A page's score for the G query heads that share its KV head is
//   max_g sum_c q_gc (q_gc > 0 ? hi_c : lo_c),
// lo and hi the least and greatest key of each channel: no logit of its rows is above
// it.  The window newest pages stay, and the budget others of the greatest score.
//
// Pages are scored in fp32, with a bound of each score's rounding error.  A CTA a unit
// then chooses: the budget-th greatest score by a histogram and a count; pages nearer
// to it than both their errors, if not all of them stay, are scored again with sums
// held in two floats, and what that leaves open in 64 bits, so that the choice is the
// definition's.  Equal scores keep the lower page, a NaN ranks above every number.
//
// Few units (latency): one launch, a cluster a unit, scores in shared memory (4 units of
// 513 pages, choice and attention: 24 us a call with scores in memory and arrivals,
// 16 so).  Many (the bounds' bytes): a launch that scores, 16 warps an SM with a page's
// bounds as whole lines straight to registers (112 units of 4,096 pages 41 us, 5.7
// TB/s; through rings of copies as in the attention 74, since a warp's 16 pages are a
// long chain of steps), and one that chooses (15 us, of dependent steps).
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

constexpr int kBlock = 256;        // threads, where no other number is given
constexpr int kBlockWarps = kBlock / 32;
constexpr int kWide = 1024;        // of a CTA that chooses alone on its SM

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

// A call's unit, and what is to be done for it.
struct Unit {
  long long at;   // of the call
  int l, s, h;    // layer of the cache, sequence, KV head
  int have, old;  // its pages; those that have to be chosen from (0: all stay)
};
__device__ __forceinline__ Unit unit_of(const SelectParams &p, long long at) {
  const View &c = p.c;
  const unsigned U = p.nl * c.H, n = (unsigned)at;  // (units are fewer than 2^31)
  Unit x;
  x.at = at;
  x.s = n / U;
  const unsigned u = n - x.s * U, lr = u / (unsigned)c.H;
  x.h = u - lr * c.H;
  x.l = p.lb + lr;
  x.have = pages_of(c, x.s);
  x.old = x.have > p.budget + p.window && p.budget > 0 ? x.have - p.window : 0;
  return x;
}

// Items: 16 pages of a unit each, unit by unit.  A warp scores an item, the one `step`
// further and so on, up to unit `units`; put(unit, page, (score, bound of its error)).
__device__ __forceinline__ int groups_of(const View &c) { return (c.tstride + 15) / 16; }

struct Items {
  int unit, group;            // the next item
  int unit_step, group_step;  // to the one after it
  int units, groups;
  __device__ __forceinline__ Items(int unit, int group, unsigned step, int units, int groups)
      : unit(unit), group(group), unit_step(step / groups), group_step(step % groups), units(units),
        groups(groups) {}
};
struct Item {
  Unit u;
  int first;
};
// The next item that has pages to score.
__device__ __forceinline__ bool next_item(const SelectParams &p, Items &it, Item &x) {
  while (it.unit < it.units) {
    x.u = unit_of(p, it.unit);
    x.first = it.group * 16;
    it.unit += it.unit_step;
    it.group += it.group_step;
    if (it.group >= it.groups) it.group -= it.groups, ++it.unit;
    if (x.first < x.u.old) return true;
  }
  return false;
}

// fp32: four pages' bounds on their way at a time; a lane sums D / 32 channels' products a
// head in a chain, then five steps between lanes, which are what it costs: 896 units of
// 60 pages at d = 128 48 us (each head summed over all lanes for itself 61, a page at a
// time 68).  A page that is none counts as one of zeros.
template <int D, typename F>
__device__ __forceinline__ void score_items(const SelectParams &p, Items it, const float *, F put) {
  constexpr int kPer = D / 32, kAhead = 4;
  const View &c = p.c;
  const int lane = threadIdx.x & 31;
  Item x;
  while (next_item(p, it, x)) {
    const Unit &u = x.u;
    const int mine =
        c.table[(long long)u.s * c.tstride + min(x.first + (lane & 15), u.old - 1)];
    if ((unsigned)mine >= (unsigned)c.n_pages) atomicOr(c.err, (unsigned)kvr::ERR_LENGTH);
    float q[kHeads][kPer];
    float most = 0.f;  // the greatest sum of |q| of a head
    const float *qs = static_cast<const float *>(p.q) + u.at * c.G * D;
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        q[g][e] = g < c.G ? qs[g * D + lane * kPer + e] : 0.f;
        sum += fabsf(q[g][e]);
      }
      most = nan_max(most, kvr::dev::warp_sum(sum));
    }
    const int many = min(16, u.old - x.first);
#pragma unroll 1
    for (int i0 = 0; i0 < many; i0 += kAhead) {
      float lo[kAhead][kPer], hi[kAhead][kPer];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int page = __shfl_sync(0xffffffffu, mine, i0 + i);
        const bool there = (unsigned)page < (unsigned)c.n_pages;
        const float *b = reinterpret_cast<const float *>(c.bounds) +
                         (((long long)u.l * c.n_pages + (there ? page : 0)) * c.H + u.h) * 2 * D +
                         lane * kPer;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          lo[i][e] = there ? __ldg(b + e) : 0.f;
          hi[i][e] = there ? __ldg(b + D + e) : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (i0 + i >= many) break;
        float score = -INFINITY, big = 0.f;
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          big = nan_max(big, nan_max(fabsf(lo[i][e]), fabsf(hi[i][e])));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) big = nan_max(big, __shfl_xor_sync(0xffffffffu, big, o));
        float y[kHeads];
#pragma unroll
        for (int g = 0; g < kHeads; ++g) {
          y[g] = 0.f;
#pragma unroll
          for (int e = 0; e < kPer; ++e)
            y[g] = fmaf(q[g][e], q[g][e] > 0.f ? hi[i][e] : lo[i][e], y[g]);
        }
        // eight sums over 32 lanes: each step halves the sums that a lane holds
#pragma unroll
        for (int n = kHeads / 2, o = 16; n > 0; n >>= 1, o >>= 1) {
          const bool upper = lane & o;
#pragma unroll
          for (int k = 0; k < n; ++k) {
            const float keep = upper ? y[k + n] : y[k], give = upper ? y[k] : y[k + n];
            y[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
          }
        }
        y[0] += __shfl_xor_sync(0xffffffffu, y[0], 2);
        y[0] += __shfl_xor_sync(0xffffffffu, y[0], 1);
        if ((lane >> 2) < c.G) score = y[0];  // the head that the lane is left with
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
          score = nan_max(score, __shfl_xor_sync(0xffffffffu, score, o));
        // Each of the D / 32 + 5 additions rounds by 2^-24 of a sum that is at most
        // sum |q| max |k|; products that underflow add 2^-149 each at most.
        if (lane == 0)
          put(u.at, x.first + i0 + i, make_float2(score, fmaf(most * big, 0x1p-20f, 1e-40f)));
      }
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

// bf16 on tensor cores: 16 pages against the 8 query heads, the positive part of q
// with the greatest keys and the negative part with the least.  A third product, |q|
// with max(|least|, |greatest|), says how large the terms of the sums are.  The pages
// of the next item are looked up while the bounds of this one come.
template <int D, typename F>
__device__ __forceinline__ void score_items(const SelectParams &p, Items it, const __nv_bfloat16 *,
                                            F put) {
  constexpr int kX = D / 64;  // 32-byte pieces of a lane in a row
  const View &c = p.c;
  const int lane = threadIdx.x & 31, row = lane >> 2, j = lane & 3;
  Item ahead;
  int page[2];
  auto look = [&]() {
    if (!next_item(p, it, ahead)) return false;
    const int32_t *table = c.table + (long long)ahead.u.s * c.tstride;
#pragma unroll
    for (int r = 0; r < 2; ++r) page[r] = table[min(ahead.first + row + 8 * r, ahead.u.old - 1)];
    return true;
  };
  for (bool more = look(); more;) {
    const long long unit = ahead.u.at;
    const int i0 = ahead.first, end = ahead.u.old;
    Words lo[2][kX], hi[2][kX];
    bool there[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      there[r] = (unsigned)page[r] < (unsigned)c.n_pages;
      const uint8_t *b = c.bounds +
                         (((long long)ahead.u.l * c.n_pages + (there[r] ? page[r] : 0)) * c.H +
                          ahead.u.h) *
                             (4 * D) +
                         j * 32;
#pragma unroll
      for (int x = 0; x < kX; ++x) {
        lo[r][x] = ld32(b + x * 128);
        hi[r][x] = ld32(b + 2 * D + x * 128);
      }
    }
    more = look();
    float up[4] = {0.f, 0.f, 0.f, 0.f}, down[4] = {0.f, 0.f, 0.f, 0.f};
    float size[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < kX; ++x) {
      Words q{};
      if (row < c.G) {  // (16-byte aligned, no more)
        const uint4 *at = reinterpret_cast<const uint4 *>(
            static_cast<const uint8_t *>(p.q) + ((unit * c.G + row) * D) * 2 + j * 32 + x * 128);
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
            big[r][y] = max2(lo[r][x].w[2 * i + y] & 0x7FFF7FFFu,
                             hi[r][x].w[2 * i + y] & 0x7FFF7FFFu);
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
      const int at = i0 + row + 8 * r;
      if (j == 0 && at < end) {
        if (!there[r]) {
          score = -INFINITY;
          err = 0.f;
          atomicOr(c.err, (unsigned)kvr::ERR_LENGTH);
        }
        // Of each of the D / 16 products of a chain, 17 terms may be cut at 2^-23 of
        // the sum of magnitudes: 136 x 2^-23 of it for d = 128, the same again for
        // the other chain and for the sum of magnitudes itself.
        put(unit, at, make_float2(score, fmaf(err, 0x1p-14f, 1e-37f)));
      }
    }
  }
}

__device__ __forceinline__ unsigned key32(float x) {
  return x != x ? 0xFFFFFFFFu : kvr::dev::ord_bits(x + 0.f);
}
__device__ __forceinline__ float value32(unsigned k) {
  return __uint_as_float((k >> 31) ? k & 0x7FFFFFFFu : ~k);
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
// `need`.  The whole CTA; hist, *s_digit and *s_left may hold what threads still read.
template <int kThreads, typename K, typename F>
__device__ K nth(int n, int need, int top, F key, unsigned *hist, int *s_digit, int *s_left,
                 int *left) {
  const int lane = threadIdx.x & 31;
  K prefix = 0, mask = 0;
  bool first = true;
  __syncthreads();
  for (int shift = top - 7; ; shift -= 8) {
    const int low = max(shift, 0), width = shift + 8 - low;
    if (threadIdx.x < 256) hist[threadIdx.x] = 0;
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

// Scoring again, a warp a page: four lanes a head, each a quarter of the channels in a
// row.  q lies on chip as fp32, quarters apart so that 32 lanes hit 32 banks.
template <int D>
__device__ __forceinline__ int q_at(int g, int channel) {
  return g * (D + 4) + channel + channel / (D / 4);
}
// f(w, k) for the lane's channels, k the bound that q's sign asks for.
template <typename T, int D, typename F>
__device__ __forceinline__ void each_term(const float *q, const T *b, int lane, F f) {
  constexpr int kN = D / 4, kVec = 16 / (int)sizeof(T);
  const float *w = q + q_at<D>(lane >> 2, (lane & 3) * kN);
  const uint4 *lo = reinterpret_cast<const uint4 *>(b + (lane & 3) * kN);
  const uint4 *hi = reinterpret_cast<const uint4 *>(b + D + (lane & 3) * kN);
#pragma unroll
  for (int i = 0; i < kN / kVec; ++i) {
    const uint4 x = lo[i], y = hi[i];
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float v = w[i * kVec + e];
      uint32_t k = v > 0.f ? ys[e * (int)sizeof(T) / 4] : xs[e * (int)sizeof(T) / 4];
      if (sizeof(T) == 2) k = e & 1 ? k & 0xFFFF0000u : k << 16;
      f(e & 1, v, __uint_as_float(k));
    }
  }
}

// A page's score in 64 bits, as a key.  No bounds: 0, below every score's.
template <typename T, int D>
__device__ __forceinline__ unsigned long long exact_key(const float *q, const T *b, int G,
                                                        int lane) {
  if (!b) return 0;
  double z = 0.0;
  each_term<T, D>(q, b, lane, [&](int, float w, float k) { z += (double)w * (double)k; });
  z += __shfl_xor_sync(0xffffffffu, z, 1);
  z += __shfl_xor_sync(0xffffffffu, z, 2);
  unsigned long long best = (lane >> 2) < G ? key64(z) : 0;
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) {
    const unsigned long long y = __shfl_xor_sync(0xffffffffu, best, o);
    best = y > best ? y : best;
  }
  return best;
}

// A page's score less t, from sums held as two floats.  Of the sum of magnitudes M:
// the errors that sums leave, 2^-24 M each, are added up over 32 terms with as many
// roundings, 2^-38 M; the difference from t, at most three bounds of a score's error
// (2^-14 M in bf16, 2^-20 of what bounds M in fp32), rounds twice.
__device__ __forceinline__ void add_exact(float &hi, float &lo, float x) {
  const float s = __fadd_rn(hi, x), b = __fsub_rn(s, hi);
  lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(s, b)), __fsub_rn(x, b)));
  hi = s;
}
template <typename T, int D>
__device__ __forceinline__ float near_offset(const float *q, const T *b, int G, float t, int lane) {
  if (!b) return -INFINITY;
  float hi[2] = {0.f, 0.f}, lo[2] = {0.f, 0.f};
  each_term<T, D>(q, b, lane, [&](int i, float w, float k) {
    const float x = __fmul_rn(w, k);
    add_exact(hi[i], lo[i], x);
    if (sizeof(T) == 4) lo[i] = __fadd_rn(lo[i], __fmaf_rn(w, k, -x));  // (bf16: exact)
  });
  lo[0] = __fadd_rn(lo[0], lo[1]);
  add_exact(hi[0], lo[0], hi[1]);
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    const float h2 = __shfl_xor_sync(0xffffffffu, hi[0], o);
    lo[0] = __fadd_rn(lo[0], __shfl_xor_sync(0xffffffffu, lo[0], o));
    add_exact(hi[0], lo[0], h2);
  }
  float best = (lane >> 2) < G ? __fadd_rn(__fsub_rn(hi[0], t), lo[0]) : -INFINITY;
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) best = nan_max(best, __shfl_xor_sync(0xffffffffu, best, o));
  return best;
}

constexpr int kHeld = 8192;    // keys of a unit that are held on chip, at most
constexpr int kOnChip = 2048;  // scores of a unit that lie on chip with them, at most
// Words of n keys, padded (threads read runs of keys) to whole vectors.
__host__ __device__ constexpr int keys_words(int n) { return (n + n / 32 + 3) / 4 * 4; }

// The choice for one unit, whose scores lie at sc: on chip (kLocal), or in memory.  The
// whole CTA.
template <typename T, int D, bool kLocal, int kThreads>
__device__ __forceinline__ void choose(const SelectParams &p, const Unit &u, float2 *sc) {
  constexpr int kWarps = kThreads / 32;
  static_assert(kThreads >= 256, "a thread a digit");
  __shared__ unsigned hist[256];
  __shared__ int s_digit, s_left, s_stay[kWarps], s_ties[kWarps], s_sure, s_few;
  __shared__ float s_err[kWarps];
  __shared__ unsigned s_least[kWarps], s_most[kWarps], s_kth;
  extern __shared__ unsigned s_held[];  // [p.held], padded
  __shared__ unsigned s_near[kThreads];  // keys of a digit; pages to be scored again
  __shared__ unsigned long long s_key[kThreads];
  __shared__ const T *s_at[kThreads];
  __shared__ float s_q[kHeads * (D + 4)];
  __shared__ float s_off[kThreads];
  __shared__ bool s_open[kThreads];
  const View &c = p.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t *table = c.table + (long long)u.s * c.tstride;
  const int have = u.have, old = u.old, B = p.budget;
  int32_t *list = p.list + u.at * p.keep;
  int32_t *chosen = p.chosen ? p.chosen + u.at * ((long long)B + p.window) : nullptr;
  const int kept = (int)min((long long)have, (long long)B + p.window);
  if (chosen)
    for (int i = kept + tid; i < B + p.window; i += kThreads) chosen[i] = -1;
  if (old == 0) {
    // all pages stay, or (no budget) the newest
    for (int i = tid; i < kept; i += kThreads) {
      list[i] = table[have - kept + i];
      if (chosen) chosen[i] = have - kept + i;
    }
    return;
  }
  auto place = [](int i) { return i + (i >> 5); };  // (threads read runs of keys)
  constexpr int kBatch = 8;  // keys of a thread that are read together
  // of a score's bound, what near_offset is within: 2^-35 and 2^-37 of what sums are
  // bounded by
  constexpr float kOff = sizeof(T) == 2 ? 0x1p-21f : 0x1p-17f;
  auto held = [&](int i) {
    return kLocal || i < p.held ? s_held[place(i)] : key32(__ldcg(sc + i).x);
  };
  // f(i, key) for the thread's share of the keys.
  auto each = [&](auto f) {
    for (int i0 = tid; i0 < old; i0 += kBatch * kThreads) {
      unsigned k[kBatch];
#pragma unroll
      for (int r = 0; r < kBatch; ++r)
        if (i0 + r * kThreads < old) k[r] = held(i0 + r * kThreads);
#pragma unroll
      for (int r = 0; r < kBatch; ++r)
        if (i0 + r * kThreads < old) f(i0 + r * kThreads, k[r]);
    }
  };
  // Keys above `top` stay, those from `low` to it do if there is room for all of
  // them; else their scores in 64 bits say which.
  unsigned low, top;
  bool settle = false;
  unsigned long long cut = 0;  // settled: the last key that stays
  int equal = 0;               // and how many with that key do
  unsigned long long *keys = reinterpret_cast<unsigned long long *>(sc);
  {
    float err = 0.f;
    unsigned least = ~0u, most = 0;
    if (tid < 256) hist[tid] = 0;
    {
      const T *q = static_cast<const T *>(p.q) + u.at * c.G * D;
      for (int i = tid; i < kHeads * D; i += kThreads)
        s_q[q_at<D>(i / D, i % D)] = i < c.G * D ? to_f(q[i]) : 0.f;
    }
    for (int i0 = 2 * tid; i0 < old; i0 += 2 * kBatch * kThreads) {
      float4 x[kBatch];
#pragma unroll
      for (int r = 0; r < kBatch; ++r)
        if (i0 + 2 * r * kThreads < old)
          x[r] = kLocal ? *reinterpret_cast<const float4 *>(sc + i0 + 2 * r * kThreads)
                         : __ldcg(reinterpret_cast<const float4 *>(sc + i0 + 2 * r * kThreads));
#pragma unroll
      for (int r = 0; r < kBatch; ++r) {
        const int i = i0 + 2 * r * kThreads;
        if (i >= old) break;
        // (the last one's neighbour is there, and not counted)
        const unsigned k0 = key32(x[r].x), k1 = i + 1 < old ? key32(x[r].z) : k0;
        if (kLocal || i < p.held) s_held[place(i)] = k0, s_held[place(i + 1)] = k1;
        err = nan_max(err, i + 1 < old ? nan_max(x[r].y, x[r].w) : x[r].y);
        least = min(least, min(k0, k1)), most = max(most, max(k0, k1));
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) err = nan_max(err, __shfl_xor_sync(0xffffffffu, err, o));
    least = __reduce_min_sync(0xffffffffu, least);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) s_err[warp] = err, s_least[warp] = least, s_most[warp] = most;
    if (tid == 0) s_sure = s_few = 0;
    __syncthreads();
    err = s_err[0], least = s_least[0], most = s_most[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
      err = nan_max(err, s_err[w]);
      least = min(least, s_least[w]), most = max(most, s_most[w]);
    }
    const float from = value32(least), to = value32(most);
    const bool all = !(fabsf(from) < INFINITY && fabsf(to) < INFINITY && err < INFINITY);
    float t = from;
    if (!all && least != most) {
      // 256 equal parts of the scores' range make a histogram, and what falls into the
      // part where the budget ends is counted out.  (Rounding keeps the order, which
      // is all that is asked of the parts.)
      const float scale = fminf(256.f / fmaxf(to - from, 0x1p-120f), 0x1p120f);
      auto part = [&](unsigned k) {
        return (unsigned)fminf(fmaxf((value32(k) - from) * scale, 0.f), 255.f);
      };
      each([&](int, unsigned k) { atomicAdd(&hist[part(k)], 1u); });
      __syncthreads();
      if (warp == 0) digit_of(hist, B, lane, &s_digit, &s_left);
      __syncthreads();
      const unsigned d = s_digit;
      const int left = s_left, in = (int)hist[d];
      if (in <= kThreads) {
        each([&](int, unsigned k) {
          if (part(k) == d) s_near[atomicAdd(&s_few, 1)] = k;
        });
        __syncthreads();
        if (tid < in) {
          const unsigned mine = s_near[tid];
          int above = 0, alike = 0;
#pragma unroll 8
          for (int k = 0; k < in; ++k) {
            above += s_near[k] > mine;
            alike += s_near[k] == mine;
          }
          if (above < left && above + alike >= left) s_kth = mine;
        }
        __syncthreads();
        if (tid == 0) s_few = 0;
        t = value32(s_kth);
      } else {
        int unused;
        t = value32(nth<kThreads, unsigned>(old, B, 31, held, hist, &s_digit, &s_left, &unused));
      }
      __syncthreads();
    }
    // twice the error on either side, rounded away from t
    top = all ? ~0u : key32(__fadd_ru(t, 2.f * err));
    low = all ? 0u : key32(__fadd_rd(t, -2.f * err));
    auto is_near = [&](unsigned x) { return all || (x >= low && x <= top); };
    int n_sure = 0;
    each([&](int i, unsigned x) {
      n_sure += !all && x > top;
      if (is_near(x)) {
        const int at = atomicAdd(&s_few, 1);
        if (at < kThreads) s_near[at] = i;
      }
    });
    n_sure = __reduce_add_sync(0xffffffffu, n_sure);
    if (lane == 0) atomicAdd(&s_sure, n_sure);
    __syncthreads();
    const int near = s_few, need = B - s_sure;
    if (near == need) {
      // all of them stay
    } else if (near <= kThreads && old <= p.held) {
      // Few: what two floats say of each, and 64 bits of those they leave open; keys
      // on chip then say who stays.  (64-bit arithmetic runs at 1/64 of the rate: ten
      // pages cost 9 us with it alone.)
      if (tid < near) s_at[tid] = bounds_of<T>(c, u.l, u.s, u.h, s_near[tid]);
      __syncthreads();
      for (int k = warp; k < near; k += kWarps) {
        const float y = near_offset<T, D>(s_q, s_at[k], c.G, t, lane);
        if (lane == 0) s_off[k] = y;
      }
      __syncthreads();
      bool in = false, open = false;
      const float off = tid < near ? s_off[tid] : 0.f, e2 = 2.f * (err * kOff + 1e-40f);
      if (tid < near) {
        int maybe = 0, surely = 0;  // that go before it
        for (int k = 0; k < near; ++k) {
          maybe += k != tid && !(s_off[k] < off - e2);
          surely += s_off[k] > off + e2;
        }
        in = maybe < need;
        open = !in && surely < need;
      }
      const int n_in = __syncthreads_count(in);
      s_open[tid] = open;
      if (__syncthreads_or(open)) {
        for (int k = warp; k < near; k += kWarps) {
          if (!s_open[k]) continue;
          const unsigned long long y = exact_key<T, D>(s_q, s_at[k], c.G, lane);
          if (lane == 0) s_key[k] = y;
        }
        __syncthreads();
        if (open) {
          const unsigned long long y = s_key[tid];
          int above = 0;
          for (int k = 0; k < near; ++k)
            above += s_open[k] && (s_key[k] > y || (s_key[k] == y && s_near[k] < s_near[tid]));
          in = above < need - n_in;
        }
      }
      if (tid < near) s_held[place(s_near[tid])] = in ? ~0u : 0u;
      low = all ? ~0u : low > 0 ? low : 1u;
      __syncthreads();
    } else {
      // Many: 64 bits for each of them, and digit by digit.  (4 units of 513 pages, of
      // which 30 and 70% are alike: 182 and 345 us a call, else 16; 112 of 4,097 pages 1.2
      // and 2.6 ms, else 88 us.)
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
              exact_key<T, D>(s_q, bounds_of<T>(c, u.l, u.s, u.h, i0 + at), c.G, lane);
          if (lane == at) key = y;
        }
        if (i < old) keys[i] = key;
      }
      __syncthreads();
      cut = nth<kThreads, unsigned long long>(old, B, 63, [&](int i) { return keys[i]; }, hist,
                                              &s_digit, &s_left, &equal);
    }
  }
  // The pages that stay, in order: a thread goes through a run of them, once to count
  // and once to write.
  const int run = (old + kThreads - 1) / kThreads;
  const int from = min(tid * run, old), upto = min(from + run, old);
  int stay = 0, ties = 0;
  if (settle) {
    for (int i = from; i < upto; ++i) stay += keys[i] > cut, ties += keys[i] == cut;
  } else {
#pragma unroll 4
    for (int i = from; i < upto; ++i) stay += held(i) >= low;
  }
  int stay_upto = stay, ties_upto = ties;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int a = __shfl_up_sync(0xffffffffu, stay_upto, o);
    const int b = __shfl_up_sync(0xffffffffu, ties_upto, o);
    if (lane >= o) stay_upto += a, ties_upto += b;
  }
  if (lane == 31) s_stay[warp] = stay_upto, s_ties[warp] = ties_upto;
  __syncthreads();
  int at = stay_upto - stay, rank = ties_upto - ties;
  for (int w = 0; w < warp; ++w) at += s_stay[w], rank += s_ties[w];
  at += min(rank, equal);  // ties stay in order of position while there is room
  const bool few = B <= kThreads;  // positions on chip, so that pages are looked up together
  auto put = [&](int at, int i) {
    list[at] = table[i];
    if (chosen) chosen[at] = i;
  };
  if (settle || stay > 0) {
#pragma unroll 4
    for (int i = from; i < upto; ++i) {
      bool in;
      if (settle) {
        in = keys[i] > cut || (keys[i] == cut && rank < equal);
        rank += keys[i] == cut;
      } else {
        in = held(i) >= low;
      }
      if (in && at < B) {
        if (few)
          s_near[at] = i;
        else
          put(at, i);
      }
      at += in;
    }
  }
  __syncthreads();
  if (few && tid < B) put(tid, s_near[tid]);
  for (int i = tid; i < p.window; i += kThreads) put(B + i, old + i);
}

// What the attention reads of each sequence: rows of the pages that stay, and the
// tiles of the sequences before it.
template <int kThreads>
__device__ void sequences(const SelectParams &p) {
  constexpr int kWarps = kThreads / 32;
  __shared__ int s_warp[kWarps];
  const View &c = p.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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
}

// A cluster a unit: its CTAs score its pages into the shared memory of the first, which
// chooses.  One cluster more: sequences().
constexpr int kUnitCtas = 8;

template <typename T, int D>
__global__ void __launch_bounds__(kBlock, 2) select_kernel(const __grid_constant__ SelectParams p) {
  kvr::pdl_begin();
  extern __shared__ __align__(16) unsigned s_dynamic[];
  const unsigned unit = blockIdx.x / kUnitCtas, rank = blockIdx.x % kUnitCtas;
  if (unit == gridDim.x / kUnitCtas - 1) {
    if (rank == 0) sequences<kBlock>(p);
    return;
  }
  // (the first CTA runs before anything is written to its memory)
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const Unit u = unit_of(p, unit);
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  // behind the keys: pairs
  float2 *sc = reinterpret_cast<float2 *>(s_dynamic + keys_words(p.held));
  if (u.old > 0) {
    uint32_t to;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(kvr::ptx::smem_u32(sc)), "r"(0));
    const int groups = groups_of(p.c);
    // (the step stays in the unit, and then leads out of it)
    for (int i = rank * kBlockWarps + (threadIdx.x >> 5); i < groups;
         i += kUnitCtas * kBlockWarps)
      score_items<D>(p, Items((int)unit, i, groups, (int)unit + 1, groups), (const T *)nullptr,
                     [&](long long, int at, float2 x) {
                       asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to + 8 * at),
                                    "f"(x.x), "f"(x.y)
                                    : "memory");
                     });
    kvr::ptx::cluster_sync();
  }
  if (rank == 0) choose<T, D, true, kBlock>(p, u, sc);
}

// The same in two launches, scores in memory.
template <typename T, int D>
__global__ void __launch_bounds__(kBlock, 2) score_kernel(const __grid_constant__ SelectParams p) {
  kvr::pdl_begin();
  const int groups = groups_of(p.c);
  const unsigned warp = blockIdx.x * kBlockWarps + (threadIdx.x >> 5);
  score_items<D>(p, Items(warp / groups, warp % groups, gridDim.x * kBlockWarps,
                          p.c.S * p.nl * p.c.H, groups),
                 (const T *)nullptr,
                 [&](long long unit, int at, float2 x) { p.score[unit * p.sstride + at] = x; });
}
template <typename T, int D, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == kWide ? 1 : 5)
    choose_kernel(const __grid_constant__ SelectParams p) {
  kvr::pdl_begin();
  if (blockIdx.x == 0) return sequences<kThreads>(p);
  const Unit u = unit_of(p, blockIdx.x - 1);
  choose<T, D, false, kThreads>(p, u, p.score + u.at * p.sstride);
}

template <typename T, int D>
cudaError_t launch(SelectParams p, int sms, cudaStream_t st, int *launches) {
  const long long units = (long long)p.c.S * p.nl * p.c.H;
  cudaError_t e;
  // (choice and attention in a graph, us a call: 4 units of 512 pages 14.1, in two launches
  // 15.5; 16 units 22.3 and 23.9; 36 units 25.9 and 25.1)
  if (units * kUnitCtas <= sms && p.sstride <= kOnChip) {
    p.held = p.sstride;
    const size_t smem = keys_words(p.held) * 4 + (size_t)p.held * 8;
    e = kvr::launch_pdl_cluster(select_kernel<T, D>, dim3((unsigned)(units + 1) * kUnitCtas),
                                dim3(kBlock), kUnitCtas, smem, st, p);
  } else {
    if (p.budget > 0) {
      const long long ctas = (units * ((p.c.tstride + 15) / 16) + kBlockWarps - 1) / kBlockWarps;
      e = kvr::launch_pdl(score_kernel<T, D>, dim3((unsigned)std::min<long long>(ctas, 2ll * sms)),
                          dim3(kBlock), 0, st, p);
      if (e != cudaSuccess) return e;
      *launches += 1;
    }
    p.held = std::min(p.sstride, kHeld);  // (both even)
    const dim3 grid((unsigned)units + 1);
    const size_t smem = keys_words(p.held) * 4;
    // (112 units of 4,096 pages: 15 us, with 256 threads 20)
    e = units < sms && p.c.tstride > kWide
            ? kvr::launch_pdl(choose_kernel<T, D, kWide>, grid, dim3(kWide), smem, st, p)
            : kvr::launch_pdl(choose_kernel<T, D, kBlock>, grid, dim3(kBlock), smem, st, p);
  }
  if (e == cudaSuccess) *launches += 1;
  return e;
}

// The wide form's lists and keys are more than a CTA gets unasked.
template <typename T, int D>
cudaError_t prepare() {
  return cudaFuncSetAttribute(choose_kernel<T, D, kWide>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize, keys_words(kHeld) * 4);
}

}  // namespace

cudaError_t prepare_select(const View &c) {
  if (c.io_bf16) return c.d == 128 ? prepare<__nv_bfloat16, 128>() : prepare<__nv_bfloat16, 64>();
  return c.d == 128 ? prepare<float, 128>() : prepare<float, 64>();
}

cudaError_t launch_select(const SelectParams &p, int sms, cudaStream_t st, int *launches) {
  if (p.c.io_bf16)
    return p.c.d == 128 ? launch<__nv_bfloat16, 128>(p, sms, st, launches)
                        : launch<__nv_bfloat16, 64>(p, sms, st, launches);
  return p.c.d == 128 ? launch<float, 128>(p, sms, st, launches)
                      : launch<float, 64>(p, sms, st, launches);
}

}  // namespace paged
}  // namespace kvr
