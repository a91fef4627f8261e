// kvr_kv4.cu -- the full context held in 4 bits (include/kvr.h, kvr_kv4_*): its
// C ABI and host state, and the kernels that write rows, read back what they
// stand for, and cut them into an evicted cache.  kvr_kv4.cuh has the layout and
// the format's arithmetic, kvr_kv4_attend.cu the attention.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/kvr.h"
#include "kvr_device.cuh"
#include "kvr_internal.h"
#include "kvr_kv4.cuh"
#include "kvr_ptx.cuh"

namespace kvr {
namespace kv4 {
namespace {

// Eight channels of a row and side are a lane's share, as they lie in a word of
// codes: lane i has channels 8 i .. 8 i + 7 of a key, and of a value the pairs
// (p, p + 1), p = 32 (i / 4) + 2 (i % 4) + {0, 16, 8, 24}, the first of each pair
// first.
template <typename T>
struct Eight {
  uint32_t w[2 * sizeof(T)];
};
__device__ __forceinline__ int pair_channel(int i, int f) {
  return 32 * (i >> 2) + 2 * (i & 3) + (f == 0 ? 0 : f == 1 ? 16 : f == 2 ? 8 : 24);
}
template <typename T>
__device__ __forceinline__ Eight<T> load_eight(const T *row, int side, int i) {
  Eight<T> a;
  if (side) {
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const T *at = row + pair_channel(i, f);
      if (sizeof(T) == 2) {
        a.w[f] = __ldcs(reinterpret_cast<const uint32_t *>(at));
      } else {
        const uint2 x = __ldcs(reinterpret_cast<const uint2 *>(at));
        a.w[2 * f % (2 * sizeof(T))] = x.x, a.w[(2 * f + 1) % (2 * sizeof(T))] = x.y;
      }
    }
  } else {
#pragma unroll
    for (int z = 0; z < (int)sizeof(T) / 2; ++z) {
      const uint4 x = __ldcs(reinterpret_cast<const uint4 *>(row + 8 * i) + z);
      a.w[4 * z] = x.x, a.w[4 * z + 1] = x.y, a.w[4 * z + 2] = x.z, a.w[4 * z + 3] = x.w;
    }
  }
  return a;
}
// In the order of a word's nibbles.
__device__ __forceinline__ void widen(const Eight<__nv_bfloat16> &a, int side, float (&x)[8]) {
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const float lo = __uint_as_float(a.w[f] << 16), hi = __uint_as_float(a.w[f] & 0xFFFF0000u);
    x[side ? f : 2 * f] = lo;
    x[side ? 4 + f : 2 * f + 1] = hi;
  }
}
__device__ __forceinline__ void widen(const Eight<float> &a, int side, float (&x)[8]) {
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    x[side ? f : 2 * f] = __uint_as_float(a.w[2 * f]);
    x[side ? 4 + f : 2 * f + 1] = __uint_as_float(a.w[2 * f + 1]);
  }
}
// The least and the greatest of a group, over its eight lanes; true if one of the
// lane's own is not finite.
__device__ __forceinline__ bool extremes(const Eight<float> &, const float (&x)[8], float &lo,
                                         float &hi) {
  float odd = 0.f;
  lo = hi = x[0];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
    odd = fmaf(x[e], 0.f, odd);  // NaN for what is not finite
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  return odd != 0.f;
}
__device__ __forceinline__ bool extremes(const Eight<__nv_bfloat16> &a, const float (&)[8],
                                         float &lo, float &hi) {
  __nv_bfloat162 w[4];
#pragma unroll
  for (int f = 0; f < 4; ++f) w[f] = *reinterpret_cast<const __nv_bfloat162 *>(&a.w[f]);
  const __nv_bfloat162 least = __hmin2(__hmin2(w[0], w[1]), __hmin2(w[2], w[3]));
  const __nv_bfloat162 most = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
  const __nv_bfloat162 zero = __float2bfloat162_rn(0.f);
  __nv_bfloat162 odd = __hfma2(w[0], zero, zero);
#pragma unroll
  for (int f = 1; f < 4; ++f) odd = __hfma2(w[f], zero, odd);
  // the least and minus the greatest as one word: an exchange and a minimum for both
  const __nv_bfloat162 l = __hmin2(least, __lowhigh2highlow(least));
  const __nv_bfloat162 h = __hmax2(most, __lowhigh2highlow(most));
  uint32_t both = (*reinterpret_cast<const uint32_t *>(&l) & 0xFFFFu) |
                  ((*reinterpret_cast<const uint32_t *>(&h) & 0xFFFF0000u) ^ 0x80000000u);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, both, o);
    const __nv_bfloat162 y = __hmin2(*reinterpret_cast<const __nv_bfloat162 *>(&both),
                                     *reinterpret_cast<const __nv_bfloat162 *>(&other));
    both = *reinterpret_cast<const uint32_t *>(&y);
  }
  lo = __uint_as_float(both << 16);
  hi = __uint_as_float((both & 0xFFFF0000u) ^ 0x80000000u);
  return (*reinterpret_cast<const uint32_t *>(&odd) & 0x7FFF7FFFu) != 0;
}
__device__ __forceinline__ void store_eight(const float (&x)[8], int side, int i,
                                            __nv_bfloat16 *row) {
  if (side) {
#pragma unroll
    for (int f = 0; f < 4; ++f)
      *reinterpret_cast<uint32_t *>(row + pair_channel(i, f)) = ptx::pack_bf16(x[f], x[4 + f]);
  } else {
    *reinterpret_cast<uint4 *>(row + 8 * i) =
        make_uint4(ptx::pack_bf16(x[0], x[1]), ptx::pack_bf16(x[2], x[3]),
                   ptx::pack_bf16(x[4], x[5]), ptx::pack_bf16(x[6], x[7]));
  }
}
__device__ __forceinline__ void store_eight(const float (&x)[8], int side, int i, float *row) {
  if (side) {
#pragma unroll
    for (int f = 0; f < 4; ++f)
      *reinterpret_cast<float2 *>(row + pair_channel(i, f)) = make_float2(x[f], x[4 + f]);
  } else {
    reinterpret_cast<float4 *>(row + 8 * i)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(row + 8 * i)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// A code by the definition's division.  Not inlined: with its divisions in every
// round the kernel outgrew the instruction cache (append of 2 x 8,191 tokens: 309 us
// against 226).
__device__ __noinline__ uint32_t divided_code(float x, uint32_t meta) {
  return code_of(x, meta, false);
}

// The codes of eight values as one word, code e in bits 4 e .. 4 e + 3.  x r - m r
// (r about 1 / s, m / s at most 64) is off by less than 2e-5, so it finds a code
// unless it lies that near to half-way between two (of bf16 values one in 450 lies
// exactly there), and it stays within -0.2 and 15.3, so that nothing needs to be
// cut to 0..15; the rest is divided.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], uint32_t meta, bool flat) {
  using namespace ptx;
  const float m = m_of(meta), r = rcp(s_of(meta)), mr = m * r;
  const uint64_t r2 = pk2(r, r), d2 = pk2(-mr, -mr), magic = pk2(12582912.f, 12582912.f);
  const uint64_t minus = pk2(-12582912.f, -12582912.f), neg = pk2(-1.f, -1.f);
  uint32_t k[8];
  float d[8], off = 0.f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const uint64_t q = fma2(pk2(x[e], x[e + 1]), r2, d2);
    const uint64_t t = add2(q, magic);  // 1.5 2^23: the code in the low bits
    float a, b;
    upk2(fma2(add2(t, minus), neg, q), d[e], d[e + 1]);
    off = fmaxf(off, fmaxf(fabsf(d[e]), fabsf(d[e + 1])));
    upk2(t, a, b);
    k[e] = __float_as_uint(a), k[e + 1] = __float_as_uint(b);
  }
  constexpr float kNear = 0.49996f;
  // (a scale that is nearly subnormal has no reciprocal, and a huge one flushes)
  const bool all = !(fabsf(mr) < 64.f) || !(r < 1e37f && r > 1e-37f);
  if (!(off < kNear) || all) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!(fabsf(d[e]) < kNear) || all) k[e] = divided_code(x[e], meta);
  }
  // low bytes, two codes a byte
  uint32_t z[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t y = __byte_perm(__byte_perm(k[4 * h], k[4 * h + 1], 0x0040),
                                   __byte_perm(k[4 * h + 2], k[4 * h + 3], 0x0040), 0x5410);
    z[h] = y | (y >> 4);
  }
  return flat ? 0 : __byte_perm(z[0], z[1], 0x6420);
}

// Where the lane finds or puts them.
template <int D>
__device__ __forceinline__ uint32_t *k_word(uint8_t *block, int r, int i) {
  int hi;
  return reinterpret_cast<uint32_t *>(block + k_byte<D>(r, 8 * i, hi));
}
template <int D>
__device__ __forceinline__ uint16_t *v_half_at(uint8_t *block, int r, int i, int c) {
  return reinterpret_cast<uint16_t *>(block + v_half<D>(r, i >> 2, c));
}
template <int D>
__device__ __forceinline__ uint32_t *meta_word(uint8_t *block, int side, int r, int i) {
  return reinterpret_cast<uint32_t *>(block + (side ? vm_off(D) : km_off(D)) +
                                      (r * (D / kGroup) + (i >> 3)) * 4);
}

// Which (unit, side, token group) a warp of a launch over units x groups x 2 is.
struct Task {
  int s, lr, h, side, group;
  bool any;
};
__device__ __forceinline__ Task task_of(const Call &k, int groups) {
  Task t;
  const unsigned w = blockIdx.x * 8 + (threadIdx.x >> 5);
  const unsigned unit = (w >> 1) / (unsigned)groups;
  t.s = blockIdx.y;
  t.side = (int)(w & 1);
  t.group = (int)((w >> 1) - unit * groups);
  t.lr = (int)(unit / (unsigned)k.c.H);
  t.h = (int)(unit - (unsigned)t.lr * k.c.H);
  t.any = t.lr < k.nl;
  return t;
}

// Quantise the new rows.  D / 8 lanes a row, eight channels a lane; a warp takes
// kRows rows of one side (key or value) at a time, their loads in flight together.
// Many tokens are bound by instructions (2 x 8,191 tokens of 28 layers, 2 KV heads: 196
// us, 3.1 TB/s read and written), few by latency (one token of 28 layers, 4 KV heads
// and its reading back: 4 us).
template <typename T, int D>
struct Append {
  static constexpr int kLanes = D / 8;             // of a row
  static constexpr int kOnce = 32 / kLanes;        // rows of a warp at once
  static constexpr int kRounds = 4;
  static constexpr int kRows = kOnce * kRounds;    // rows of a warp
};
template <typename T, int D, int SIDE>
__device__ __forceinline__ void append_rows(const Call &k, const Seqs &q, const Task &at,
                                            const T *src, long long token_stride) {
  using A = Append<T, D>;
  const View &c = k.c;
  const int lane = threadIdx.x & 31, i = lane % A::kLanes;
  const int count = q.count[at.s], t0 = at.group * A::kRows;
  Eight<T> in[A::kRounds];
#pragma unroll
  for (int n = 0; n < A::kRounds; ++n) {
    const int t = min(t0 + n * A::kOnce + lane / A::kLanes, count - 1);
    in[n] = load_eight(src + t * token_stride, SIDE, i);
  }
  const size_t u = unit_at(c, k.s0 + at.s, k.lb, at.lr, at.h);
  const int r0 = q.len[at.s] - count;
#pragma unroll
  for (int n = 0; n < A::kRounds; ++n) {
    if (t0 + n * A::kOnce >= count) break;
    const int t = t0 + n * A::kOnce + lane / A::kLanes;
    float x[8], lo, hi;
    widen(in[n], SIDE, x);
    const bool odd = extremes(in[n], x, lo, hi);
    const unsigned bad = __ballot_sync(0xffffffffu, odd);
    bool flat;
    const uint32_t meta =
        group_meta(lo, hi, ((bad >> (lane & ~7)) & 255u) == 0, flat);
    const uint32_t word = codes_of(x, meta, flat);
    if (t < count) {
      const int r = r0 + t, rb = r % kBlock;
      uint8_t *block = block_at(c, u, r);
      if (SIDE) {
        const int y = i & 3;
        *v_half_at<D>(block, rb, i, 2 * y) = (uint16_t)word;
        *v_half_at<D>(block, rb, i, 2 * y + 1) = (uint16_t)(word >> 16);
      } else {
        *k_word<D>(block, rb, i) = word;
      }
      if (i % 8 == 0) *meta_word<D>(block, SIDE, rb, i) = meta;
      if (SIDE == 0 && i == 0) c.score[u * c.sstride + r] = 0.f;
    }
  }
}
template <typename T, int D>
__global__ void __launch_bounds__(256)
    append_kernel(const __grid_constant__ Call k, const __grid_constant__ Seqs q, int groups,
                  const T *key, const T *val, RowStrides st) {
  pdl_begin();
  const Task at = task_of(k, groups);
  if (!at.any || at.group * Append<T, D>::kRows >= q.count[at.s]) return;
  const long long from = (at.s + k.s0) * st.seq + at.lr * st.layer + at.h * st.head;
  if (at.side)
    append_rows<T, D, 1>(k, q, at, val + from, st.token);
  else
    append_rows<T, D, 0>(k, q, at, key + from, st.token);
}

// The lane's word of codes and its (m, s), and what they stand for.
struct RowWords {
  uint32_t w, meta;
};
template <int D>
__device__ __forceinline__ RowWords row_words(const uint8_t *block, int side, int r, int i) {
  uint8_t *at = const_cast<uint8_t *>(block);
  RowWords x;
  if (side) {
    const int y = i & 3;
    x.w = *v_half_at<D>(at, r, i, 2 * y) |
          ((uint32_t)*v_half_at<D>(at, r, i, 2 * y + 1) << 16);
  } else {
    x.w = *k_word<D>(at, r, i);
  }
  x.meta = *meta_word<D>(at, side, r, i);
  return x;
}
__device__ __forceinline__ void word_values(const RowWords &a, float (&x)[8]) {
  const float m = m_of(a.meta), s = s_of(a.meta);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t c = ((a.w >> (4 * e)) & 15u) | 0x4B000000u;  // 2^23 + c
    x[e] = fmaf(__uint_as_float(c) - 8388608.f, s, m);
  }
}

// What the newest rows stand for: D / 8 lanes a row and side.  Bound by the bytes: the
// same 2 x 8,191 rows 123 us, 4.9 TB/s.
template <typename T, int D>
__global__ void __launch_bounds__(256)
    read_kernel(const __grid_constant__ Call k, const __grid_constant__ Seqs q, int groups,
                int rows, T *key, T *val) {
  pdl_begin();
  using A = Append<T, D>;
  const View &c = k.c;
  const int lane = threadIdx.x & 31, i = lane % A::kLanes;
  const Task at = task_of(k, groups);
  if (!at.any) return;
  const int count = q.count[at.s], r0 = q.len[at.s] - count, t0 = at.group * A::kRows;
  const size_t u = unit_at(c, k.s0 + at.s, k.lb, at.lr, at.h);
  T *to = (at.side ? val : key) +
          (((size_t)(at.s + k.s0) * k.nl + at.lr) * c.H + at.h) * rows * D;
  RowWords words[A::kRounds];
#pragma unroll
  for (int n = 0; n < A::kRounds; ++n) {
    const int r = r0 + min(t0 + n * A::kOnce + lane / A::kLanes, count - 1);
    words[n] = RowWords{0, 0};
    if (count > 0) words[n] = row_words<D>(block_at(c, u, r), at.side, r % kBlock, i);
  }
#pragma unroll
  for (int n = 0; n < A::kRounds; ++n) {
    const int t = t0 + n * A::kOnce + lane / A::kLanes;
    if (t >= rows) break;
    float x[8];
    if (t >= count) words[n] = RowWords{0, 0};
    word_values(words[n], x);
    if (at.side)
      store_eight(x, 1, i, to + (size_t)t * D);
    else
      store_eight(x, 0, i, to + (size_t)t * D);
  }
}

// A score's rank, higher first: -0 counts as 0, and every NaN as one above every
// number.
__device__ __forceinline__ uint32_t score_rank(float x) {
  const uint32_t b = __float_as_uint(x), a = b & 0x7FFFFFFFu;
  return a > 0x7F800000u ? 0xFFFFFFFFu : a == 0 ? 0x80000000u : b != a ? ~b : (b | 0x80000000u);
}

// Cut a unit into dst: one CTA a unit, whose scores' ranks lie in shared memory
// (or are formed from the scores anew, where a unit has too many rows).  Three
// passes of 11, 11 and 10 bits find the rank of the budget-th row before the
// window; of the rows of that rank the first ones are kept.  (Attention leaves
// scores within a few octaves: bins of a quarter octave keep the lanes of a warp
// off each other's counters.)  The kept rows are listed in order, in dst's
// positions, and their values written from there, D / 8 lanes a row and side.
// What costs is latency: every step has its loads in flight together.  One sequence
// of 2,048 rows (28 layers, 4 KV heads) cut to 64 + 8: 7 us; four of 4,000 to 16,384
// cut to 512 + 128: 66 us, of which the bytes need 30.
constexpr int kEvictThreads = 512;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictBins = 2048;
constexpr int kEvictSmemRows = 24576;

template <typename T, int D, bool IN_SMEM>
__global__ void __launch_bounds__(kEvictThreads, 2)
    evict_kernel(const __grid_constant__ Call k, const __grid_constant__ Seqs q,
                 const __grid_constant__ CacheView dst, int budget, int window) {
  extern __shared__ uint32_t s_rank[];
  __shared__ unsigned s_hist[kEvictBins];
  __shared__ int s_count[kEvictWarps], s_ties[kEvictWarps];
  __shared__ unsigned s_digit, s_need;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_begin();
  const View &c = k.c;
  const int h = blockIdx.x % c.H, l = blockIdx.x / c.H;
  const int s = q.count[blockIdx.y];  // the longest sequences first
  const size_t u = unit_at(c, k.s0 + s, 0, l, h);
  const float *score = c.score + u * c.sstride;
  const int n = q.len[s], first = max(0, n - window);  // rows [first, n): the window
  const int keep = min(n, budget + window);
  const bool cut = first > budget;
  if (IN_SMEM && cut) {
    // rows of 16 floats start on 64 bytes, so whole vectors are within the row; what
    // is beyond `first` gets rank 0, which no score has
#pragma unroll 8
    for (int i = tid; 4 * i < first; i += kEvictThreads) {
      const float4 x = __ldg(reinterpret_cast<const float4 *>(score) + i);
      *reinterpret_cast<uint4 *>(s_rank + 4 * i) =
          make_uint4(score_rank(x.x), 4 * i + 1 < first ? score_rank(x.y) : 0u,
                     4 * i + 2 < first ? score_rank(x.z) : 0u,
                     4 * i + 3 < first ? score_rank(x.w) : 0u);
    }
  }
  auto rank = [&](int i) { return IN_SMEM ? s_rank[i] : score_rank(score[i]); };
  // The rank of the last row kept, and how many rows of that rank are kept.
  uint32_t least = 0, mask = 0;
  int need = budget;
  if (cut && budget > 0) {
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t digits = pass == 2 ? 1023u : 2047u;
      for (int i = tid; i < kEvictBins; i += kEvictThreads) s_hist[i] = 0;
      __syncthreads();
      auto count = [&](uint32_t x) {
        if ((x & mask) == least && x) atomicAdd(&s_hist[(x >> shift) & digits], 1u);
      };
      if (IN_SMEM) {
#pragma unroll 4
        for (int i = tid; 4 * i < first; i += kEvictThreads) {
          const uint4 x = *reinterpret_cast<const uint4 *>(s_rank + 4 * i);
          count(x.x), count(x.y), count(x.z), count(x.w);
        }
      } else {
#pragma unroll 4
        for (int i = tid; i < first; i += kEvictThreads) count(rank(i));
      }
      __syncthreads();
      // a thread's four digits, counted from the top
      constexpr int kPer = kEvictBins / kEvictThreads;
      unsigned d[kPer], sum = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        d[e] = s_hist[kEvictBins - 1 - kPer * tid - e];
        sum += d[e];
      }
      unsigned above = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned x = __shfl_up_sync(0xffffffffu, above, o);
        if (lane >= o) above += x;
      }
      if (lane == 31) s_count[warp] = (int)above;
      __syncthreads();
      above += __reduce_add_sync(0xffffffffu,
                                 lane < warp ? (unsigned)s_count[lane % kEvictWarps] : 0u) -
               sum;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        if (above < (unsigned)need && above + d[e] >= (unsigned)need) {
          s_digit = kEvictBins - 1 - kPer * tid - e;
          s_need = need - above;
        }
        above += d[e];
      }
      __syncthreads();
      least |= s_digit << shift;
      need = s_need;
      mask |= digits << shift;
    }
  }
  // List the kept rows in order: each warp counts those of its own stretch, and
  // then knows where they go.
  int32_t *pos = dst.pos + u * dst.sstride;
  float *to_score = dst.score + u * dst.sstride;
  const int stretch = (n + 32 * kEvictWarps - 1) / (32 * kEvictWarps) * 32;
  const int i0 = min(n, warp * stretch), i1 = min(n, i0 + stretch);
  const unsigned lower = (1u << lane) - 1u;
  auto look = [&](int i, unsigned &over, unsigned &tie) {  // ballots of 32 rows
    bool o = i < n && (i >= first || !cut), t = false;
    if (cut && budget > 0 && i < first) {
      const uint32_t x = rank(i);
      o = x > least;
      t = x == least;
    }
    over = __ballot_sync(0xffffffffu, o);
    tie = __ballot_sync(0xffffffffu, t);
  };
  int overs = 0, ties = 0;
#pragma unroll 4
  for (int b = i0; b < i1; b += 32) {
    unsigned over, tie;
    look(b + lane, over, tie);
    overs += __popc(over);
    ties += __popc(tie);
  }
  if (lane == 0) {
    s_count[warp] = overs;
    s_ties[warp] = ties;
  }
  __syncthreads();
  overs = __reduce_add_sync(0xffffffffu, lane < warp ? s_count[lane % kEvictWarps] : 0);
  ties = __reduce_add_sync(0xffffffffu, lane < warp ? s_ties[lane % kEvictWarps] : 0);
#pragma unroll 4
  for (int b = i0; b < i1; b += 32) {
    unsigned over, tie;
    look(b + lane, over, tie);
    const int tied = ties + __popc(tie & lower);
    const bool kept = (over >> lane & 1u) || ((tie >> lane & 1u) && tied < need);
    const int at = overs + __popc(over & lower) + min(tied, need);
    if (kept && at < keep) pos[at] = b + lane;
    overs += __popc(over);
    ties += __popc(tie);
  }
  if (tid == kEvictThreads - 1 && overs + min(ties, need) != keep && cut)
    atomicOr(c.err, ERR_LENGTH);
  __syncthreads();
  for (int j = tid; j < keep; j += kEvictThreads) to_score[j] = score[pos[j]];
  // Their values: D / 8 lanes a row, kBatch rows of each in flight.
  constexpr int kLanes = D / 8, kOnce = 32 / kLanes, kBatch = 8;
  constexpr int kStride = kEvictWarps * kOnce;
  const int m = keep, ch = lane % kLanes;
  for (int j0 = warp * kOnce; j0 < m; j0 += kBatch * kStride) {
    RowWords kw[kBatch], vw[kBatch];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
      const int r = pos[min(j0 + e * kStride + lane / kLanes, m - 1)];
      const uint8_t *block = block_at(c, u, r);
      kw[e] = row_words<D>(block, 0, r % kBlock, ch);
      vw[e] = row_words<D>(block, 1, r % kBlock, ch);
    }
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
      const int j = j0 + e * kStride + lane / kLanes;
      if (j >= m) continue;
      const size_t to = (u * (size_t)dst.cap + j) * D;
      float x[8];
      word_values(kw[e], x);
      store_eight(x, 0, ch, static_cast<T *>(dst.K) + to);
      word_values(vw[e], x);
      store_eight(x, 1, ch, static_cast<T *>(dst.V) + to);
    }
  }
  if (tid == 0) {
    dst.state[4 * u] = m;
    dst.state[4 * u + 1] = n;
    dst.state[4 * u + 2] = 0;  // no R-KV key sum yet
  }
}

// Grid of a launch of eight warps a CTA, kRows rows of one side a warp.
template <typename T, int D>
bool row_grid(const Call &k, int rows, int *groups, dim3 *grid) {
  constexpr int kRows = Append<T, D>::kRows;
  *groups = (rows + kRows - 1) / kRows;
  const long long warps = 2ll * k.nl * k.c.H * *groups;
  *grid = dim3((unsigned)((warps + 7) / 8), k.n);
  return warps + 7 <= UINT32_MAX;
}
template <typename T, int D>
cudaError_t launch_read(const Call &k, const Seqs &q, int rows, void *key, void *val,
                        cudaStream_t stream) {
  dim3 grid;
  int groups;
  if (!row_grid<T, D>(k, rows, &groups, &grid)) return cudaErrorInvalidValue;
  return launch_pdl(read_kernel<T, D>, grid, dim3(256), 0, stream, k, q, groups, rows,
                    static_cast<T *>(key), static_cast<T *>(val));
}

template <typename T, int D>
cudaError_t launch_append_as(const Call &k, const Seqs &q, int tokens, const void *key,
                             const void *val, const RowStrides &st, cudaStream_t stream) {
  dim3 grid;
  int groups;
  if (!row_grid<T, D>(k, tokens, &groups, &grid)) return cudaErrorInvalidValue;
  return launch_pdl(append_kernel<T, D>, grid, dim3(256), 0, stream, k, q, groups,
                    static_cast<const T *>(key), static_cast<const T *>(val), st);
}

template <typename T, int D>
cudaError_t launch_evict(const Call &k, Seqs q, const CacheView &dst, int budget, int window,
                         cudaStream_t stream) {
  for (int i = 0; i < k.n; ++i) q.count[i] = i;
  std::sort(q.count, q.count + k.n, [&](int a, int b) { return q.len[a] > q.len[b]; });
  const int most = std::max(0, q.len[q.count[0]] - window);
  const dim3 grid(k.c.L * k.c.H, k.n);
  if (most > kEvictSmemRows)
    return launch_pdl(evict_kernel<T, D, false>, grid, dim3(kEvictThreads), 0, stream, k, q, dst,
                      budget, window);
  auto kern = evict_kernel<T, D, true>;
  const int bytes = most > budget ? round_up16(most) * 4 : 0;
  return launch_pdl(kern, grid, dim3(kEvictThreads), bytes, stream, k, q, dst, budget, window);
}

// The destination may be of either type.
template <int D>
cudaError_t prepare_evict() {
  cudaError_t e = cudaFuncSetAttribute(evict_kernel<__nv_bfloat16, D, true>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       kEvictSmemRows * 4);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(evict_kernel<float, D, true>,
                             cudaFuncAttributeMaxDynamicSharedMemorySize, kEvictSmemRows * 4);
  return e;
}

}  // namespace

cudaError_t launch_append(const Call &k, const Seqs &q, int tokens, const void *key,
                          const void *val, const RowStrides &st, cudaStream_t stream) {
  if (k.c.io_bf16)
    return k.c.d == 128
               ? launch_append_as<__nv_bfloat16, 128>(k, q, tokens, key, val, st, stream)
               : launch_append_as<__nv_bfloat16, 64>(k, q, tokens, key, val, st, stream);
  return k.c.d == 128 ? launch_append_as<float, 128>(k, q, tokens, key, val, st, stream)
                      : launch_append_as<float, 64>(k, q, tokens, key, val, st, stream);
}

}  // namespace kv4
}  // namespace kvr

using kvr::report_error;
using kvr::kv4::Call;
using kvr::kv4::Seqs;
using kvr::kv4::View;

struct kvr_kv4 {
  kvr_cache_desc desc;
  View view;
  kvr::kv4::Device device;
  std::vector<int32_t> len;  // [S][L]
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

struct Layout {
  size_t blocks, score, ticket, err, total;
  int nb, sstride;
};

// The descriptor's checks are those of an evicted cache.
bool layout_of(const kvr_cache_desc *d, Layout *l) {
  if (!kvr_cache_required_bytes(d)) return false;
  const size_t units = (size_t)d->n_seq * d->n_layers * d->n_kv_heads;
  l->nb = (d->capacity + kvr::kv4::kBlock - 1) / kvr::kv4::kBlock;
  l->sstride = kvr::round_up16(d->capacity);
  size_t off = 0;
  l->blocks = off;
  off = align_up(off + units * l->nb * (size_t)kvr::kv4::block_bytes(d->head_dim));
  l->score = off;
  off = align_up(off + units * l->sstride * sizeof(float));
  l->ticket = off;
  off = align_up(off + units * kvr::kv4::kMaxTiles * sizeof(unsigned));
  l->err = off;
  off = align_up(off + 16);
  l->total = off;
  return true;
}

bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// The layers' common length of every sequence, plus `grow` tokens where counts
// allows, in spans of kMaxSeqs sequences; fn(call, seqs) for each.
template <typename F>
kvr_status each_span(const kvr_kv4 *c, int lb, int le, int tokens, const int32_t *counts,
                     int grow, F fn) {
  const int S = c->desc.n_seq, L = c->desc.n_layers;
  Seqs q;
  for (int s0 = 0; s0 < S; s0 += kvr::kv4::kMaxSeqs) {
    Call k{c->view, s0, std::min(S - s0, kvr::kv4::kMaxSeqs), lb, le - lb};
    for (int i = 0; i < k.n; ++i) {
      q.count[i] = counts ? counts[s0 + i] : tokens;
      q.len[i] = c->len[(size_t)(s0 + i) * L + lb] + (grow ? q.count[i] : 0);
    }
    const kvr_status st = fn(k, q);
    if (st != KVR_OK) return st;
  }
  return KVR_OK;
}

kvr_status check_call(const kvr_kv4 *c, int lb, int le, int tokens, const int32_t *counts) {
  if (!c) return fail(KVR_EINVAL, "null cache");
  const int S = c->desc.n_seq, L = c->desc.n_layers;
  if (lb < 0 || le > L || lb >= le)
    return fail(KVR_EINVAL, "layer range [%d, %d) outside [0, %d)", lb, le, L);
  if (tokens < 1 || tokens > (1 << 24)) return fail(KVR_EINVAL, "%d tokens", tokens);
  for (int s = 0; s < S; ++s) {
    if (counts && (counts[s] < 0 || counts[s] > tokens))
      return fail(KVR_EINVAL, "sequence %d: %d of %d tokens", s, counts[s], tokens);
    for (int l = lb + 1; l < le; ++l)
      if (c->len[(size_t)s * L + l] != c->len[(size_t)s * L + lb])
        return fail(KVR_ESTATE, "sequence %d: layers %d and %d differ in length", s, lb, l);
  }
  return KVR_OK;
}

// Of a workspace for statistics of n_q tokens and so many floats of partial results.
size_t bytes_of(const kvr_kv4 *c, int nl, int n_q, size_t parts) {
  return std::max<size_t>(16, (kvr::kv4::attend_stat_floats(c->view, nl, n_q) + parts) *
                                  sizeof(float));
}

}  // namespace

extern "C" {

size_t kvr_kv4_required_bytes(const kvr_cache_desc *desc) {
  Layout l;
  return layout_of(desc, &l) ? l.total : 0;
}

kvr_status kvr_kv4_create(const kvr_cache_desc *desc, void *dev_buf, size_t bytes,
                          void *stream, kvr_kv4 **out) {
  if (!out) return fail(KVR_EINVAL, "null output handle");
  *out = nullptr;
  Layout l;
  if (!layout_of(desc, &l)) return fail(KVR_EINVAL, "invalid cache descriptor");
  if (!dev_buf) return fail(KVR_EINVAL, "null device buffer");
  if (reinterpret_cast<uintptr_t>(dev_buf) % kAlign)
    return fail(KVR_EINVAL, "device buffer not %zu-byte aligned", kAlign);
  if (bytes < l.total)
    return fail(KVR_ENOMEM, "buffer of %zu bytes < required %zu", bytes, l.total);
  kvr_kv4 *c = new (std::nothrow) kvr_kv4();
  if (!c) return fail(KVR_ENOMEM, "host allocation failed");
  c->desc = *desc;
  uint8_t *b = static_cast<uint8_t *>(dev_buf);
  View &v = c->view;
  v.blocks = b + l.blocks;
  v.score = reinterpret_cast<float *>(b + l.score);
  v.ticket = reinterpret_cast<unsigned *>(b + l.ticket);
  v.err = reinterpret_cast<unsigned *>(b + l.err);
  v.S = desc->n_seq;
  v.L = desc->n_layers;
  v.H = desc->n_kv_heads;
  v.G = desc->group;
  v.d = desc->head_dim;
  v.cap = desc->capacity;
  v.nb = l.nb;
  v.sstride = l.sstride;
  v.scale = desc->softmax_scale > 0.f ? desc->softmax_scale
                                      : 1.0f / std::sqrt((float)desc->head_dim);
  v.io_bf16 = desc->kv_dtype == KVR_BF16;
  v.out_bf16 = desc->out_dtype == KVR_BF16;
  try {
    c->len.assign((size_t)v.S * v.L, 0);
  } catch (const std::bad_alloc &) {
    delete c;
    return fail(KVR_ENOMEM, "host allocation failed");
  }
  cudaError_t e = kvr::kv4::prepare_attend(v, &c->device);
  if (e == cudaSuccess)
    e = v.d == 128 ? kvr::kv4::prepare_evict<128>() : kvr::kv4::prepare_evict<64>();
  // scores, tickets and the error word lie side by side
  if (e == cudaSuccess)
    e = cudaMemsetAsync(b + l.score, 0, l.total - l.score, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) {
    delete c;
    return cuda_fail("kvr_kv4_create", e);
  }
  *out = c;
  return KVR_OK;
}

void kvr_kv4_destroy(kvr_kv4 *cache) { delete cache; }

kvr_status kvr_kv4_load(kvr_kv4 *c, int seq, const void *k, const void *v, int n_rows,
                        void *stream) {
  if (!c) return fail(KVR_EINVAL, "null cache");
  const kvr_cache_desc &d = c->desc;
  if (seq < 0 || seq >= d.n_seq)
    return fail(KVR_EINVAL, "sequence %d outside [0, %d)", seq, d.n_seq);
  if (n_rows < 0) return fail(KVR_EINVAL, "%d rows", n_rows);
  if (n_rows > d.capacity)
    return fail(KVR_ECAPACITY, "%d rows > capacity %d", n_rows, d.capacity);
  if (n_rows > 0) {
    if (!k || !v) return fail(KVR_EINVAL, "null k or v");
    if (!aligned16(k) || !aligned16(v))
      return fail(KVR_EINVAL, "k and v must be 16-byte aligned");
    Call call{c->view, seq, 1, 0, d.n_layers};
    Seqs q;
    q.len[0] = q.count[0] = n_rows;
    // one sequence: its stride is never used, so the base stands for sequence seq
    kvr::kv4::RowStrides st{0, (long long)d.n_kv_heads * n_rows * d.head_dim, d.head_dim,
                            (long long)n_rows * d.head_dim};
    const cudaError_t e = kvr::kv4::launch_append(call, q, n_rows, k, v, st,
                                                  static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail("kvr_kv4_load", e);
    c->launches += 1;
  }
  std::fill_n(c->len.begin() + (size_t)seq * d.n_layers, d.n_layers, n_rows);
  return KVR_OK;
}

kvr_status kvr_kv4_append(kvr_kv4 *c, int lb, int le, int n_new, const int32_t *counts,
                          const void *k, const void *v, void *stream) {
  kvr_status st = check_call(c, lb, le, n_new, counts);
  if (st != KVR_OK) return st;
  if (!k || !v) return fail(KVR_EINVAL, "null k or v");
  if (!aligned16(k) || !aligned16(v))
    return fail(KVR_EINVAL, "k and v must be 16-byte aligned");
  const kvr_cache_desc &d = c->desc;
  for (int s = 0; s < d.n_seq; ++s) {
    const int n = c->len[(size_t)s * d.n_layers + lb], more = counts ? counts[s] : n_new;
    if (more > d.capacity - n)
      return fail(KVR_ECAPACITY, "sequence %d: %d rows and %d more > capacity %d", s, n, more,
                  d.capacity);
  }
  const long long dd = d.head_dim;
  const kvr::kv4::RowStrides rs{(le - lb) * n_new * d.n_kv_heads * dd,
                                n_new * d.n_kv_heads * dd, d.n_kv_heads * dd, dd};
  st = each_span(c, lb, le, n_new, counts, 1, [&](const Call &call, const Seqs &q) {
    const cudaError_t e = kvr::kv4::launch_append(call, q, n_new, k, v, rs,
                                                  static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail("kvr_kv4_append", e);
    c->launches += 1;
    return KVR_OK;
  });
  if (st != KVR_OK) return st;
  for (int s = 0; s < d.n_seq; ++s)
    for (int l = lb; l < le; ++l)
      c->len[(size_t)s * d.n_layers + l] += counts ? counts[s] : n_new;
  return KVR_OK;
}

kvr_status kvr_kv4_truncate(kvr_kv4 *c, const int32_t *lens) {
  if (!c || !lens) return fail(KVR_EINVAL, "null cache or lengths");
  const int S = c->desc.n_seq, L = c->desc.n_layers;
  for (int s = 0; s < S; ++s)
    for (int l = 0; l < L; ++l)
      if (lens[s] < 0 || lens[s] > c->len[(size_t)s * L + l])
        return fail(KVR_EINVAL, "sequence %d: %d rows of %d", s, lens[s],
                    c->len[(size_t)s * L + l]);
  for (int s = 0; s < S; ++s) std::fill_n(c->len.begin() + (size_t)s * L, L, lens[s]);
  return KVR_OK;
}

kvr_status kvr_kv4_lengths(const kvr_kv4 *c, int32_t *host_len) {
  if (!c || !host_len) return fail(KVR_EINVAL, "null argument");
  std::copy(c->len.begin(), c->len.end(), host_len);
  return KVR_OK;
}

kvr_status kvr_kv4_read(kvr_kv4 *c, int lb, int le, int n_rows, const int32_t *counts, void *k,
                        void *v, void *stream) {
  kvr_status st = check_call(c, lb, le, n_rows, counts);
  if (st != KVR_OK) return st;
  if (!k || !v) return fail(KVR_EINVAL, "null k or v");
  if (!aligned16(k) || !aligned16(v))
    return fail(KVR_EINVAL, "k and v must be 16-byte aligned");
  for (int s = 0; s < c->desc.n_seq; ++s) {
    const int n = c->len[(size_t)s * c->desc.n_layers + lb], want = counts ? counts[s] : n_rows;
    if (want > n) return fail(KVR_EINVAL, "sequence %d: %d rows of %d", s, want, n);
  }
  return each_span(c, lb, le, n_rows, counts, 0, [&](const Call &call, const Seqs &q) {
    const cudaStream_t cs = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (call.c.io_bf16)
      e = call.c.d == 128 ? kvr::kv4::launch_read<__nv_bfloat16, 128>(call, q, n_rows, k, v, cs)
                          : kvr::kv4::launch_read<__nv_bfloat16, 64>(call, q, n_rows, k, v, cs);
    else
      e = call.c.d == 128 ? kvr::kv4::launch_read<float, 128>(call, q, n_rows, k, v, cs)
                          : kvr::kv4::launch_read<float, 64>(call, q, n_rows, k, v, cs);
    if (e != cudaSuccess) return cuda_fail("kvr_kv4_read", e);
    c->launches += 1;
    return KVR_OK;
  });
}

size_t kvr_kv4_attend_workspace_bytes(const kvr_kv4 *c, int lb, int le, int n_q) {
  if (!c || lb < 0 || le > c->desc.n_layers || lb >= le || n_q < 1 || n_q > (1 << 24)) return 0;
  // Partial results depend on how query rows are tiled, so that fewer tokens may need
  // more of them; there are none above kMaxTiles tiles, of 64 rows at most.
  size_t parts = 0;
  for (int n = std::min(n_q, 64 * kvr::kv4::kMaxTiles); n > 0; --n)
    parts = std::max(parts, kvr::kv4::attend_part_floats(c->view, le - lb, n));
  return bytes_of(c, le - lb, n_q, parts);
}

kvr_status kvr_kv4_attend(kvr_kv4 *c, int lb, int le, int n_q, const int32_t *counts,
                          const void *q, void *out, int add_scores, void *workspace,
                          size_t workspace_bytes, void *stream) {
  kvr_status st = check_call(c, lb, le, n_q, counts);
  if (st != KVR_OK) return st;
  if (!q || !out || !workspace) return fail(KVR_EINVAL, "null q, out or workspace");
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace))
    return fail(KVR_EINVAL, "q, out and workspace must be 16-byte aligned");
  const size_t need = bytes_of(c, le - lb, n_q,
                               kvr::kv4::attend_part_floats(c->view, le - lb, n_q));
  if (workspace_bytes < need)
    return fail(KVR_ENOMEM, "workspace of %zu bytes < required %zu", workspace_bytes, need);
  kvr::kv4::AttendParams p{};
  p.n_q = n_q;
  p.q = q;
  p.out = out;
  float *ws = static_cast<float *>(workspace);
  p.stats = add_scores ? ws : nullptr;
  p.parts = ws + kvr::kv4::attend_stat_floats(c->view, le - lb, n_q);
  return each_span(c, lb, le, n_q, counts, 0, [&](const Call &call, const Seqs &sq) {
    p.k = call;
    int n = 0;
    const cudaError_t e =
        kvr::kv4::launch_attend(p, sq, c->device, static_cast<cudaStream_t>(stream), &n);
    c->launches += n;
    return e == cudaSuccess ? KVR_OK : cuda_fail("kvr_kv4_attend", e);
  });
}

kvr_status kvr_kv4_evict(kvr_kv4 *c, kvr_cache *dst, int budget, int window, void *stream) {
  if (!dst) return fail(KVR_EINVAL, "null destination");
  if (!c) return fail(KVR_EINVAL, "null cache");
  kvr_status st = check_call(c, 0, c->desc.n_layers, 1, nullptr);
  if (st != KVR_OK) return st;
  if (budget < 0 || window < 0 || (long long)budget + window < 1 ||
      (long long)budget + window > (1 << 24))
    return fail(KVR_EINVAL, "bad budget %d / window %d", budget, window);
  const kvr::CacheView &v = kvr::cache_view(dst);
  const View &w = c->view;
  if (v.S != w.S || v.L != w.L || v.H != w.H || v.d != w.d)
    return fail(KVR_EINVAL, "the caches' sequences, layers, KV heads or head_dim differ");
  if (kvr::cache_forked(dst)) return fail(KVR_ESTATE, "the destination has a live fork");
  for (int s = 0; s < w.S; ++s) {
    const int keep = std::min(c->len[(size_t)s * w.L], budget + window);
    if (keep > v.cap)
      return fail(KVR_ECAPACITY, "sequence %d: %d rows > the destination's capacity %d", s, keep,
                  v.cap);
  }
  st = each_span(c, 0, w.L, 1, nullptr, 0, [&](const Call &call, const Seqs &q) {
    const cudaStream_t cs = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (v.kv_bf16)
      e = w.d == 128
              ? kvr::kv4::launch_evict<__nv_bfloat16, 128>(call, q, v, budget, window, cs)
              : kvr::kv4::launch_evict<__nv_bfloat16, 64>(call, q, v, budget, window, cs);
    else
      e = w.d == 128 ? kvr::kv4::launch_evict<float, 128>(call, q, v, budget, window, cs)
                     : kvr::kv4::launch_evict<float, 64>(call, q, v, budget, window, cs);
    if (e != cudaSuccess) return cuda_fail("kvr_kv4_evict", e);
    c->launches += 1;
    return KVR_OK;
  });
  if (st != KVR_OK) return st;
  for (int s = 0; s < w.S; ++s) {
    const int n = c->len[(size_t)s * w.L];
    kvr::cache_set_length(dst, s, std::min(n, budget + window), n);
  }
  return KVR_OK;
}

kvr_status kvr_kv4_scores(const kvr_kv4 *c, float **score, int64_t *row_stride) {
  if (!c) return fail(KVR_EINVAL, "null cache");
  if (score) *score = c->view.score;
  if (row_stride) *row_stride = c->view.sstride;
  return KVR_OK;
}

kvr_status kvr_kv4_launch_count(const kvr_kv4 *c, uint64_t *count) {
  if (!c || !count) return fail(KVR_EINVAL, "null argument");
  *count = c->launches;
  return KVR_OK;
}

kvr_status kvr_kv4_sync_status(kvr_kv4 *c, void *stream) {
  if (!c) return fail(KVR_EINVAL, "null cache");
  // All on the caller's stream: one that does not wait for the default stream would
  // not wait for what is cleared there either.
  const cudaStream_t cs = static_cast<cudaStream_t>(stream);
  unsigned word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, c->view.err, sizeof word, cudaMemcpyDeviceToHost, cs);
  if (e == cudaSuccess) e = cudaStreamSynchronize(cs);
  if (e != cudaSuccess) return cuda_fail("kvr_kv4_sync_status: read", e);
  if (!word) return KVR_OK;
  // The tickets lie ahead of the word, and a launch that gave up a wait may have
  // left some of its arrivals there.
  auto *from = reinterpret_cast<uint8_t *>(c->view.ticket);
  e = cudaMemsetAsync(from, 0, reinterpret_cast<uint8_t *>(c->view.err) + sizeof word - from, cs);
  if (e == cudaSuccess) e = cudaStreamSynchronize(cs);
  if (e != cudaSuccess) return cuda_fail("kvr_kv4_sync_status: clear", e);
  return fail(KVR_EDEVICE, "device error word 0x%x (%s%s%s)", word,
              word & kvr::ERR_NONFINITE ? "non-finite " : "",
              word & kvr::ERR_LENGTH ? "length " : "",
              word & kvr::ERR_TIMEOUT ? "timeout" : "");
}

}  // extern "C"
