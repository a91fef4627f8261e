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

template <typename T>
struct Eight {  // eight channels in memory
  uint4 w[sizeof(T) / 2];
};
__device__ __forceinline__ void widen(const Eight<float> &a, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[4 * i] = __uint_as_float(a.w[i].x), x[4 * i + 1] = __uint_as_float(a.w[i].y);
    x[4 * i + 2] = __uint_as_float(a.w[i].z), x[4 * i + 3] = __uint_as_float(a.w[i].w);
  }
}
__device__ __forceinline__ void widen(const Eight<__nv_bfloat16> &a, float (&x)[8]) {
  const uint32_t w[4] = {a.w[0].x, a.w[0].y, a.w[0].z, a.w[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void narrow(const float (&x)[8], Eight<float> &a) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    a.w[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]),
                        __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
}
__device__ __forceinline__ void narrow(const float (&x)[8], Eight<__nv_bfloat16> &a) {
  a.w[0] = make_uint4(ptx::pack_bf16(x[0], x[1]), ptx::pack_bf16(x[2], x[3]),
                      ptx::pack_bf16(x[4], x[5]), ptx::pack_bf16(x[6], x[7]));
}

// The codes of eight values as one word, code e in bits 4 e .. 4 e + 3.  A product
// with 1 / s finds a code unless it lies within 2e-5 of half-way between two (the
// product is off by less than 2^-21 of 15); those few are divided.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], uint32_t meta, bool flat) {
  const float m = m_of(meta), r = ptx::rcp(s_of(meta));
  uint32_t w = 0;
  float off = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = fminf(fmaxf(__fmul_rn(__fsub_rn(x[e], m), r), 0.f), 15.f);
    const float k = __fadd_rn(q, 12582912.f);  // 1.5 2^23: the code in the low bits
    off = fmaxf(off, fabsf(__fsub_rn(q, __fsub_rn(k, 12582912.f))));
    w |= (__float_as_uint(k) & 15u) << (4 * e);
  }
  // a scale that is nearly subnormal has no reciprocal, and a huge one flushes
  if (off > 0.49998f || !(r < 1e37f && r > 1e-37f)) {
    w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= code_of(x[e], meta, flat) << (4 * e);
  }
  return flat ? 0 : w;
}

// Between a word of eight neighbouring channels' codes of a row and V's halves:
// the four lanes of 32 channels hold channels 8 y .. 8 y + 7, and lane y ends up
// with the halves of c = 2 y (low) and 2 y + 1, whose nibbles are c + {0, 16, 8,
// 24}.  The same exchange takes the halves back.
__device__ __forceinline__ uint32_t to_halves(uint32_t w) {
  const int y = threadIdx.x & 3;
  uint32_t z = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t v = i == 0 ? w : __shfl_xor_sync(0xffffffffu, w, i);
    const int from = y ^ i;  // the lane that v comes from: channels 8 from + c
    const int f = 4 * (((from & 1) << 1) | (from >> 1));
    z |= ((v >> (8 * y)) & 15u) << f;
    z |= ((v >> (8 * y + 4)) & 15u) << (16 + f);
  }
  return z;
}
__device__ __forceinline__ uint32_t from_halves(uint32_t z) {
  const int y = threadIdx.x & 3, f = 4 * (((y & 1) << 1) | (y >> 1));
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t v = i == 0 ? z : __shfl_xor_sync(0xffffffffu, z, i);
    const int from = y ^ i;  // channels c = 2 from, 2 from + 1
    w |= ((v >> f) & 15u) << (8 * from);
    w |= ((v >> (16 + f)) & 15u) << (8 * from + 4);
  }
  return w;
}

// Where a lane that holds channels 8 i .. 8 i + 7 of row r finds or puts them.
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

// Quantise the new rows.  D / 8 lanes a row, eight channels a lane; a warp takes
// kRows rows of one side (key or value) at a time, their loads in flight together.
// Bound by the bytes read and written where tokens are many, else by latency.
template <typename T, int D>
struct Append {
  static constexpr int kLanes = D / 8;             // of a row
  static constexpr int kOnce = 32 / kLanes;        // rows of a warp at once
  static constexpr int kRounds = 4;
  static constexpr int kRows = kOnce * kRounds;    // rows of a warp
};
template <typename T, int D>
__global__ void __launch_bounds__(256)
    append_kernel(const __grid_constant__ Call k, const __grid_constant__ Seqs q, int tokens,
                  const T *key, const T *val, RowStrides st) {
  pdl_begin();
  using A = Append<T, D>;
  const View &c = k.c;
  const int lane = threadIdx.x & 31, i = lane % A::kLanes;
  // a warp: (sequence, layer, head), side, kRows tokens
  const int groups = (tokens + A::kRows - 1) / A::kRows;
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int side = (int)(w & 1);
  const int tg = (int)((w >> 1) % groups);
  const long long unit = (w >> 1) / groups;
  const int h = (int)(unit % c.H), lr = (int)(unit / c.H % k.nl);
  const long long s = unit / c.H / k.nl;
  if (s >= k.n) return;
  const int count = q.count[s], t0 = tg * A::kRows;
  if (t0 >= count) return;
  const T *src = (side ? val : key) + (s + k.s0) * st.seq + lr * st.layer + h * st.head + 8 * i;
  Eight<T> in[A::kRounds];
#pragma unroll
  for (int n = 0; n < A::kRounds; ++n) {
    const int t = min(t0 + n * A::kOnce + lane / A::kLanes, count - 1);
    const uint4 *at = reinterpret_cast<const uint4 *>(src + t * st.token);
#pragma unroll
    for (int e = 0; e < (int)sizeof(T) / 2; ++e) in[n].w[e] = __ldcs(at + e);
  }
  const size_t u = unit_at(c, k.s0 + (int)s, k.lb, lr, h);
  const int r0 = q.len[s] - count;
#pragma unroll
  for (int n = 0; n < A::kRounds; ++n) {
    if (t0 + n * A::kOnce >= count) break;
    const int t = t0 + n * A::kOnce + lane / A::kLanes;
    float x[8];
    widen(in[n], x);
    float lo = x[0], hi = x[0], odd = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo = fminf(lo, x[e]);
      hi = fmaxf(hi, x[e]);
      odd = fmaf(x[e], 0.f, odd);  // NaN for what is not finite
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {  // the eight lanes of a group
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const unsigned bad = __ballot_sync(0xffffffffu, odd != 0.f);
    bool flat;
    const uint32_t meta =
        group_meta(lo, hi, ((bad >> (lane & ~7)) & 255u) == 0, flat);
    uint32_t word = codes_of(x, meta, flat);
    if (side) word = to_halves(word);
    if (t < count) {
      const int r = r0 + t, rb = r % kBlock;
      uint8_t *block = block_at(c, u, r);
      if (side) {
        const int y = i & 3;
        *v_half_at<D>(block, rb, i, 2 * y) = (uint16_t)word;
        *v_half_at<D>(block, rb, i, 2 * y + 1) = (uint16_t)(word >> 16);
      } else {
        *k_word<D>(block, rb, i) = word;
      }
      if (i % 8 == 0) *meta_word<D>(block, side, rb, i) = meta;
      if (side == 0 && i == 0) c.score[u * c.sstride + r] = 0.f;
    }
  }
}

// The codes and (m, s) of channels 8 i .. 8 i + 7 of row r of a block (V's codes
// as halves), and what they stand for.  All lanes call word_values.
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
__device__ __forceinline__ void word_values(const RowWords &a, int side, float (&x)[8]) {
  const uint32_t w = side ? from_halves(a.w) : a.w;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = value_of((w >> (4 * e)) & 15u, a.meta);
}

// What the newest rows stand for: D / 8 lanes a row and side.
template <typename T, int D>
__global__ void __launch_bounds__(256)
    read_kernel(const __grid_constant__ Call k, const __grid_constant__ Seqs q, int rows, T *key,
                T *val) {
  pdl_begin();
  using A = Append<T, D>;
  const View &c = k.c;
  const int lane = threadIdx.x & 31, i = lane % A::kLanes;
  const int groups = (rows + A::kRows - 1) / A::kRows;
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int side = (int)(w & 1);
  const int tg = (int)((w >> 1) % groups);
  const long long unit = (w >> 1) / groups;
  const int h = (int)(unit % c.H), lr = (int)(unit / c.H % k.nl);
  const long long s = unit / c.H / k.nl;
  if (s >= k.n) return;
  const int count = q.count[s], r0 = q.len[s] - count;
  const size_t u = unit_at(c, k.s0 + (int)s, k.lb, lr, h);
  T *to = (side ? val : key) +
          (((size_t)(s + k.s0) * k.nl + lr) * c.H + h) * rows * D + 8 * i;
  RowWords words[A::kRounds];
#pragma unroll
  for (int n = 0; n < A::kRounds; ++n) {
    const int r = r0 + min(tg * A::kRows + n * A::kOnce + lane / A::kLanes, count - 1);
    words[n] = RowWords{0, 0};
    if (count > 0) words[n] = row_words<D>(block_at(c, u, r), side, r % kBlock, i);
  }
#pragma unroll
  for (int n = 0; n < A::kRounds; ++n) {
    const int t = tg * A::kRows + n * A::kOnce + lane / A::kLanes;
    float x[8];
    word_values(words[n], side, x);
    if (t >= count)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
    Eight<T> o;
    narrow(x, o);
    if (t < rows)
#pragma unroll
      for (int e = 0; e < (int)sizeof(T) / 2; ++e)
        __stcs(reinterpret_cast<uint4 *>(to + (size_t)t * D) + e, o.w[e]);
  }
}

// A score's rank, higher first: -0 counts as 0, and every NaN as one above every
// number.
__device__ __forceinline__ uint32_t score_rank(float x) {
  const uint32_t b = __float_as_uint(x), a = b & 0x7FFFFFFFu;
  return a > 0x7F800000u ? 0xFFFFFFFFu : a == 0 ? 0x80000000u : b != a ? ~b : (b | 0x80000000u);
}

// Cut a unit into dst: one CTA a unit, whose scores' ranks lie in shared memory
// (or are formed from the scores anew, where a unit has too many rows).  Four
// passes of eight bits find the rank of the budget-th row before the window, with
// a histogram a warp; of the rows of that rank the first ones are kept.  The kept
// rows are listed in order, in dst's positions, and their values written from
// there, D / 8 lanes a row and side.
constexpr int kEvictThreads = 1024;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictHists = 8;  // histograms: one for every four warps
constexpr int kEvictSmemRows = 24576;

template <typename T, int D, bool IN_SMEM>
__global__ void __launch_bounds__(kEvictThreads)
    evict_kernel(const __grid_constant__ Call k, const __grid_constant__ Seqs q,
                 const __grid_constant__ CacheView dst, int budget, int window) {
  extern __shared__ uint32_t s_rank[];
  __shared__ unsigned s_hist[kEvictHists][256];
  __shared__ int s_count[kEvictWarps], s_ties[kEvictWarps];
  __shared__ unsigned s_digit, s_need;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_begin();
  const View &c = k.c;
  const int h = blockIdx.x % c.H, l = blockIdx.x / c.H, s = blockIdx.y;
  const size_t u = unit_at(c, k.s0 + s, 0, l, h);
  const float *score = c.score + u * c.sstride;
  const int n = q.len[s], first = max(0, n - window);  // rows [first, n): the window
  const int keep = min(n, budget + window);
  const bool cut = first > budget;
  if (IN_SMEM && cut) {
    // rows of 16 floats start on 64 bytes, so whole vectors are within the row
    for (int i = tid; 4 * i < first; i += kEvictThreads) {
      const float4 x = __ldg(reinterpret_cast<const float4 *>(score) + i);
      *reinterpret_cast<uint4 *>(s_rank + 4 * i) =
          make_uint4(score_rank(x.x), score_rank(x.y), score_rank(x.z), score_rank(x.w));
    }
  }
  auto rank = [&](int i) { return IN_SMEM ? s_rank[i] : score_rank(score[i]); };
  // The rank of the last row kept, and how many rows of that rank are kept.
  uint32_t least = 0, mask = 0;
  int need = budget;
  if (cut && budget > 0) {
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < kEvictHists * 256; i += kEvictThreads) (&s_hist[0][0])[i] = 0;
      __syncthreads();
      unsigned *hist = s_hist[warp % kEvictHists];
      for (int i = tid; i < first; i += kEvictThreads) {
        const uint32_t x = rank(i);
        if ((x & mask) == least) atomicAdd(&hist[(x >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (warp == 0) {
        // lane j: digits 255 - 8 j .. 248 - 8 j, counted from the top
        unsigned d[8], sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          d[e] = 0;
#pragma unroll
          for (int z = 0; z < kEvictHists; ++z) d[e] += s_hist[z][255 - 8 * lane - e];
          sum += d[e];
        }
        unsigned above = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned x = __shfl_up_sync(0xffffffffu, above, o);
          if (lane >= o) above += x;
        }
        above -= sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (above < (unsigned)need && above + d[e] >= (unsigned)need) {
            s_digit = 255 - 8 * lane - e;
            s_need = need - above;
          }
          above += d[e];
        }
      }
      __syncthreads();
      least |= s_digit << shift;
      need = s_need;
      mask |= 255u << shift;
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
  overs = __reduce_add_sync(0xffffffffu, lane < warp ? s_count[lane] : 0);
  ties = __reduce_add_sync(0xffffffffu, lane < warp ? s_ties[lane] : 0);
  for (int b = i0; b < i1; b += 32) {
    unsigned over, tie;
    look(b + lane, over, tie);
    const int tied = ties + __popc(tie & lower);
    const bool kept = (over >> lane & 1u) || ((tie >> lane & 1u) && tied < need);
    const int at = overs + __popc(over & lower) + min(tied, need);
    if (kept && at < keep) {
      pos[at] = b + lane;
      to_score[at] = score[b + lane];
    }
    overs += __popc(over);
    ties += __popc(tie);
  }
  if (tid == kEvictThreads - 1 && overs + min(ties, need) != keep && cut)
    atomicOr(c.err, ERR_LENGTH);
  __syncthreads();
  // Their values: D / 8 lanes a row, kBatch rows of each in flight.
  constexpr int kLanes = D / 8, kOnce = 32 / kLanes, kBatch = 4;
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
      float x[8];
      Eight<T> o;
      const size_t to = (u * (size_t)dst.cap + j) * D + 8 * ch;
      word_values(kw[e], 0, x);
      narrow(x, o);
      if (j < m)
#pragma unroll
        for (int z = 0; z < (int)sizeof(T) / 2; ++z)
          reinterpret_cast<uint4 *>(static_cast<T *>(dst.K) + to)[z] = o.w[z];
      word_values(vw[e], 1, x);
      narrow(x, o);
      if (j < m)
#pragma unroll
        for (int z = 0; z < (int)sizeof(T) / 2; ++z)
          reinterpret_cast<uint4 *>(static_cast<T *>(dst.V) + to)[z] = o.w[z];
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
bool row_grid(const Call &k, int rows, dim3 *grid) {
  constexpr int kRows = Append<T, D>::kRows;
  const long long warps = 2ll * k.n * k.nl * k.c.H * ((rows + kRows - 1) / kRows);
  *grid = dim3((unsigned)((warps + 7) / 8));
  return (warps + 7) / 8 <= INT32_MAX;
}
template <typename T, int D>
cudaError_t launch_read(const Call &k, const Seqs &q, int rows, void *key, void *val,
                        cudaStream_t stream) {
  dim3 grid;
  if (!row_grid<T, D>(k, rows, &grid)) return cudaErrorInvalidValue;
  return launch_pdl(read_kernel<T, D>, grid, dim3(256), 0, stream, k, q, rows,
                    static_cast<T *>(key), static_cast<T *>(val));
}

template <typename T, int D>
cudaError_t launch_append_as(const Call &k, const Seqs &q, int tokens, const void *key,
                             const void *val, const RowStrides &st, cudaStream_t stream) {
  dim3 grid;
  if (!row_grid<T, D>(k, tokens, &grid)) return cudaErrorInvalidValue;
  return launch_pdl(append_kernel<T, D>, grid, dim3(256), 0, stream, k, q, tokens,
                    static_cast<const T *>(key), static_cast<const T *>(val), st);
}

template <typename T, int D>
cudaError_t launch_evict(const Call &k, const Seqs &q, const CacheView &dst, int budget,
                         int window, cudaStream_t stream) {
  int most = 0;
  for (int i = 0; i < k.n; ++i) most = std::max(most, q.len[i] - window);
  const dim3 grid(k.c.L * k.c.H, k.n);
  if (most > kEvictSmemRows)
    return launch_pdl(evict_kernel<T, D, false>, grid, dim3(kEvictThreads), 0, stream, k, q, dst,
                      budget, window);
  auto kern = evict_kernel<T, D, true>;
  static bool ready = false;
  if (!ready) {
    const cudaError_t e = cudaFuncSetAttribute(
        kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kEvictSmemRows * 4);
    if (e != cudaSuccess) return e;
    ready = true;
  }
  const int bytes = most > budget ? round_up16(most) * 4 : 0;
  return launch_pdl(kern, grid, dim3(kEvictThreads), bytes, stream, k, q, dst, budget, window);
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
  // scores, tickets and the error word lie side by side
  const cudaError_t e = cudaMemsetAsync(b + l.score, 0, l.total - l.score,
                                        static_cast<cudaStream_t>(stream));
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
  return std::max<size_t>(16, (kvr::kv4::attend_stat_floats(c->view, le - lb, n_q) +
                               kvr::kv4::attend_part_floats(c->view, le - lb, n_q)) *
                                  sizeof(float));
}

kvr_status kvr_kv4_attend(kvr_kv4 *c, int lb, int le, int n_q, const int32_t *counts,
                          const void *q, void *out, int add_scores, void *workspace,
                          size_t workspace_bytes, void *stream) {
  kvr_status st = check_call(c, lb, le, n_q, counts);
  if (st != KVR_OK) return st;
  if (!q || !out || !workspace) return fail(KVR_EINVAL, "null q, out or workspace");
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace))
    return fail(KVR_EINVAL, "q, out and workspace must be 16-byte aligned");
  const size_t need = kvr_kv4_attend_workspace_bytes(c, lb, le, n_q);
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
        kvr::kv4::launch_attend(p, sq, static_cast<cudaStream_t>(stream), &n);
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
  cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail("kvr_kv4_sync_status: sync", e);
  unsigned word = 0;
  e = cudaMemcpy(&word, c->view.err, sizeof word, cudaMemcpyDeviceToHost);
  if (e != cudaSuccess) return cuda_fail("kvr_kv4_sync_status: read", e);
  if (!word) return KVR_OK;
  e = cudaMemset(c->view.err, 0, sizeof word);
  if (e != cudaSuccess) return cuda_fail("kvr_kv4_sync_status: clear", e);
  return fail(KVR_EDEVICE, "device error word 0x%x (%s%s%s)", word,
              word & kvr::ERR_NONFINITE ? "non-finite " : "",
              word & kvr::ERR_LENGTH ? "length " : "",
              word & kvr::ERR_TIMEOUT ? "timeout" : "");
}

}  // extern "C"
