// kvr_kv4_attend.cu -- attention over the 4-bit cache (kvr_kv4.cuh has its
// layout).
//
// A unit's query rows (token, head of the group) are the columns of two small
// matrix products per 16 cached tokens on warp-level tensor cores:
//   S  [tokens x columns]  = K [tokens x d] Q^T
//   O^T [d x columns]     += V^T [d x tokens] P^T
// with the 4-bit codes as the A operand of both.  A code needs no conversion: a
// masked nibble in a 16-bit half is the half-precision subnormal c 2^-24 (or
// c 2^-20, one nibble up), which tensor cores multiply exactly; the powers of two
// are taken up by q and by the epilogue.  The group's (m, s) enter outside the
// product, in fp32:
//   q . k = sum over groups of  s (c . q) + m sum(q)
//   p . v = sum over tokens of  (p s) c + p m
// so K's logits are formed from a product per group, and V's probabilities are
// multiplied by s before they are rounded to 16 bits, w = half(p s).  With bf16
// tensors the second term is w (m / s), so that a token's channels all have the
// weight w / s and what the rounding costs is to scale with its values; with
// fp32 tensors q and p s have two 16-bit terms, the second term is p m, and codes
// are converted and count from 8 (m + 8 s in the place of m), so that sums do not
// cancel.
//
// Rows stream through a ring of bulk copies for each warp, one 32-token block
// (4,608 B at d = 128) a copy.  Units are cut into equal pieces of at most four
// blocks, and the list of all pieces into equal spans, one a CTA, so that lengths
// of any mix fill the GPU; a unit that spans share is joined by the last of them
// to finish, in order of the spans, so that results do not depend on scheduling.
//
// Bound by the bytes of the cache where it is long: one token of 16 sequences of
// 16,384 rows (28 layers, 2 KV heads, G = 6) 380 us, 5.6 TB/s.  Small calls are bound
// by latency: a layer of one sequence of 4,099 rows (4 KV heads, G = 7) 10.6 us, and
// a call from Python takes the host about as long.
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "kvr_device.cuh"
#include "kvr_internal.h"
#include "kvr_kv4.cuh"
#include "kvr_kv4_attend.cuh"
#include "kvr_ptx.cuh"

namespace kvr {
namespace kv4 {
namespace {

using namespace ptx;

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kStages = 2;      // blocks in flight a warp
constexpr int kMinSpan = 3;     // pieces of a span, at least (2 to 4: within 3% for 28 small calls)
// Pieces that a turn to another item is worth: a call is cut into parts rather than
// spans where these are at most as much longer (28 calls of a layer each, one
// sequence of 4,099 rows, on the GPU: 293 us in parts, 381 in spans).
constexpr int kTurn = 3;
constexpr int kMaxGrid = 1024;  // CTAs of a split call, at most

// How a launch is cut.  An item (unit, tile of query rows) of sequence s has
// pieces_of(blocks_of(s)) pieces.
//  kSpans: all pieces form one list, and a CTA takes `span` of them, whatever
//    items they belong to; base[s] pieces precede sequence s.
//  kParts: an item is cut into as few equal parts as keep each within `span`
//    pieces, and a CTA takes one; base[s] parts precede sequence s.  No CTA turns
//    from one item to another, which costs as much as a few pieces.
//  kItems: a CTA takes an item.
enum Cut { kSpans, kParts, kItems };
struct Plan {
  int32_t base[kMaxSeqs + 1];
  int32_t cut, span, tiles;
};

__host__ __device__ inline int pieces_of(int nb) { return (nb + kPiece - 1) / kPiece; }
__host__ __device__ inline int parts_of(int np, int span) { return (np + span - 1) / span; }
// First block of piece i of np.
// (nb is at most 2^19, so np * nb fits 36 bits: where it does not fit 32, in 64.)
__device__ __forceinline__ int piece_at(int nb, int np, int i) {
  if (nb > 65535) return (int)((long long)i * nb / np);
  return (int)((unsigned)i * (unsigned)nb / (unsigned)np);
}

// A run of blocks [begin, end) of one item, which are pieces [piece, piece + n).
struct Run {
  int s, item;        // sequence of the launch, item of the sequence
  int begin, end, nb; // nb: all blocks of the item
  int n;
  int at;             // list index of the first piece
};

template <int D, int NT>
struct Smem {
  static constexpr int kCols = 8 * NT;
  static constexpr int kRow = D + 4;  // floats of an exchanged column
  static constexpr int kRing = kWarps * kStages * block_bytes(D);
  // sums of the warps, (maximum, normaliser) of them and of all, their factors
  static constexpr int kExch = kWarps * kCols * (kRow + 2) * 4 + kCols * 8 + kWarps * kCols * 4;
  static constexpr int kBars = kRing + kExch;
  static constexpr int kTable = kBars + kWarps * kStages * 8 + 16;
  static constexpr int kBytes = kTable + kCols * 16;
};

// The forms of K and V.
__host__ __device__ constexpr Codes k_codes(int terms) { return terms == 2 ? kCentred : kRough; }
__host__ __device__ constexpr Codes v_codes(int terms) { return terms == 2 ? kCentred : kEven; }

template <int W>
__device__ __forceinline__ void lds_words(uint32_t at, uint32_t (&x)[W]) {
  if (W == 4)
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2 % W]), "=r"(x[3 % W])
                 : "r"(at));
  else
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(at));
}
template <int N>
__device__ __forceinline__ void lds_meta(uint32_t at, uint32_t (&x)[N]) {
  if (N == 2)
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(x[0]), "=r"(x[1 % N]) : "r"(at));
  else
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x[0]) : "r"(at));
}

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack_half(uint32_t x) {
  return __half22float2(*reinterpret_cast<const __half2 *>(&x));
}

// A warp's query columns as B fragments.  TERMS == 2: the second holds what
// rounding to 16 bits left of the first.
template <int D, int NT, int TERMS>
struct Query {
  uint32_t f[NT][TERMS][D / 16][2];
  float sum[NT][D / kGroup][2];  // of the lane's two columns: sum of q, scaled as f
  float unit[NT][2];             // what a scaled product is to be multiplied by
  int limit[NT][2];              // last row that the column sees, or -1
};

template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4 *>(p)[0];
  const float4 b = reinterpret_cast<const float4 *>(p)[1];
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
  x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
template <>
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float (&x)[8]) {
  const uint4 a = *reinterpret_cast<const uint4 *>(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// q's columns [col0, col0 + 8 NT) of a unit.  Each column is scaled by a power of
// two that puts its largest value in [2^14, 2^15): exact, and a 16-bit half then
// holds all that matters of a bf16 value.
template <typename T, Codes M, int D, int NT, int TERMS>
__device__ __forceinline__ void load_query(Query<D, NT, TERMS> &q, const AttendParams &p,
                                           const Seqs &sq, int s, int lr, int h, int col0) {
  const View &c = p.k.c;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int count = sq.count[s], before = sq.len[s] - count;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int col = col0 + 8 * n + g, tok = col / c.G;
    // (a token that the sequence has not may hold anything: its columns are zeros)
    const bool live = tok < count;
    const T *src = static_cast<const T *>(p.q) +
                   (((((size_t)(p.k.s0 + s) * p.k.nl + lr) * p.n_q + tok) * c.H + h) * c.G +
                    (col - tok * c.G)) *
                       D;
    float x[D / 32][8], top = 0.f;
    bool fine = true;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
      if (live)
        load8<T>(src + 64 * (w >> 1) + 16 * t + 8 * (w & 1), x[w]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) x[w][e] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        top = fmaxf(top, fabsf(x[w][e]));
        fine &= isfinite(x[w][e]);
      }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const unsigned bad = __ballot_sync(0xffffffffu, !fine);
    fine = ((bad >> (lane & ~3)) & 15u) == 0;
    int k = 14 - ((int)(__float_as_uint(top) >> 23) - 127);
    k = top == 0.f || !fine ? 0 : max(-90, min(k, 100));
    const float up = __uint_as_float((unsigned)(127 + k) << 23);
    float sum[D / kGroup] = {};
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[w][e] *= up;
        sum[w >> 1] += x[w][e];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        // the odd nibbles stand for 2^4 times their code
        const float f = M == kRough && e == 1 ? 0.0625f : 1.f;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float lo = x[w][2 * b + e] * f, hi = x[w][2 * b + 4 + e] * f;
          uint32_t y = pack_half(lo, hi);
          q.f[n][0][2 * w + e][b] = y;
          if (TERMS == 2) {
            const float2 z = unpack_half(y);
            q.f[n][TERMS - 1][2 * w + e][b] = pack_half(lo - z.x, hi - z.y);
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < D / kGroup; ++j) {
      sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 1);
      sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 2);
      sum[j] *= 1.f / field_unit(M);
    }
    const float unit =
        field_unit(M) * __uint_as_float((unsigned)(127 - k) << 23) * (c.scale * kLog2e);
    const int limit = live ? before + tok : -1;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int from = 8 * t + 4 * e;  // a lane of column 2 t + e
#pragma unroll
      for (int j = 0; j < D / kGroup; ++j)
        q.sum[n][j][e] = __shfl_sync(0xffffffffu, sum[j], from);
      q.unit[n][e] = __shfl_sync(0xffffffffu, unit, from);
      q.limit[n][e] = __shfl_sync(0xffffffffu, limit, from);
    }
  }
}

// A token's (m, s) as the products take them: with centred codes m stands for
// code 8.  `gone`: the token does not exist.
template <bool CENTRED>
__device__ __forceinline__ void meta_of(uint32_t w, bool gone, float &m, float &s) {
  if (gone) w = 0;
  m = m_of(w);
  s = s_of(w);
  if (CENTRED) m = fmaf(8.f, s, m);
}

// The logits (base 2) of a block's 32 tokens: l[tile][n][0, 1]: token g of the
// 16-token tile, columns 2 t and 2 t + 1; [2, 3]: token g + 8.
template <Codes M, int D, int NT, int TERMS, bool MASK>
__device__ __forceinline__ void block_logits(const Query<D, NT, TERMS> &q, uint32_t block,
                                             int row0, int len, float (&l)[2][NT][4]) {
  constexpr int W = D / 32, GR = D / kGroup;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int r = 16 * tt + g;
    uint32_t x[W], y[W], mx[GR], my[GR];
    lds_words<W>(block + k_off() + r * (D / 2) + k_chunk(r, t) * (D / 8), x);
    lds_words<W>(block + k_off() + (r + 8) * (D / 2) + k_chunk(r + 8, t) * (D / 8), y);
    lds_meta<GR>(block + km_off(D) + r * GR * 4, mx);
    lds_meta<GR>(block + km_off(D) + (r + 8) * GR * 4, my);
    float acc[NT][GR][4] = {};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      uint32_t a[4], b[4];
      fields<M>(x[w], a);
      fields<M>(y[w], b);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int z = 0; z < TERMS; ++z) {
          mma_f16(acc[n][w >> 1], a[0], b[0], a[2], b[2], q.f[n][z][2 * w][0],
                  q.f[n][z][2 * w][1]);
          mma_f16(acc[n][w >> 1], a[1], b[1], a[3], b[3], q.f[n][z][2 * w + 1][0],
                  q.f[n][z][2 * w + 1][1]);
        }
    }
    float m[2][GR], sc[2][GR];
#pragma unroll
    for (int j = 0; j < GR; ++j) {
      meta_of<M == kCentred>(mx[j], MASK && row0 + r >= len, m[0][j], sc[0][j]);
      meta_of<M == kCentred>(my[j], MASK && row0 + r + 8 >= len, m[1][j], sc[1][j]);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v = 0.f;
#pragma unroll
        for (int j = 0; j < GR; ++j) {
          v = j == 0 ? m[i >> 1][j] * q.sum[n][j][i & 1]
                     : fmaf(m[i >> 1][j], q.sum[n][j][i & 1], v);
          v = fmaf(sc[i >> 1][j], acc[n][j][i], v);
        }
        v *= q.unit[n][i & 1];
        if (MASK && row0 + r + 8 * (i >> 1) > q.limit[n][i & 1]) v = -INFINITY;
        l[tt][n][i] = v;
      }
  }
}

// A warp's running result: columns 2 t, 2 t + 1 of each 8.
template <int D, int NT, int TERMS>
struct State {
  float o[NT][D / 16][4];        // channels 16 i + g, + 8; scaled by 2^(6 - ref)
  float bias[NT][D / kGroup][2]; // the lane's share of what the codes leave out
  float top[NT][2], z[NT][2];
  float ref;                     // 2^(6 - e), e the exponent of the largest scale of V
  float back;                    // 1 / ref
  uint32_t most;                 // scales up to these bits fit that ref
};

template <int D, int NT, int TERMS>
__device__ __forceinline__ void clear(State<D, NT, TERMS> &a) {
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) a.o[n][i][e] = 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      a.top[n][e] = kNone;
      a.z[n][e] = 0.f;
#pragma unroll
      for (int j = 0; j < D / kGroup; ++j) a.bias[n][j][e] = 0.f;
    }
  }
  a.ref = a.back = 1.f;
  a.most = 0;
}

// One block: logits, their exponentials against a running maximum that may lag by
// 2^8 (p s is scaled so that a half holds it all the same), and V's product.
template <int D, int NT, int TERMS, bool MASK>
__device__ __forceinline__ void block_step(State<D, NT, TERMS> &a, const Query<D, NT, TERMS> &q,
                                           uint32_t block, int row0, int len) {
  constexpr Codes kV = v_codes(TERMS);
  constexpr int W = D / 32, GR = D / kGroup;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  float l[2][NT][4];
  block_logits<k_codes(TERMS), D, NT, TERMS, MASK>(q, block, row0, len, l);

  uint32_t vm[2][2][GR];
  uint32_t scale = 0;
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int r = 16 * tt + g + 8 * b;
      lds_meta<GR>(block + vm_off(D) + r * GR * 4, vm[tt][b]);
#pragma unroll
      for (int j = 0; j < GR; ++j) {
        if (MASK && row0 + r >= len) vm[tt][b][j] = 0;
        scale = max(scale, vm[tt][b][j] & 0xFFFF0000u);
      }
    }
  bool grow = scale > a.most;
  float best[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      best[n][e] = fmaxf(fmaxf(l[0][n][e], l[0][n][2 + e]), fmaxf(l[1][n][e], l[1][n][2 + e]));
      grow |= best[n][e] > a.top[n][e] + 8.f;
    }
  if (__any_sync(0xffffffffu, grow)) {
    scale = __reduce_max_sync(0xffffffffu, scale);
    float shrink = 1.f;
    if (scale > a.most) {
      const int e = max((int)(scale >> 23) - 127, -110);
      const float ref = __uint_as_float((unsigned)(127 + 6 - e) << 23);
      shrink = a.most ? ref / a.ref : 0.f;
      a.ref = ref;
      a.back = __uint_as_float((unsigned)(127 - 6 + e) << 23);
      a.most = ((unsigned)(127 + e) << 23) | 0x007FFFFFu;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = best[n][e];
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
        x = fmaxf(x, a.top[n][e]);
        const float f = ex2(a.top[n][e] - x);
        a.top[n][e] = x;
        a.z[n][e] *= f;
#pragma unroll
        for (int j = 0; j < GR; ++j) a.bias[n][j][e] *= f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          a.o[n][i][e] *= f * shrink;
          a.o[n][i][2 + e] *= f * shrink;
        }
      }
  }

  // P^T, times s, as B fragments
  uint32_t pf[2][NT][GR][TERMS][2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      float m[GR], sc[GR];
#pragma unroll
      for (int j = 0; j < GR; ++j) {
        meta_of<kV == kCentred>(vm[tt][b][j], false, m[j], sc[j]);
        // m / s over what has been held against a.ref: a step that is subnormal itself
        // has no reciprocal, 2^116 times it has.  Below 2^-126, half precision leaves
        // nothing of p s, and any finite number will do.
        sc[j] *= a.ref;
        if (TERMS == 1) m[j] *= rcp(fmaxf(sc[j], 0x1p-126f));
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float pr[2];
        bool hidden[2];  // a hidden row's m may be NaN
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float x = l[tt][n][2 * b + e];
          hidden[e] = MASK && x == -INFINITY;
          pr[e] = ex2(x - a.top[n][e]);
          a.z[n][e] += pr[e];
        }
#pragma unroll
        for (int j = 0; j < GR; ++j) {
          const float x = pr[0] * sc[j], y = pr[1] * sc[j];
          const uint32_t w = pack_half(x, y);
          pf[tt][n][j][0][b] = movm_t(w);
          const float2 z = unpack_half(w);
          if (TERMS == 2) pf[tt][n][j][TERMS - 1][b] = movm_t(pack_half(x - z.x, y - z.y));
          a.bias[n][j][0] =
              fmaf(TERMS == 2 ? pr[0] : z.x, hidden[0] ? 0.f : m[j], a.bias[n][j][0]);
          a.bias[n][j][1] =
              fmaf(TERMS == 2 ? pr[1] : z.y, hidden[1] ? 0.f : m[j], a.bias[n][j][1]);
        }
      }
    }

  // V's product.  A block's sum is formed from zero and added in fp32: the tensor
  // core's accumulator rounds towards zero, which over a long context would
  // drift.
  uint32_t v[2][2][W];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int pr = 8 * tt + t + 4 * b;
      lds_words<W>(block + v_off(D) + pr * D + v_chunk<D>(pr, g) * (D / 8), v[tt][b]);
    }
#pragma unroll
  for (int w = 0; w < W; ++w) {
    uint32_t x[2][2][4];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int b = 0; b < 2; ++b) fields<kV>(v[tt][b][w], x[tt][b]);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float sum[4] = {};
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int z = 0; z < TERMS; ++z)
            mma_f16(sum, x[tt][0][i], x[tt][0][2 + i], x[tt][1][i], x[tt][1][2 + i],
                    pf[tt][n][w >> 1][z][0], pf[tt][n][w >> 1][z][1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) a.o[n][2 * w + i][e] += sum[e];
      }
  }
}

template <typename T, typename O, int D, int NT, int TERMS>
__global__ void __launch_bounds__(kThreads, NT * TERMS == 1 ? 4 : 2)
    attend_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ Seqs sq,
                  const __grid_constant__ Plan plan) {
  using S = Smem<D, NT>;
  constexpr int kCols = S::kCols, GR = D / kGroup;
  constexpr uint32_t kBytes = block_bytes(D);
  extern __shared__ __align__(128) uint8_t smem[];
  float *exch = reinterpret_cast<float *>(smem + S::kRing);  // [warp][col][kRow]
  float *stat = exch + kWarps * kCols * S::kRow;             // [warp][col][2]
  float2 *col_stat = reinterpret_cast<float2 *>(stat + kWarps * kCols * 2);
  float *factor = reinterpret_cast<float *>(col_stat + kCols);
  int *flag = reinterpret_cast<int *>(smem + S::kBars + kWarps * kStages * 8);
  Place *place = reinterpret_cast<Place *>(smem + S::kTable);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t ring = smem_u32(smem) + warp * kStages * kBytes;
  const uint32_t bars = smem_u32(smem) + S::kBars + warp * kStages * 8;
  volatile int *abort = flag + 1;
  const View &c = p.k.c;
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(bars + 8 * i, 1);
    fence_mbar_init();
  }
  if (threadIdx.x == 0) flag[1] = 0;
  __syncthreads();

  const int per_seq = p.k.nl * c.H * plan.tiles;
  int last;  // list index behind the CTA's last piece
  Run run;
  if (plan.cut != kItems) {
    run.at = plan.cut == kSpans ? (int)blockIdx.x * plan.span : (int)blockIdx.x;
    last = min(run.at + plan.span, plan.base[p.k.n]);
    int lo = 0, hi = p.k.n;  // the sequence that holds run.at
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.base[mid] <= run.at) lo = mid; else hi = mid;
    }
    run.s = lo;
    run.nb = blocks_of(sq.len[lo]);
    const int np = pieces_of(run.nb);
    const int rest = run.at - plan.base[lo];
    if (plan.cut == kSpans) {
      run.item = rest / np;
      const int piece = rest - run.item * np;
      run.n = min(np - piece, last - run.at);
      run.begin = piece_at(run.nb, np, piece);
      run.end = piece_at(run.nb, np, piece + run.n);
    } else {
      const int parts = parts_of(np, plan.span);
      run.item = rest / parts;
      const int part = rest - run.item * parts;
      run.begin = piece_at(run.nb, np, piece_at(np, parts, part));
      run.end = piece_at(run.nb, np, piece_at(np, parts, part + 1));
      run.n = 1;
      last = run.at + 1;
    }
  } else {
    run.s = blockIdx.x / per_seq;
    run.item = blockIdx.x - run.s * per_seq;
    // no block past the last row that the tile's last token sees
    const int tok = min(sq.count[run.s], ((run.item % plan.tiles + 1) * kCols - 1) / c.G + 1);
    run.nb = blocks_of(sq.len[run.s] - sq.count[run.s] + tok);
    run.begin = 0;
    run.end = run.nb;
    run.at = 0;
    run.n = 1;
    last = 1;
  }
  // The run behind r; false at the end of the span.
  auto next_run = [&](Run &r) {
    r.at += r.n;
    if (r.at >= last) return false;
    if (++r.item == per_seq) {
      r.item = 0;
      ++r.s;
      r.nb = blocks_of(sq.len[r.s]);
    }
    const int np = pieces_of(r.nb);
    r.n = min(np, last - r.at);
    r.begin = 0;
    r.end = piece_at(r.nb, np, r.n);
    return true;
  };
  auto unit_of = [&](const Run &r) {
    const int unit = r.item / plan.tiles;
    return unit_at(c, p.k.s0 + r.s, p.k.lb, unit / c.H, unit % c.H);
  };

  // The warp's blocks: every fourth of each run.  `ahead` runs before the
  // consumer by up to kStages blocks.
  Run ahead = run;
  int ahead_blk = run.begin + warp;
  bool more = true;
  const uint8_t *ahead_at = c.blocks + unit_of(ahead) * c.nb * (size_t)kBytes;
  int issued = 0, taken = 0;
  auto issue = [&]() {
    while (more && ahead_blk >= ahead.end) {
      more = next_run(ahead);
      if (more) {
        ahead_blk = ahead.begin + warp;
        ahead_at = c.blocks + unit_of(ahead) * c.nb * (size_t)kBytes;
      }
    }
    if (!more) return;
    if (lane == 0) {
      const uint32_t bar = bars + 8 * (issued % kStages);
      mbar_expect_tx(bar, kBytes);
      bulk_load(ring + (issued % kStages) * kBytes, ahead_at + (size_t)ahead_blk * kBytes,
                kBytes, bar);
    }
    ++issued;
    ahead_blk += kWarps;
  };
  // Nothing before this read what earlier launches write.
  pdl_begin();
  for (int i = 0; i < kStages; ++i) issue();

  bool ok = true;
  do {
    const int unit = run.item / plan.tiles, tile = run.item % plan.tiles;
    const int lr = unit / c.H, h = unit % c.H, col0 = tile * kCols;
    const int len = sq.len[run.s];
    if (threadIdx.x < kCols)
      place[threadIdx.x] = place_of(p, sq, run.s, lr, h, col0 + threadIdx.x);
    Query<D, NT, TERMS> q;
    load_query<T, k_codes(TERMS)>(q, p, sq, run.s, lr, h, col0);
    State<D, NT, TERMS> a;
    clear(a);
    // rows below `full` are seen by every column that has a token
    const int first = col0 / c.G;
    const int full = first < sq.count[run.s] ? len - sq.count[run.s] + first + 1 : len;
    for (int blk = run.begin + warp; blk < run.end; blk += kWarps) {
      if (ok) {
        ok = warp_wait(bars + 8 * (taken % kStages), (taken / kStages) & 1, abort);
        if (!ok && lane == 0) {
          atomicOr(c.err, ERR_TIMEOUT);
          *abort = 1;
        }
      }
      if (!ok) break;
      const uint32_t at = ring + (taken % kStages) * kBytes;
      const int row0 = blk * kBlock;
      if (row0 + kBlock <= full)
        block_step<D, NT, TERMS, false>(a, q, at, row0, len);
      else
        block_step<D, NT, TERMS, true>(a, q, at, row0, len);
      ++taken;
      __syncwarp();
      issue();
    }
    // Join the warps.
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          a.z[n][e] += __shfl_xor_sync(0xffffffffu, a.z[n][e], o);
#pragma unroll
          for (int j = 0; j < GR; ++j)
            a.bias[n][j][e] += __shfl_xor_sync(0xffffffffu, a.bias[n][j][e], o);
        }
        const int col = 8 * n + 2 * t + e;
        float *to = exch + (warp * kCols + col) * S::kRow;
        const float f = field_unit(v_codes(TERMS)) * a.back;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          to[16 * i + g] = fmaf(a.o[n][i][e], f, a.bias[n][i >> 2][e]);
          to[16 * i + g + 8] = fmaf(a.o[n][i][2 + e], f, a.bias[n][i >> 2][e]);
        }
        if (g == 0) {
          stat[(warp * kCols + col) * 2] = a.top[n][e];
          stat[(warp * kCols + col) * 2 + 1] = a.z[n][e];
        }
      }
    __syncthreads();
    const bool whole = run.end - run.begin == run.nb;
    // Each column's maximum and normaliser over the warps, and the warps' factors;
    // stat[0 .. kCols) then holds (maximum, normaliser), factor[warp][column].
    float2 joined = make_float2(kNone, 0.f);
    if (threadIdx.x < kCols) {
      const float2 *of = reinterpret_cast<const float2 *>(stat) + threadIdx.x;
      float2 x[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        x[w] = of[w * kCols];
        joined.x = fmaxf(joined.x, x[w].x);
      }
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        x[w].x = ex2(x[w].x - joined.x);
        joined.y = fmaf(x[w].y, x[w].x, joined.y);
      }
#pragma unroll
      for (int w = 0; w < kWarps; ++w) factor[w * kCols + threadIdx.x] = x[w].x;
      col_stat[threadIdx.x] = joined;
    }
    __syncthreads();
    constexpr int kPer = kCols * D / 4 / kThreads;  // groups of four channels a thread
    const size_t call_unit = ((size_t)(p.k.s0 + run.s) * p.k.nl + lr) * c.H + h;
    // a CTA's first run may lack its beginning, its last one its end
    const int slot = blockIdx.x * 2 + (run.begin > 0 ? 0 : 1);
    float *part = p.parts + (size_t)slot * kCols * (D + 2);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = threadIdx.x + j * kThreads, col = 4 * i / D, x = 4 * i % D;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w)
        add4(o, *reinterpret_cast<const float4 *>(&exch[(w * kCols + col) * S::kRow + x]),
             factor[w * kCols + col]);
      if (whole)
        finish<O>(p, place[col], x, o, col_stat[col].x, col_stat[col].y, call_unit);
      else
        __stcg(reinterpret_cast<float4 *>(part) + i, o);
    }
    if (!whole) {
      if (threadIdx.x < kCols)
        __stcg(reinterpret_cast<float2 *>(part + kCols * D) + threadIdx.x, joined);
      // The last of the item's spans to finish joins them, in order.
      const int np = pieces_of(run.nb), parts = parts_of(np, plan.span);
      const int i0 = plan.base[run.s] + run.item * (plan.cut == kSpans ? np : parts);
      const int c0 = plan.cut == kSpans ? i0 / plan.span : i0;
      const int c1 = plan.cut == kSpans ? (i0 + np - 1) / plan.span : i0 + parts - 1;
      unsigned *ticket = c.ticket + unit_of(run) * kMaxTiles + tile;
      __syncthreads();
      if (threadIdx.x == 0) flag[0] = take_ticket(ticket) == (unsigned)(c1 - c0);
      __syncthreads();
      if (flag[0]) {
        if (threadIdx.x == 0) *ticket = 0;
        auto part_of = [&](int w) {
          return p.parts + ((size_t)w * 2 + (w == c0 ? 1 : 0)) * kCols * (D + 2);
        };
        // kSome contributors at a time, all their loads in flight together.
        constexpr int kSome = NT == 1 ? 8 : NT == 2 ? 4 : 2;
        float4 sum[kPer];
        float top[kPer], z[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          sum[j] = make_float4(0.f, 0.f, 0.f, 0.f);
          top[j] = kNone;
          z[j] = 0.f;
        }
        for (int w0 = c0; w0 <= c1; w0 += kSome) {
          float2 st[kSome][kPer];
          float4 x[kSome][kPer];
#pragma unroll
          for (int w = 0; w < kSome; ++w)
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
              const int i = threadIdx.x + j * kThreads;
              const float *from = part_of(min(c1, w0 + w));
              st[w][j] = __ldcg(reinterpret_cast<const float2 *>(from + kCols * D) + 4 * i / D);
              x[w][j] = __ldcg(reinterpret_cast<const float4 *>(from) + i);
            }
#pragma unroll
          for (int j = 0; j < kPer; ++j) {
            float m = top[j];
#pragma unroll
            for (int w = 0; w < kSome; ++w) m = fmaxf(m, st[w][j].x);
            const float f = ex2(top[j] - m);
            top[j] = m;
            z[j] *= f;
            sum[j].x *= f, sum[j].y *= f, sum[j].z *= f, sum[j].w *= f;
#pragma unroll
            for (int w = 0; w < kSome; ++w) {
              if (w0 + w > c1) break;
              const float g = ex2(st[w][j].x - m);
              z[j] = fmaf(st[w][j].y, g, z[j]);
              add4(sum[j], x[w][j], g);
            }
          }
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const int i = threadIdx.x + j * kThreads;
          finish<O>(p, place[4 * i / D], 4 * i % D, sum[j], top[j], z[j], call_unit);
        }
      }
    }
    __syncthreads();  // the exchange area is free again
  } while (next_run(run));
  if (!ok) {  // copies in flight end before the CTA does
    volatile int never = 0;
    for (; taken < issued; ++taken)
      mbar_wait(bars + 8 * (taken % kStages), (taken / kStages) & 1, &never);
  }
}

// Adds every row's probabilities to its score, after the attention has left each
// column's maximum and normaliser.  K alone is read again: a unit's logits would
// take 4 G bytes a row and token to keep, its K half takes 72.  A CTA has a span
// of one unit's blocks and all columns, whose fragments lie in shared memory; a
// warp loads a block's K into registers, its next one ahead, and goes through the
// columns, so that a row's sum stays with one warp and its order is fixed.
template <int D, int TERMS>
struct ScoreSmem {
  static constexpr int kTiles = TERMS == 1 ? 16 : 8;         // tiles of 8 columns at once
  static constexpr int kFrag = TERMS * (D / 16) * 2;         // words a lane and tile
  static constexpr int kSide = 2 * (D / kGroup) + 8;         // floats a column pair
  static constexpr int kBytes = kTiles * (32 * kFrag + 4 * kSide) * 4;
};
template <typename T, int D, int TERMS>
__global__ void __launch_bounds__(kThreads)
    score_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ Seqs sq,
                 int span) {
  using S = ScoreSmem<D, TERMS>;
  constexpr Codes M = TERMS == 2 ? kCentred : kEven;
  constexpr int W = D / 32, GR = D / kGroup;
  extern __shared__ __align__(128) uint8_t smem[];
  uint4 *frag = reinterpret_cast<uint4 *>(smem);  // [tile][word / 4][lane]
  float *side = reinterpret_cast<float *>(smem + S::kTiles * 32 * S::kFrag * 4);
  pdl_begin();
  const View &c = p.k.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int h = blockIdx.y % c.H, lr = blockIdx.y / c.H, s = blockIdx.z;
  const int len = sq.len[s], count = sq.count[s];
  const int first = blockIdx.x * span, nb = (len + kBlock - 1) / kBlock;
  if (first >= nb || count == 0) return;
  const int end = min(nb, first + span);
  const size_t u = unit_at(c, p.k.s0 + s, p.k.lb, lr, h);
  const uint8_t *blocks = c.blocks + u * c.nb * (size_t)block_bytes(D);
  float *score = c.score + u * c.sstride;
  const int rows = p.n_q * c.G;
  const float2 *stats = reinterpret_cast<const float2 *>(p.stats) +
                        (((size_t)(p.k.s0 + s) * p.k.nl + lr) * c.H + h) * rows;
  // the columns that have a token, then as many whole tiles
  const int tiles = (count * c.G + 7) / 8;
  for (int t0 = 0; t0 < tiles; t0 += S::kTiles) {
    const int tn = min(S::kTiles, tiles - t0);
    __syncthreads();
    for (int i = warp; i < tn; i += kWarps) {
      Query<D, 1, TERMS> q;
      load_query<T, M>(q, p, sq, s, lr, h, 8 * (t0 + i));
      const uint32_t *f = &q.f[0][0][0][0];
#pragma unroll
      for (int w = 0; w < S::kFrag; w += 4)
        frag[(i * (S::kFrag / 4) + w / 4) * 32 + lane] =
            make_uint4(f[w], f[w + 1], f[w + 2], f[w + 3]);
      if (g == 0) {
        float *to = side + (4 * i + t) * S::kSide;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = 8 * (t0 + i) + 2 * t + e;
          const bool live = q.limit[0][e] >= 0;
          const float2 st = live ? stats[col] : make_float2(-kNone, 0.f);
          to[e] = q.unit[0][e];
          to[2 + e] = st.x;
          to[4 + e] = st.y;
          to[6 + e] = __int_as_float(q.limit[0][e]);
#pragma unroll
          for (int j = 0; j < GR; ++j) to[8 + 2 * j + e] = q.sum[0][j][e];
        }
      }
    }
    __syncthreads();
    uint32_t next[2][2][W], next_m[2][2][GR];
    auto load = [&](int blk) {
      const uint8_t *at = blocks + (size_t)blk * block_bytes(D);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int r = 16 * tt + 8 * b + g;
          const uint32_t *k = reinterpret_cast<const uint32_t *>(
              at + k_off() + r * (D / 2) + k_chunk(r, t) * (D / 8));
          if (W == 4) {
            const uint4 x = __ldg(reinterpret_cast<const uint4 *>(k));
            next[tt][b][0] = x.x, next[tt][b][1] = x.y;
            next[tt][b][2 % W] = x.z, next[tt][b][3 % W] = x.w;
          } else {
            const uint2 x = __ldg(reinterpret_cast<const uint2 *>(k));
            next[tt][b][0] = x.x, next[tt][b][1] = x.y;
          }
          const uint32_t *m = reinterpret_cast<const uint32_t *>(at + km_off(D)) + r * GR;
#pragma unroll
          for (int j = 0; j < GR; ++j) next_m[tt][b][j] = __ldg(m + j);
        }
    };
    if (first + warp < end) load(first + warp);
    for (int blk = first + warp; blk < end; blk += kWarps) {
      uint32_t a[2][2][W][4];
      float m[2][2][GR], sc[2][2][GR], sum[2][2] = {};
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
          for (int w = 0; w < W; ++w) fields<M>(next[tt][b][w], a[tt][b][w]);
#pragma unroll
          for (int j = 0; j < GR; ++j)
            meta_of<M == kCentred>(next_m[tt][b][j],
                                   blk * kBlock + 16 * tt + 8 * b + g >= len, m[tt][b][j],
                                   sc[tt][b][j]);
        }
      if (blk + kWarps < end) load(blk + kWarps);
      const bool all = (blk + 1) * kBlock <= len - count;  // every token sees the block
#pragma unroll 1
      for (int i = 0; i < tn; ++i) {
        const float *at = side + (4 * i + t) * S::kSide;
        float acc[2][GR][4] = {};
#pragma unroll
        for (int z = 0; z < TERMS; ++z)
#pragma unroll
          for (int w = 0; w < W; ++w) {
            const uint4 f = frag[(i * (S::kFrag / 4) + z * W + w) * 32 + lane];
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
              mma_f16(acc[tt][w >> 1], a[tt][0][w][0], a[tt][1][w][0], a[tt][0][w][2],
                      a[tt][1][w][2], f.x, f.y);
              mma_f16(acc[tt][w >> 1], a[tt][0][w][1], a[tt][1][w][1], a[tt][0][w][3],
                      a[tt][1][w][3], f.z, f.w);
            }
          }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float unit = at[e], top = at[2 + e], inv = at[4 + e];
          const int limit = __float_as_int(at[6 + e]);
          float qs[GR];
#pragma unroll
          for (int j = 0; j < GR; ++j) qs[j] = at[8 + 2 * j + e];
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              float v = 0.f;
#pragma unroll
              for (int j = 0; j < GR; ++j) {
                v = j == 0 ? m[tt][b][j] * qs[j] : fmaf(m[tt][b][j], qs[j], v);
                v = fmaf(sc[tt][b][j], acc[tt][j][2 * b + e], v);
              }
              v = ex2(fmaf(v, unit, -top));
              if (!all && blk * kBlock + 16 * tt + 8 * b + g > limit) v = 0.f;
              sum[tt][b] = fmaf(v, inv, sum[tt][b]);
            }
        }
      }
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float x = sum[tt][b];
          x += __shfl_xor_sync(0xffffffffu, x, 1);
          x += __shfl_xor_sync(0xffffffffu, x, 2);
          const int r = blk * kBlock + 16 * tt + 8 * b + g;
          if (t == 0 && r < len) score[r] += x;
        }
    }
  }
}

// Tiles of 8 query rows that a kernel takes at once.
int tile_cols(const View &c, int n_q) {
  const long long rows = (long long)n_q * c.G;
  return rows <= 8 ? 8 : rows <= 16 || !(c.io_bf16 && c.out_bf16) ? 16 : 24;
}
long long tiles_of(const View &c, int n_q) {
  const int cols = tile_cols(c, n_q);
  return ((long long)n_q * c.G + cols - 1) / cols;
}

template <typename T, int D, int TERMS>
cudaError_t launch_scores(const AttendParams &p, const Seqs &q, const Device &dev,
                          cudaStream_t stream) {
  constexpr int kBytes = ScoreSmem<D, TERMS>::kBytes;
  auto kern = score_kernel<T, D, TERMS>;
  const int sms = dev.sms;
  const long long units = (long long)p.k.nl * p.k.c.H;
  long long total = 0;
  int most = 1;
  for (int i = 0; i < p.k.n; ++i) {
    total += units * blocks_of(q.len[i]);
    most = std::max(most, blocks_of(q.len[i]));
  }
  // about twelve CTAs an SM, a block a warp at least
  const int span = (int)std::max<long long>(kWarps, total / (12 * sms));
  return launch_pdl(kern, dim3((most + span - 1) / span, (unsigned)units, p.k.n), dim3(kThreads),
                    kBytes, stream, p, q, span);
}

template <typename T, typename O, int D, int NT, int TERMS>
cudaError_t prepare_as(Device *dev) {
  using S = Smem<D, NT>;
  auto kern = attend_kernel<T, O, D, NT, TERMS>;
  int per = 0;
  cudaError_t e =
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
  if (e == cudaSuccess)
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kern, kThreads, S::kBytes);
  dev->resident[NT - 1] = std::max(1, std::min(kMaxGrid, dev->sms * std::max(1, per)));
  return e;
}
template <typename T, typename O, int D, int TERMS>
cudaError_t prepare_tiles(Device *dev) {
  cudaError_t e = prepare_as<T, O, D, 1, TERMS>(dev);
  if (e == cudaSuccess) e = prepare_as<T, O, D, 2, TERMS>(dev);
  if (e == cudaSuccess && TERMS == 1) e = prepare_as<T, O, D, TERMS == 1 ? 3 : 2, TERMS>(dev);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(score_kernel<T, D, TERMS>,
                             cudaFuncAttributeMaxDynamicSharedMemorySize,
                             ScoreSmem<D, TERMS>::kBytes);
  return e;
}
template <typename T, typename O, int TERMS>
cudaError_t prepare_io(const View &c, Device *dev) {
  return c.d == 128 ? prepare_tiles<T, O, 128, TERMS>(dev) : prepare_tiles<T, O, 64, TERMS>(dev);
}

template <typename T, typename O, int D, int NT, int TERMS>
cudaError_t launch_as(const AttendParams &p, const Seqs &q, const Device &dev,
                      cudaStream_t stream) {
  using S = Smem<D, NT>;
  const View &c = p.k.c;
  auto kern = attend_kernel<T, O, D, NT, TERMS>;
  const int resident = dev.resident[NT - 1];  // CTAs that the device holds at once
  Plan plan;
  const long long tiles = tiles_of(c, p.n_q), per_seq = (long long)p.k.nl * c.H * tiles;
  if (tiles > INT32_MAX || per_seq > INT32_MAX) return cudaErrorInvalidValue;
  plan.tiles = (int)tiles;
  auto total_of = [&](int span) {  // parts, or pieces for span == 1
    long long n = 0;
    for (int i = 0; i < p.k.n; ++i) {
      plan.base[i] = (int32_t)std::min<long long>(n, INT32_MAX);
      n += per_seq * parts_of(pieces_of(blocks_of(q.len[i])), span);
    }
    plan.base[p.k.n] = (int32_t)std::min<long long>(n, INT32_MAX);
    return n;
  };
  const long long total = total_of(1);
  long long grid;
  if (tiles <= kMaxTiles && total <= INT32_MAX) {
    const int even = (int)std::max<long long>(kMinSpan, (total + resident - 1) / resident);
    plan.cut = kSpans;
    plan.span = even;
    grid = (total + even - 1) / even;
    // parts where they fit on the GPU at once and are not much longer
    for (int span = even; span <= even + kTurn; ++span) {
      const long long parts = total_of(span);
      if (parts > resident) continue;
      plan.cut = kParts;
      plan.span = span;
      grid = parts;
      break;
    }
    if (plan.cut == kSpans) total_of(1);
  } else {
    plan.cut = kItems;
    plan.span = 1;
    grid = per_seq * p.k.n;
  }
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  return launch_pdl(kern, dim3((unsigned)grid), dim3(kThreads), S::kBytes, stream, p, q, plan);
}
template <typename T, typename O, int D, int TERMS>
cudaError_t launch_tiles(const AttendParams &p, const Seqs &q, const Device &dev,
                         cudaStream_t stream) {
  switch (tile_cols(p.k.c, p.n_q)) {
    case 8: return launch_as<T, O, D, 1, TERMS>(p, q, dev, stream);
    case 16: return launch_as<T, O, D, 2, TERMS>(p, q, dev, stream);
    default: return launch_as<T, O, D, TERMS == 1 ? 3 : 2, TERMS>(p, q, dev, stream);
  }
}
template <typename T, typename O, int TERMS>
cudaError_t launch_io(const AttendParams &p, const Seqs &q, const Device &dev,
                      cudaStream_t stream, int *launches) {
  const bool wide = p.k.c.d == 128;
  cudaError_t e = tile_applies(p.k.c, p.n_q) ? launch_tile_attend(p, q, dev, stream)
                  : wide                     ? launch_tiles<T, O, 128, TERMS>(p, q, dev, stream)
                                             : launch_tiles<T, O, 64, TERMS>(p, q, dev, stream);
  *launches = 1;
  if (e != cudaSuccess || !p.stats) return e;
  *launches = 2;
  if (tile_applies(p.k.c, p.n_q)) return launch_tile_scores(p, q, dev, stream);
  return wide ? launch_scores<T, 128, TERMS>(p, q, dev, stream)
              : launch_scores<T, 64, TERMS>(p, q, dev, stream);
}

}  // namespace

size_t attend_stat_floats(const View &c, int nl, int n_q) {
  return ((size_t)c.S * nl * c.H * n_q * c.G * 2 + 3) / 4 * 4;
}
size_t attend_part_floats(const View &c, int nl, int n_q) {
  if (tile_applies(c, n_q)) return tile_part_floats(c, nl, n_q);
  const long long tiles = tiles_of(c, n_q);
  if (tiles > kMaxTiles) return 0;
  const size_t pieces = (size_t)std::min(c.S, kMaxSeqs) * nl * c.H * tiles * pieces_of(c.nb);
  return 2 * std::min<size_t>(kMaxGrid, pieces) * tile_cols(c, n_q) * (c.d + 2);
}

cudaError_t prepare_attend(const View &c, Device *dev) {
  *dev = Device{};
  int id = 0;
  cudaError_t e = cudaGetDevice(&id);
  if (e == cudaSuccess)
    e = cudaDeviceGetAttribute(&dev->sms, cudaDevAttrMultiProcessorCount, id);
  if (e != cudaSuccess) return e;
  if (c.io_bf16)
    e = c.out_bf16 ? prepare_io<__nv_bfloat16, __nv_bfloat16, 1>(c, dev)
                   : prepare_io<__nv_bfloat16, float, 2>(c, dev);
  else
    e = c.out_bf16 ? prepare_io<float, __nv_bfloat16, 2>(c, dev)
                   : prepare_io<float, float, 2>(c, dev);
  // (whether the tensor-memory kernels apply depends on a call's tokens: many, here)
  return e == cudaSuccess && tile_applies(c, 1 << 10) ? prepare_tile() : e;
}

cudaError_t launch_attend(const AttendParams &p, const Seqs &q, const Device &dev,
                          cudaStream_t stream, int *launches) {
  const bool ob = p.k.c.out_bf16;
  if (p.k.c.io_bf16)
    return ob ? launch_io<__nv_bfloat16, __nv_bfloat16, 1>(p, q, dev, stream, launches)
              : launch_io<__nv_bfloat16, float, 2>(p, q, dev, stream, launches);
  return ob ? launch_io<float, __nv_bfloat16, 2>(p, q, dev, stream, launches)
            : launch_io<float, float, 2>(p, q, dev, stream, launches);
}

}  // namespace kv4
}  // namespace kvr
