// kvr_paged_attend.cu -- attention of one new token a sequence over the paged
// cache (include/kvr.h, kvr_paged_attend): out = softmax(scale q K^T) V, every row of
// K and V read once.
//
// The call's rows are tiles of 16, in order of sequence, layer, head and position;
// every warp of the grid takes an equal span of them, whatever units (sequence,
// layer, head) it runs through, so that lengths on the device alone decide who does
// what.  A warp copies its own tiles ahead, by cp.async, and waits for nobody.  A
// copy instruction takes 512 bytes in a row from memory, whole lines, and puts each
// vector where the lane that needs it reads without bank conflicts: with the
// lanes fetching their own 64 bytes of eight rows instead, 16 sequences of 16,384
// rows (1.5B geometry) took 1,348 us, now 1,096 (6.86 TB/s).  A unit that lies in one warp's span is written
// out by it; the pieces (greatest logit, sum, weighted values) of one that does not
// are joined in the CTA in order, and where it goes on in another CTA by the last of
// its CTAs to arrive, in order again, so that results do not depend on who is last.
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

using namespace kvr::ptx;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxCtas = kMostCtas;  // whose weights the last one holds for 8 heads
constexpr int kLeast = 3;       // tiles of a warp, where there are as many

// 16 bytes to shared memory, zeros where `bytes` is 0 (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <typename T>
struct Elems;
template <>
struct Elems<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4 &w, float (&x)[4]) {
    x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y);
    x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
  }
};
template <>
struct Elems<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4 &w, float (&x)[8]) {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(a[i] << 16);
      x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
  }
};

__device__ __forceinline__ void put4(float *p, float4 x) { *reinterpret_cast<float4 *>(p) = x; }
__device__ __forceinline__ void put4(__nv_bfloat16 *p, float4 x) {
  *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
}

// What a lane copies and reads of a tile: its x-th vector of K and of V.
template <typename T, int D>
struct Shape {
  static constexpr int kRow = D * (int)sizeof(T);  // bytes of a row
  static constexpr int kVecs = kRow / 16;
  static constexpr int kPer = kVecs / 2;           // vectors of a lane, K or V
  static constexpr int kStage = 2 * kTile * kRow;
  static constexpr int E = Elems<T>::N;
};

// Plain arithmetic in fp32, for fp32 rows.  Logits: four lanes share a row, each a
// quarter of its channels.  Values: a lane owns E channels.
template <typename T, int D>
struct Fma : Shape<T, D> {
  using S = Shape<T, D>;
  static constexpr int kWarps = 4, kStages = 3;
  static constexpr int kRowsAtOnce = 32 / S::kVecs;
  // of a warp: q fp32 [8][D], probabilities [16][8], the rescaling [8]
  static constexpr int kOwn = (kHeads * D + kTile * kHeads + kHeads) * 4;
  float *q, *p, *up;
  float scale;
  float m[2], l[2];          // heads 2 j, 2 j + 1
  float o[kHeads][S::E];

  // Where a row's vector lies in its half of the stage.
  static __device__ __forceinline__ int k_at(int row, int vec) {
    return (2 * (vec >> 2) + (row >> 3)) * 512 + ((row & 7) * 4 + (vec & 3)) * 16;
  }
  static __device__ __forceinline__ int v_at(int row, int vec) {
    return (row * S::kVecs + vec) * 16;
  }
  static __device__ __forceinline__ int v_row(int lane, int x) {
    return lane / S::kVecs + kRowsAtOnce * x;
  }

  __device__ __forceinline__ void init(uint8_t *own, float scale_log2e) {
    q = reinterpret_cast<float *>(own);
    p = q + kHeads * D;
    up = p + kTile * kHeads;
    scale = scale_log2e;
  }
  __device__ __forceinline__ void start(const T *from, int G, int lane) {
    __syncwarp();
    for (int i = lane; i < kHeads * D; i += 32)
      q[i] = i < G * D ? kvr::dev::to_f(from[i]) * scale : 0.f;
    __syncwarp();
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
#pragma unroll
    for (int g = 0; g < kHeads; ++g)
#pragma unroll
      for (int e = 0; e < S::E; ++e) o[g][e] = 0.f;
  }
  // One tile; rows from `limit` on do not exist.
  __device__ __forceinline__ void step(const uint4 *stage, int limit, int lane) {
    const int j = lane & 3;
    float x[2][kHeads];
#pragma unroll
    for (int g = 0; g < kHeads; ++g) x[0][g] = x[1][g] = 0.f;
#pragma unroll 2
    for (int i = 0; i < S::kPer / 2; ++i) {
      float a[S::E], b[S::E];
      Elems<T>::get(stage[(2 * i) * 32 + lane], a);
      Elems<T>::get(stage[(2 * i + 1) * 32 + lane], b);
      const float *qc = q + (j + 4 * i) * S::E;
#pragma unroll
      for (int g = 0; g < kHeads; ++g)
#pragma unroll
        for (int e = 0; e < S::E; e += 4) {
          const float4 w = *reinterpret_cast<const float4 *>(qc + g * D + e);
          x[0][g] = fmaf(a[e], w.x, x[0][g]), x[1][g] = fmaf(b[e], w.x, x[1][g]);
          x[0][g] = fmaf(a[e + 1], w.y, x[0][g]), x[1][g] = fmaf(b[e + 1], w.y, x[1][g]);
          x[0][g] = fmaf(a[e + 2], w.z, x[0][g]), x[1][g] = fmaf(b[e + 2], w.z, x[1][g]);
          x[0][g] = fmaf(a[e + 3], w.w, x[0][g]), x[1][g] = fmaf(b[e + 3], w.w, x[1][g]);
        }
    }
    float mine[2][2];
#pragma unroll
    for (int g = 0; g < kHeads; ++g)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float y = x[r][g];
        y += __shfl_xor_sync(0xffffffffu, y, 1);
        y += __shfl_xor_sync(0xffffffffu, y, 2);
        if ((g >> 1) == j) mine[r][g & 1] = (lane >> 2) + 8 * r < limit ? y : -INFINITY;
      }
    __syncwarp();  // the last tile's probabilities have been read
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      float t = fmaxf(mine[0][g], mine[1][g]);
#pragma unroll
      for (int s = 4; s < 32; s <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, s));
      const float now = fmaxf(m[g], t), ref = now == -INFINITY ? 0.f : now;
      const float a = ex2(m[g] - ref);
      m[g] = now;
      const float p0 = ex2(mine[0][g] - ref), p1 = ex2(mine[1][g] - ref);
      l[g] = fmaf(l[g], a, p0 + p1);
      p[(lane >> 2) * kHeads + 2 * j + g] = p0;
      p[((lane >> 2) + 8) * kHeads + 2 * j + g] = p1;
      if (lane < 4) up[2 * j + g] = a;
    }
    __syncwarp();
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
      const float a = up[g];
#pragma unroll
      for (int e = 0; e < S::E; ++e) o[g][e] *= a;
    }
    const uint4 *vs = stage + S::kPer * 32;
#pragma unroll 4
    for (int i = 0; i < S::kPer; ++i) {
      float v[S::E];
      Elems<T>::get(vs[i * 32 + lane], v);
      const float4 *pr = reinterpret_cast<const float4 *>(p + v_row(lane, i) * kHeads);
      const float4 pa = pr[0], pb = pr[1];
      const float w[kHeads] = {pa.x, pa.y, pa.z, pa.w, pb.x, pb.y, pb.z, pb.w};
#pragma unroll
      for (int g = 0; g < kHeads; ++g)
#pragma unroll
        for (int e = 0; e < S::E; ++e) o[g][e] = fmaf(w[g], v[e], o[g][e]);
    }
  }
  // Sums over the lanes; then f(head, channel, four weighted sums, greatest logit,
  // sum of weights) for every head and channel, once each.
  template <typename F>
  __device__ __forceinline__ void finish(int lane, F f) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int s = 4; s < 32; s <<= 1) l[g] += __shfl_xor_sync(0xffffffffu, l[g], s);
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
      const float mg = __shfl_sync(0xffffffffu, m[g & 1], g >> 1);
      const float lg = __shfl_sync(0xffffffffu, l[g & 1], g >> 1);
#pragma unroll
      for (int e = 0; e < S::E; ++e)
#pragma unroll
        for (int s = S::kVecs; s < 32; s <<= 1) o[g][e] += __shfl_xor_sync(0xffffffffu, o[g][e], s);
      if (lane < S::kVecs)
#pragma unroll
        for (int e = 0; e < S::E; e += 4)
          f(g, lane * S::E + e, make_float4(o[g][e], o[g][e + 1], o[g][e + 2], o[g][e + 3]), mg,
            lg);
    }
  }
};

// bf16 on warp-level tensor cores (a unit has eight query rows at most: what binds is
// bytes).  Products run over 16 channels or 16 rows whatever their order, so a lane's
// 16-byte vectors are fragments as they come: of K, eight channels of a row, which are
// two steps' share of a lane; of V, eight channels of four rows, whose halves are
// paired by byte permutation.  Probabilities go in as two bf16 numbers each (the 8
// rows that heads leave free hold the low ones), which keeps 2^-16 of them; a tile's
// sum is formed from zero and added in fp32, because the accumulator truncates.
template <int D>
struct Mma : Shape<__nv_bfloat16, D> {
  using S = Shape<__nv_bfloat16, D>;
  static constexpr int kWarps = 4, kStages = D == 128 ? 3 : 6;
  static constexpr int kOwn = 0;
  static constexpr int kK = D / 32, kV = D / 64;  // vectors of a row, K or V
  uint4 q[kK];
  float scale;
  float m, l;          // head lane / 4
  float o[kV][8][2];   // channels 64 v + 8 (2 (lane & 3) + i) + e at [v][e][i]

  static __device__ __forceinline__ int k_slot(int t, int j, int i) {
    return (t >> 1) * 8 + (((t & 1) * 4 + j) ^ (4 * (i & 1)));
  }
  static __device__ __forceinline__ int v_slot(int j, int g) { return j * 8 + (g ^ (2 * j)); }
  static __device__ __forceinline__ int k_at(int row, int vec) {
    return (2 * (vec >> 2) + (row >> 3)) * 512 + k_slot(row & 7, vec & 3, vec >> 2) * 16;
  }
  static __device__ __forceinline__ int v_at(int row, int vec) {
    return (4 * (vec >> 3) + 2 * (row >> 3) + (row & 1)) * 512 + v_slot((row & 7) >> 1, vec & 7) * 16;
  }

  __device__ __forceinline__ void init(uint8_t *, float scale_log2e) { scale = scale_log2e; }
  __device__ __forceinline__ void start(const __nv_bfloat16 *from, int G, int lane) {
    const int g = lane >> 2;
#pragma unroll
    for (int i = 0; i < kK; ++i)
      q[i] = g < G ? __ldg(reinterpret_cast<const uint4 *>(from + g * D) + (lane & 3) + 4 * i)
                   : make_uint4(0, 0, 0, 0);
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int v = 0; v < kV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) o[v][e][0] = o[v][e][1] = 0.f;
  }
  __device__ __forceinline__ void step(const uint4 *stage, int limit, int lane) {
    float s[2][4];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[r][i] = 0.f;
#pragma unroll
      for (int i = 0; i < kK; ++i) {
        const uint4 k = stage[(2 * i + r) * 32 + k_slot(lane >> 2, lane & 3, i)];
        mma_bf16(s[r], q[i].x, 0u, q[i].y, 0u, k.x, k.y);
        mma_bf16(s[r], q[i].z, 0u, q[i].w, 0u, k.z, k.w);
      }
    }
    // rows 8 r + 2 (lane & 3) + i at [r][i]
    float x[2][2];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        x[r][i] = 8 * r + 2 * (lane & 3) + i < limit ? s[r][i] * scale : -INFINITY;
    float t = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1]));
    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
    const float now = fmaxf(m, t), ref = now == -INFINITY ? 0.f : now;
    const float a = ex2(m - ref);
    m = now;
    uint32_t hi[2], lo[2];
    l *= a;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float p0 = ex2(x[r][0] - ref), p1 = ex2(x[r][1] - ref);
      l += p0 + p1;
      hi[r] = pack_bf16(p0, p1);
      lo[r] = pack_bf16(p0 - __uint_as_float(hi[r] << 16),
                        p1 - __uint_as_float(hi[r] & 0xFFFF0000u));
    }
    const uint4 *vs = stage + S::kPer * 32 + v_slot(lane & 3, lane >> 2);
    // what the accumulators of head lane / 4 are multiplied by is the lane's own a
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const uint4 w0 = vs[(4 * v) * 32], w1 = vs[(4 * v + 1) * 32];
      const uint4 w2 = vs[(4 * v + 2) * 32], w3 = vs[(4 * v + 3) * 32];
      const uint32_t b[4][4] = {{w0.x, w0.y, w0.z, w0.w},
                                {w1.x, w1.y, w1.z, w1.w},
                                {w2.x, w2.y, w2.z, w2.w},
                                {w3.x, w3.y, w3.z, w3.w}};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t sel = e & 1 ? 0x7632u : 0x5410u;
        float d[4] = {0.f, 0.f, 0.f, 0.f};
        mma_bf16(d, hi[0], lo[0], hi[1], lo[1], __byte_perm(b[0][e >> 1], b[1][e >> 1], sel),
                 __byte_perm(b[2][e >> 1], b[3][e >> 1], sel));
        o[v][e][0] = fmaf(o[v][e][0], a, d[0] + d[2]);
        o[v][e][1] = fmaf(o[v][e][1], a, d[1] + d[3]);
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void finish(int lane, F f) {
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
#pragma unroll
    for (int v = 0; v < kV; ++v)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 8; e += 4)
          f(lane >> 2, 64 * v + 16 * (lane & 3) + 8 * i + e,
            make_float4(o[v][e][i], o[v][e + 1][i], o[v][e + 2][i], o[v][e + 3][i]), m, l);
  }
};

// A place in the list of tiles.
struct Place {
  int s, u, tile, n, rows;  // unit u of the sequence's nl * H; its tiles and rows
};

// A piece of a unit: tiles [first, first + count) of the n of unit `unit`.
struct Piece {
  long long unit;
  int first, count, n;
};

template <typename T, int D, typename P, typename O>
__global__ void __launch_bounds__(P::kWarps * 32) attend_kernel(const __grid_constant__ AttendParams p) {
  kvr::pdl_begin();
  using S = Shape<T, D>;
  constexpr int kWarps = P::kWarps, kStages = P::kStages, kPart = part_floats(D);
  static_assert(kStages * S::kStage >= kPart * 4, "a warp's last piece takes its copies' place");
  static_assert(kWarps * kStages * S::kStage >= kHeads * (kMaxCtas + 1) * 4,
                "the weights of a unit's parts");
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Piece s_piece[2 * kWarps];
  __shared__ int s_last[2];
  const View &c = p.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint8_t *ring = smem + warp * (kStages * S::kStage);
  float *early = reinterpret_cast<float *>(smem + kWarps * kStages * S::kStage) + warp * kPart;
  uint8_t *own = smem + kWarps * (kStages * S::kStage + kPart * 4) + warp * P::kOwn;
  const uint32_t ring32 = smem_u32(ring);
  const int U = p.nl * c.H;  // units of a sequence
  const long long total = (long long)p.src.tiles[c.S] * U;
  const long long warps = (long long)gridDim.x * kWarps;
  const long long span = max((long long)kLeast, (total + warps - 1) / warps);
  const long long cta_span = span * kWarps;
  const long long t0 = min(total, ((long long)blockIdx.x * kWarps + warp) * span);
  const long long t1 = min(total, t0 + span);

  // sequences without rows: zeros
  for (int s = blockIdx.x; s < c.S; s += gridDim.x) {
    if (p.src.tiles[s + 1] != p.src.tiles[s]) continue;
    uint4 *o = reinterpret_cast<uint4 *>(static_cast<O *>(p.out) + (long long)s * U * c.G * D);
    for (long long i = threadIdx.x; i < (long long)U * c.G * D * (int)sizeof(O) / 16;
         i += kWarps * 32)
      o[i] = make_uint4(0, 0, 0, 0);
  }

  auto locate = [&](long long t) {
    // the last sequence that starts at or before t (32 of them asked at a time)
    const int key = (int)(t / U);
    int lo = 0, hi = c.S;
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, at = lo + lane * step;
      const unsigned in = __ballot_sync(0xffffffffu, at < hi && p.src.tiles[at] <= key);
      lo += (__popc(in) - 1) * step;
      hi = min(hi, lo + step);
    }
    Place x;
    x.s = lo;
    const int base = p.src.tiles[lo];
    x.n = p.src.tiles[lo + 1] - base;
    x.rows = p.src.rows[lo];
    const long long off = t - (long long)base * U;
    x.u = (int)(off / x.n);
    x.tile = (int)(off - (long long)x.u * x.n);
    return x;
  };
  auto page_of = [&](const Place &x) {
    return p.src.pages[x.s * p.src.seq_stride + x.u * p.src.unit_stride +
                       ((long long)x.tile * kTile >> c.psh)];
  };
  auto advance = [&](Place &x, long long next) {
    if (++x.tile < x.n) return;
    if (x.u + 1 < U)
      x.tile = 0, x.u += 1;
    else if (next < t1)
      x = locate(next);
  };

  Place at{}, ahead{};
  long long issued = t0;
  int page = 0;
  bool bad_page = false;
  auto issue = [&]() {
    if (issued < t1) {
      const uint32_t dst = ring32 + (uint32_t)((issued - t0) % kStages) * S::kStage;
      const bool there = (unsigned)page < (unsigned)c.n_pages;
      bad_page |= !there;
      const int row = ahead.tile * kTile, limit = there ? ahead.rows - row : 0;
      const int lr = ahead.u / c.H, h = ahead.u - lr * c.H;
      const long long from =
          (pool_row(c, p.lb + lr, there ? page : 0, h) + (row & (c.P - 1))) * S::kRow;
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        const int r = (x * 32 + lane) / S::kVecs, v = lane % S::kVecs;
        copy16(dst + P::k_at(r, v), c.K + from + (x * 32 + lane) * 16, r < limit ? 16 : 0);
      }
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        const int r = (x * 32 + lane) / S::kVecs, v = lane % S::kVecs;
        copy16(dst + S::kPer * 512 + P::v_at(r, v), c.V + from + (x * 32 + lane) * 16,
               r < limit ? 16 : 0);
      }
      ++issued;
      advance(ahead, issued);
      if (issued < t1) page = page_of(ahead);
    }
    copies_end();
  };

  P work;
  work.init(own, c.scale * kLog2e);
  if (lane < 2) s_piece[2 * warp + lane] = Piece{-1, 0, 0, 0};
  __syncwarp();
  bool infinite = false;
  auto out_of = [&](long long unit) {
    return static_cast<O *>(p.out) + unit * c.G * D;
  };
  if (t0 < t1) {
    at = ahead = locate(t0);
    page = page_of(ahead);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) issue();
    int first = at.tile;
    work.start(static_cast<const T *>(p.q) + ((long long)at.s * U + at.u) * c.G * D, c.G, lane);
    for (long long t = t0; t < t1; ++t) {
      copies_wait<kStages - 2>();
      __syncwarp();
      issue();  // where tile t - 1 was, which the warp has read
      work.step(reinterpret_cast<const uint4 *>(ring + (uint32_t)((t - t0) % kStages) * S::kStage),
                at.rows - at.tile * kTile, lane);
      const bool last = t + 1 == t1;
      if (at.tile + 1 < at.n && !last) {
        ++at.tile;
        continue;
      }
      const long long unit = (long long)at.s * U + at.u;
      if (first == 0 && at.tile + 1 == at.n) {
        O *o = out_of(unit);
        work.finish(lane, [&](int g, int ch, float4 v, float, float s) {
          if (g >= c.G) return;
          const float r = 1.f / s;
          infinite |= !(fabsf(s) < INFINITY) || s == 0.f;
          put4(o + g * D + ch, make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
        });
      } else {
        // a warp's first piece beside its copies, its last one in their place
        if (lane == 0)
          s_piece[2 * warp + last] = Piece{unit, first, at.tile + 1 - first, at.n};
        if (last) {
          copies_wait<0>();
          __syncwarp();
        }
        float *dst = last ? reinterpret_cast<float *>(ring) : early;
        work.finish(lane, [&](int g, int ch, float4 v, float m, float s) {
          put4(dst + g * D + ch, v);
          if (ch == 0) dst[kHeads * D + g] = m, dst[kHeads * D + kHeads + g] = s;
        });
      }
      if (!last) {
        advance(at, t + 1);
        first = 0;
        work.start(static_cast<const T *>(p.q) + ((long long)at.s * U + at.u) * c.G * D, c.G,
                   lane);
      }
    }
  }
  copies_wait<0>();
  __syncthreads();

  // Join the pieces that lie side by side.  Thread x owns 4 channels of a head.
  auto piece_at = [&](int i) {
    return reinterpret_cast<const float *>(
        (i & 1) ? smem + (i >> 1) * (kStages * S::kStage)
                : smem + kWarps * kStages * S::kStage + (i >> 1) * kPart * 4);
  };
  constexpr int kMine = kHeads * D / 4 / (kWarps * 32) > 0 ? kHeads * D / 4 / (kWarps * 32) : 1;
  const bool busy = (int)threadIdx.x < kHeads * D / 4;
  if (threadIdx.x < 2) s_last[threadIdx.x] = 0;
  long long owed[2] = {-1, -1};  // units that go on in other CTAs: before, behind
  int owed_first[2], owed_n[2];
  for (int i = 0; i < 2 * kWarps;) {
    const Piece a = s_piece[i];
    if (a.unit < 0) {
      ++i;
      continue;
    }
    int end = i, upto = 0;
    for (int k = i; k < 2 * kWarps; ++k)
      if (s_piece[k].unit == a.unit)
        end = k + 1, upto = s_piece[k].first + s_piece[k].count;
      else if (s_piece[k].unit >= 0)
        break;
    const bool whole = a.first == 0 && upto == a.n;
    const int which = a.first == 0 ? 1 : 0;
    float *part = p.parts + (2ll * blockIdx.x + which) * kPart;
    if (busy)
#pragma unroll
      for (int y = 0; y < kMine; ++y) {
        const int x = threadIdx.x + y * kWarps * 32, g = x / (D / 4);
        float m = -INFINITY;
        for (int k = i; k < end; ++k)
          if (s_piece[k].unit >= 0) m = fmaxf(m, piece_at(k)[kHeads * D + g]);
        const float ref = m == -INFINITY ? 0.f : m;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float s = 0.f;
        for (int k = i; k < end; ++k) {
          if (s_piece[k].unit < 0) continue;
          const float *from = piece_at(k);
          const float a = ex2(from[kHeads * D + g] - ref);
          const float4 w = reinterpret_cast<const float4 *>(from)[x];
          v.x = fmaf(w.x, a, v.x), v.y = fmaf(w.y, a, v.y);
          v.z = fmaf(w.z, a, v.z), v.w = fmaf(w.w, a, v.w);
          s = fmaf(from[kHeads * D + kHeads + g], a, s);
        }
        if (!whole) {
          put4(part + 4 * x, v);
          if (x % (D / 4) == 0) part[kHeads * D + g] = m, part[kHeads * D + kHeads + g] = s;
        } else if (g < c.G) {
          const float r = 1.f / s;
          infinite |= !(fabsf(s) < INFINITY) || s == 0.f;
          put4(out_of(a.unit) + 4 * x, make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
        }
      }
    if (!whole) {
      owed[which] = a.unit;
      owed_first[which] = a.first;
      owed_n[which] = a.n;
    }
    i = end;
  }
  if (bad_page && lane == 0) atomicOr(c.err, (unsigned)kvr::ERR_LENGTH);
  if (owed[0] >= 0 || owed[1] >= 0) {
    // position of the unit's first tile, and with it the CTAs that share it
    long long from[2], upto[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if (owed[w] < 0) continue;
      const int s = (int)(owed[w] / U);
      const long long begin = (long long)p.src.tiles[s] * U + (owed[w] - (long long)s * U) * owed_n[w];
      from[w] = begin / cta_span;
      upto[w] = (begin + owed_n[w] - 1) / cta_span;
    }
    __syncthreads();
    if (threadIdx.x < 2 && owed[threadIdx.x] >= 0) {
      const int w = threadIdx.x;
      // (the barrier and this fence order every thread's part before the arrival)
      __threadfence();
      const unsigned there = (unsigned)(upto[w] - from[w]);
      if (atomicAdd(c.ticket + from[w], 1u) == there) {
        c.ticket[from[w]] = 0;
        s_last[w] = 1;
      }
      __threadfence();
    }
    __syncthreads();
    // Shared memory is free now: the weights of all parts there, while the first
    // parts' values are on their way.
    float *weight = reinterpret_cast<float *>(smem), *sum = weight + kHeads * kMaxCtas;
    constexpr int kAhead = 8;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if (owed[w] < 0 || !s_last[w]) continue;
      const int many = (int)(upto[w] - from[w]) + 1;
      auto part = [&](int k) { return p.parts + (2 * (from[w] + k) + (k == 0)) * kPart; };
      float4 z[kMine][kAhead];
      auto fetch = [&](int k0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
          for (int y = 0; y < kMine; ++y)
            if (busy && k0 + k < many)
              z[y][k] = __ldcg(reinterpret_cast<const float4 *>(part(k0 + k)) + threadIdx.x +
                               y * kWarps * 32);
      };
      fetch(0);
      __syncthreads();
      for (int g = warp; g < c.G; g += kWarps) {
        float m = -INFINITY;
        for (int k = lane; k < many; k += 32) {
          const float x = __ldcg(part(k) + kHeads * D + g);
          weight[g * kMaxCtas + k] = x;
          m = fmaxf(m, x);
        }
        m = kvr::dev::warp_max(m);
        const float ref = m == -INFINITY ? 0.f : m;
        float s = 0.f;
        for (int k = lane; k < many; k += 32) {
          const float a = ex2(weight[g * kMaxCtas + k] - ref);
          weight[g * kMaxCtas + k] = a;
          s = fmaf(__ldcg(part(k) + kHeads * D + kHeads + g), a, s);
        }
        s = kvr::dev::warp_sum(s);
        if (lane == 0) sum[g] = s;
      }
      __syncthreads();
      if (!busy) continue;
      float4 v[kMine];
#pragma unroll
      for (int y = 0; y < kMine; ++y) v[y] = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k0 = 0;;) {
#pragma unroll
        for (int y = 0; y < kMine; ++y) {
          const int g = (threadIdx.x + y * kWarps * 32) / (D / 4);
#pragma unroll
          for (int k = 0; k < kAhead; ++k) {
            if (k0 + k >= many || g >= c.G) continue;
            const float a = weight[g * kMaxCtas + k0 + k];
            v[y].x = fmaf(z[y][k].x, a, v[y].x), v[y].y = fmaf(z[y][k].y, a, v[y].y);
            v[y].z = fmaf(z[y][k].z, a, v[y].z), v[y].w = fmaf(z[y][k].w, a, v[y].w);
          }
        }
        k0 += kAhead;
        if (k0 >= many) break;
        fetch(k0);
      }
#pragma unroll
      for (int y = 0; y < kMine; ++y) {
        const int x = threadIdx.x + y * kWarps * 32, g = x / (D / 4);
        if (g >= c.G) continue;
        const float s = sum[g], r = 1.f / s;
        infinite |= !(fabsf(s) < INFINITY) || s == 0.f;
        put4(out_of(owed[w]) + 4 * x,
             make_float4(v[y].x * r, v[y].y * r, v[y].z * r, v[y].w * r));
      }
    }
  }
  if (infinite) atomicOr(c.err, (unsigned)kvr::ERR_NONFINITE);
}

template <typename T, int D, typename P>
constexpr size_t smem_bytes() {
  return (size_t)P::kWarps * (P::kStages * Shape<T, D>::kStage + part_floats(D) * 4 + P::kOwn);
}

template <typename T, int D>
struct Choice {
  using P = Fma<T, D>;
};
template <int D>
struct Choice<__nv_bfloat16, D> {
  using P = Mma<D>;
};

template <typename T, int D>
cudaError_t prepare() {
  using P = typename Choice<T, D>::P;
  constexpr size_t bytes = smem_bytes<T, D, P>();
  static_assert(bytes + 2 * P::kWarps * sizeof(Piece) + 64 <= 227 * 1024, "shared memory");
  cudaError_t e = cudaFuncSetAttribute(attend_kernel<T, D, P, float>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(attend_kernel<T, D, P, __nv_bfloat16>,
                             cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  return e;
}

// CTAs of a launch: as many as run at once, or several times as many, where the
// largest call would still give every warp 24 tiles: SMs do not get the same share of
// the memory's rate, and shorter spans even that out.
template <typename T, int D>
int ctas_of(const AttendParams &p, int sms) {
  using P = typename Choice<T, D>::P;
  // (of an SM's 228 KB a CTA takes 1 KB more than it asks for)
  constexpr int kResident =
      228 * 1024 / (int)(smem_bytes<T, D, P>() + 2 * P::kWarps * sizeof(Piece) + 64 + 1024);
  static_assert(kResident >= 1, "shared memory");
  const int at_once = std::min(sms * kResident, kMaxCtas);
  const long long waves = p.most / ((long long)at_once * P::kWarps * 24);
  return at_once * (int)std::max(1ll, std::min<long long>(waves, std::min(8, kMaxCtas / at_once)));
}

template <typename T, int D>
cudaError_t launch(const AttendParams &p, int sms, cudaStream_t st) {
  using P = typename Choice<T, D>::P;
  const dim3 grid(ctas_of<T, D>(p, sms)), block(P::kWarps * 32);
  return p.c.out_bf16 ? kvr::launch_pdl(attend_kernel<T, D, P, __nv_bfloat16>, grid, block,
                                        smem_bytes<T, D, P>(), st, p)
                      : kvr::launch_pdl(attend_kernel<T, D, P, float>, grid, block,
                                        smem_bytes<T, D, P>(), st, p);
}

}  // namespace

int attend_ctas(const AttendParams &p, int sms) {
  if (p.c.io_bf16)
    return p.c.d == 128 ? ctas_of<__nv_bfloat16, 128>(p, sms) : ctas_of<__nv_bfloat16, 64>(p, sms);
  return p.c.d == 128 ? ctas_of<float, 128>(p, sms) : ctas_of<float, 64>(p, sms);
}

cudaError_t prepare_attend(const View &c) {
  if (c.io_bf16) return c.d == 128 ? prepare<__nv_bfloat16, 128>() : prepare<__nv_bfloat16, 64>();
  return c.d == 128 ? prepare<float, 128>() : prepare<float, 64>();
}

cudaError_t launch_attend(const AttendParams &p, int sms, cudaStream_t st) {
  if (p.c.io_bf16)
    return p.c.d == 128 ? launch<__nv_bfloat16, 128>(p, sms, st)
                        : launch<__nv_bfloat16, 64>(p, sms, st);
  return p.c.d == 128 ? launch<float, 128>(p, sms, st) : launch<float, 64>(p, sms, st);
}

}  // namespace paged
}  // namespace kvr
