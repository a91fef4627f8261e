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
// rows (1.5B geometry) took 1,348 us, now 1,076 (6.99 TB/s; bound by those bytes).
//
// A unit that lies in one warp's span is written out by it; the pieces (greatest
// logit, sum, weighted values) of one that does not are joined in the CTA in order,
// and where it goes on in another CTA by the last of its CTAs to arrive, in order
// again, so that results do not depend on who is last.  A call of few units and tiles
// takes a cluster a unit instead, whose CTAs' parts meet in shared memory: 28 calls of
// a layer, one sequence of 4,099 rows (7B), in a graph 335 us with arrivals and 253 so.
// What is left there is latency: lengths, pages and rows one after the other, tiles of
// 0.4 us, and three joins.
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
constexpr int kMaxCtas = kMostCtas;  // whose logits the last one holds for 8 heads
// Tiles of a warp, where there are as many: what its copies hold.  (28 calls of 257
// tiles a unit with 2, 3, 4 and 6: 348, 335, 333 and 376 us.)
constexpr int kLeast = 3;

// 16 bytes to shared memory, zeros where `bytes` is 0 (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void copies_end() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A place in the shared memory of a CTA of the cluster, and what lies there.
__device__ __forceinline__ uint32_t in_cta(uint32_t here, unsigned rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(here), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 ld4_cluster(uint32_t at) {
  float4 x;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
               : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w)
               : "r"(at)
               : "memory");
  return x;
}
__device__ __forceinline__ float2 ld2_cluster(uint32_t at) {
  float2 x;
  asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];"
               : "=f"(x.x), "=f"(x.y)
               : "r"(at)
               : "memory");
  return x;
}
__device__ __forceinline__ void get4(const uint4 &w, float (&x)[4]) {
  x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y);
  x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
}

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
};

// Plain arithmetic in fp32, for fp32 rows.  Logits: four lanes share a row, each a
// quarter of its channels.  Values: a lane owns E channels.
template <int D>
struct Fma : Shape<float, D> {
  using S = Shape<float, D>;
  static constexpr int E = 4;
  static constexpr int kWarps = 4, kStages = 3;
  static constexpr int kRowsAtOnce = 32 / S::kVecs;
  static constexpr int kOwn = kHeads * D * 4;  // of a warp: q fp32 [8][D]
  static constexpr int kUnroll = D == 128 ? 4 : 2;
  float *q;
  float scale;
  float m[2], l[2];          // heads 2 j, 2 j + 1
  float o[kHeads][E];

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
    scale = scale_log2e;
  }
  __device__ __forceinline__ void start(const float *from, int G, int lane) {
    __syncwarp();
    for (int i = lane; i < kHeads * D; i += 32)
      q[i] = i < G * D ? from[i] * scale : 0.f;
    __syncwarp();
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
#pragma unroll
    for (int g = 0; g < kHeads; ++g)
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] = 0.f;
  }
  // One tile; rows from `limit` on do not exist.  Probabilities [16][8] and the
  // rescaling [8] take the place of K, once it has been read: two CTAs fit an SM at d =
  // 64 so.
  __device__ __forceinline__ void step(uint4 *stage, int limit, int lane) {
    const int j = lane & 3;
    float *p = reinterpret_cast<float *>(stage), *up = p + kTile * kHeads;
    static_assert(S::kPer * 512 >= (kTile * kHeads + kHeads) * 4, "room in K's place");
    float x[2][kHeads];
#pragma unroll
    for (int g = 0; g < kHeads; ++g) x[0][g] = x[1][g] = 0.f;
#pragma unroll kUnroll
    for (int i = 0; i < S::kPer / 2; ++i) {
      float a[E], b[E];
      get4(stage[(2 * i) * 32 + lane], a);
      get4(stage[(2 * i + 1) * 32 + lane], b);
      const float *qc = q + (j + 4 * i) * E;
#pragma unroll
      for (int g = 0; g < kHeads; ++g)
#pragma unroll
        for (int e = 0; e < E; e += 4) {
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
    __syncwarp();  // K has been read
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
      for (int e = 0; e < E; ++e) o[g][e] *= a;
    }
    const uint4 *vs = stage + S::kPer * 32;
#pragma unroll 2 * kUnroll
    for (int i = 0; i < S::kPer; ++i) {
      float v[E];
      get4(vs[i * 32 + lane], v);
      const float4 *pr = reinterpret_cast<const float4 *>(p + v_row(lane, i) * kHeads);
      const float4 pa = pr[0], pb = pr[1];
      const float w[kHeads] = {pa.x, pa.y, pa.z, pa.w, pb.x, pb.y, pb.z, pb.w};
#pragma unroll
      for (int g = 0; g < kHeads; ++g)
#pragma unroll
        for (int e = 0; e < E; ++e) o[g][e] = fmaf(w[g], v[e], o[g][e]);
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
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int s = S::kVecs; s < 32; s <<= 1) o[g][e] += __shfl_xor_sync(0xffffffffu, o[g][e], s);
      if (lane < S::kVecs)
#pragma unroll
        for (int e = 0; e < E; e += 4)
          f(g, lane * E + e, make_float4(o[g][e], o[g][e + 1], o[g][e + 2], o[g][e + 3]), mg,
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
    return (4 * (vec >> 3) + 2 * (row >> 3) + (row & 1)) * 512 +
           v_slot((row & 7) >> 1, vec & 7) * 16;
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
  __device__ __forceinline__ void step(uint4 *stage, int limit, int lane) {
    float s[2][4], s2[2][4];  // two chains a row of the tile
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[r][i] = s2[r][i] = 0.f;
#pragma unroll
    for (int i = 0; i < kK; ++i)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint4 k = stage[(2 * i + r) * 32 + k_slot(lane >> 2, lane & 3, i)];
        mma_bf16(s[r], q[i].x, 0u, q[i].y, 0u, k.x, k.y);
        mma_bf16(s2[r], q[i].z, 0u, q[i].w, 0u, k.z, k.w);
      }
    // rows 8 r + 2 (lane & 3) + i at [r][i]
    float x[2][2];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        x[r][i] = 8 * r + 2 * (lane & 3) + i < limit ? (s[r][i] + s2[r][i]) * scale : -INFINITY;
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

// A piece of a unit: tiles [first, upto) of the n of unit `unit`, whose first is tile
// `begin` of the call.
struct Piece {
  int unit, first, upto, n;
  unsigned begin;
};

// kCluster > 1: a cluster a unit, whose parts are joined through the CTAs' shared
// memory.
template <typename T, int D, typename P, typename O, int kCluster>
__global__ void __launch_bounds__(P::kWarps * 32)
    attend_kernel(const __grid_constant__ AttendParams p) {
  kvr::pdl_begin();
  using S = Shape<T, D>;
  constexpr int kWarps = P::kWarps, kStages = P::kStages, kPart = part_floats(D);
  constexpr int kThreads = kWarps * 32, kStats = kHeads * D;
  static_assert(kStages * S::kStage >= kPart * 4, "a warp's last piece takes its copies' place");
  static_assert(kWarps * kStages * S::kStage >= kHeads * kMaxCtas * 4, "logits of a unit's parts");
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Piece s_piece[2 * kWarps];
  __shared__ int s_last[2];
  __shared__ float2 s_stat[kWarps][kHeads];
  const View &c = p.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // All that is known of sequences is asked for at once: the end of the list, and a
  // first probe of where sequences start in it.
  const int stride = (c.S + 31) / 32;
  const unsigned tiles = p.src.tiles[c.S];
  const unsigned probe = p.src.tiles[min(lane * stride, c.S)];
  const int probe_rows = p.src.rows[min(lane, c.S - 1)];
  uint8_t *ring = smem + warp * (kStages * S::kStage);
  float *early = reinterpret_cast<float *>(smem + kWarps * kStages * S::kStage) + warp * kPart;
  uint8_t *own = smem + kWarps * (kStages * S::kStage + kPart * 4) + warp * P::kOwn;
  const uint32_t ring32 = smem_u32(ring);
  const unsigned U = p.nl * c.H;  // units of a sequence
  unsigned t0, t1, span;  // the warp's tiles
  int many = 0;           // CTAs of the cluster that have any
  if constexpr (kCluster > 1) {
    const unsigned unit = blockIdx.x / kCluster, s = unit / U, base = p.src.tiles[s];
    const unsigned n = p.src.tiles[s + 1] - base, from = base * U + (unit - s * U) * n;
    const unsigned mine = blockIdx.x % kCluster * kWarps + warp;
    span = max((n + kCluster * kWarps - 1) / (kCluster * kWarps), 1u);
    t0 = from + min(n, mine * span);
    t1 = from + min(n, (mine + 1) * span);
    many = (n + span * kWarps - 1) / (span * kWarps);
  } else {
    const unsigned total = tiles * U, warps = gridDim.x * kWarps;
    span = max((unsigned)kLeast, (total + warps - 1) / warps);
    t0 = min(total, (blockIdx.x * kWarps + warp) * span);
    t1 = min(total, t0 + span);
  }

  auto locate = [&](unsigned t) {
    // the last sequence that starts at or before t, 32 of them asked at a time
    const unsigned key = t / U;
    const int m = __popc(__ballot_sync(0xffffffffu, lane * stride < c.S && probe <= key)) - 1;
    Place x;
    x.s = m * stride;
    unsigned base = __shfl_sync(0xffffffffu, probe, m), next;
    if (stride == 1) {
      next = __shfl_sync(0xffffffffu, probe, (m + 1) & 31);
      if (m + 1 >= c.S) next = tiles;
      x.rows = __shfl_sync(0xffffffffu, probe_rows, m);
    } else {
      int hi = min(c.S, x.s + stride);
      while (hi - x.s > 1) {
        const int step = (hi - x.s + 31) / 32, at = x.s + lane * step;
        const unsigned in =
            __ballot_sync(0xffffffffu, at < hi && (unsigned)p.src.tiles[at] <= key);
        x.s += (__popc(in) - 1) * step;
        hi = min(hi, x.s + step);
      }
      base = p.src.tiles[x.s];
      next = p.src.tiles[x.s + 1];
      x.rows = p.src.rows[x.s];
    }
    x.n = next - base;
    const unsigned off = t - base * U;
    x.u = off / (unsigned)x.n;
    x.tile = off - x.u * x.n;
    return x;
  };
  auto page_of = [&](const Place &x) {
    return p.src.pages[x.s * p.src.seq_stride + x.u * p.src.unit_stride +
                       (x.tile * kTile >> c.psh)];
  };
  auto advance = [&](Place &x, unsigned next) {
    if (++x.tile < x.n) return;
    if (x.u + 1 < (int)U)
      x.tile = 0, x.u += 1;
    else if (next < t1)
      x = locate(next);
  };

  Place ahead{};
  unsigned issued = t0;
  int page = 0, to = 0;  // to: the stage that the next copies go to
  bool bad_page = false;
  auto issue = [&]() {
    if (issued < t1) {
      const uint32_t dst = ring32 + (uint32_t)to * S::kStage;
      const bool there = (unsigned)page < (unsigned)c.n_pages;
      bad_page |= !there;
      const int row = ahead.tile * kTile, limit = there ? ahead.rows - row : 0;
      const int lr = ahead.u / c.H, h = ahead.u - lr * c.H;
      const long long from =
          (pool_row(c, p.lb + lr, there ? page : 0, h) + (row & (c.P - 1))) * S::kRow + lane * 16;
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        const int r = (x * 32 + lane) / S::kVecs, v = lane % S::kVecs;
        copy16(dst + P::k_at(r, v), c.K + from + x * 512, r < limit ? 16 : 0);
      }
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        const int r = (x * 32 + lane) / S::kVecs, v = lane % S::kVecs;
        copy16(dst + S::kPer * 512 + P::v_at(r, v), c.V + from + x * 512, r < limit ? 16 : 0);
      }
      to = to + 1 == kStages ? 0 : to + 1;
      ++issued;
      advance(ahead, issued);
      if (issued < t1) page = page_of(ahead);
    }
    copies_end();
  };

  P work;
  work.init(own, c.scale * kLog2e);
  if (lane < 2) s_piece[2 * warp + lane] = Piece{-1, 0, 0, 0, 0};
  __syncwarp();
  bool infinite = false;
  auto out_of = [&](int unit) { return static_cast<O *>(p.out) + (long long)unit * c.G * D; };
  // Four channels of a head, normalised.
  auto put = [&](O *o, float4 v, float s) {
    const float r = 1.f / s;
    infinite |= !(fabsf(s) < INFINITY) || s == 0.f;
    put4(o, make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
  };
  // (one copy of everything below: a call of a few tiles spends its time on fetching
  // instructions)
  if (t0 < t1) {
    Place at = locate(t0);
    ahead = at;
    page = page_of(ahead);
    int first = at.tile, stage = 0;
    bool fresh = true;
#pragma unroll 1
    for (int k = 1 - kStages; t0 + k != t1; ++k) {
      if (k >= 0) {
        if (fresh) {
          work.start(static_cast<const T *>(p.q) + ((long long)at.s * U + at.u) * c.G * D, c.G,
                     lane);
          fresh = false;
        }
        copies_wait<kStages - 2>();
        __syncwarp();
      }
      issue();  // where tile k - 1 was, which the warp has read
      if (k < 0) continue;
      work.step(reinterpret_cast<uint4 *>(ring + (uint32_t)stage * S::kStage),
                at.rows - at.tile * kTile, lane);
      stage = stage + 1 == kStages ? 0 : stage + 1;
      const bool last = t0 + k + 1 == t1;
      if (at.tile + 1 < at.n && !last) {
        ++at.tile;
        continue;
      }
      const int unit = at.s * U + at.u;
      const bool whole = first == 0 && at.tile + 1 == at.n;
      // a warp's first piece goes beside its copies, its last one takes their place
      if (last) {
        copies_wait<0>();
        __syncwarp();
      }
      float *dst = last ? reinterpret_cast<float *>(ring) : early;
      if (!whole && lane == 0)
        s_piece[2 * warp + last] = Piece{unit, first, at.tile + 1, at.n, t0 + k - at.tile};
      O *o = out_of(unit);
      work.finish(lane, [&](int g, int ch, float4 v, float m, float s) {
        if (!whole) {
          put4(dst + g * D + ch, v);
          if (ch == 0) reinterpret_cast<float2 *>(dst + kStats)[g] = make_float2(m, s);
        } else if (g < c.G) {
          put(o + g * D + ch, v, s);
        }
      });
      if (!last) {
        advance(at, t0 + k + 1);
        first = 0;
        fresh = true;
      }
    }
  }
  copies_wait<0>();
  __syncthreads();

  // Join the pieces that lie side by side.  A thread owns 4 channels of a head, or of
  // kMine heads.
  auto piece_at = [&](int i) {
    return reinterpret_cast<const float *>(
        (i & 1) ? smem + (i >> 1) * (kStages * S::kStage)
                : smem + kWarps * kStages * S::kStage + (i >> 1) * kPart * 4);
  };
  constexpr int kMine = (kHeads * D / 4 + kThreads - 1) / kThreads;
  static_assert(kHeads * D / 4 % kThreads == 0, "all threads own the same");
  if (threadIdx.x < 2) s_last[threadIdx.x] = 0;
  Piece mine{-1, 0, 0, 0, 0};
  if (lane < 2 * kWarps) mine = s_piece[lane];
  int owed[2] = {-1, -1}, owed_n[2] = {0, 0};  // units that go on in CTAs before, behind
  unsigned owed_begin[2] = {0, 0};
#pragma unroll 1
  for (unsigned left = __ballot_sync(0xffffffffu, mine.unit >= 0); left;) {
    const int i = __ffs(left) - 1, unit = __shfl_sync(0xffffffffu, mine.unit, i);
    const unsigned same = __ballot_sync(0xffffffffu, mine.unit == unit);
    left &= ~same;
    const int n = __shfl_sync(0xffffffffu, mine.n, i);
    const int first = __shfl_sync(0xffffffffu, mine.first, i);
    const unsigned begin = __shfl_sync(0xffffffffu, mine.begin, i);
    const int upto = __shfl_sync(0xffffffffu, mine.upto, 31 - __clz(same));
    const bool whole = first == 0 && upto == n;
    const int which = first == 0;
    // (in a cluster nobody has an early piece: the CTA's part goes there)
    float *part = kCluster > 1 ? reinterpret_cast<float *>(smem + kWarps * kStages * S::kStage)
                               : p.parts + (2ll * blockIdx.x + which) * kPart;
#pragma unroll
    for (int y = 0; y < kMine; ++y) {
      const int x = threadIdx.x + y * kThreads, g = x / (D / 4);
      float2 ms[2 * kWarps];
      float4 w[2 * kWarps];
#pragma unroll
      for (int k = 0; k < 2 * kWarps; ++k) {
        ms[k] = make_float2(-INFINITY, 0.f);
        w[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (same >> k & 1) {
          ms[k] = reinterpret_cast<const float2 *>(piece_at(k) + kStats)[g];
          w[k] = reinterpret_cast<const float4 *>(piece_at(k))[x];
        }
      }
      float m = -INFINITY;
#pragma unroll
      for (int k = 0; k < 2 * kWarps; ++k) m = fmaxf(m, ms[k].x);
      const float ref = m == -INFINITY ? 0.f : m;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < 2 * kWarps; ++k) {
        const float a = ex2(ms[k].x - ref);
        v.x = fmaf(w[k].x, a, v.x), v.y = fmaf(w[k].y, a, v.y);
        v.z = fmaf(w[k].z, a, v.z), v.w = fmaf(w[k].w, a, v.w);
        s = fmaf(ms[k].y, a, s);
      }
      if (!whole) {
        put4(part + 4 * x, v);
        if (x % (D / 4) == 0) reinterpret_cast<float2 *>(part + kStats)[g] = make_float2(m, s);
      } else if (g < c.G) {
        put(out_of(unit) + 4 * x, v, s);
      }
    }
    if (!whole) {
      // (no dynamic index: which is 0 or 1)
      owed[0] = which ? owed[0] : unit, owed[1] = which ? unit : owed[1];
      owed_n[0] = which ? owed_n[0] : n, owed_n[1] = which ? n : owed_n[1];
      owed_begin[0] = which ? owed_begin[0] : begin, owed_begin[1] = which ? begin : owed_begin[1];
    }
  }
  if constexpr (kCluster > 1) {
    if (many > 1) {
      cluster_sync();
      constexpr int kSlice = kHeads * D / 4 / kCluster;  // of the outputs, a CTA's
      static_assert(kHeads * D / 4 % kCluster == 0 && kSlice <= kThreads, "slices");
      const unsigned here = smem_u32(smem + kWarps * kStages * S::kStage);
      const int x = blockIdx.x % kCluster * kSlice + threadIdx.x, g = x / (D / 4);
      if ((int)threadIdx.x < kSlice && g < c.G) {
        float2 ms[kCluster];
        float4 w[kCluster];
#pragma unroll
        for (int k = 0; k < kCluster; ++k) {
          ms[k] = make_float2(-INFINITY, 0.f);
          w[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (k < many) {
            const uint32_t at = in_cta(here, k);
            ms[k] = ld2_cluster(at + (kStats + 2 * g) * 4);
            w[k] = ld4_cluster(at + x * 16);
          }
        }
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < kCluster; ++k) m = fmaxf(m, ms[k].x);
        const float ref = m == -INFINITY ? 0.f : m;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kCluster; ++k) {
          const float a = ex2(ms[k].x - ref);
          v.x = fmaf(w[k].x, a, v.x), v.y = fmaf(w[k].y, a, v.y);
          v.z = fmaf(w[k].z, a, v.z), v.w = fmaf(w[k].w, a, v.w);
          s = fmaf(ms[k].y, a, s);
        }
        put(out_of(blockIdx.x / kCluster) + 4 * x, v, s);
      }
      cluster_sync();  // nobody leaves while its part is read
    }
  } else if (owed[0] >= 0 || owed[1] >= 0) {
    // CTAs that share the unit: the first has its part behind, the others before
    unsigned from[2], many[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      from[w] = owed_begin[w] / (span * kWarps);
      many[w] = (owed_begin[w] + owed_n[w] - 1) / (span * kWarps) - from[w] + 1;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
      const int w = threadIdx.x;
      if ((w ? owed[1] : owed[0]) >= 0) {
        unsigned *ticket = c.ticket + (w ? from[1] : from[0]);
        // (the barrier and this fence order every thread's part before the arrival)
        __threadfence();
        if (atomicAdd(ticket, 1u) == (w ? many[1] : many[0]) - 1) {
          *ticket = 0;
          s_last[w] = 1;
        }
        __threadfence();
      }
    }
    __syncthreads();
    // Shared memory is free now, for the greatest logits of all parts.
    float *logit = reinterpret_cast<float *>(smem);
    constexpr int kAhead = 12;
#pragma unroll 1
    for (int w = 0; w < 2; ++w) {
      if (!s_last[w]) continue;
      const int N = w ? many[1] : many[0], first = w ? from[1] : from[0];
      auto part = [&](int k) { return p.parts + (2ll * (first + k) + (k == 0)) * kPart; };
      // values of the first parts are on their way meanwhile
      float4 z[kMine][kAhead];
      auto fetch = [&](int k0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
          for (int y = 0; y < kMine; ++y)
            if (k0 + k < N)
              z[y][k] = __ldcg(reinterpret_cast<const float4 *>(part(k0 + k)) + threadIdx.x +
                               y * kThreads);
      };
      fetch(0);
      {
        const int g = lane & 7;
        float m = -INFINITY, s = 0.f;
        for (int k0 = threadIdx.x >> 3; k0 < N; k0 += 4 * (kThreads / 8)) {
          float2 ms[4];
          float now = m;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = k0 + i * (kThreads / 8);
            ms[i] = k < N ? __ldcg(reinterpret_cast<const float2 *>(part(k) + kStats) + g)
                          : make_float2(-INFINITY, 0.f);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = k0 + i * (kThreads / 8);
            if (k < N) logit[k * kHeads + g] = ms[i].x;
            now = fmaxf(now, ms[i].x);
          }
          const float ref = now == -INFINITY ? 0.f : now;
          s *= ex2(m - ref);
#pragma unroll
          for (int i = 0; i < 4; ++i) s = fmaf(ms[i].y, ex2(ms[i].x - ref), s);
          m = now;
        }
#pragma unroll
        for (int o = 8; o < 32; o <<= 1) {
          const float m2 = __shfl_xor_sync(0xffffffffu, m, o);
          const float s2 = __shfl_xor_sync(0xffffffffu, s, o);
          const float now = fmaxf(m, m2), ref = now == -INFINITY ? 0.f : now;
          s = s * ex2(m - ref) + s2 * ex2(m2 - ref);
          m = now;
        }
        if (lane < kHeads) s_stat[warp][lane] = make_float2(m, s);
      }
      __syncthreads();
      float4 v[kMine];
      float ref[kMine], sum[kMine];
#pragma unroll
      for (int y = 0; y < kMine; ++y) {
        const int g = (threadIdx.x + y * kThreads) / (D / 4);
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) m = fmaxf(m, s_stat[i][g].x);
        ref[y] = m == -INFINITY ? 0.f : m;
        sum[y] = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i)
          sum[y] = fmaf(s_stat[i][g].y, ex2(s_stat[i][g].x - ref[y]), sum[y]);
        v[y] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll 1
      for (int k0 = 0;;) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          if (k0 + k >= N) break;
#pragma unroll
          for (int y = 0; y < kMine; ++y) {
            const int g = (threadIdx.x + y * kThreads) / (D / 4);
            const float a = ex2(logit[(k0 + k) * kHeads + g] - ref[y]);
            v[y].x = fmaf(z[y][k].x, a, v[y].x), v[y].y = fmaf(z[y][k].y, a, v[y].y);
            v[y].z = fmaf(z[y][k].z, a, v[y].z), v[y].w = fmaf(z[y][k].w, a, v[y].w);
          }
        }
        k0 += kAhead;
        if (k0 >= N) break;
        fetch(k0);
      }
#pragma unroll
      for (int y = 0; y < kMine; ++y) {
        const int x = threadIdx.x + y * kThreads, g = x / (D / 4);
        if (g < c.G) put(out_of(w ? owed[1] : owed[0]) + 4 * x, v[y], sum[y]);
      }
      __syncthreads();  // the logits are read
    }
  }

  // sequences without rows: zeros
  for (int s = blockIdx.x; s < c.S; s += gridDim.x) {
    if (p.src.rows[s] > 0) continue;
    uint4 *o = reinterpret_cast<uint4 *>(out_of(s * U));
    for (int i = threadIdx.x; i < (int)U * c.G * D * (int)sizeof(O) / 16; i += kThreads)
      o[i] = make_uint4(0, 0, 0, 0);
  }
  if (bad_page && lane == 0) atomicOr(c.err, (unsigned)kvr::ERR_LENGTH);
  if (infinite) atomicOr(c.err, (unsigned)kvr::ERR_NONFINITE);
}

template <typename T, int D, typename P>
constexpr size_t smem_bytes() {
  return (size_t)P::kWarps * (P::kStages * Shape<T, D>::kStage + part_floats(D) * 4 + P::kOwn);
}

template <typename T, int D>
struct Choice {
  using P = Fma<D>;
};
template <int D>
struct Choice<__nv_bfloat16, D> {
  using P = Mma<D>;
};

// CTAs of a unit's cluster, where the call has few tiles: the first that fits.
constexpr int kUnitCtas[] = {16, 8};

// How many clusters of N CTAs run at once (SMs lie differently in clusters' reach from
// device to device).
template <typename T, int D, typename O, int N>
cudaError_t prepare_unit(int *clusters) {
  using P = typename Choice<T, D>::P;
  constexpr size_t bytes = smem_bytes<T, D, P>();
  constexpr auto unit = attend_kernel<T, D, P, O, N>;
  cudaError_t e =
      cudaFuncSetAttribute(unit, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(unit, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(N);
  cfg.blockDim = dim3(P::kWarps * 32);
  cfg.dynamicSmemBytes = bytes;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = N;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaOccupancyMaxActiveClusters(clusters, unit, &cfg);
}

template <typename T, int D, typename O>
cudaError_t prepare_as(Device *dev) {
  using P = typename Choice<T, D>::P;
  constexpr size_t bytes = smem_bytes<T, D, P>();
  static_assert(bytes + 2 * P::kWarps * (sizeof(Piece) + 32) + 64 <= 227 * 1024, "shared memory");
  cudaError_t e = cudaFuncSetAttribute(attend_kernel<T, D, P, O, 1>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) e = prepare_unit<T, D, O, kUnitCtas[0]>(&dev->clusters[0]);
  if (e == cudaSuccess) e = prepare_unit<T, D, O, kUnitCtas[1]>(&dev->clusters[1]);
  return e;
}

template <typename T, int D>
cudaError_t prepare(bool bf16_out, Device *dev) {
  return bf16_out ? prepare_as<T, D, __nv_bfloat16>(dev) : prepare_as<T, D, float>(dev);
}

// CTAs of a launch: as many as run at once.  (Two, four and eight times as many, so that
// SMs with a smaller share of the memory's rate do less: 1,067, 1,074 and 1,074 us
// against 1,070 for 16 sequences of 16,384 rows, and 274, 279 and 282 against 269 for
// chosen pages of six.)
template <typename T, int D>
int ctas_of(const Device &dev) {
  using P = typename Choice<T, D>::P;
  // (of an SM's 228 KB a CTA takes 1 KB more than it asks for)
  constexpr int kResident =
      228 * 1024 / (int)(smem_bytes<T, D, P>() + 2 * P::kWarps * (sizeof(Piece) + 32) + 64 + 1024);
  static_assert(kResident >= 1, "shared memory");
  return std::min(dev.sms * kResident, kMaxCtas);
}

// A cluster of n CTAs a unit: where all of them run at once and even the largest call
// gives a warp no more than 8 tiles on average, and none more than 16.  Parts then meet
// in shared memory and not across the L2's halves.  us a call in a graph, 4 units (7B, a
// layer of one sequence) of 32, 128, 512 and 1,500 tiles: 5.2, 6.5, 11.3 and 26.0, by
// spans 9.5, 10.3, 16.0 and 21.3; 16 units of 32 and 128, in clusters of 8, 6.0 and 9.6,
// by spans 10.6 and 12.9.  Lengths are the device's, and one sequence may hold nearly
// all of the pool, which is then one cluster's work: 18 units that share 288, 576, 1,152
// and 4,608 tiles, alike 5.3, 5.6, 6.8 and 13.6 (by spans 10.8, 10.5, 10.7 and 11.8),
// all in one unit 11.8, 19.6, 35.0 and 127 (11.5, 12.7, 18.5 and 33.2).  The bound of
// 16 lies where a wrong guess costs about as much either way; tables no longer than the
// sequences get keep batches that are alike in clusters.
bool fits(const AttendParams &p, int clusters, int n) {
  const long long units = (long long)p.c.S * p.nl * p.c.H, warps = n * 4;
  return units <= clusters && p.most <= units * warps * 8 && p.longest <= warps * 16;
}

template <typename T, int D, typename O, int N>
cudaError_t launch_units(const AttendParams &p, cudaStream_t st) {
  using P = typename Choice<T, D>::P;
  return kvr::launch_pdl_cluster(attend_kernel<T, D, P, O, N>, dim3(p.c.S * p.nl * p.c.H * N),
                                 dim3(P::kWarps * 32), N, smem_bytes<T, D, P>(), st, p);
}

template <typename T, int D, typename O>
cudaError_t launch_as(const AttendParams &p, const Device &dev, cudaStream_t st) {
  using P = typename Choice<T, D>::P;
  if (fits(p, dev.clusters[0], kUnitCtas[0])) return launch_units<T, D, O, kUnitCtas[0]>(p, st);
  if (fits(p, dev.clusters[1], kUnitCtas[1])) return launch_units<T, D, O, kUnitCtas[1]>(p, st);
  return kvr::launch_pdl(attend_kernel<T, D, P, O, 1>, dim3(ctas_of<T, D>(dev)),
                         dim3(P::kWarps * 32), smem_bytes<T, D, P>(), st, p);
}

template <typename T, int D>
cudaError_t launch(const AttendParams &p, const Device &dev, cudaStream_t st) {
  return p.c.out_bf16 ? launch_as<T, D, __nv_bfloat16>(p, dev, st)
                      : launch_as<T, D, float>(p, dev, st);
}

}  // namespace

int attend_ctas(const View &c, const Device &dev) {
  if (c.io_bf16)
    return c.d == 128 ? ctas_of<__nv_bfloat16, 128>(dev) : ctas_of<__nv_bfloat16, 64>(dev);
  return c.d == 128 ? ctas_of<float, 128>(dev) : ctas_of<float, 64>(dev);
}

cudaError_t prepare_attend(const View &c, Device *dev) {
  int now = 0;
  cudaError_t e = cudaGetDevice(&now);
  if (e == cudaSuccess)
    e = cudaDeviceGetAttribute(&dev->sms, cudaDevAttrMultiProcessorCount, now);
  if (e != cudaSuccess) return e;
  const bool out = c.out_bf16 != 0;
  if (c.io_bf16)
    return c.d == 128 ? prepare<__nv_bfloat16, 128>(out, dev)
                      : prepare<__nv_bfloat16, 64>(out, dev);
  return c.d == 128 ? prepare<float, 128>(out, dev)
                    : prepare<float, 64>(out, dev);
}

cudaError_t launch_attend(const AttendParams &p, const Device &dev, cudaStream_t st) {
  if (p.c.io_bf16)
    return p.c.d == 128 ? launch<__nv_bfloat16, 128>(p, dev, st)
                        : launch<__nv_bfloat16, 64>(p, dev, st);
  return p.c.d == 128 ? launch<float, 128>(p, dev, st) : launch<float, 64>(p, dev, st);
}

}  // namespace paged
}  // namespace kvr
