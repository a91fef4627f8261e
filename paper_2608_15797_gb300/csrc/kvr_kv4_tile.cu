// kvr_kv4_tile.cu -- attention over the 4-bit cache for more than a few query rows
// a unit, on 5th-generation tensor cores (bf16, d = 128; kvr_kv4.cuh has the
// cache's layout, kvr_kv4_attend.cu the kernel for fewer rows).
//
// Columns are (token, head) pairs of a unit, N <= 64 of them a tile, and rows the
// 128 cached tokens of four blocks:
//   S_j [tokens x N] = K_j Q_j^T for the two channel groups j, in tensor memory
//   P   [tokens x N] = 2^(logit - reference of the column), 16 bits, in shared memory
//   O^T [d x N]     += V^T P, in tensor memory
// With tokens as rows a thread of the softmax owns a token: the scales and minima
// of its key are registers, and a column's maximum, which would need the other
// lanes, is only checked (P must not pass 2^15): the reference is a maximum over
// some of a run's first tile, and raised when a logit outgrows it.  K's operand is
// its codes as they are (half-precision subnormals, scaled back by q and s), in
// tensor memory; V's is m + s c rounded to half precision once, relative to the
// token's largest value 2^e, and the power of two that takes this back goes into the
// token's logits.  P is rounded to half precision once; its sums are fp32.  Below
// 2^-14 that rounding is 2^-25 of the reference and no longer of P, so that rows which
// all weigh 2^-20 of the greatest and less are summed to a few percent of themselves
// (1e-3 of the output and less).  References 2^4 to 2^8 lower would move that limit as
// far, but are outgrown more often: 5 tokens of 16 sequences, keys of uneven size, 722
// and 908 us against 640.  Values below 2^-84 count as zero.
//
// One CTA an SM, its warps in roles with bounded waits on mbarriers between them:
//   8 softmax   two groups of four warps (4 x 32 tokens), each with half of the
//               tile's columns: a thread then holds its columns' sums of q and its
//               normalisers in registers.  (Groups that took turns by tile, with
//               all columns each, loaded the sums of q for every element: 16
//               sequences of 512 to 16,384 rows, 35 columns, 741 us against 672.)
//   4 K         codes -> K's operand, the keys' constants
//   4 V         codes -> V's operand in shared memory, the values' constants
//   1 issuer    the matrix products
//   1 loader    raw blocks, kRing tiles ahead
// K's and V's warps in one role, seven warps that loaded for themselves, made K's
// next tile wait for the softmax: 845 us against 750.
// As in the other kernel, CTAs take equal spans of the list of all tiles and the
// last of those that share a unit joins their results in order.
//
// Bound by latency: a tile of 48 columns takes about 2,400 cycles, of which the
// softmax of a group works 1,900 and the tensor core 1,400 (its operands come out of
// the shared memory that everything else uses too).  Measured (28 layers, 4 KV heads,
// G = 7): 5 tokens of 16 sequences of 512 to 16,384 rows 619 us (2.0 TB/s of the
// cache's bytes), of 8 sequences of 8,192 493 us (2.1 TB/s), of 64 of 512 498 us; 32
// tokens of 2 sequences of 8,191 561 us (375 TFLOP/s).
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "kvr_kv4_attend.cuh"
#include "kvr_tmem.cuh"

namespace kvr {
namespace kv4 {
namespace {

constexpr int kD = 128;
constexpr int kTok = 128;                   // tokens of a tile
constexpr int kTileBlocks = kTok / kBlock;
constexpr int kMaxN = 64;                   // columns of a tile
// Warps, in warpgroups of four: softmax (two), K, V, and one with the issuer and the
// loader.
constexpr int kSoft = 8, kKey = 4, kVal = 4;
constexpr int kIssuer = kSoft + kKey + kVal, kLoader = kIssuer + 1;
constexpr int kThr = 32 * (kIssuer + 4);
// Registers a thread: at launch, then for the softmax and for the others (168 and 48:
// 672 us where 144 and 64 took 703; 64 columns 606 against 598).
constexpr int kRegs = 96, kRegsSoft = 168, kRegsRest = 48;
static_assert(32 * kSoft * kRegsSoft + (kThr - 32 * kSoft) * kRegsRest <= kThr * kRegs,
              "the shares come out of what the CTA was launched with");
constexpr int kRing = 4;                    // raw tiles in flight
static_assert(kVal == kTileBlocks && kKey == 4, "a warp's 32 tokens");
constexpr int kConst = 4;                   // tiles whose tokens' constants are held
constexpr int kTileGrid = 256;              // CTAs of a split call, at most
constexpr uint32_t kRaw = kTileBlocks * block_bytes(kD);
constexpr uint32_t kHalf = kTok * 128;      // one 64-element half of an operand
constexpr uint32_t kCols = 512;             // tensor memory: S (2 x 2 x 64), O (64),
constexpr uint32_t kColO = 256;             // K (2 x 64)
constexpr uint32_t kColK = 384;
constexpr float kUnit = field_unit(kRough);  // of K's codes

// An item's place in the list counts its tiles and, before them, kSwitch more for
// what a CTA spends on an item whatever its length (its queries, the first
// maxima, the result).  One of kWhole tiles or fewer is not cut, but its first
// tile's CTA has all of it: that is one result instead of a join.
constexpr int kSwitch = 5;
constexpr int kWhole = 4;
struct TilePlan {
  int32_t base[kMaxSeqs + 1];
  int32_t span;    // of a CTA, or 0: one item a CTA
  int32_t tiles;   // column tiles of a unit
};

struct __align__(16) Side {
  float4 key[kConst][kTok];     // s0, s1, m0, m1 of a token's key
  float2 val[kConst][kTok];     // e + 1, 2^-(e + 1) of its value
  uint2 vc[2][kTok / 2];        // [group][pair]: s 2^(18 - e - 1), m 2^-(e + 1), halves
  float4 qs[kMaxN / 2];         // sums of q: group 0 of two columns, group 1
  float ntop[kMaxN];            // minus the columns' references
  float factor[kMaxN];
  float wmax[4][kMaxN], zsum[4][kMaxN];
  int limit[kMaxN];             // last row a column sees, or -1
  float2 stat[kMaxN];
  Place place[kMaxN];
  float qmax[kSoft];
  int nan_row[16][2];           // [run % 16][group]: first row whose value is NaN
  uint64_t raw_full[kRing], raw_free[kRing];
  uint64_t cf[kConst], c_free[kConst], kf[2], vf[2], pv[2], sf[2], s_free[2], pf[2], qf, drain;
  uint32_t tmem;
  int abort, flag;
};

constexpr uint32_t kOffV = 0, kOffP = kOffV + 4 * kHalf, kOffQ = kOffP + 2 * kHalf,
                   kOffRaw = kOffQ + 2 * kMaxN * 128, kOffSide = kOffRaw + kRing * kRaw;
constexpr uint32_t kSmem = kOffSide + sizeof(Side);
static_assert(kSmem <= 227 * 1024, "shared memory");

// Instruction descriptor of kind::f16 with half-precision A and B, fp32 D, A
// K-major.
__device__ __forceinline__ uint32_t idesc_f16(int M, int N, bool b_mn_major) {
  return (1u << 4) | (b_mn_major ? 1u << 16 : 0u) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void tmem_ld8(uint32_t ta, float (&v)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]),
        "=f"(v[7])
      : "r"(ta));
}
__device__ __forceinline__ void tmem_st8(uint32_t ta, const float (&v)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(ta),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
      : "memory");
}
// Barrier `id` of n threads with the OR of their predicates.
__device__ __forceinline__ bool bar_any(int id, int n, bool x) {
  int y;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, %3, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
      : "=r"(y)
      : "r"((int)x), "r"(id), "r"(n)
      : "memory");
  return y != 0;
}
// Operands are written for the tensor cores alone, and a fence that orders memory
// follows: no clobber here, so that loads may run ahead of these stores.
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c,
                                       uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d));
}
// True for one lane of a whole warp, the same one every time.  (The tensor cores'
// instructions take their operands from uniform registers; under lane == 0 eight
// products took the issuer some 1,000 cycles.)
__device__ __forceinline__ bool elect_one() {
  uint32_t y;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}"
               : "=r"(y));
  return y != 0;
}
// Gives registers of a warpgroup to the softmax.
__device__ __forceinline__ void give_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRest));
}
// As tmem_wait_ld, but only what was loaded waits: memory's loads may pass it.
__device__ __forceinline__ void tmem_landed(float (&a)[8], float (&b)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(a[0]), "+f"(a[1]), "+f"(a[2]), "+f"(a[3]), "+f"(a[4]), "+f"(a[5]),
                 "+f"(a[6]), "+f"(a[7]), "+f"(b[0]), "+f"(b[1]), "+f"(b[2]), "+f"(b[3]),
                 "+f"(b[4]), "+f"(b[5]), "+f"(b[6]), "+f"(b[7]));
}
// A token's products with N columns, where some columns do not see it: they get
// minus infinity (what multiplies it is above zero), which keeps the mask out of the
// loops over all tiles.  A key that stands for NaN gives it to those who see it, and
// its constants are made harmless.
__device__ __forceinline__ void mask_row(uint32_t ts, int n, const int *limit, int row,
                                         float4 &key) {
  const bool bad = key.z != key.z || key.w != key.w;
#pragma unroll 1
  for (int k = 0; k < n; k += 8) {
    float a[8];
    tmem_ld8(ts + k, a);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = row > limit[k + e] ? -INFINITY : bad ? NAN : a[e];
    tmem_st8(ts + k, a);
  }
  tmem_wait_st();
  if (bad) key = make_float4(1.f, 1.f, 0.f, 0.f);
}
__device__ __forceinline__ uint32_t half2_bits(__half2 x) {
  return *reinterpret_cast<const uint32_t *>(&x);
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<__half2 *>(&x); }

// A run of tiles [t0, t1) of one item; np: all it has; at: the item's place.
struct TileRun {
  int s, item, t0, t1, np, at;
};

struct Walk {
  const Seqs &sq;
  const TilePlan &plan;
  int per_seq, last;  // the end of the CTA's span
  __device__ static int tiles_of(int nb) { return (nb + kTileBlocks - 1) / kTileBlocks; }
  __device__ int end_of(const TileRun &r) const {
    return r.np <= kWhole ? r.np : min(r.np, last - r.at - kSwitch);
  }
  // The span's first item with a tile in it.
  __device__ bool first(TileRun &r, int seqs) {
    const int from = blockIdx.x * plan.span;
    last = min(from + plan.span, plan.base[seqs]);
    int lo = 0, hi = seqs;  // the sequence that holds the span's start
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.base[mid] <= from) lo = mid; else hi = mid;
    }
    r.s = lo;
    r.np = tiles_of(blocks_of(sq.len[lo]));
    const int rest = from - plan.base[lo], cost = kSwitch + r.np;
    r.item = rest / cost;
    r.at = plan.base[lo] + r.item * cost;
    r.t0 = max(0, from - r.at - kSwitch);
    if (r.t0 > 0 && r.np <= kWhole) return next(r);
    if (r.at + kSwitch >= last) return false;  // a short span may lie before the tile
    r.t1 = end_of(r);
    return true;
  }
  __device__ bool next(TileRun &r) const {
    r.at += kSwitch + r.np;
    if (r.at + kSwitch >= last) return false;
    if (++r.item == per_seq) {
      r.item = 0;
      ++r.s;
      r.np = tiles_of(blocks_of(sq.len[r.s]));
    }
    r.t0 = 0;
    r.t1 = end_of(r);
    return true;
  }
};

// CH: groups of eight columns of a tile.
template <int CH>
__global__ void __launch_bounds__(kThr, 1)
    tile_attend_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ Seqs sq,
                       const __grid_constant__ TilePlan plan) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char *smem = smem_raw;
  Side &S = *reinterpret_cast<Side *>(smem + kOffSide);
  const View &c = p.k.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int N = 8 * CH;
  const uint32_t base = smem_u32(smem);
  volatile int *abort = &S.abort;
  // A whole warp's bounded wait for completion n of a barrier.
  auto wait = [&](uint64_t &bar, int n) {
    return warp_wait(smem_u32(&bar), (uint32_t)(n & 1), abort);
  };
  // Completion n of a barrier, and a wait for up to three of them.
  auto at = [&](uint64_t &bar, int n) { return Phase{smem_u32(&bar), (uint32_t)(n & 1)}; };
  auto wait_for = [&](Phase a, Phase b, Phase c, int n) { return warp_wait(a, b, c, n, abort); };
  auto give_up = [&]() {
    if (lane == 0) {
      if (!*abort) atomicOr(c.err, ERR_TIMEOUT);
      *abort = 1;
    }
  };
  if (warp == kSoft) tmem_alloc(smem_u32(&S.tmem), kCols);
  if (tid == 0) {
    for (int b = 0; b < kRing; ++b) {
      mbar_init(smem_u32(&S.raw_full[b]), 1);
      mbar_init(smem_u32(&S.raw_free[b]), kKey + kVal);
    }
    for (int b = 0; b < kConst; ++b) {
      mbar_init(smem_u32(&S.cf[b]), kKey + kVal);
      mbar_init(smem_u32(&S.c_free[b]), kSoft);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&S.kf[b]), kKey);
      mbar_init(smem_u32(&S.vf[b]), kVal);
      mbar_init(smem_u32(&S.sf[b]), 1);
      mbar_init(smem_u32(&S.s_free[b]), kSoft);
      mbar_init(smem_u32(&S.pf[b]), 2);
      mbar_init(smem_u32(&S.pv[b]), 1);
    }
    mbar_init(smem_u32(&S.qf), 1);
    mbar_init(smem_u32(&S.drain), 1);
    S.abort = 0;
    for (int i = 0; i < 16; ++i) S.nan_row[i][0] = S.nan_row[i][1] = INT32_MAX;
    fence_mbar_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_begin();
  const uint32_t tm = S.tmem;

  // The CTA's first run.
  Walk walk{sq, plan, p.k.nl * c.H * plan.tiles, 0};
  TileRun run;
  bool any = true;
  if (plan.span) {
    any = walk.first(run, p.k.n);
  } else {
    run.s = blockIdx.x / walk.per_seq;
    run.item = blockIdx.x - run.s * walk.per_seq;
    // no tile past the last row that the column tile's last token sees
    const int tok = min(sq.count[run.s], ((run.item % plan.tiles + 1) * N - 1) / c.G + 1);
    run.np = Walk::tiles_of(blocks_of(sq.len[run.s] - sq.count[run.s] + tok));
    run.at = 0;
    run.t0 = 0;
    run.t1 = run.np;
    walk.last = 0;
  }
  auto unit_of = [&](const TileRun &r) {
    const int unit = r.item / plan.tiles;
    return unit_at(c, p.k.s0 + r.s, p.k.lb, unit / c.H, unit % c.H);
  };

  if (!any) {
    // no work
  } else if (warp >= kIssuer) {
    give_registers();
    if (warp == kIssuer) {
      // ---- issuer
      const uint32_t id_s = idesc_f16(kTok, N, false), id_o = idesc_f16(kD, N, true);
      const uint64_t dq = sdesc_sw128(base + kOffQ, 16, 1024);
      const uint64_t dv = sdesc_sw128(base + kOffV, 16, 1024);
      const uint64_t dp = sdesc_sw128(base + kOffP, kHalf, 1024);
      int i = 0, runs = 0;
      bool ok = true;
      auto issue_pv = [&](int j, bool first) {  // tile j's P and V are there
        ok = ok && wait_for(at(S.vf[j & 1], j / 2), at(S.pf[j & 1], j / 2), {}, 2);
        if (!ok) return;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t a = dv + (uint64_t)(((j & 1) * 2 * kHalf) >> 4);
          const uint64_t b = dp + (uint64_t)(((j & 1) * kHalf) >> 4);
  #pragma unroll
          for (int k = 0; k < 8; ++k)
            tc_mma(tm + kColO, a + (uint64_t)(((k >> 2) * kHalf + (k & 3) * 32) >> 4),
                   b + (uint64_t)(k * 128), id_o, !(first && k == 0));
          tc_commit(smem_u32(&S.pv[j & 1]));
        }
        __syncwarp();
      };
      do {
        for (int t = run.t0; t < run.t1 && ok; ++t, ++i) {
          ok = wait_for(at(S.kf[i & 1], i / 2), at(S.qf, runs), at(S.s_free[i & 1], i / 2 - 1),
                        i < 2 ? 2 : 3);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
  #pragma unroll
            for (int j = 0; j < 2; ++j)
  #pragma unroll
              for (int k = 0; k < 4; ++k)
                tc_mma_ts(tm + (i & 1) * 128 + j * 64, tm + kColK + (i & 1) * 64 + j * 32 + k * 8,
                          dq + (uint64_t)((j * N * 128 + k * 32) >> 4), id_s, k > 0);
            tc_commit(smem_u32(&S.sf[i & 1]));
          }
          __syncwarp();
          if (t > run.t0) issue_pv(i - 1, t - 1 == run.t0);
        }
        issue_pv(i - 1, run.t1 - 1 == run.t0);
        ++runs;
      } while (ok && walk.next(run));
      if (!ok) give_up();
      __syncwarp();
      // Every product is done before tensor memory is freed.  (A commit covers what its
      // own lane issued: the same one is elected every time.)
      if (elect_one()) {
        volatile int never = 0;
        tc_commit(smem_u32(&S.drain));
        mbar_wait(smem_u32(&S.drain), 0, &never);
      }
    } else if (warp == kLoader) {
      // ---- loader: raw tiles, kRing ahead of their use
      int issued = 0;
      bool ok = true;
      do {
        const int unit = run.item / plan.tiles;
        const uint8_t *blocks =
            c.blocks + unit_at(c, p.k.s0 + run.s, p.k.lb, unit / c.H, unit % c.H) * c.nb *
                           (size_t)block_bytes(kD);
        const int nb = blocks_of(sq.len[run.s]);
        for (int t = run.t0; t < run.t1 && ok; ++t) {
          const int rb = issued % kRing;
          if (issued >= kRing) ok = wait(S.raw_free[rb], issued / kRing - 1);
          if (!ok) break;
          if (lane == 0) {
            const uint32_t bytes =
                (uint32_t)min(kTileBlocks, nb - t * kTileBlocks) * block_bytes(kD);
            mbar_expect_tx(smem_u32(&S.raw_full[rb]), bytes);
            bulk_load(base + kOffRaw + rb * kRaw, blocks + (size_t)t * kRaw, bytes,
                      smem_u32(&S.raw_full[rb]));
          }
          __syncwarp();
          ++issued;
        }
      } while (ok && walk.next(run));
      if (!ok) give_up();
      if (lane == 0) {  // every copy lands before the shared memory is given back
        volatile int never = 0;
        for (int j = max(0, issued - kRing); j < issued; ++j)
          mbar_wait(smem_u32(&S.raw_full[j % kRing]), (uint32_t)((j / kRing) & 1), &never);
      }
    }
  } else if (warp >= kSoft + kKey) {
    // ---- V
    give_registers();
    const int vw = warp - kSoft - kKey, vt = tid - 32 * (kSoft + kKey);
    int i = 0, runs = 0;
    bool ok = true;
    do {
      const int len = sq.len[run.s];
      for (int t = run.t0; t < run.t1; ++t, ++i) {
        const int b = i & 1, cb = i % kConst, rb = i % kRing;
        const unsigned char *raw = smem + kOffRaw + rb * kRaw;
        ok = ok && wait_for(at(S.raw_full[rb], i / kRing), at(S.c_free[cb], i / kConst - 1), {},
                            i < kConst ? 1 : 2);
        if (!ok) break;
        // The slot of eight runs ahead: none of this role has reached it, and the
        // softmax, at most four tiles behind, has left the run that had it.
        if (vt == 0 && t == run.t0)
          S.nan_row[(runs + 8) & 15][0] = S.nan_row[(runs + 8) & 15][1] = INT32_MAX;
        {  // a token's constants
          const int row = t * kTok + vt;
          uint2 vm = *reinterpret_cast<const uint2 *>(raw + vw * block_bytes(kD) + vm_off(kD) +
                                                      lane * 8);
          if (row >= len) vm = make_uint2(0, 0);
          float m[2] = {m_of(vm.x), m_of(vm.y)}, s[2] = {s_of(vm.x), s_of(vm.y)};
          float top = 0.f;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (m[g] != m[g]) {  // the group stands for NaN: told to those who see it
              atomicMin(&S.nan_row[runs & 15][g], row);
              m[g] = s[g] = 0.f;
            }
            top = fmaxf(top, fmaxf(fabsf(m[g]), fabsf(fmaf(15.f, s[g], m[g]))));
          }
          const int e = max(-60, min((int)(__float_as_uint(top) >> 23) - 127, 120)) + 1;
          const float down = __uint_as_float((unsigned)(127 - e) << 23);
          S.val[cb][vt] = make_float2((float)e, down);
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            __half *h = reinterpret_cast<__half *>(&S.vc[g][vt >> 1]) + (vt & 1);
            h[0] = __float2half_rn(s[g] * down * 0x1p18f);
            h[2] = __float2half_rn(m[g] * down);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&S.cf[cb]));
        ok = i < 2 || wait(S.pv[b], i / 2 - 1);
        if (!ok) break;
        // Eight tokens (tg) of chunk ch a lane, a channel group (w, w + 1) at a time; the
        // warp's tokens are those of one block.
        const int tg = vw * 4 + (lane >> 3), ch = lane & 7;
#pragma unroll
        for (int w = 0; w < 4; w += 2) {
          uint2 v[4];
          __half2 sc[4], mn[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int pr = tg * 4 + k, pb = pr % (kBlock / 2);
            v[k] = *reinterpret_cast<const uint2 *>(raw + vw * block_bytes(kD) + v_off(kD) +
                                                    pb * kD + v_chunk<kD>(pb, ch) * 16 + w * 4);
            const uint2 x = S.vc[w >> 1][pr];
            sc[k] = as_half2(x.x);
            mn[k] = as_half2(x.y);
          }
          // (ch: the row within eight)
          const uint32_t to = base + kOffV + b * 2 * kHalf + (tg >> 3) * kHalf +
                              (32 * w + ch) * 128 + (((tg & 7) ^ ch) << 4);
#pragma unroll
          for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int f = 0; f < 4; ++f) {
              uint32_t o[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t x = z ? v[k].y : v[k].x;
                const uint32_t y =
                    (f == 0 ? x << 6 : f == 1 ? x << 2 : f == 2 ? x >> 2 : x >> 6) & 0x03C003C0u;
                o[k] = half2_bits(__hfma2(as_half2(y), sc[k], mn[k]));  // c 2^-18
              }
              sts128(to + (32 * z + (f == 0 ? 0 : f == 1 ? 16 : f == 2 ? 8 : 24)) * 128, o[0],
                     o[1], o[2], o[3]);
            }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&S.vf[b]));
          mbar_arrive(smem_u32(&S.raw_free[rb]));
        }
      }
      ++runs;
    } while (ok && walk.next(run));
    if (!ok) give_up();
  } else if (warp >= kSoft) {
    // ---- K: a token a thread, into tensor memory
    give_registers();
    const int dt = tid - 32 * kSoft, dw = warp - kSoft;
    int i = 0;
    bool ok = true;
    do {
      const int len = sq.len[run.s];
      for (int t = run.t0; t < run.t1; ++t, ++i) {
        const int b = i & 1, cb = i % kConst, rb = i % kRing;
        const unsigned char *blk = smem + kOffRaw + rb * kRaw + (dt / kBlock) * block_bytes(kD);
        // (its place is free once tile i - 2's product is there)
        ok = ok && wait_for(at(S.raw_full[rb], i / kRing), at(S.sf[b], i / 2 - 1),
                            at(S.c_free[cb], i / kConst - 1), i < 2 ? 1 : i < kConst ? 2 : 3);
        if (!ok) break;
        const int r = dt % kBlock;
        uint2 km = *reinterpret_cast<const uint2 *>(blk + km_off(kD) + r * 8);
        if (t * kTok + dt >= len) km = make_uint2(0, 0);
        S.key[cb][dt] = make_float4(s_of(km.x), s_of(km.y), m_of(km.x), m_of(km.y));
        uint4 w[4];
#pragma unroll
        for (int t4 = 0; t4 < 4; ++t4)
          w[t4] = *reinterpret_cast<const uint4 *>(blk + k_off() + r * (kD / 2) +
                                                   k_chunk(r, t4) * 16);
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&S.raw_free[rb]));
          mbar_arrive(smem_u32(&S.cf[cb]));
        }
        tc_fence_after();
        // A word's fields are the pairs of nibbles 0 4, 1 5, 2 6, 3 7; channels 64 j ..
        // are words 2 j, 2 j + 1 of each chunk.
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            uint32_t o[16];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint4 &c4 = w[2 * y + (x >> 1)];
              const uint32_t v = j == 0 ? (x & 1 ? c4.y : c4.x) : (x & 1 ? c4.w : c4.z);
              fields<kRough>(v, o + 4 * x);
            }
            tmem_st16(tm + ((uint32_t)(dw * 32) << 16) + kColK + b * 64 + j * 32 + y * 16, o);
          }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&S.kf[b]));
      }
    } while (ok && walk.next(run));
    if (!ok) give_up();
  } else {
    // ---- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
    const int wq = warp & 3, grp = warp >> 2;
    const uint32_t lanes = (uint32_t)(wq * 32) << 16;
    const int tok = wq * 32 + lane, gt = tid & 127;  // of the group's threads
    constexpr int NG = N / 2, CG = CH / 2;  // columns of the group, and their eights
    const int c0 = grp * NG;
    const uint32_t to = tm + kColO + c0 + lanes;
    float *const ntop = S.ntop + c0, *const factor = S.factor + c0;
    auto all_ok = [&](bool ok) { return !bar_any(2, 32 * kSoft, !ok); };
    auto group_ok = [&](bool ok) { return !bar_any(3 + grp, 16 * kSoft, !ok); };
    int i = 0, runs = 0;  // i: tiles before the run
    bool ok = true, more = true;
    // A run's queries, eight channels (ci) of every sixteenth column a thread.
    const int ci = tid & 15;
    uint4 raw[CH / 2];
    auto load_q = [&](const TileRun &r) {
      const int unit = r.item / plan.tiles, col0 = (r.item % plan.tiles) * N;
#pragma unroll
      for (int z = 0; z < CH / 2; ++z) {
        const Place a = place_of(p, sq, r.s, unit / c.H, unit % c.H, col0 + (tid >> 4) + 16 * z);
        raw[z] = make_uint4(0, 0, 0, 0);
        if (a.out >= 0 && a.live)
          raw[z] = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.q) +
                                                    a.out + 8 * ci);
      }
    };
    load_q(run);
    do {
      // ---- a run's queries, scaled by one power of two for all columns, and columns
      const int unit = run.item / plan.tiles, col0 = (run.item % plan.tiles) * N;
      const int lr = unit / c.H, h = unit % c.H;
      const int len = sq.len[run.s], count = sq.count[run.s];
      if (tid < N) {
        const Place a = place_of(p, sq, run.s, lr, h, col0 + tid);
        S.place[tid] = a;
        S.ntop[tid] = -kNone;
        S.limit[tid] = a.out >= 0 && a.live ? len - count + (col0 + tid) / c.G : -1;
      }
      float x[CH / 2][8];
      float top = 0.f;
#pragma unroll
      for (int z = 0; z < CH / 2; ++z) {
        const uint32_t ws[4] = {raw[z].x, raw[z].y, raw[z].z, raw[z].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[z][2 * e] = __uint_as_float(ws[e] << 16);
          x[z][2 * e + 1] = __uint_as_float(ws[e] & 0xFFFF0000u);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = fabsf(x[z][e]);
          if (y < INFINITY) top = fmaxf(top, y);
        }
      }
      top = dev::warp_max(top);
      if (lane == 0) S.qmax[warp] = top;
      ok = all_ok(ok);
      if (!ok) break;
#pragma unroll
      for (int w = 0; w < kSoft; ++w) top = fmaxf(top, S.qmax[w]);
      int k2 = 14 - ((int)(__float_as_uint(top) >> 23) - 127);
      k2 = top == 0.f ? 0 : max(-90, min(k2, 100));
      const float up = __uint_as_float((unsigned)(127 + k2) << 23);
      const float unit_s = kUnit * __uint_as_float((unsigned)(127 - k2) << 23) * (c.scale * kLog2e);
#pragma unroll
      for (int z = 0; z < CH / 2; ++z) {
        const int col = (tid >> 4) + 16 * z;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[z][e] *= up;
          sum += x[z][e];
          if (e & 1) x[z][e] *= 0.0625f;  // the odd nibbles stand for 2^4 their code
        }
        const uint32_t at =
            base + kOffQ + (ci >> 3) * N * 128 + col * 128 + (((ci & 7) ^ (col & 7)) << 4);
        sts128(at, half2_bits(__floats2half2_rn(x[z][0], x[z][4])),
               half2_bits(__floats2half2_rn(x[z][1], x[z][5])),
               half2_bits(__floats2half2_rn(x[z][2], x[z][6])),
               half2_bits(__floats2half2_rn(x[z][3], x[z][7])));
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if ((ci & 7) == 0) {
          float *q = reinterpret_cast<float *>(&S.qs[col >> 1]) + 2 * (ci >> 3) + (col & 1);
          *q = sum * (1.f / kUnit);
        }
      }
      fence_proxy_async();
      ok = all_ok(ok);
      if (!ok) break;
      if (tid == 0) mbar_arrive(smem_u32(&S.qf));

      // rows below `full` are seen by every column that has a token
      const int first = col0 / c.G;
      const int full = first < count ? len - count + first + 1 : len;
      uint64_t z2[4 * CG], q0[4 * CG], q1[4 * CG];
#pragma unroll
      for (int e = 0; e < 4 * CG; ++e) {
        const float4 q = S.qs[c0 / 2 + e];
        q0[e] = pk2(q.x, q.y), q1[e] = pk2(q.z, q.w);
        z2[e] = 0;
      }
      for (int t = run.t0; t < run.t1; ++t) {
        const int n = i + t - run.t0, b = n & 1, cb = n % kConst, row = t * kTok + tok;
        const uint32_t ts = tm + b * 128 + c0 + lanes;
        unsigned char *const prow = smem + kOffP + b * kHalf + tok * 128;
        // the constants, S and P's place
        if (ok) ok = wait_for(at(S.cf[cb], n / kConst), at(S.sf[b], n / 2),
                              at(S.pv[b], n / 2 - 1), n < 2 ? 2 : 3);
        tc_fence_after();
        float4 key = S.key[cb][tok];
        const float2 val = S.val[cb][tok];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&S.c_free[cb]));
        if (ok && (t + 1) * kTok > full) mask_row(ts, NG, S.limit + c0, row, key);
        const float k0 = fmaxf(key.x * unit_s, 0x1p-126f);
        const uint64_t s0 = pk2(k0, k0);
        const uint64_t s1 = pk2(key.y * unit_s, key.y * unit_s);
        const uint64_t m0 = pk2(key.z * unit_s, key.z * unit_s);
        const uint64_t m1 = pk2(key.w * unit_s, key.w * unit_s);
        const uint64_t e2 = pk2(val.x, val.x), down2 = pk2(val.y, val.y);
        // Logits plus e, less the reference, of column pairs 4 k .. 4 k + 3.
        auto logits = [&](int k, bool less, const float (&a0)[8], const float (&a1)[8],
                          uint64_t (&l)[4]) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 nt = *reinterpret_cast<const float2 *>(&ntop[8 * k + 2 * e]);
            uint64_t y = less ? add2(pk2(nt.x, nt.y), e2) : e2;
            y = fma2(m1, q1[4 * k + e], y);
            y = fma2(m0, q0[4 * k + e], y);
            y = fma2(s1, pk2(a1[2 * e], a1[2 * e + 1]), y);
            l[e] = fma2(s0, pk2(a0[2 * e], a0[2 * e + 1]), y);
          }
        };
        // P of the tile against the present references; true if one is too large.
        // `again`: the references were raised; the lane's sums hold the tile already,
        // but for the columns (a bit each) of `anew`.
        auto probabilities = [&](bool again, uint32_t anew) {
          __half2 most = __float2half2_rn(0.f);
          float a0[8], a1[8];
          tmem_ld8(ts, a0);
          tmem_ld8(ts + 64, a1);
#pragma unroll
          for (int k = 0; k < CG; ++k) {
            uint64_t l[4];
            uint32_t w[4];
            tmem_landed(a0, a1);
            logits(k, true, a0, a1, l);
            if (k + 1 < CG) {  // the next columns come while these are worked on
              tmem_ld8(ts + 8 * k + 8, a0);
              tmem_ld8(ts + 64 + 8 * k + 8, a1);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float u, v;
              upk2(l[e], u, v);
              u = ex2(u), v = ex2(v);
              const __half2 ph = __floats2half2_rn(u, v);
              most = __hmax2(most, ph);
              w[e] = half2_bits(ph);
              uint64_t p2 = pk2(u, v);
              if (again) {
                const uint32_t mine = anew >> (8 * k + 2 * e);
                p2 = pk2(mine & 1 ? u : 0.f, mine & 2 ? v : 0.f);
              }
              z2[4 * k + e] = fma2(p2, down2, z2[4 * k + e]);
            }
            *reinterpret_cast<uint4 *>(prow + (((grp * CG + k) ^ (tok & 7)) << 4)) =
                make_uint4(w[0], w[1], w[2], w[3]);
          }
          fence_proxy_async();
          return __hgt(__hmax(__low2half(most), __high2half(most)), __float2half_rn(32768.f));
        };
        // The largest of column chunk k's logits over the warp's tokens, to `to`.
        auto chunk_max = [&](int k, float *to) {
          uint64_t l[4];
          float a0[8], a1[8];
          tmem_ld8(ts + 8 * k, a0);
          tmem_ld8(ts + 64 + 8 * k, a1);
          tmem_wait_ld();
          logits(k, false, a0, a1, l);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float u[2];
            upk2(l[e], u[0], u[1]);
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const unsigned o = dev::ord_bits(u[z] == u[z] ? u[z] : -INFINITY);
              const unsigned most = __reduce_max_sync(0xffffffffu, o);
              if (lane == 0)
                to[8 * k + 2 * e + z] =
                    __uint_as_float(most & 0x80000000u ? most & 0x7FFFFFFFu : ~most);
            }
          }
        };
        const bool begin = t == run.t0;
        bool grow = begin;
        if (grow && (t + 1) * kTok <= full) {
          // A run's first references: a column's largest over 32 of the tokens will
          // do, so that a warp has a quarter of the columns.
          grow = false;
          if (ok) {
#pragma unroll
            for (int k = 0; k < CG; ++k)
              if (k == wq) chunk_max(k, S.wmax[0] + c0);
          }
          ok = group_ok(ok);
          if (!ok) break;
          if (gt < NG) ntop[gt] = -fmaxf(kNone, S.wmax[0][c0 + gt]);
          ok = group_ok(ok);
          if (!ok) break;
        }
        if (ok && !grow) {
          grow = probabilities(false, 0);
          tc_fence_before();
        }
        if (bar_any(3 + grp, 16 * kSoft, grow || !ok)) {
          // Raise the references to the columns' maxima so far.
          ok = group_ok(ok);
          if (!ok) break;
#pragma unroll
          for (int k = 0; k < CG; ++k) chunk_max(k, S.wmax[wq] + c0);
          ok = group_ok(ok);
          if (!ok) break;
          if (gt < NG) {
            const float old = -ntop[gt];
            float now = old;
#pragma unroll
            for (int w = 0; w < 4; ++w) now = fmaxf(now, S.wmax[w][c0 + gt]);
            factor[gt] = ex2(old - now);
            ntop[gt] = -now;
          }
          ok = group_ok(ok);
          if (!ok) break;
          if (!begin) {
            ok = wait(S.pv[b ^ 1], (n - 1) / 2);
            tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < CG; ++k) {
              float o[8];
              tmem_ld8(to + 8 * k, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 8; ++e) o[e] *= factor[8 * k + e];
              tmem_st8(to + 8 * k, o);
            }
            tmem_wait_st();
          }
          // A sum that the tile made infinite is begun anew.  Against its token's
          // probability, 2^(128 - e) of the old reference's or more, what it held was
          // nothing: 2^15 a tile for values like that token's, and 2^74 where they are
          // next to nothing (e = -59).
          uint32_t anew = 0;
#pragma unroll
          for (int e = 0; e < 4 * CG; ++e) {
            const float2 f = *reinterpret_cast<const float2 *>(&factor[2 * e]);
            float u, v;
            upk2(z2[e], u, v);
            const bool fu = begin || u == INFINITY, fv = begin || v == INFINITY;
            anew |= (fu ? 1u : 0u) << (2 * e) | (fv ? 2u : 0u) << (2 * e);
            z2[e] = pk2(fu ? 0.f : u * f.x, fv ? 0.f : v * f.y);
          }
          probabilities(true, anew);
          tc_fence_before();
          ok = group_ok(ok);
          if (!ok) break;
        }
        if (lane == 0) mbar_arrive(smem_u32(&S.s_free[b]));
        if (gt == 0) mbar_arrive(smem_u32(&S.pf[b]));
      }
      // ---- the run's result: each group's columns
      const bool whole = run.t1 - run.t0 == run.np;
      i += run.t1 - run.t0;
      if (ok) ok = wait(S.pv[(i - 1) & 1], (i - 1) / 2);
      tc_fence_after();
      // Sums over the warp's tokens, eight columns at a time: each exchange halves a
      // lane's columns and doubles the tokens in its sums.
#pragma unroll
      for (int k = 0; k < CG; ++k) {
        float u[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) upk2(z2[4 * k + e], u[2 * e], u[2 * e + 1]);
#pragma unroll
        for (int o = 16, n = 4; n > 0; o >>= 1, n >>= 1)
#pragma unroll
          for (int e = 0; e < n; ++e) {
            const bool high = lane & o;
            const float give = high ? u[e] : u[e + n];
            u[e] = (high ? u[e + n] : u[e]) + __shfl_xor_sync(0xffffffffu, give, o);
          }
        u[0] += __shfl_xor_sync(0xffffffffu, u[0], 2);
        u[0] += __shfl_xor_sync(0xffffffffu, u[0], 1);
        if ((lane & 3) == 0) S.zsum[wq][c0 + 8 * k + (lane >> 2)] = u[0];
      }
      TileRun then = run;
      more = walk.next(then);
      if (more) load_q(then);  // on its way during what follows
      ok = all_ok(ok);
      if (!ok) break;
      if (gt < NG) {
        const int col = c0 + gt;
        const float z = (S.zsum[0][col] + S.zsum[1][col]) + (S.zsum[2][col] + S.zsum[3][col]);
        // a whole run's factors normalise, and make zeros of a column without a token
        factor[gt] = !whole ? 1.f : S.place[col].live && z != 0.f ? 1.f / z : 0.f;
        S.stat[col] = make_float2(-ntop[gt], z);
      }
      ok = group_ok(ok);
      if (!ok) break;
      const size_t call_unit = ((size_t)(p.k.s0 + run.s) * p.k.nl + lr) * c.H + h;
      // a CTA's first run may lack its beginning, its last one its end
      const int slot = blockIdx.x * 2 + (run.t0 > 0 ? 0 : 1);
      float *part = p.parts + (size_t)slot * N * (kD + 2);
      const int nan_row = S.nan_row[runs & 15][wq >> 1];  // dims 32 wq .. + 31: their group
#pragma unroll 1
      for (int k = 0; k < CG; ++k) {
        float o[8];
        tmem_ld8(to + 8 * k, o);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float f = factor[8 * k + e];
          o[e] = f != 0.f ? o[e] * f : 0.f;  // (0: a column without a token)
          if (nan_row <= S.limit[c0 + 8 * k + e]) o[e] = NAN;
        }
        if (whole) {
          long long out[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) out[e] = S.place[c0 + 8 * k + e].out;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (out[e] >= 0)
              static_cast<__nv_bfloat16 *>(p.out)[out[e] + tok] = __float2bfloat16_rn(o[e]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) __stcg(&part[(c0 + 8 * k + e) * kD + tok], o[e]);
        }
      }
      if (whole) {
        const int col = c0 + gt;
        if (gt < NG && S.place[col].out >= 0) {
          const float z = S.stat[col].y;
          const bool live = S.place[col].live && z != 0.f;
          if (live && !isfinite(z)) atomicOr(c.err, ERR_NONFINITE);
          if (p.stats)
            reinterpret_cast<float2 *>(p.stats)[call_unit * (p.n_q * c.G) + S.place[col].stat] =
                make_float2(S.stat[col].x, live ? 1.f / (z * c.G) : 0.f);
        }
      } else {
        if (gt < NG) __stcg(reinterpret_cast<float2 *>(part + N * kD) + c0 + gt, S.stat[c0 + gt]);
        const int i0 = run.at + kSwitch;  // the first tile's place
        const int w0 = i0 / plan.span, w1 = (i0 + run.np - 1) / plan.span;
        unsigned *ticket = c.ticket + unit_of(run) * kMaxTiles + run.item % plan.tiles;
        ok = all_ok(ok);
        if (!ok) break;
        if (tid == 0) S.flag = take_ticket(ticket) == (unsigned)(w1 - w0);
        ok = all_ok(ok);
        if (!ok) break;
        if (S.flag) {
          if (tid == 0) *ticket = 0;
          auto part_of = [&](int w) {
            return p.parts + ((size_t)w * 2 + (w == w0 ? 1 : 0)) * N * (kD + 2);
          };
          for (int col = warp; col < N; col += kSoft) {
            float mx = kNone, z = 0.f;
            for (int w = w0 + lane; w <= w1; w += 32) {
              const float2 y =
                  __ldcg(reinterpret_cast<const float2 *>(part_of(w) + N * kD) + col);
              const float m = fmaxf(mx, y.x);
              z = fmaf(z, ex2(mx - m), y.y * ex2(y.x - m));
              mx = m;
            }
            const float all = dev::warp_max(mx);
            z = dev::warp_sum(z * ex2(mx - all));
            if (lane == 0) S.stat[col] = make_float2(all, z);
          }
          ok = all_ok(ok);
          if (!ok) break;
          // a thread has N / 8 groups of four channels, kSome at a time
          constexpr int kSome = 2;
          for (int j0 = 0; 8 * j0 < N; j0 += kSome) {
            float4 sum[kSome];
            float mx[kSome];
#pragma unroll
            for (int j = 0; j < kSome; ++j) {
              sum[j] = make_float4(0.f, 0.f, 0.f, 0.f);
              mx[j] = S.stat[(tid + (j0 + j) * 32 * kSoft) * 4 / kD].x;
            }
#pragma unroll 4
            for (int w = w0; w <= w1; ++w) {
              const float *from = part_of(w);
#pragma unroll
              for (int j = 0; j < kSome; ++j) {
                const int at = tid + (j0 + j) * 32 * kSoft;
                add4(sum[j], __ldcg(reinterpret_cast<const float4 *>(from) + at),
                     ex2(__ldcg(from + N * kD + 2 * (at * 4 / kD)) - mx[j]));
              }
            }
#pragma unroll
            for (int j = 0; j < kSome; ++j) {
              const int at = 4 * (tid + (j0 + j) * 32 * kSoft), col = at / kD;
              finish<__nv_bfloat16>(p, S.place[col], at % kD, sum[j], S.stat[col].x,
                                    S.stat[col].y, call_unit);
            }
          }
        }
      }
      tc_fence_before();
      ok = all_ok(ok);  // the columns' arrays are free again
      if (!ok) break;
      ++runs;
      run = then;
    } while (more);
    if (!ok) give_up();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kSoft) tmem_dealloc(tm, kCols);
}

// ---- accumulated weights -----------------------------------------------------

// Adds to each row's score what the attention's columns gave it: 2^(logit - top)
// / (z G) over all columns, from their statistics.  K alone is read, once for all
// columns (kScoreCols at a time); S comes as in the attention, and as a thread has a
// token, its sum needs no other thread but the one of the other group, which has
// the odd column tiles.  K's codes are 2^-20 c here: all of their bits count.
// Bound by the exponentials' loop, about 12 instructions an element: 32 tokens of 2
// sequences of 8,191 rows (28 layers, 4 KV heads, G = 7) 320 us, 400 with mma.sync.
constexpr int kScoreTiles = 4;
constexpr int kScoreCols = kScoreTiles * kMaxN;
constexpr int kScoreThr = 32 * (kSoft + 4 + 1);
constexpr uint32_t kScoreColK = 256;  // of tensor memory: S (2 x 2 x 64), K (2 x 64)

struct __align__(16) ScoreSide {
  float4 key[2][kTok];              // s0, s1, m0, m1 of a token's key
  float4 qs[kScoreCols / 2];        // sums of q: group 0 of two columns, group 1
  float4 ref[kScoreCols / 2];       // minus the references of two columns, 1 / (z G)
  int limit[kScoreCols];
  float part[2][kTok];
  float qmax[kSoft];
  uint64_t raw_full[kRing], kf[2], k_free[2], t_free[2], sf[2], s_free[2], qf, drain;
  uint32_t tmem;
  int abort;
};
constexpr uint32_t kScoreOffRaw = kScoreCols * 256, kScoreOffSide = kScoreOffRaw + kRing * kRaw;
constexpr uint32_t kScoreSmem = kScoreOffSide + sizeof(ScoreSide);
static_assert(kScoreSmem <= 227 * 1024, "shared memory");

template <int CH>
__global__ void __launch_bounds__(kScoreThr, 1)
    tile_score_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ Seqs sq,
                      const __grid_constant__ TilePlan plan) {
  constexpr int N = 8 * CH;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char *smem = smem_raw;
  ScoreSide &S = *reinterpret_cast<ScoreSide *>(smem + kScoreOffSide);
  const View &c = p.k.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t base = smem_u32(smem);
  volatile int *abort = &S.abort;
  auto wait = [&](uint64_t &bar, int n) {
    return warp_wait(smem_u32(&bar), (uint32_t)(n & 1), abort);
  };
  auto give_up = [&]() {
    if (lane == 0) {
      if (!*abort) atomicOr(c.err, ERR_TIMEOUT);
      *abort = 1;
    }
  };
  if (warp == kSoft) tmem_alloc(smem_u32(&S.tmem), kCols);
  if (tid == 0) {
    for (int b = 0; b < kRing; ++b) mbar_init(smem_u32(&S.raw_full[b]), 1);
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&S.kf[b]), 4);
      mbar_init(smem_u32(&S.k_free[b]), 1);
      mbar_init(smem_u32(&S.t_free[b]), kSoft);
      mbar_init(smem_u32(&S.sf[b]), 1);
      mbar_init(smem_u32(&S.s_free[b]), kSoft / 2);
    }
    mbar_init(smem_u32(&S.qf), 1);
    mbar_init(smem_u32(&S.drain), 1);
    S.abort = 0;
    fence_mbar_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();

  // Spans of the list of all units' tiles; a unit's columns are taken kScoreCols at a
  // time by the CTA that has its tiles.
  Walk walk{sq, plan, p.k.nl * c.H, 0};
  TileRun first;
  const bool any = walk.first(first, p.k.n);
  pdl_begin();
  const uint32_t tm = S.tmem;
  // A run's passes over its tiles, and the column tiles of pass g.
  auto passes_of = [&](const TileRun &r) {
    return (sq.count[r.s] * c.G + kScoreTiles * N - 1) / (kScoreTiles * N);
  };
  auto chunks_of = [&](const TileRun &r, int g) {
    return min(kScoreTiles, (sq.count[r.s] * c.G - g * kScoreTiles * N + N - 1) / N);
  };
  // With one column tile the groups take turns by tile, else by column tile.
  auto owner = [](int chunks, int tile, int ch) { return (chunks == 1 ? tile : ch) & 1; };

  if (!any) {
    // no work
  } else if (warp == kSoft + 4) {
    // ---- issuer
    const uint32_t id_s = idesc_f16(kTok, N, false);
    const uint64_t dq = sdesc_sw128(base, 16, 1024);
    int i = 0, passes = 0, m[2] = {0, 0};
    bool ok = true;
    TileRun run = first;
    do {
      const int np = passes_of(run);
      for (int g = 0; g < np && ok; ++g, ++passes) {
        const int chunks = chunks_of(run, g);
        ok = wait(S.qf, passes);
        for (int t = run.t0; t < run.t1 && ok; ++t, ++i) {
          ok = wait(S.kf[i & 1], i / 2);
          for (int ch = 0; ch < chunks && ok; ++ch) {
            const int w = owner(chunks, i, ch);
            if (m[w] > 0) ok = wait(S.s_free[w], m[w] - 1);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  tc_mma_ts(tm + w * 128 + j * 64, tm + kScoreColK + (i & 1) * 64 + j * 32 + k * 8,
                            dq + (uint64_t)(((ch * 2 + j) * N * 128 + k * 32) >> 4), id_s, k > 0);
              tc_commit(smem_u32(&S.sf[w]));
              if (ch + 1 == chunks) tc_commit(smem_u32(&S.k_free[i & 1]));
            }
            __syncwarp();
            ++m[w];
          }
        }
      }
    } while (ok && walk.next(run));
    if (!ok) give_up();
    __syncwarp();
    if (elect_one()) {  // every product is done before tensor memory is freed
      volatile int never = 0;
      tc_commit(smem_u32(&S.drain));
      mbar_wait(smem_u32(&S.drain), 0, &never);
    }
  } else if (warp >= kSoft) {
    // ---- dequant: a token a thread, K's half of the raw blocks alone
    const int dt = tid - 32 * kSoft, dw = warp - kSoft;
    int i = 0, issued = 0;
    bool ok = true, more = true;
    TileRun ahead = first, run = first;
    int ahead_t = first.t0, ahead_g = 0;
    auto skip_empty = [&]() {  // runs without a token have no pass
      while (more && passes_of(ahead) == 0) {
        more = walk.next(ahead);
        ahead_t = ahead.t0;
      }
    };
    auto load_next = [&]() {  // dt == 0
      if (!more) return;
      const int nb = min(kTileBlocks, blocks_of(sq.len[ahead.s]) - ahead_t * kTileBlocks);
      const uint32_t bar = smem_u32(&S.raw_full[issued % kRing]);
      constexpr uint32_t kCodes = kBlock * kD / 2, kMeta = kBlock * (kD / kGroup) * 4;
      mbar_expect_tx(bar, (uint32_t)nb * (kCodes + kMeta));
      const int unit = ahead.item;
      const uint8_t *at =
          c.blocks + unit_at(c, p.k.s0 + ahead.s, p.k.lb, unit / c.H, unit % c.H) * c.nb *
                         (size_t)block_bytes(kD) +
          (size_t)ahead_t * kRaw;
      const uint32_t to = base + kScoreOffRaw + (issued % kRing) * kRaw;
      for (int b = 0; b < nb; ++b) {
        bulk_load(to + b * block_bytes(kD), at + b * block_bytes(kD), kCodes, bar);
        bulk_load(to + b * block_bytes(kD) + km_off(kD), at + b * block_bytes(kD) + km_off(kD),
                  kMeta, bar);
      }
      ++issued;
      if (++ahead_t == ahead.t1) {
        ahead_t = ahead.t0;
        if (++ahead_g == passes_of(ahead)) {
          ahead_g = 0;
          more = walk.next(ahead);
          ahead_t = ahead.t0;
          skip_empty();
        }
      }
    };
    if (dt == 0) {
      skip_empty();
      for (int j = 0; j < kRing; ++j) load_next();
    }
    do {
      const int len = sq.len[run.s], np = passes_of(run);
      for (int g = 0; g < np && ok; ++g)
        for (int t = run.t0; t < run.t1; ++t, ++i) {
          const int b = i & 1, rb = i % kRing;
          const unsigned char *blk =
              smem + kScoreOffRaw + rb * kRaw + (dt / kBlock) * block_bytes(kD);
          ok = ok && wait(S.raw_full[rb], i / kRing) &&
               (i < 2 || (wait(S.t_free[b], i / 2 - 1) && wait(S.k_free[b], i / 2 - 1)));
          ok = !bar_any(1, 128, !ok);
          if (!ok) break;
          if (dt == 0 && i > 0) load_next();  // in the place of tile i - 1
          tc_fence_after();
          const int r = dt % kBlock;
          uint2 km = *reinterpret_cast<const uint2 *>(blk + km_off(kD) + r * 8);
          if (t * kTok + dt >= len) km = make_uint2(0, 0);
          S.key[b][dt] = make_float4(s_of(km.x), s_of(km.y), m_of(km.x), m_of(km.y));
          uint4 w[4];
#pragma unroll
          for (int t4 = 0; t4 < 4; ++t4)
            w[t4] = *reinterpret_cast<const uint4 *>(blk + k_off() + r * (kD / 2) +
                                                     k_chunk(r, t4) * 16);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t o[32];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              const uint4 &c4 = w[x >> 1];
              const uint32_t v = j == 0 ? (x & 1 ? c4.y : c4.x) : (x & 1 ? c4.w : c4.z);
              fields<kEven>(v, o + 4 * x);
            }
            tmem_st32(tm + ((uint32_t)(dw * 32) << 16) + kScoreColK + b * 64 + j * 32, o);
          }
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&S.kf[b]));
        }
    } while (ok && walk.next(run));
    if (!ok) give_up();
    if (dt == 0) {  // every copy lands before the shared memory is given back
      volatile int never = 0;
      for (int j = max(0, issued - kRing); j < issued; ++j)
        mbar_wait(smem_u32(&S.raw_full[j % kRing]), (uint32_t)((j / kRing) & 1), &never);
    }
  } else {
    // ---- sums
    const int wq = warp & 3, grp = warp >> 2, tok = wq * 32 + lane;
    const uint32_t ts = tm + grp * 128 + ((uint32_t)(wq * 32) << 16);
    auto all_ok = [&](bool ok) { return !bar_any(2, 32 * kSoft, !ok); };
    int i = 0, m = 0;
    bool ok = true, more = true;
    TileRun run = first;
    do {
      const int lr = run.item / c.H, h = run.item % c.H;
      const int len = sq.len[run.s], count = sq.count[run.s];
      const size_t call_unit = ((size_t)(p.k.s0 + run.s) * p.k.nl + lr) * c.H + h;
      float *score = c.score + unit_at(c, p.k.s0 + run.s, p.k.lb, lr, h) * c.sstride;
      const int np = passes_of(run);
      for (int g = 0; g < np; ++g) {
        const int chunks = chunks_of(run, g), col0 = g * kScoreTiles * N;
        // ---- the pass's queries, scaled by one power of two for all columns
        if (tid < chunks * N) {
          const int col = col0 + tid, k = tid >> 1;
          const Place a = place_of(p, sq, run.s, lr, h, col);
          const bool live = a.out >= 0 && a.live;
          const float2 st = live ? reinterpret_cast<const float2 *>(
                                       p.stats)[call_unit * (p.n_q * c.G) + a.stat]
                                 : make_float2(-kNone, 0.f);
          S.limit[tid] = live ? len - count + col / c.G : -1;
          float *ref = reinterpret_cast<float *>(&S.ref[k]) + (tid & 1);
          ref[0] = -st.x;
          ref[2] = st.y;
        }
        float top = 0.f;
        const int ci = tid & 15;
        auto load_q = [&](int col, float (&x)[8]) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = 0.f;
          const Place a = place_of(p, sq, run.s, lr, h, col0 + col);
          if (a.out < 0 || !a.live) return;
          const uint4 w = *reinterpret_cast<const uint4 *>(
              static_cast<const __nv_bfloat16 *>(p.q) + a.out + 8 * ci);
          const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(ws[e] << 16);
            x[2 * e + 1] = __uint_as_float(ws[e] & 0xFFFF0000u);
          }
        };
#pragma unroll 2
        for (int col = tid >> 4; col < chunks * N; col += 16) {
          float x[8];
          load_q(col, x);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (fabsf(x[e]) < INFINITY) top = fmaxf(top, fabsf(x[e]));
        }
        top = dev::warp_max(top);
        if (lane == 0) S.qmax[warp] = top;
        ok = all_ok(ok);
        if (!ok) break;
#pragma unroll
        for (int w = 0; w < kSoft; ++w) top = fmaxf(top, S.qmax[w]);
        int k2 = 14 - ((int)(__float_as_uint(top) >> 23) - 127);
        k2 = top == 0.f ? 0 : max(-90, min(k2, 100));
        const float up = __uint_as_float((unsigned)(127 + k2) << 23);
        constexpr float kEvenUnit = field_unit(kEven);
        const float unit_s =
            kEvenUnit * __uint_as_float((unsigned)(127 - k2) << 23) * (c.scale * kLog2e);
#pragma unroll 2
        for (int col = tid >> 4; col < chunks * N; col += 16) {
          float x[8], sum = 0.f;
          load_q(col, x);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] *= up;
            sum += x[e];
          }
          const int ch = col / N, cc = col % N;
          sts128(base + (ch * 2 + (ci >> 3)) * N * 128 + cc * 128 + (((ci & 7) ^ (cc & 7)) << 4),
                 half2_bits(__floats2half2_rn(x[0], x[4])),
                 half2_bits(__floats2half2_rn(x[1], x[5])),
                 half2_bits(__floats2half2_rn(x[2], x[6])),
                 half2_bits(__floats2half2_rn(x[3], x[7])));
#pragma unroll
          for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          if ((ci & 7) == 0) {
            float *q = reinterpret_cast<float *>(&S.qs[col >> 1]) + 2 * (ci >> 3) + (col & 1);
            *q = sum * (1.f / kEvenUnit);
          }
        }
        fence_proxy_async();
        ok = all_ok(ok);
        if (!ok) break;
        if (tid == 0) mbar_arrive(smem_u32(&S.qf));

        // rows up to the first of the pass's tokens are seen by all its columns
        const int all_rows = len - count + col0 / c.G + 1;
        for (int t = run.t0; t < run.t1; ++t, ++i) {
          const int b = i & 1, row = t * kTok + tok;
          const bool mask = (t + 1) * kTok > all_rows;
          if (ok) ok = wait(S.kf[b], i / 2);
          const float4 key = S.key[b][tok];
          uint64_t sum[2] = {0, 0};
          bool mine = false;
#pragma unroll 1
          for (int ch = 0; ch < chunks; ++ch) {
            if (owner(chunks, i, ch) != grp) continue;
            mine = true;
            if (ok) ok = wait(S.sf[grp], m);
            if (!ok) break;
            ++m;
            tc_fence_after();
            const float4 *qs = S.qs + ch * (N / 2), *ref = S.ref + ch * (N / 2);
            float4 y = key;
            if (mask) mask_row(ts, N, S.limit + ch * N, row, y);
            const float k0 = fmaxf(y.x * unit_s, 0x1p-126f), k1 = y.y * unit_s;
            const uint64_t s0 = pk2(k0, k0), s1 = pk2(k1, k1);
            const uint64_t m0 = pk2(y.z * unit_s, y.z * unit_s);
            const uint64_t m1 = pk2(y.w * unit_s, y.w * unit_s);
            float a0[8], a1[8];
            tmem_ld8(ts, a0);
            tmem_ld8(ts + 64, a1);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
              uint64_t l[4], inv[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float4 f = ref[4 * k + e], q = qs[4 * k + e];
                inv[e] = pk2(f.z, f.w);
                l[e] = fma2(m1, pk2(q.z, q.w), fma2(m0, pk2(q.x, q.y), pk2(f.x, f.y)));
              }
              tmem_landed(a0, a1);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                l[e] = fma2(s0, pk2(a0[2 * e], a0[2 * e + 1]),
                            fma2(s1, pk2(a1[2 * e], a1[2 * e + 1]), l[e]));
              if (k + 1 < CH) {
                tmem_ld8(ts + 8 * k + 8, a0);
                tmem_ld8(ts + 64 + 8 * k + 8, a1);
              }
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float u, v;
                upk2(l[e], u, v);
                sum[e & 1] = fma2(pk2(ex2(u), ex2(v)), inv[e], sum[e & 1]);
              }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&S.s_free[grp]));
          }
          float u, v;
          upk2(add2(sum[0], sum[1]), u, v);
          float add = u + v;
          if (chunks > 1) {
            if (grp == 1) S.part[b][tok] = add;
            ok = all_ok(ok);
            if (!ok) break;
            if (grp == 0) add += S.part[b][tok];
            mine = grp == 0;
          }
          if (mine && row < len) score[row] += add;
          if (lane == 0) mbar_arrive(smem_u32(&S.t_free[b]));
        }
        ok = all_ok(ok);  // the pass's arrays are free again
        if (!ok) break;
      }
      if (ok) more = walk.next(run);
    } while (ok && more);
    if (!ok) give_up();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kSoft) tmem_dealloc(tm, kCols);
}

int tile_n(const View &c, int n_q) {
  const long long rows = (long long)n_q * c.G, tiles = (rows + kMaxN - 1) / kMaxN;
  return (int)(((rows + tiles - 1) / tiles + 15) / 16 * 16);
}
long long col_tiles(const View &c, int n_q) {
  return ((long long)n_q * c.G + tile_n(c, n_q) - 1) / tile_n(c, n_q);
}

}  // namespace

// More than 24 query rows a unit.  Over 8 sequences of 8,192 rows (28 layers, 4 KV
// heads) 28 rows take 428 us here and 790 in the kernel for fewer rows; 21 rows 426
// and 405; 14 rows 394 and 281.  Over 64 sequences of 512: 28 rows 443 and 699, 21
// rows 440 and 404; over one of 4,099, 21 rows 41.0 and 42.6, 14 rows 36.6 and 31.3.
bool tile_applies(const View &c, int n_q) {
  return c.d == kD && c.io_bf16 && c.out_bf16 && (long long)n_q * c.G > 24;
}

size_t tile_part_floats(const View &c, int nl, int n_q) {
  const long long tiles = col_tiles(c, n_q);
  if (tiles > kMaxTiles) return 0;
  const size_t all = (size_t)std::min(c.S, kMaxSeqs) * nl * c.H * tiles *
                     ((c.nb + kTileBlocks - 1) / kTileBlocks);
  return 2 * std::min<size_t>(kTileGrid, all) * tile_n(c, n_q) * (kD + 2);
}

template <int CH>
cudaError_t prepare_ch() {
  auto kern = tile_attend_kernel<CH>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  // (the kernel's split of the registers counts on as many at launch)
  cudaFuncAttributes attr;
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&attr, kern);
  if (e == cudaSuccess && attr.numRegs != kRegs) e = cudaErrorInvalidConfiguration;
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(tile_score_kernel<CH>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             kScoreSmem);
  return e;
}
cudaError_t prepare_tile() {
  cudaError_t e = prepare_ch<4>();
  if (e == cudaSuccess) e = prepare_ch<6>();
  if (e == cudaSuccess) e = prepare_ch<8>();
  return e;
}

template <int CH>
cudaError_t launch_ch(const AttendParams &p, const Seqs &q, const Device &dev,
                      cudaStream_t stream) {
  const View &c = p.k.c;
  auto kern = tile_attend_kernel<CH>;
  const int sms = std::min(dev.sms, kTileGrid);
  TilePlan plan;
  const long long tiles = col_tiles(c, p.n_q), per_seq = (long long)p.k.nl * c.H * tiles;
  if (tiles > INT32_MAX || per_seq > INT32_MAX) return cudaErrorInvalidValue;
  plan.tiles = (int)tiles;
  long long total = 0;
  for (int i = 0; i < p.k.n; ++i) {
    plan.base[i] = (int32_t)total;
    total += per_seq * (kSwitch + (blocks_of(q.len[i]) + kTileBlocks - 1) / kTileBlocks);
  }
  plan.base[p.k.n] = (int32_t)total;
  long long grid;
  if (tiles <= kMaxTiles && total <= INT32_MAX) {
    plan.span = (int32_t)std::max<long long>(kSwitch + 1, (total + sms - 1) / sms);
    grid = (total + plan.span - 1) / plan.span;
  } else {
    plan.span = 0;
    grid = per_seq * p.k.n;
  }
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  return launch_pdl(kern, dim3((unsigned)grid), dim3(kThr), kSmem, stream, p, q, plan);
}

template <int CH>
cudaError_t launch_score_ch(const AttendParams &p, const Seqs &q, const Device &dev,
                            cudaStream_t stream) {
  const View &c = p.k.c;
  auto kern = tile_score_kernel<CH>;
  const int sms = dev.sms;
  TilePlan plan;
  plan.tiles = 1;
  long long total = 0;
  for (int i = 0; i < p.k.n; ++i) {
    plan.base[i] = (int32_t)std::min<long long>(total, INT32_MAX);
    total += (long long)p.k.nl * c.H *
             (kSwitch + (blocks_of(q.len[i]) + kTileBlocks - 1) / kTileBlocks);
  }
  if (total > INT32_MAX) return cudaErrorInvalidValue;
  plan.base[p.k.n] = (int32_t)total;
  plan.span = (int32_t)std::max<long long>(kSwitch + 1, (total + sms - 1) / sms);
  return launch_pdl(kern, dim3((unsigned)((total + plan.span - 1) / plan.span)), dim3(kScoreThr),
                    kScoreSmem, stream, p, q, plan);
}

cudaError_t launch_tile_scores(const AttendParams &p, const Seqs &q, const Device &dev,
                               cudaStream_t stream) {
  switch (tile_n(p.k.c, p.n_q)) {
    case 32: return launch_score_ch<4>(p, q, dev, stream);
    case 48: return launch_score_ch<6>(p, q, dev, stream);
    default: return launch_score_ch<8>(p, q, dev, stream);
  }
}

cudaError_t launch_tile_attend(const AttendParams &p, const Seqs &q, const Device &dev,
                               cudaStream_t stream) {
  switch (tile_n(p.k.c, p.n_q)) {
    case 32: return launch_ch<4>(p, q, dev, stream);
    case 48: return launch_ch<6>(p, q, dev, stream);
    default: return launch_ch<8>(p, q, dev, stream);
  }
}

}  // namespace kv4
}  // namespace kvr
