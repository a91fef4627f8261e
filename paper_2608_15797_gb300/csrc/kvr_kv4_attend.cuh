// kvr_kv4_attend.cuh -- what the kernels of the 4-bit cache's attention share: codes
// as 16-bit operands, how a column (a token's query head) is addressed, and how its
// partial results are joined and written.
#pragma once

#include <cuda_fp16.h>

#include "kvr_device.cuh"
#include "kvr_internal.h"
#include "kvr_kv4.cuh"
#include "kvr_ptx.cuh"

namespace kvr {
namespace kv4 {
namespace {

using namespace ptx;

constexpr float kNone = -1e30f; // a maximum over nothing
constexpr float kLog2e = 1.4426950408889634f;

// 16-bit pairs of codes: field f (0..3) of a word, f + 4 in the high half.
//  kRough: c 2^-24 (f even) or c 2^-20 (f odd): the fewest instructions, but the
//    tensor core aligns products by their operands' exponents, a subnormal
//    counting as 2^-14, and cuts below 2^-24 of the largest; a leading bit at
//    2^-21 costs up to seven bits of that.  Enough for logits of bf16 outputs.
//  kEven: c 2^-20; as exact as normal numbers.
//  kCentred: c - 8.
enum Codes { kRough, kEven, kCentred };
template <Codes M>
__device__ __forceinline__ void fields(uint32_t x, uint32_t *f) {
  if (M == kCentred) {
    const __half2 off = __float2half2_rn(1032.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t y = ((x >> (4 * i)) & 0x000F000Fu) | 0x64006400u;  // 1024 + c
      const __half2 z = __hsub2(*reinterpret_cast<__half2 *>(&y), off);
      f[i] = *reinterpret_cast<const uint32_t *>(&z);
    }
  } else if (M == kRough) {
    const uint32_t y = x >> 8;
    f[0] = x & 0x000F000Fu;
    f[1] = x & 0x00F000F0u;
    f[2] = y & 0x000F000Fu;
    f[3] = y & 0x00F000F0u;
  } else {
    f[0] = (x << 4) & 0x00F000F0u;
    f[1] = x & 0x00F000F0u;
    f[2] = (x >> 4) & 0x00F000F0u;
    f[3] = (x >> 8) & 0x00F000F0u;
  }
}
// What field f of 1 stands for, inverted.
__host__ __device__ constexpr float field_unit(Codes m) {
  return m == kCentred ? 1.f : m == kEven ? 0x1p20f : 0x1p24f;
}

__host__ __device__ inline int blocks_of(int len) {
  return len > kBlock ? (len + kBlock - 1) / kBlock : 1;
}

// A whole warp's bounded wait for phases of up to three barriers, each asked by one
// lane: 32 lanes' questions are as many turns at the barrier, and lanes that ask one
// barrier after the other wait for as many answers.  No branch parts the lanes.
// (Three waits a tile of the tensor-memory kernel's softmax took 600 cycles when all
// lanes asked.)
__device__ __forceinline__ bool ask(uint32_t bar, uint32_t parity, bool mine) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %3, 0;\n\tsetp.eq.b32 p, %3, 0;\n\t"
      "@q mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity), "r"((uint32_t)mine)
      : "memory");
  return ok != 0;
}
struct Phase {
  uint32_t bar, parity;
};
__device__ __forceinline__ bool warp_wait(Phase a, Phase b, Phase c, int n, volatile int *abort) {
  const int lane = threadIdx.x & 31;
  const uint32_t bar = lane == 0 ? a.bar : lane == 1 ? b.bar : c.bar;
  const uint32_t parity = lane == 0 ? a.parity : lane == 1 ? b.parity : c.parity;
  if (!__all_sync(0xffffffffu, ask(bar, parity, lane < n))) {
    const uint64_t t0 = global_ns();
    while (!__all_sync(0xffffffffu, ask(bar, parity, lane < n)))
      if (__any_sync(0xffffffffu, *abort || global_ns() - t0 > kWaitNs)) return false;
  }
  __syncwarp();
  return true;
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abort) {
  const Phase a{bar, parity};
  return warp_wait(a, a, a, 1, abort);
}

// Where a column's result goes.
struct Place {
  long long out;  // element of `out`, or -1: no such column
  int stat;       // index of its statistics (its row in the unit)
  int live;       // 0: no token, zeros
};
__device__ __forceinline__ Place place_of(const AttendParams &p, const Seqs &sq, int s, int lr,
                                          int h, int col) {
  const View &c = p.k.c;
  Place a;
  const int tok = col / c.G;
  const size_t call = (size_t)(p.k.s0 + s) * p.k.nl + lr;
  a.out = tok < p.n_q ? (long long)((((call * p.n_q + tok) * c.H + h) * c.G + (col - tok * c.G)) *
                                    c.d)
                      : -1;
  a.stat = col;
  a.live = tok < sq.count[s];
  return a;
}
// Four channels of a finished column, normalised and written.
template <typename O>
__device__ __forceinline__ void finish(const AttendParams &p, const Place &a, int x, float4 o,
                                       float top, float z, size_t unit) {
  if (a.out < 0) return;
  const bool live = a.live && z != 0.f;
  const float f = live ? 1.f / z : 0.f;
  if (!live) o = make_float4(0.f, 0.f, 0.f, 0.f);
  o.x *= f, o.y *= f, o.z *= f, o.w *= f;
  O *to = static_cast<O *>(p.out) + a.out + x;
  if (sizeof(O) == 2)
    *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
  else
    *reinterpret_cast<float4 *>(to) = o;
  if (x == 0) {
    if (live && !isfinite(z)) atomicOr(p.k.c.err, ERR_NONFINITE);
    if (p.stats)
      reinterpret_cast<float2 *>(p.stats)[unit * (p.n_q * p.k.c.G) + a.stat] =
          make_float2(top, f / p.k.c.G);
  }
}
__device__ __forceinline__ void add4(float4 &a, const float4 &b, float f) {
  a.x = fmaf(b.x, f, a.x), a.y = fmaf(b.y, f, a.y);
  a.z = fmaf(b.z, f, a.z), a.w = fmaf(b.w, f, a.w);
}
// Adds one to *at, behind all the CTA has written before the barrier that precedes
// it and ahead of what it reads after the one that follows.
__device__ __forceinline__ unsigned take_ticket(unsigned *at) {
  unsigned old;
  asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(old) : "l"(at) : "memory");
  return old;
}

}  // namespace
}  // namespace kv4
}  // namespace kvr
