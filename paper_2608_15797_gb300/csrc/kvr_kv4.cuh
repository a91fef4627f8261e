// kvr_kv4.cuh -- the layout of the 4-bit cache (include/kvr.h, kvr_kv4_*) and
// the arithmetic that defines it, shared by the kernels that write and read it.
//
// A unit's rows are held in blocks of 32 tokens, each one contiguous piece of
// memory, so that one bulk copy fetches all that a step of the attention needs:
//   K codes [32 tokens][d/2 B] | V codes [16 token pairs][d B]
//   | K (m, s) [32][d/64] | V (m, s) [32][d/64]      (bf16 pairs, m low)
// Within them the codes lie where tensor-core fragments want them, so that a
// thread loads its fragment's words whole and masks give 16-bit pairs:
//  - K word: 8 channels of one token, channel 64 j + 16 t + 8 i + e of a row
//    in chunk t (of four), word 2 j + i, bits 4 e .. 4 e + 3.  Thread t of a
//    fragment's row owns chunk t; its words 2 j, 2 j + 1 belong to group j.  Chunks
//    lie permuted by the row (k_chunk), so that threads that read one chunk of
//    eight neighbouring rows hit different banks.
//  - V word: 4 channels of two tokens (even token low half): the row of chunk c
//    (of eight), word w holds channels 32 w + c + {0, 16, 8, 24}, in order of
//    bits.  Chunks lie permuted by the pair's index (v_chunk), so that the
//    eight threads of one wavefront hit different banks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace kvr {
namespace kv4 {

constexpr int kGroup = 64;   // channels that share a scale
constexpr int kBlock = 32;   // tokens of a block
constexpr int kMaxSeqs = 128;  // sequences of one launch
constexpr int kPiece = 4;      // blocks of a piece of a unit, at most
constexpr int kMaxTiles = 16;  // query tiles of a unit whose rows are split over CTAs

__host__ __device__ constexpr int k_off() { return 0; }
__host__ __device__ constexpr int v_off(int d) { return kBlock * d / 2; }
__host__ __device__ constexpr int km_off(int d) { return kBlock * d; }
__host__ __device__ constexpr int vm_off(int d) {
  return kBlock * d + kBlock * (d / kGroup) * 4;
}
__host__ __device__ constexpr int block_bytes(int d) {
  return kBlock * d + 2 * kBlock * (d / kGroup) * 4;
}

// Device view of a 4-bit cache.  A unit u = (s * L + l) * H + h.
struct View {
  uint8_t *blocks;    // [u][nb][block_bytes(d)]
  float *score;       // [u][sstride]
  unsigned *err;      // device error word
  unsigned *ticket;   // [u][kMaxTiles] arrivals of a split unit, 0 between calls
  int S, L, H, G, d, cap;
  int nb;             // blocks of a unit
  int sstride;
  float scale;
  int io_bf16, out_bf16;
};

// What a launch needs of its sequences, [0, n) of the launch.
struct Seqs {
  int32_t len[kMaxSeqs];    // rows, with the call's tokens
  int32_t count[kMaxSeqs];  // the call's tokens
};

// Physical chunk of chunk c in the line of token pair p.
template <int D>
__device__ __forceinline__ int v_chunk(int p, int c) {
  return D == 128 ? c ^ ((p & 3) << 1) : c ^ (((p >> 1) & 1) << 2);
}

// Physical chunk of chunk t of row r.
__device__ __forceinline__ int k_chunk(int r, int t) { return t ^ ((r >> 1) & 3); }

// Byte of the block, and whether it is the high nibble, of a channel's code.
template <int D>
__device__ __forceinline__ int k_byte(int r, int x, int &hi) {
  const int j = x >> 6, t = (x >> 4) & 3, i = (x >> 3) & 1, e = x & 7;
  hi = e & 1;
  return k_off() + r * (D / 2) + k_chunk(r, t) * (D / 8) + (2 * j + i) * 4 + (e >> 1);
}
// 16-bit half (byte offset of the block) that holds channels
// 32 w + c + {0, 16, 8, 24} of token r.
template <int D>
__device__ __forceinline__ int v_half(int r, int w, int c) {
  const int p = r >> 1;
  return v_off(D) + p * D + v_chunk<D>(p, c) * (D / 8) + w * 4 + (r & 1) * 2;
}

__device__ __forceinline__ float m_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float s_of(uint32_t w) {
  return __uint_as_float(w & 0xFFFF0000u);
}

// A group's (m, s) from its least and greatest value; `fine`: every value is
// finite.  Each rounding is written out: the definition is fp32 arithmetic,
// and no fused multiply-add may change it.  `flat`: the group has one value
// (s is 0 by definition) or none (m = NaN), and every code is 0.  What is held
// as its s then multiplies 0 alone; it is |m| / 8, so that the attention can
// write a value as s (c + m / s) for every group.
__device__ __forceinline__ uint32_t group_meta(float lo, float hi, bool fine, bool &flat) {
  const uint32_t least = 0x0080u;  // 2^-126
  flat = true;
  if (!fine) return 0x7FC0u | (least << 16);
  const float f = 1.0f / 15.0f;
  const float s = __fsub_rn(__fmul_rn(hi, f), __fmul_rn(lo, f));
  const uint32_t mb = __bfloat16_as_ushort(__float2bfloat16_rn(lo));
  uint32_t sb = __bfloat16_as_ushort(__float2bfloat16_rn(s));
  flat = sb == 0;
  if (flat) {
    sb = mb & 0x7FFFu;                      // |m|
    sb = sb > 0x0180u + least ? sb - 0x0180u : least;  // three exponents down
  }
  return mb | (sb << 16);
}
// The code of x, 0..15, by the definition's division.
__device__ __forceinline__ uint32_t code_of(float x, uint32_t meta, bool flat) {
  if (flat) return 0;
  const float c = rintf(__fdiv_rn(__fsub_rn(x, m_of(meta)), s_of(meta)));
  return (uint32_t)fminf(fmaxf(c, 0.f), 15.f);
}
// Unit x in [0, n * nl * H) of a launch over sequences [s0, s0 + n) and layers
// [lb, lb + nl): its index in the cache.
__device__ __forceinline__ size_t unit_at(const View &c, int s, int lb, int lr, int h) {
  return ((size_t)s * c.L + lb + lr) * c.H + h;
}
__device__ __forceinline__ uint8_t *block_at(const View &c, size_t u, int r) {
  return c.blocks + (u * c.nb + r / kBlock) * (size_t)block_bytes(c.d);
}

// One launch's share of a call over sequences [s0, s0 + n): layers
// [lb, lb + nl).
struct Call {
  View c;
  int s0, n, lb, nl;
};

// kvr_kv4.cu.  Strides in elements; `tokens` rows a sequence at most, the new
// rows of sequence s being [len - count, len).
struct RowStrides {
  long long seq, layer, token, head;
};
cudaError_t launch_append(const Call &k, const Seqs &q, int tokens, const void *key,
                          const void *val, const RowStrides &st, cudaStream_t stream);

// kvr_kv4_attend.cu
struct AttendParams {
  Call k;
  int n_q;
  const void *q;
  void *out;
  float *stats;  // [unit of the call][n_q * G][2], or null: no scores
  float *parts;  // partial results
};
// What launches need to know of the handle's device, which is the current one when
// the handle is made.  (Limits of shared memory are raised then too, as they belong
// to the device.)
struct Device {
  int sms;
  int resident[3];  // CTAs of the kernel for few query rows, by tiles of 8 columns
};
cudaError_t prepare_attend(const View &c, Device *dev);
cudaError_t launch_attend(const AttendParams &p, const Seqs &q, const Device &dev,
                          cudaStream_t stream, int *launches);
// kvr_kv4_tile.cu: the same, on 5th-generation tensor cores, where it applies
// (bf16, d = 128, more than a few query rows a unit), and the scores' sums.
bool tile_applies(const View &c, int n_q);
size_t tile_part_floats(const View &c, int nl, int n_q);
cudaError_t prepare_tile();
cudaError_t launch_tile_attend(const AttendParams &p, const Seqs &q, const Device &dev,
                               cudaStream_t stream);
cudaError_t launch_tile_scores(const AttendParams &p, const Seqs &q, const Device &dev,
                               cudaStream_t stream);
// Floats of workspace: statistics of every query row, then partial results.
size_t attend_stat_floats(const View &c, int nl, int n_q);
size_t attend_part_floats(const View &c, int nl, int n_q);

}  // namespace kv4
}  // namespace kvr
