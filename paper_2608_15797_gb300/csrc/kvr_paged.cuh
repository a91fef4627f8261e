// kvr_paged.cuh -- the paged full-context cache (include/kvr.h, kvr_paged_*):
// its device view, shared by the kernels that plan, fill and read it.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace kvr {
namespace paged {

constexpr int kTile = 16;   // rows that a warp of the attention takes at a time
constexpr int kHeads = 8;   // query heads of a unit, at most

// Device view.  A page holds page_rows rows of every layer and KV head; a row
// of layer l, head h in page p is row ((l * n_pages + p) * H + h) * P + r.
struct View {
  uint8_t *K, *V;    // [L][n_pages][H][P][d]
  uint8_t *bounds;   // [L][n_pages][H][2][d]: least and greatest keys of full pages
  int32_t *table;    // [S][tstride], -1 behind a sequence's pages
  int32_t *len;      // [S]
  int32_t *from;     // [S] rows that the last plan kept: its new tokens follow them
  int32_t *first;    // [S] where in the stack the last plan's new pages of s begin
  int32_t *tiles;    // [S + 1] tiles of the sequences before s
  int32_t *stack;    // [n_pages] free pages, the next one to go at free[0] - 1
  int32_t *free;     // [0]: how many; [1]: whether the last plan was carried out
  unsigned *ticket;  // [CTAs] arrivals of a unit split over CTAs, 0 between calls
  unsigned *err;     // device error word
  int S, L, H, G, d, P, n_pages, tstride;
  int psh;           // log2(P)
  float scale;
  int io_bf16, out_bf16;
};

// What is read of a sequence: its table (or, page by page, the list chosen for a
// unit), how many rows that stands for, and the tiles of those before it.
struct Source {
  const int32_t *pages;  // pool pages
  long long seq_stride, unit_stride;
  const int32_t *rows;   // [S]
  const int32_t *tiles;  // [S + 1]
};

// One launch of the attention over layers [lb, lb + nl).
struct AttendParams {
  View c;
  Source src;
  int lb, nl;
  const void *q;   // [S][nl][H * G][d]
  void *out;
  float *parts;    // [2 * CTAs][part_floats(d)]
  long long most;  // tiles that the call can have, whatever the lengths
  long long longest;  // and one unit of it
};
__host__ __device__ constexpr int part_floats(int d) { return kHeads * d + 2 * kHeads; }

// What launches need to know of the handle's device, which is the current one when
// the handle is made (limits of shared memory are raised then too).
struct Device {
  int sms;
  int clusters[2];  // of 16 and of 8 CTAs, that run at once
};
// CTAs of a launch.
constexpr int kMostCtas = 1024;
int attend_ctas(const View &c, const Device &dev);
cudaError_t prepare_attend(const View &c, Device *dev);
cudaError_t launch_attend(const AttendParams &p, const Device &dev, cudaStream_t st);

// The choice of pages over layers [lb, lb + nl): scores, then each unit's list of
// pool pages in ascending order of position, and what the attention reads of it.
struct SelectParams {
  View c;
  int lb, nl;
  const void *q;
  int budget, window;
  int keep;           // pages of a list
  float2 *score;      // [unit of the call][sstride]: score, bound of its error
  int sstride;        // even
  int held;           // keys of a unit that are held on chip, even
  int32_t *list;      // [unit][keep]
  int32_t *rows;      // [S]
  int32_t *tiles;     // [S + 1]
  int32_t *chosen;    // [unit][budget + window] or null: positions, then -1
};
cudaError_t prepare_select(const View &c);
cudaError_t launch_select(const SelectParams &p, int sms, cudaStream_t st, int *launches);

__host__ __device__ __forceinline__ long long pool_row(const View &c, int l, int page, int h) {
  return (((long long)l * c.n_pages + page) * c.H + h) << c.psh;
}

}  // namespace paged
}  // namespace kvr
