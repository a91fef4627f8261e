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

namespace kvr {
namespace kv4 {
namespace {

template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}

// Quantise the new rows.  One warp a (sequence, layer, head, token) and side
// (key or value): its lanes hold D / 32 neighbouring channels each, agree on the
// groups' extremes by shuffles, leave the codes in shared memory and write the
// row's words from there.
template <typename T, int D>
__global__ void __launch_bounds__(256)
    append_kernel(const Call k, const __grid_constant__ Seqs q, int tokens, const T *key,
                  const T *val, RowStrides st) {
  pdl_begin();
  const View &c = k.c;
  __shared__ uint8_t s_code[8][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 8 + warp;  // [seq][layer][token][head][side]
  const int side = (int)(row & 1);
  const int h = (int)((row >> 1) % c.H);
  const long long rest = (row >> 1) / c.H;
  const int t = (int)(rest % tokens);
  const int lr = (int)(rest / tokens % k.nl);
  const long long s = rest / tokens / k.nl;
  if (s >= k.n || t >= q.count[s]) return;
  constexpr int E = D / 32;
  const T *src = (side ? val : key) + (s + k.s0) * st.seq + lr * st.layer + t * st.token +
                 h * st.head + lane * E;
  float x[E];
  bool fine = true;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] = dev::to_f(src[e]);
    fine &= isfinite(x[e]);
  }
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int e = 1; e < E; ++e) {
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
  }
  constexpr int kLanes = kGroup / E;  // lanes of a group: 16 or 32
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    fine &= __shfl_xor_sync(0xffffffffu, (int)fine, o) != 0;
  }
  bool flat;
  const uint32_t meta = group_meta(lo, hi, fine, flat);
#pragma unroll
  for (int e = 0; e < E; ++e) s_code[warp][lane * E + e] = (uint8_t)code_of(x[e], meta, flat);
  __syncwarp();
  const int r = q.len[s] - q.count[s] + t, rb = r % kBlock;
  const size_t u = unit_at(c, k.s0 + (int)s, k.lb, lr, h);
  uint8_t *block = block_at(c, u, r);
  if (lane % kLanes == 0)
    *reinterpret_cast<uint32_t *>(block + (side ? vm_off(D) : km_off(D)) +
                                  (rb * (D / kGroup) + lane / kLanes) * 4) = meta;
  if (lane < D / 4) {  // four codes a lane, one 16-bit store
    const uint8_t *z = s_code[warp];
    uint32_t w;
    int at;
    if (side) {
      const int x0 = 32 * (lane >> 3) + (lane & 7);
      w = z[x0] | (z[x0 + 16] << 4) | (z[x0 + 8] << 8) | (z[x0 + 24] << 12);
      at = v_half<D>(rb, lane >> 3, lane & 7);
    } else {
      int hi4;
      w = z[4 * lane] | (z[4 * lane + 1] << 4) | (z[4 * lane + 2] << 8) |
          (z[4 * lane + 3] << 12);
      at = k_byte<D>(rb, 4 * lane, hi4);
    }
    *reinterpret_cast<uint16_t *>(block + at) = (uint16_t)w;
  }
  if (side == 0 && lane == 0) c.score[u * c.sstride + r] = 0.f;
}

// What the newest rows stand for: one warp a (unit, row).
template <typename T, int D>
__global__ void __launch_bounds__(256)
    read_kernel(const Call k, const __grid_constant__ Seqs q, int rows, T *key, T *val) {
  pdl_begin();
  const View &c = k.c;
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);  // [seq][layer][head][row]
  const int lane = threadIdx.x & 31;
  const int t = (int)(w % rows);
  const long long rest = w / rows;
  const int h = (int)(rest % c.H), lr = (int)(rest / c.H % k.nl);
  const long long s = rest / c.H / k.nl;
  if (s >= k.n) return;
  const size_t to = ((((size_t)(s + k.s0) * k.nl + lr) * c.H + h) * rows + t) * D;
  if (t >= q.count[s]) {
    for (int x = lane; x < D; x += 32) {
      key[to + x] = from_f<T>(0.f);
      val[to + x] = from_f<T>(0.f);
    }
    return;
  }
  const int r = q.len[s] - q.count[s] + t;
  const uint8_t *block = block_at(c, unit_at(c, k.s0 + (int)s, k.lb, lr, h), r);
  for (int x = lane; x < D; x += 32) {
    key[to + x] = from_f<T>(k_value<D>(block, r % kBlock, x));
    val[to + x] = from_f<T>(v_value<D>(block, r % kBlock, x));
  }
}

// A row's rank: higher score first, then lower position.  -0 counts as 0, and
// every NaN as one above every number.
__device__ __forceinline__ unsigned long long row_key(float x, int i) {
  const unsigned b = __float_as_uint(x), a = b & 0x7FFFFFFFu;
  const unsigned o = a > 0x7F800000u ? 0xFFFFFFFFu : a == 0 ? 0x80000000u
                     : b != a        ? ~b
                                     : (b | 0x80000000u);
  return ((unsigned long long)o << 32) | (0xFFFFFFFFu - (unsigned)i);
}

// Cut a unit into dst: one CTA a unit.  A radix select finds the budget-th
// largest (score, lower position) among the rows before the window; the kept
// rows are then listed in order, in dst's positions, and their values written.
template <typename T, int D>
__global__ void __launch_bounds__(dev::kThreads)
    evict_kernel(const Call k, const __grid_constant__ Seqs q, const CacheView dst, int budget,
                 int window) {
  pdl_begin();
  const View &c = k.c;
  __shared__ unsigned s_hist[256];
  __shared__ unsigned long long s_prefix;
  __shared__ int s_need, s_base, s_wsum[dev::kWarps];
  const int h = blockIdx.x % c.H, l = blockIdx.x / c.H, s = blockIdx.y;
  const size_t u = unit_at(c, k.s0 + s, 0, l, h);
  const float *score = c.score + u * c.sstride;
  const int n = q.len[s], first = max(0, n - window);  // rows [first, n): the window
  const int keep = min(n, budget + window);
  auto key = [&](int i) { return row_key(score[i], i); };
  unsigned long long least = 0;
  if (first > budget) {
    if (budget > 0)
      least = dev::block_select(first, budget, [](int) { return true; }, key, s_hist,
                                &s_prefix, &s_need);
    else
      least = ~0ull;
  }
  const bool none = first > budget && budget == 0;
  int32_t *pos = dst.pos + u * dst.sstride;
  const int got = dev::block_collect(
      0, n, [&](int i) { return i >= first || (!none && key(i) >= least); }, pos, s_wsum,
      &s_base);
  if (got != keep && threadIdx.x == 0) atomicOr(c.err, ERR_LENGTH);
  const int m = min(got, keep);
  float *to_score = dst.score + u * dst.sstride;
  for (int i = threadIdx.x; i < m; i += dev::kThreads) to_score[i] = score[pos[i]];
  T *K = static_cast<T *>(dst.K) + u * (size_t)dst.cap * D;
  T *V = static_cast<T *>(dst.V) + u * (size_t)dst.cap * D;
  for (int i = threadIdx.x / 32; i < m; i += dev::kWarps) {
    const int r = pos[i];
    const uint8_t *block = block_at(c, u, r);
    for (int x = threadIdx.x & 31; x < D; x += 32) {
      K[(size_t)i * D + x] = from_f<T>(k_value<D>(block, r % kBlock, x));
      V[(size_t)i * D + x] = from_f<T>(v_value<D>(block, r % kBlock, x));
    }
  }
  if (threadIdx.x == 0) {
    dst.state[4 * u] = m;
    dst.state[4 * u + 1] = n;
    dst.state[4 * u + 2] = 0;  // no R-KV key sum yet
  }
}

template <typename T, int D>
cudaError_t launch_read(const Call &k, const Seqs &q, int rows, void *key, void *val,
                        cudaStream_t stream) {
  const long long warps = (long long)k.n * k.nl * k.c.H * rows;
  return launch_pdl(read_kernel<T, D>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, stream,
                    k, q, rows, static_cast<T *>(key), static_cast<T *>(val));
}

template <typename T, int D>
cudaError_t launch_append_as(const Call &k, const Seqs &q, int tokens, const void *key,
                             const void *val, const RowStrides &st, cudaStream_t stream) {
  const long long warps = 2ll * k.n * k.nl * k.c.H * tokens;
  return launch_pdl(append_kernel<T, D>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0,
                    stream, k, q, tokens, static_cast<const T *>(key),
                    static_cast<const T *>(val), st);
}

template <typename T, int D>
cudaError_t launch_evict(const Call &k, const Seqs &q, const CacheView &dst, int budget,
                         int window, cudaStream_t stream) {
  return launch_pdl(evict_kernel<T, D>, dim3(k.c.L * k.c.H, k.n), dim3(dev::kThreads), 0,
                    stream, k, q, dst, budget, window);
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
