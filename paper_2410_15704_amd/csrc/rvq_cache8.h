// The paged cache of 8-bit codes as its kernels see it (device code shared by append, read and attention).
#pragma once

#include "rvq_rows.h"

// what a kernel is given of a cache and of a step
struct CacheView {
  uint8_t *pages;
  float *scales;
  const int32_t *table, *lengths, *cu;
  int64_t n_pages, rows;
  int heads, hd, table_pages, n_seqs;
};

namespace {

constexpr int PAGE = RVQ_PAGE_TOKENS;

// rows of sequence b in this step; whatever the array holds, they lie inside [0, rows)
struct SeqRows {
  int64_t row;
  int n;
};
__device__ __forceinline__ SeqRows rows_of(const CacheView &c, int b) {
  int64_t lo = c.cu[b], hi = c.cu[b + 1];
  lo = lo < 0 ? 0 : lo > c.rows ? c.rows : lo;
  hi = hi < lo ? lo : hi > c.rows ? c.rows : hi;
  return {lo, (int)(hi - lo)};
}

// the page behind an entry of a sequence's table, or -1: there is none
__device__ __forceinline__ int page_of(const CacheView &c, int b, int64_t entry) {
  if (entry < 0 || entry >= c.table_pages) return -1;
  const int id = c.table[(int64_t)b * c.table_pages + entry];
  return id >= 0 && id < c.n_pages ? id : -1;
}

__device__ __forceinline__ uint8_t *codes_of(const CacheView &c, int64_t page, int head, int values) {
  return c.pages + ((page * c.heads + head) * 2 + values) * (int64_t)(PAGE * c.hd);
}
__device__ __forceinline__ float *scale_of(const CacheView &c, int64_t page, int head, int values) {
  return c.scales + (page * c.heads + head) * 2 + values;
}

// Finds the piece `at` of the sequences' pieces in order: sequence and place inside it.  Every wavefront does
// it for itself, 64 sequences per trip: a prefix sum over the lanes and the first lane that passes `at`.
// count(b) is called with b < n_seqs.  false: there are not so many.
template <typename N, typename Count>
__device__ __forceinline__ bool find_piece(int n_seqs, N at, Count count, int &seq, N &inside) {
  const int lane = threadIdx.x & 63;
  N before = 0;
  for (int b0 = 0; b0 < n_seqs; b0 += 64) {
    const int b = b0 + lane;
    N c = b < n_seqs ? count(b) : 0, sum = c;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const N o = __shfl_up(sum, d, 64);
      if (lane >= d) sum += o;
    }
    const unsigned long long past = __ballot(before + sum > at);
    if (past) {
      const int l = __ffsll(past) - 1;
      seq = b0 + l;
      inside = at - before - __shfl(sum - c, l, 64);
      return true;
    }
    before += __shfl(sum, 63, 64);
  }
  return false;
}

// The same by the whole workgroup, THREADS sequences per trip, for more than 64 sequences: a trip is a chain of loads (cu, lengths),
// and it is these chains, not the additions, that many sequences cost.  For 64 and less the barriers are saved.
template <int THREADS, typename N> struct Together {
  N sums[THREADS / 64], inside;
  int seq;
};
// Inclusive prefix sum over the workgroup's threads, and the sum of all.  Ends behind a barrier; another one has to come before
// the next call.
template <int THREADS, typename N> __device__ __forceinline__ N scan_all(N x, Together<THREADS, N> &sh, N &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const N o = __shfl_up(x, d, 64);
    if (lane >= d) x += o;
  }
  if (lane == 63) sh.sums[wave] = x;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    const N s = sh.sums[w];
    if (w < wave) x += s;
    total += s;
  }
  return x;
}
template <int THREADS, typename N, typename Count>
__device__ __forceinline__ bool find_piece_together(int n_seqs, N at, Count count, Together<THREADS, N> &sh, int &seq, N &inside) {
  N before = 0;
  for (int b0 = 0; b0 < n_seqs; b0 += THREADS) {
    const int b = b0 + (int)threadIdx.x;
    const N c = b < n_seqs ? count(b) : 0;
    N total;
    const N upto = before + scan_all<THREADS, N>(c, sh, total);
    if (upto > at && upto - c <= at) {
      sh.seq = b;
      sh.inside = at - (upto - c);
    }
    __syncthreads();
    before += total;
    if (before > at) {  // the same in every thread
      seq = sh.seq;
      inside = sh.inside;
      return true;
    }
  }
  return false;
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// smallest power of two >= 2^-100 with which `amax` (finite, >= 0) is at most 448 = 1.75 2^8
__device__ __forceinline__ float code_scale(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = e < -100 ? -100 : e;
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// four codes: nearest e4m3 numbers, ties to even; |x| <= 448
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// the same where some may not be finite: those become the code 0x7f
__device__ __forceinline__ uint32_t encode4_any(float a, float b, float c, float d) {
  const bool na = not_finite(a), nb = not_finite(b), nc = not_finite(c), nd = not_finite(d);
  const uint32_t w = encode4(na ? 0.0f : a, nb ? 0.0f : b, nc ? 0.0f : c, nd ? 0.0f : d);
  return w | (na ? 0x7fu : 0u) | (nb ? 0x7f00u : 0u) | (nc ? 0x7f0000u : 0u) | (nd ? 0x7f000000u : 0u);
}
__device__ __forceinline__ void decode4(uint32_t w, float (&v)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = lo[0]; v[1] = lo[1]; v[2] = hi[0]; v[3] = hi[1];
}

}  // namespace

// host side: the arguments that every call on a cache shares
inline bool rvq_cache8_ok(const rvq_cache8 *c) {
  if (!c || c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return false;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return false;
  if (c->table_pages < 1 || c->table_pages > INT32_MAX / RVQ_PAGE_TOKENS || c->n_seqs < 1 || c->n_seqs > 65535) return false;
  return c->n_pages <= INT64_MAX / 8 / ((int64_t)c->n_kv_heads * c->head_dim * RVQ_PAGE_TOKENS);
}
inline bool rvq_aligned(const void *p, uintptr_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool rvq_cache8_pointers_ok(const rvq_cache8 *c) {
  return rvq_aligned(c->pages, 16) && rvq_aligned(c->scales, 8) && rvq_aligned(c->table, 4) && rvq_aligned(c->lengths, 4);
}
// rows of [rows][heads][hd] that are moved 16 bytes at a time
inline bool rvq_rows16_ok(const void *p, int32_t dtype, int64_t rows, int64_t heads, int64_t hd, int64_t ld, int64_t hs) {
  const int64_t e = dtype == RVQ_F32 ? 4 : 2;
  if (!rvq_aligned(p, 16) || !rvq_rows_fit(rows, heads, hd, ld, hs)) return false;
  return ((rows > 1 ? ld : 0) * e) % 16 == 0 && ((heads > 1 ? hs : 0) * e) % 16 == 0;  // one row, one head: no stride
}
namespace {
inline CacheView view_of(const rvq_cache8 *c, const int32_t *cu, int64_t rows) {
  CacheView v;
  v.pages = c->pages; v.scales = c->scales; v.table = c->table; v.lengths = c->lengths; v.cu = cu;
  v.n_pages = c->n_pages; v.rows = rows;
  v.heads = c->n_kv_heads; v.hd = c->head_dim; v.table_pages = c->table_pages; v.n_seqs = c->n_seqs;
  return v;
}
}  // namespace
