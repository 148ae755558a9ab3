// What the two attention kernels over the paged cache share: arguments, which pages a query sees, conversions.
#pragma once

#include "rvq_cache8.h"

struct AttnArgs {
  CacheView c;
  const void *q;
  void *out;
  int64_t ldq, hsq, ldo, hso;
  int rep, window, sinks;
  float scale;      // log2(e) times the softmax scale
  float *part;      // [2 * groups][COLS or MANY][HD + 2]
  int64_t *header;  // [groups][8]
  int groups;       // workgroups that share the pages in equal runs
};

// the kernel for many columns; half: fp16 queries, else bf16
enum ItemPlan { ITEMS_RUNS, ITEMS_WHOLE, ITEMS_EITHER };
void rvq_launch_cache8_chunk(const AttnArgs &a, bool half, int64_t grid, ItemPlan items, hipStream_t s);

namespace {

constexpr float NEG = -3.402823466e38f;  // "nothing yet": finite, so that differences are numbers
constexpr int COLS = 16;                 // columns of an item of the kernel for few columns
constexpr int MANY = 128;                // and of the kernel for many
constexpr int WAVES = 4;

// Positions, rows and entries of a table fit 32 bits: a sequence has at most 2^31 - 1 tokens and a step as many rows.
struct Seq {
  int row, n;  // its rows of the step
  int p0;      // position of the first of them
  int tokens;  // its tokens that have an entry in the table
};
__device__ __forceinline__ Seq seq_of(const AttnArgs &a, int b) {
  const SeqRows r = rows_of(a.c, b);
  const int len = a.c.lengths[b] < 0 ? 0 : a.c.lengths[b], room = a.c.table_pages * PAGE;
  return {(int)r.row, r.n, len - r.n, len < room ? len : room};
}

// The pages that the query tokens at positions first .. last see: [0, sink_pages) and pages - sink_pages from `begin` on;
// at least one, since rows that see nothing are written too.
struct Span {
  int sink_pages, begin, pages;
  __device__ __forceinline__ int entry(int i) const { return i < sink_pages ? i : begin + i - sink_pages; }
};
// the last position that the window of a query at p hides
__device__ __forceinline__ int hidden_to(const AttnArgs &a, int p) {
  const int64_t x = (int64_t)p - a.window;
  return a.window > 0 && x >= 0 ? (int)x : -1;
}
__device__ __forceinline__ Span span_of(const AttnArgs &a, const Seq &s, int first, int last) {
  Span k;
  k.begin = (hidden_to(a, first) + 1) / PAGE;
  const int seen = last < s.tokens - 1 ? last : s.tokens - 1;
  const int end = seen < 0 ? 0 : seen / PAGE + 1;
  const int sink = a.window > 0 ? (int)(((int64_t)a.sinks + PAGE - 1) / PAGE) : 0;
  k.sink_pages = min(min(sink, k.begin), end);
  k.pages = max(1, k.sink_pages + max(0, end - k.begin));
  return k;
}

// Columns col0 .. col0 + cols - 1 of a sequence, by query token and then by head.
struct Block {
  int col0, cols;
  int first, last;  // positions of the first and the last query token
};
__device__ __forceinline__ int columns_of(const AttnArgs &a, int n) { return n * a.rep; }
__device__ __forceinline__ int blocks_of(const AttnArgs &a, int n, int width) { return (columns_of(a, n) + width - 1) / width; }
__device__ __forceinline__ Block block_of(const AttnArgs &a, const Seq &s, int col0, int width) {
  Block k;
  k.col0 = col0;
  k.cols = min(width, columns_of(a, s.n) - col0);
  k.first = s.p0 + (int)((uint32_t)col0 / (uint32_t)a.rep);
  k.last = s.p0 + (int)((uint32_t)(col0 + k.cols - 1) / (uint32_t)a.rep);
  return k;
}

// which tokens a column sees: t <= to, and t > hidden or t < sinks
struct Sight {
  int to, hidden;
};
__device__ __forceinline__ Sight sight_of(const AttnArgs &a, const Seq &s, int p) {
  return {p < s.tokens - 1 ? p : s.tokens - 1, hidden_to(a, p)};
}
// bit i: this lane's column sees token t0 + i, i < 32
__device__ __forceinline__ uint32_t ones(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t seen_bits(const AttnArgs &a, const Sight &x, int t0) {
  return ones(x.to - t0 + 1) & (~ones(x.hidden - t0 + 1) | ones(a.sinks - t0));
}
// all bits of the result are bit i of x
__device__ __forceinline__ uint32_t spread_bit(uint32_t x, int i) { return (uint32_t)((int)(x << (31 - i)) >> 31); }
// none or all of the page at t0 is seen by all columns of a block
__device__ __forceinline__ bool none_sees(const AttnArgs &a, const Seq &s, const Block &k, int t0) {
  return t0 > k.last || t0 >= s.tokens || (t0 + PAGE - 1 <= hidden_to(a, k.first) && t0 >= a.sinks);
}
__device__ __forceinline__ bool all_see(const AttnArgs &a, const Seq &s, const Block &k, int t0) {
  return t0 + PAGE - 1 <= k.first && t0 + PAGE - 1 < s.tokens && (t0 > hidden_to(a, k.last) || t0 + PAGE - 1 < a.sinks);
}

__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x) |
                   ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32));
}
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// 8 codes -> 8 fp16 numbers, exactly
__device__ __forceinline__ f16x8 widen8(uint32_t lo, uint32_t hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  f16x8 r;
  r[0] = a[0]; r[1] = a[1]; r[2] = b[0]; r[3] = b[1];
  r[4] = c[0]; r[5] = c[1]; r[6] = d[0]; r[7] = d[1];
  return r;
}
// bytes that are NaN codes, as 0x80 in their place
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// nearest of eight floats as fp16, or what that leaves
__device__ __forceinline__ f16x8 half8(const float (&x)[8]) {
  f16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (_Float16)x[i];
  return r;
}
__device__ __forceinline__ f16x8 rest8(const float (&x)[8], f16x8 hi) {
  f16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (_Float16)(x[i] - (float)hi[i]);
  return r;
}

// header of a workgroup whose last item goes on in the next runs: what the joining kernel needs
enum { H_PARTS = 0, H_FIRST, H_ROW, H_COLS, H_HEAD, H_COL0 };

}  // namespace
