// Attention over the paged cache of 8-bit codes, for the query tokens of a step.
//
// Work.  The query heads that share a kv head, times the query tokens of a sequence, are columns; an item is a
// block of columns of one (sequence, kv head), a unit one page of an item.  Units are numbered sequence by
// sequence, and every workgroup takes an equal run of them, whatever the lengths: it walks the run
// item by item, and where it holds all pages of an item it writes the rows, else a partial result (maximum, sum,
// weighted values of every column), which a second kernel joins.  The numbering needs the lengths, which only
// the device knows, so every workgroup computes it: a prefix sum over the sequences.
//
// Arithmetic of a page (64 tokens) and 16 columns, all in one wavefront and without any exchange but two lane
// moves for the maximum:
//   scores^T = K q^T    16x16x32 products, rows = tokens, columns = query heads
//   weights             2^(s - m) of the same registers
//   out^T += V^T w^T    rows = channels, contraction over tokens
// A lane of the first product's result holds 4 tokens of its column per tile; the tokens are dealt to the tiles' rows
// so that the four tiles give a lane of group g (lane / 16) the tokens 16 g .. 16 g + 15, which is what it feeds the
// second product.  The cache's layout is made for it: a lane reads 16 bytes of a key (channels 16 g ..) or of a
// value channel (tokens 16 g ..) and converts them in pairs to fp16, which holds every e4m3 number exactly.
//
// Roundings.  Queries: scaled by a power of two to a largest element in [2^8, 2^9) and rounded to fp16 (exact for bf16 and
// fp16 but for elements below 2^-22 of the largest); fp32 queries are split into two fp16 terms, 22 bits.  Weights: 2^14 2^(s - m), so
// that fp16 holds them with 11 bits down to 2^-28 of the largest; with fp32 queries two terms of them as
// well.  Sums in fp32 (weights before their rounding), products accumulate in fp32.
//
// The scale of a page's keys enters the scores' factor.  Its values' scale becomes the unit of the accumulators,
// which are multiplied by the powers of two between units along with the correction of the maximum.
#include <cmath>

#include "rvq_cache8.h"

namespace {

constexpr float NEG = -3.402823466e38f;  // "nothing yet": finite, so that differences are numbers
constexpr float WEIGHT_BITS = 14.0f;     // weights are held as 2^14 2^(s - m)
constexpr int COLS = 16;                 // columns of an item of the kernel for few columns
constexpr int MANY = 128;                // and of the kernel for many
constexpr int WAVES = 4;

struct AttnArgs {
  CacheView c;
  const void *q;
  void *out;
  int64_t ldq, hsq, ldo, hso;
  int rep, window, sinks;
  float scale;  // log2(e) times the softmax scale
  float *part;      // [2 * workgroups][COLS or MANY][HD + 2]
  int64_t *header;  // [workgroups][8]
  int64_t least;    // fewest units of a workgroup
};

// what a sequence's queries see: pages [0, sink_pages) and [begin, end) of its table
struct Seen {
  SeqRows r;
  int64_t p0;     // position of the first query token
  int64_t tokens; // tokens that have an entry in the table
  int64_t sink_pages, begin, pages;
  int blocks;     // of columns
};
__device__ __forceinline__ Seen seen_by(const AttnArgs &a, int b) {
  Seen s;
  s.r = rows_of(a.c, b);
  const int64_t len = a.c.lengths[b] < 0 ? 0 : a.c.lengths[b], room = (int64_t)a.c.table_pages * PAGE;
  s.p0 = len - s.r.n;
  s.tokens = len < room ? len : room;
  int64_t begin = a.window > 0 ? s.p0 - a.window + 1 : 0;
  s.begin = (begin < 0 ? 0 : begin) / PAGE;
  const int64_t end = (s.tokens + PAGE - 1) / PAGE;
  int64_t sink = a.window > 0 ? ((int64_t)a.sinks + PAGE - 1) / PAGE : 0;
  sink = sink < s.begin ? sink : s.begin;
  s.sink_pages = sink < end ? sink : end;
  const int64_t windowed = end > s.begin ? end - s.begin : 0;
  s.pages = s.sink_pages + windowed;
  if (s.pages < 1) s.pages = 1;  // rows that see nothing are written too
  s.blocks = (int)(((int64_t)s.r.n * a.rep + COLS - 1) / COLS);
  return s;
}
__device__ __forceinline__ int64_t units_of(const AttnArgs &a, int b) {
  const Seen s = seen_by(a, b);
  return (int64_t)s.blocks * a.c.heads * s.pages;
}

// units of a workgroup's run, computed by every wavefront
__device__ __forceinline__ int64_t run_length(const AttnArgs &a) {
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  for (int b = lane; b < a.c.n_seqs; b += 64) total += units_of(a, b);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d, 64);
  const int64_t even = (total + gridDim.x - 1) / gridDim.x;
  return even > a.least ? even : a.least;
}

__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x) |
                   ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32));
}

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

template <typename T, int HD> struct Columns {
  static constexpr bool SPLIT = std::is_same<T, float>::value;
  static constexpr int PARTS = HD / 32;  // products of 32 channels
  f16x8 hi[PARTS], lo[SPLIT ? PARTS : 1];
  float factor;  // of a score, but for the keys' scale
  int64_t p;     // position of this lane's column; -1: no such column
};

template <typename T, int HD>
__device__ __forceinline__ void load_columns(const AttnArgs &a, const Seen &s, int head, int block, Columns<T, HD> &k) {
  typedef Columns<T, HD> C;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int64_t c = (int64_t)block * COLS + (lane & 15), token = c / a.rep;
  const bool valid = token < s.r.n;
  float x[C::PARTS][8];
  float amax = 0.0f;
  if (valid) {
    const T *q = (const T *)a.q + (s.r.row + token) * a.ldq + ((int64_t)head * a.rep + (c - token * a.rep)) * a.hsq;
#pragma unroll
    for (int m = 0; m < C::PARTS; ++m) load8<T>(q + (m >> 1) * 64 + g * 16 + (m & 1) * 8, x[m]);
  } else {
#pragma unroll
    for (int m = 0; m < C::PARTS; ++m)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[m][i] = 0.0f;
  }
#pragma unroll
  for (int m = 0; m < C::PARTS; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(x[m][i]));
  amax = fmaxf(amax, __shfl_xor(amax, 16, 64));
  amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
  int e = (int)(__float_as_uint(amax) >> 23) - 127 - 8;  // largest element to [2^8, 2^9)
  e = e < -118 ? -118 : e;
  const float down = __uint_as_float((uint32_t)(127 - e) << 23);
  k.factor = ldexpf(a.scale, e);
  k.p = valid ? s.p0 + token : -1;
#pragma unroll
  for (int m = 0; m < C::PARTS; ++m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[m][i] *= down;
    k.hi[m] = half8(x[m]);
    if constexpr (C::SPLIT) k.lo[m] = rest8(x[m], k.hi[m]);
  }
}

// one wavefront's running result of 16 columns: lane (column n, group g) holds channels 16 t + 4 g + r
template <int HD> struct State {
  f32x4 acc[HD / 16];
  float m, l, unit;  // maximum (base 2), sum of this lane's weights, scale of the accumulators
};

template <typename T, int HD>
__device__ __forceinline__ void take_page(const AttnArgs &a, const Columns<T, HD> &k, State<HD> &st, int64_t page, int head,
                                          int64_t t0, int64_t tokens, bool whole) {
  typedef Columns<T, HD> C;
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const uint8_t *kc = codes_of(a.c, page, head, 0), *vc = codes_of(a.c, page, head, 1);
  const f32x2 scales = *reinterpret_cast<const f32x2 *>(scale_of(a.c, page, head, 0));
  u32x4 kw[4][HD / 64], vw[HD / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < HD / 64; ++j)  // row n of tile i is token 16 (n / 4) + 4 i + n % 4
      kw[i][j] = *reinterpret_cast<const u32x4 *>(kc + ((n >> 2) * 16 + i * 4 + (n & 3)) * HD + j * 64 + g * 16);
#pragma unroll
  for (int t = 0; t < HD / 16; ++t) vw[t] = *reinterpret_cast<const u32x4 *>(vc + (t * 16 + n) * PAGE + g * 16);

  const float factor = k.factor * scales[0];
  float s[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x4 d = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) {
      const f16x8 x = widen8(kw[i][j][0], kw[i][j][1]), y = widen8(kw[i][j][2], kw[i][j][3]);
      if constexpr (C::SPLIT) {
        d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, k.lo[2 * j], d, 0, 0, 0);
        d = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, k.lo[2 * j + 1], d, 0, 0, 0);
      }
      d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, k.hi[2 * j], d, 0, 0, 0);
      d = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, k.hi[2 * j + 1], d, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) s[4 * i + r] = d[r] * factor;
  }
  bool visible[16];
  if (!whole) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int64_t t = t0 + g * 16 + i;
      visible[i] = t <= k.p && t < tokens && (a.window <= 0 || t > k.p - a.window || t < a.sinks);
      s[i] = visible[i] ? s[i] : -INFINITY;
    }
  }
  float top = st.m;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
  float fix = __builtin_amdgcn_exp2f(st.m - top);
  st.m = top;
  st.l *= fix;
  // the accumulators' unit becomes this page's scale; a step of more than 2^40 downwards is left to the weights
  float unit = scales[1], rest = 1.0f;
  if (unit < st.unit * 0x1p-40f) {
    unit = st.unit * 0x1p-40f;
    rest = scales[1] / unit;
  }
  fix *= st.unit / unit;
  st.unit = unit;
  float w[2][8];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float x = __builtin_amdgcn_exp2f(s[i] - (top - WEIGHT_BITS));
    st.l += x;
    w[i >> 3][i & 7] = x * rest;
  }
  f16x8 hi[2], lo[C::SPLIT ? 2 : 1];
  hi[0] = half8(w[0]);
  hi[1] = half8(w[1]);
  if constexpr (C::SPLIT) {
    lo[0] = rest8(w[0], hi[0]);
    lo[1] = rest8(w[1], hi[1]);
  }
  // A NaN in a slot that a column does not see must not meet its weight of 0: take such codes out, and count, for
  // each (channel, column), the NaN that it does see.
  uint32_t bad = 0;
  if (!whole) {
#pragma unroll
    for (int t = 0; t < HD / 16; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) bad |= nan_bytes(vw[t][i]);
    bad = __ballot(bad != 0) != 0;
  }
  if (bad) {
    f16x8 sees[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) sees[i >> 3][i & 7] = visible[i] ? (_Float16)1.0f : (_Float16)0.0f;
#pragma unroll
    for (int t = 0; t < HD / 16; ++t) {
      u32x4 mark;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t b = nan_bytes(vw[t][i]) >> 7;  // 1 in the place of a NaN
        mark[i] = b * 0x38u;                          // the code of 1.0
        vw[t][i] &= ~(b * 0xffu);
      }
      f32x4 d = {0, 0, 0, 0};
      d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(mark[0], mark[1]), sees[0], d, 0, 0, 0);
      d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(mark[2], mark[3]), sees[1], d, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (d[r] > 0.0f) st.acc[t][r] = __uint_as_float(0x7fc00000u);
    }
  }
#pragma unroll
  for (int t = 0; t < HD / 16; ++t) {
    const f16x8 x = widen8(vw[t][0], vw[t][1]), y = widen8(vw[t][2], vw[t][3]);
    f32x4 d = st.acc[t] * fix;
    if constexpr (C::SPLIT) {
      d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, lo[0], d, 0, 0, 0);
      d = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, lo[1], d, 0, 0, 0);
    }
    d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, hi[0], d, 0, 0, 0);
    d = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, hi[1], d, 0, 0, 0);
    st.acc[t] = d;
  }
}

// header of a workgroup whose last item goes on in the next runs: what the joining kernel needs
enum { H_PARTS = 0, H_FIRST, H_ROW, H_COLS, H_HEAD, H_COL0 };

template <typename T, int HD>
__global__ __launch_bounds__(64 * WAVES, HD == 256 ? 1 : 2) void cache8_attn_kernel(const AttnArgs a) {
  __shared__ float sh_acc[WAVES][COLS][HD + 4];
  __shared__ float sh_m[WAVES][COLS], sh_l[WAVES][COLS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, n = lane & 15;
  const int64_t run = run_length(a), w = blockIdx.x;
  const int64_t u0 = w * run;
  int b;
  int64_t inside;
  if (threadIdx.x == 0) a.header[w * 8 + H_PARTS] = 0;
  if (!find_piece(a.c.n_seqs, u0, [&](int i) { return units_of(a, i); }, b, inside)) return;
  b = __builtin_amdgcn_readfirstlane(b);
  inside = uniform(inside);
  int64_t left = run;
  bool at_start = true;
  while (left > 0 && b < a.c.n_seqs) {
    const Seen s = seen_by(a, b);
    const int64_t items = (int64_t)s.blocks * a.c.heads;
    int64_t item = inside / s.pages, x = inside - item * s.pages;
    for (; item < items && left > 0; ++item, x = 0) {
      const int head = (int)(item / s.blocks), block = (int)(item - (int64_t)head * s.blocks);
      const int64_t end = x + left < s.pages ? x + left : s.pages;
      left -= end - x;
      Columns<T, HD> k;
      load_columns<T, HD>(a, s, head, block, k);
      const int64_t col0 = (int64_t)block * COLS, most = (int64_t)s.r.n * a.rep - col0;
      const int cols = most < COLS ? (int)most : COLS;
      const int64_t first = s.p0 + col0 / a.rep, last = s.p0 + (col0 + cols - 1) / a.rep;
      State<HD> st;
#pragma unroll
      for (int t = 0; t < HD / 16; ++t) st.acc[t] = f32x4{0, 0, 0, 0};
      st.m = NEG;
      st.l = 0.0f;
      st.unit = 1.0f;
      for (int64_t i = x + wave; i < end; i += WAVES) {
        const int64_t entry = i < s.sink_pages ? i : s.begin + i - s.sink_pages, t0 = entry * PAGE;
        if (t0 > last || t0 >= s.tokens) continue;
        if (a.window > 0 && t0 + PAGE <= first - a.window + 1 && t0 >= a.sinks) continue;
        const int64_t page = page_of(a.c, b, entry);
        if (page < 0) continue;
        const bool whole = t0 + PAGE - 1 <= first && t0 + PAGE <= s.tokens &&
                           (a.window <= 0 || t0 > last - a.window || t0 + PAGE <= a.sinks);
        take_page<T, HD>(a, k, st, uniform(page), head, t0, s.tokens, whole);
      }
      // the wavefronts' results together
      st.l += __shfl_xor(st.l, 16, 64);
      st.l += __shfl_xor(st.l, 32, 64);
      if (g == 0) {
        sh_m[wave][n] = st.m;
        sh_l[wave][n] = st.l;
      }
#pragma unroll
      for (int t = 0; t < HD / 16; ++t)
        *reinterpret_cast<f32x4 *>(&sh_acc[wave][n][t * 16 + g * 4]) = st.acc[t] * st.unit;
      __syncthreads();
      const int c = threadIdx.x >> 4, ch0 = (threadIdx.x & 15) * (HD / 16);
      float top = NEG, sum = 0.0f, weight[WAVES];
#pragma unroll
      for (int v = 0; v < WAVES; ++v) top = fmaxf(top, sh_m[v][c]);
#pragma unroll
      for (int v = 0; v < WAVES; ++v) {
        weight[v] = __builtin_amdgcn_exp2f(sh_m[v][c] - top);
        sum += weight[v] * sh_l[v][c];
      }
      float o[HD / 16];
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        o[i] = 0.0f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) o[i] += weight[v] * sh_acc[v][c][ch0 + i];
      }
      const bool all = x == 0 && end == s.pages;
      if (c < cols) {
        if (all) {
          const int64_t token = (col0 + c) / a.rep, h = (int64_t)head * a.rep + (col0 + c - token * a.rep);
          T *out = (T *)a.out + (s.r.row + token) * a.ldo + h * a.hso + ch0;
          const float over = sum != 0.0f ? 1.0f / sum : 0.0f;  // nothing seen: 0
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) out[i] = (T)(sum != 0.0f ? o[i] * over : 0.0f);
        } else {
          float *p = a.part + ((2 * w + (at_start ? 0 : 1)) * COLS + c) * (HD + 2);
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) p[ch0 + i] = o[i];
          if ((threadIdx.x & 15) == 0) {
            p[HD] = top;
            p[HD + 1] = sum;
          }
        }
      }
      if (x == 0 && end < s.pages && threadIdx.x == 0) {
        int64_t *hd = a.header + w * 8;
        hd[H_PARTS] = 1 + (s.pages - end + run - 1) / run;
        hd[H_FIRST] = 2 * w + (at_start ? 0 : 1);
        hd[H_ROW] = s.r.row;
        hd[H_COLS] = cols;
        hd[H_HEAD] = head;
        hd[H_COL0] = col0;
      }
      at_start = false;
      __syncthreads();
    }
    ++b;
    inside = 0;
  }
}

// ---- many columns: chunks of prompts ---------------------------------------------------------------
// The same arithmetic with 32x32x16 products: an item has 128 columns, 32 for each wavefront, and the four
// share the page's 16 KiB of codes, which are copied to LDS a page ahead (straight from memory, 16 bytes a lane; pieces of
// a row change places so that the wavefront's reads of neighbouring rows hit different banks).  A lane holds one
// column and, of the two tiles of 32 tokens, the tokens 32 h .. 32 h + 31 (h = lane / 32): its weights are again what the
// second product takes from it.
//
// What bounds it is the vector pipe: per page and wavefront 32 matrix instructions of 32 clocks stand against 128 conversions
// and some 8 operations, one of them an exponential, for each of a lane's 32 scores.  So the maximum that weights
// refer to moves only when a score passes it by more than 2^7 (the accumulators are not touched otherwise), weights being
// held as 2^8 2^(s - m) in fp16: at most 2^15, exact to 11 bits down to 2^-22 of the largest.

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float CHUNK_BITS = 8.0f, CHUNK_SLACK = 7.0f;

// pages that a block of columns sees: [0, sink_pages) and `pages - sink_pages` from `begin` on
struct Block {
  int64_t first, last;  // positions of its first and last query token
  int64_t sink_pages, begin, pages;
  int cols;
};
__device__ __forceinline__ Block block_of(const AttnArgs &a, const Seen &s, int64_t j, int width) {
  Block k;
  const int64_t col0 = j * width, most = (int64_t)s.r.n * a.rep - col0;
  k.cols = most < width ? (int)most : width;
  k.first = s.p0 + col0 / a.rep;
  k.last = s.p0 + (col0 + k.cols - 1) / a.rep;
  const int64_t low = a.window > 0 ? k.first - a.window + 1 : 0;
  k.begin = (low < 0 ? 0 : low) / PAGE;
  const int64_t seen = k.last + 1 < s.tokens ? k.last + 1 : s.tokens;
  const int64_t end = seen < 0 ? 0 : (seen + PAGE - 1) / PAGE;
  int64_t sink = a.window > 0 ? ((int64_t)a.sinks + PAGE - 1) / PAGE : 0;
  sink = sink < k.begin ? sink : k.begin;
  k.sink_pages = sink < end ? sink : end;
  k.pages = k.sink_pages + (end > k.begin ? end - k.begin : 0);
  if (k.pages < 1) k.pages = 1;
  return k;
}
__device__ __forceinline__ int64_t blocks_of(const AttnArgs &a, int b) {
  return ((int64_t)rows_of(a.c, b).n * a.rep + MANY - 1) / MANY;
}

// Units (pages) of all items, or, with FIND, the block and place of unit `target`.  256 blocks per trip: their sequence
// by bisection of the sequences' prefix sums in LDS, then a prefix sum of their units.
struct WalkShared {
  int64_t before[257], wave[4];
  int64_t found[4];
};
__device__ __forceinline__ int64_t scan256(int64_t x, int64_t *wave, int64_t &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t sum = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t o = __shfl_up(sum, d, 64);
    if (lane >= d) sum += o;
  }
  __syncthreads();
  if (lane == 63) wave[w] = sum;
  __syncthreads();
  int64_t add = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < w) add += wave[i];
    total += wave[i];
  }
  return sum + add;
}
template <bool FIND> __device__ __forceinline__ int64_t walk(const AttnArgs &a, WalkShared &sh, int64_t target) {
  const int t = threadIdx.x;
  int64_t base = 0, total;
  if (FIND && t == 0) sh.found[0] = -1;
  for (int b0 = 0; b0 < a.c.n_seqs; b0 += 256) {
    const int64_t upto = scan256(b0 + t < a.c.n_seqs ? blocks_of(a, b0 + t) : 0, sh.wave, total);
    sh.before[t + 1] = upto;
    if (t == 0) sh.before[0] = 0;
    __syncthreads();
    const int64_t blocks = total;
    for (int64_t k0 = 0; k0 < blocks; k0 += 256) {
      const int64_t k = k0 + t;
      int64_t units = 0, j = 0;
      int s = 0;
      if (k < blocks) {
#pragma unroll
        for (int d = 128; d; d /= 2)
          if (sh.before[s + d] <= k) s += d;
        j = k - sh.before[s];
        units = block_of(a, seen_by(a, b0 + s), j, MANY).pages * a.c.heads;
      }
      const int64_t sum = scan256(units, sh.wave, total);
      if (FIND) {
        const int64_t at = base + sum - units;
        if (at <= target && target < at + units) {
          sh.found[0] = b0 + s;
          sh.found[1] = j;
          sh.found[2] = target - at;
        }
        __syncthreads();
        if (sh.found[0] >= 0) return 0;
      }
      base += total;
    }
    __syncthreads();
  }
  return base;
}

template <typename T, int HD> struct Chunk {
  static constexpr int BYTES = 2 * PAGE * HD;  // of a page and kv head
  f16x8 q[HD / 16];  // product 2 c + i takes channels 32 c + 16 h + 8 i ..
  f32x16 acc[HD / 32];
  float factor, m, l, unit;
  int64_t p;
};

template <typename T, int HD>
__device__ __forceinline__ void load_chunk(const AttnArgs &a, const Seen &s, int head, int64_t col, Chunk<T, HD> &k) {
  const int h = (threadIdx.x >> 5) & 1;
  const int64_t token = col / a.rep;
  const bool valid = token < s.r.n;
  float x[HD / 16][8];
  float amax = 0.0f;
  const T *q = (const T *)a.q + (s.r.row + token) * a.ldq + ((int64_t)head * a.rep + (col - token * a.rep)) * a.hsq;
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) {
    if (valid) {
      load8<T>(q + (i >> 1) * 32 + h * 16 + (i & 1) * 8, x[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(x[i][j]));
  }
  amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
  int e = (int)(__float_as_uint(amax) >> 23) - 127 - 8;
  e = e < -118 ? -118 : e;
  // a factor >= 0, so that the largest product is the largest score; not 0, which would make a number of a hidden one
  const float down = __uint_as_float((uint32_t)(127 - e) << 23) * (a.scale < 0.0f ? -1.0f : 1.0f);
  k.factor = fmaxf(ldexpf(fabsf(a.scale), e), 1e-37f);
  k.p = valid ? s.p0 + token : -1;
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[i][j] *= down;
    k.q[i] = half8(x[i]);
  }
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) k.acc[i] = f32x16{};
  k.m = NEG;
  k.l = 0.0f;
  k.unit = 1.0f;
}

// Where 16-byte piece c of a row lies in LDS: rows of keys (HD bytes, HD / 16 pieces) and of values (64 bytes, 4
// pieces).  A wavefront reads one piece column of 32 rows at a time.
template <int PIECES> __device__ __forceinline__ int piece(int row, int c) {
  return PIECES == 4 ? c ^ ((row >> 1) & 3) : c ^ (row & 7);
}

// copies a page's codes of one kv head to LDS; complete for a wavefront's own part after vmcnt(0)
template <int HD> __device__ __forceinline__ void fetch_page(const uint8_t *codes, uint8_t *to) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 2 * HD / 64; ++i) {  // 1024 bytes per wavefront and step, keys first
    const int at = (i * WAVES + wave) * 64 + lane;  // 16-byte piece in LDS
    int from;
    if (i < HD / 64) {
      const int row = at / (HD / 16), c = at % (HD / 16);
      from = row * (HD / 16) + piece<HD / 16>(row, c);
    } else {
      const int v = at - 4 * HD, row = v >> 2, c = v & 3;
      from = 4 * HD + row * 4 + piece<4>(row, c);
    }
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(codes + from * 16),
                                     (__attribute__((address_space(3))) void *)(to + (i * WAVES + wave) * 1024), 16, 0, 0);
  }
}

template <typename T, int HD>
__device__ __forceinline__ void take_chunk_page(const AttnArgs &a, Chunk<T, HD> &k, const uint8_t *codes, f32x2 scales, int64_t t0,
                                                int64_t tokens, bool whole) {
  const int lane = threadIdx.x & 63, h = lane >> 5, n = lane & 31;
  const uint8_t *kc = codes, *vc = codes + PAGE * HD;
  f32x16 s[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    // row n of tile i is token 32 ((n / 4) % 2) + 16 i + 4 (n / 8) + n % 4
    const int row = ((n >> 2) & 1) * 32 + i * 16 + (n >> 3) * 4 + (n & 3);
    s[i] = f32x16{};
#pragma unroll
    for (int c = 0; c < HD / 32; ++c) {
      const u32x4 w = *reinterpret_cast<const u32x4 *>(kc + row * HD + piece<HD / 16>(row, 2 * c + h) * 16);
      s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(w[0], w[1]), k.q[2 * c], s[i], 0, 0, 0);
      s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(w[2], w[3]), k.q[2 * c + 1], s[i], 0, 0, 0);
    }
  }
  uint32_t sees = 0xffffffffu;  // bit i: token 32 h + i
  if (!whole) {
    sees = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const int64_t t = t0 + h * 32 + i;
      const bool v = t <= k.p && t < tokens && (a.window <= 0 || t > k.p - a.window || t < a.sinks);
      sees |= v ? 1u << i : 0u;
      s[i >> 4][i & 15] = v ? s[i >> 4][i & 15] : -INFINITY;
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = fmaxf(top, fmaxf(s[0][i], s[1][i]));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
  const float factor = k.factor * scales[0];
  top = fmaxf(k.m, top * factor);
  const bool up = top > k.m + CHUNK_SLACK;
  if (__any(up) || scales[1] > k.unit || scales[1] < k.unit * 0x1p-6f) {
    // the accumulators' unit: this page's scale, but no more than 2^40 below the last one
    const float low = k.unit * 0x1p-40f, unit = scales[1] < low ? low : scales[1];
    const float fix = __builtin_amdgcn_exp2f(k.m - top);
    k.m = top;
    k.l *= fix;
    const float all = fix * (k.unit / unit);
    k.unit = unit;
#pragma unroll
    for (int c = 0; c < HD / 32; ++c) k.acc[c] *= all;
  }
  const float rest = scales[1] / k.unit;  // at most 1
  const float ref = CHUNK_BITS - k.m;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float x = __builtin_amdgcn_exp2f(fmaf(s[i][j], factor, ref));
      sum += x;
      s[i][j] = x;
    }
  k.l += sum;
  if (rest != 1.0f) {
#pragma unroll
    for (int i = 0; i < 2; ++i) s[i] *= rest;
  }
  f16x8 w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 two = {s[i >> 1][(i & 1) * 8 + 2 * j], s[i >> 1][(i & 1) * 8 + 2 * j + 1]};
      const f16x2 r = __builtin_convertvector(two, f16x2);
      w[i][2 * j] = r[0];
      w[i][2 * j + 1] = r[1];
    }
  bool bad = false;
  if (!whole) {  // NaN codes that some column must not see: as in take_page
    uint32_t any = 0;
    for (int c = 0; c < HD / 16; ++c) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(vc + (c * 64 + lane) * 16);
      any |= nan_bytes(v[0]) | nan_bytes(v[1]) | nan_bytes(v[2]) | nan_bytes(v[3]);
    }
    bad = __ballot(any != 0) != 0;
  }
#pragma unroll
  for (int c = 0; c < HD / 32; ++c) {
    const int row = c * 32 + n;
    u32x4 v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = *reinterpret_cast<const u32x4 *>(vc + row * PAGE + piece<4>(row, 2 * h + i) * 16);
    if (bad) {
      f32x16 d = f32x16{};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f16x8 one;
#pragma unroll
        for (int j = 0; j < 8; ++j) one[j] = (sees >> (i * 8 + j)) & 1u ? (_Float16)1.0f : (_Float16)0.0f;
        uint32_t mark[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int at = (i & 1) * 2 + j;
          const uint32_t b = nan_bytes(v[i >> 1][at]) >> 7;
          mark[j] = b * 0x38u;
          v[i >> 1][at] &= ~(b * 0xffu);
        }
        d = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(mark[0], mark[1]), one, d, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (d[r] > 0.0f) k.acc[c][r] = __uint_as_float(0x7fc00000u);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      k.acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(v[i >> 1][(i & 1) * 2], v[i >> 1][(i & 1) * 2 + 1]), w[i], k.acc[c], 0, 0, 0);
  }
}

// `whole`: a workgroup takes one item, blockIdx.x / heads counting blocks from the last of every sequence (the longest) on;
// else an equal run of the items' pages, as in the kernel for few columns.
template <typename T, int HD>
__global__ __launch_bounds__(64 * WAVES, HD == 256 ? 1 : 2) void cache8_chunk_kernel(const AttnArgs a, int whole_items) {
  typedef Chunk<T, HD> C;
  __shared__ __align__(16) uint8_t tile[2][C::BYTES];
  __shared__ WalkShared sh;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, n = lane & 31;
  const int64_t w = blockIdx.x;
  int b, head = 0;
  int64_t j, x = 0, left, run = 0;
  if (whole_items) {
    if (!find_piece(a.c.n_seqs, w / a.c.heads, [&](int i) { return blocks_of(a, i); }, b, j)) return;
    head = (int)(w % a.c.heads);
    j = blocks_of(a, b) - 1 - j;
    left = INT64_MAX;
  } else {
    if (threadIdx.x == 0) a.header[w * 8 + H_PARTS] = 0;
    const int64_t total = walk<false>(a, sh, 0), even = (total + gridDim.x - 1) / gridDim.x;
    run = even > a.least ? even : a.least;
    if (w * run >= total) return;
    walk<true>(a, sh, w * run);
    b = (int)sh.found[0];
    j = sh.found[1];
    left = run;
    const int64_t pages = block_of(a, seen_by(a, b), j, MANY).pages;
    head = (int)(sh.found[2] / pages);
    x = sh.found[2] % pages;
  }
  b = __builtin_amdgcn_readfirstlane(b);
  head = __builtin_amdgcn_readfirstlane(head);
  j = uniform(j);
  x = uniform(x);
  bool at_start = true;
  while (true) {
    const Seen s = seen_by(a, b);
    const Block k = block_of(a, s, j, MANY);
    const int64_t end = x + left < k.pages && left < k.pages ? x + left : k.pages;
    left -= end - x;
    C c;
    const int64_t col0 = j * MANY;
    load_chunk<T, HD>(a, s, head, col0 + wave * 32 + n, c);
    // this wavefront's columns
    const bool busy = wave * 32 < k.cols;
    const int64_t first = s.p0 + (col0 + wave * 32) / a.rep;
    const int64_t last = s.p0 + (col0 + (wave * 32 + 31 < k.cols ? wave * 32 + 31 : k.cols - 1)) / a.rep;
    const auto entry_of = [&](int64_t i) { return i < k.sink_pages ? i : k.begin + i - k.sink_pages; };
    // the page in hand, the next one, on its way to LDS while the wavefronts work on this, and the entry behind it
    const auto scales_of = [&](int64_t id) { return id >= 0 ? *reinterpret_cast<const f32x2 *>(scale_of(a.c, id, head, 0)) : f32x2{0, 0}; };
    int64_t page = uniform(page_of(a.c, b, entry_of(x))), next = x + 1 < end ? page_of(a.c, b, entry_of(x + 1)) : -1;
    f32x2 scales = scales_of(page);
    __syncthreads();  // the tiles are free
    if (page >= 0) fetch_page<HD>(codes_of(a.c, page, head, 0), tile[0]);
    for (int64_t i = x; i < end; ++i) {
      const int cur = (int)(i - x) & 1;
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wavefront's part of the page has landed
      __syncthreads();
      next = uniform(next);
      const int64_t after = i + 2 < end ? page_of(a.c, b, entry_of(i + 2)) : -1;
      const f32x2 next_scales = scales_of(next);
      if (next >= 0) fetch_page<HD>(codes_of(a.c, next, head, 0), tile[cur ^ 1]);
      const int64_t t0 = entry_of(i) * PAGE;
      if (page >= 0 && busy && t0 <= last && t0 < s.tokens &&
          !(a.window > 0 && t0 + PAGE <= first - a.window + 1 && t0 >= a.sinks)) {
        const bool all = t0 + PAGE - 1 <= first && t0 + PAGE <= s.tokens &&
                         (a.window <= 0 || t0 > last - a.window || t0 + PAGE <= a.sinks);
        take_chunk_page<T, HD>(a, c, tile[cur], scales, t0, s.tokens, all);
      }
      page = next;
      next = after;
      scales = next_scales;
    }
    c.l += __shfl_xor(c.l, 32, 64);
    const bool all = x == 0 && end == k.pages;
    const int col = wave * 32 + n;
    if (col < k.cols) {
      if (all) {
        const int64_t token = (col0 + col) / a.rep, hq = (int64_t)head * a.rep + (col0 + col - token * a.rep);
        T *out = (T *)a.out + (s.r.row + token) * a.ldo + hq * a.hso;
        const float over = c.l != 0.0f ? c.unit / c.l : 0.0f;
#pragma unroll
        for (int t = 0; t < HD / 32; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) out[t * 32 + q * 8 + h * 4 + r] = (T)(c.l != 0.0f ? c.acc[t][q * 4 + r] * over : 0.0f);
      } else {
        float *p = a.part + ((2 * w + (at_start ? 0 : 1)) * MANY + col) * (HD + 2);
#pragma unroll
        for (int t = 0; t < HD / 32; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) p[t * 32 + q * 8 + h * 4 + r] = c.acc[t][q * 4 + r] * c.unit;
        if (h == 0) {
          p[HD] = c.m;
          p[HD + 1] = c.l;
        }
      }
    }
    if (x == 0 && end < k.pages && threadIdx.x == 0) {
      int64_t *hd = a.header + w * 8;
      hd[H_PARTS] = 1 + (k.pages - end + run - 1) / run;
      hd[H_FIRST] = 2 * w + (at_start ? 0 : 1);
      hd[H_ROW] = s.r.row;
      hd[H_COLS] = k.cols;
      hd[H_HEAD] = head;
      hd[H_COL0] = col0;
    }
    at_start = false;
    if (whole_items || left <= 0) return;
    // the next item: the next head, block, sequence with rows
    x = 0;
    if (++head < a.c.heads) continue;
    head = 0;
    if (++j < blocks_of(a, b)) continue;
    j = 0;
    do {
      if (++b >= a.c.n_seqs) return;
    } while (rows_of(a.c, b).n == 0);
  }
}

// Joins the parts of the item that begins in run blockIdx.x and goes on: a wavefront per column.  The first part lies at
// H_FIRST, the others at the beginnings of the following runs.
template <typename T, int HD, int WIDTH> __global__ __launch_bounds__(256) void cache8_join_kernel(const AttnArgs a) {
  const int64_t w = blockIdx.x;
  const int64_t *hd = a.header + w * 8;
  const int64_t parts = hd[H_PARTS];
  const int c = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (!parts || c >= hd[H_COLS]) return;
  const auto part = [&](int64_t i) { return a.part + ((i ? 2 * (w + i) : hd[H_FIRST]) * WIDTH + c) * (HD + 2); };
  float top = NEG;
  for (int64_t i = lane; i < parts; i += 64) top = fmaxf(top, part(i)[HD]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
  float sum = 0.0f, o[HD / 64];
#pragma unroll
  for (int j = 0; j < HD / 64; ++j) o[j] = 0.0f;
#pragma unroll 8
  for (int64_t i = 0; i < parts; ++i) {
    const float *p = part(i);
    const float x = __builtin_amdgcn_exp2f(p[HD] - top);
    sum += x * p[HD + 1];
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) o[j] += x * p[j * 64 + lane];
  }
  const int64_t col = hd[H_COL0] + c, token = col / a.rep, h = hd[H_HEAD] * a.rep + (col - token * a.rep);
  T *out = (T *)a.out + (hd[H_ROW] + token) * a.ldo + h * a.hso;
  const float over = sum != 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
  for (int j = 0; j < HD / 64; ++j) out[j * 64 + lane] = (T)(sum != 0.0f ? o[j] * over : 0.0f);
}

int attn_cus() {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1) {
    (void)hipGetLastError();
    return 0;
  }
  return cus;
}

// How a call is run, from what the host knows: rows, sequences and heads, not the lengths.
struct Plan {
  bool many;       // the kernel for many columns
  bool whole;      // its form in which a workgroup takes one item
  int64_t groups;  // workgroups
};
Plan plan_of(int cus, int32_t dtype, int64_t rows, int n_seqs, int heads, int rep, int hd) {
  Plan p;
  const int64_t seqs = rows < n_seqs ? rows : n_seqs, cols = rows * rep;
  p.many = dtype != RVQ_F32 && cols > 2 * COLS * seqs;
  const int per_cu = p.many && hd == 256 ? 1 : 2;
  p.groups = per_cu * cus;
  const int64_t items = cols / MANY * heads;  // at least
  p.whole = p.many && items >= 2 * p.groups && (cols / MANY + seqs) * heads <= INT32_MAX;
  if (p.whole) p.groups = (cols / MANY + seqs) * heads;
  return p;
}

template <typename T, int HD> void launch_attn(const AttnArgs &a, const Plan &p, hipStream_t s) {
  const dim3 grid((unsigned)p.groups);
  if constexpr (!std::is_same<T, float>::value) {
    if (p.many) {
      hipLaunchKernelGGL((cache8_chunk_kernel<T, HD>), grid, dim3(64 * WAVES), 0, s, a, (int)p.whole);
      if (!p.whole) hipLaunchKernelGGL((cache8_join_kernel<T, HD, MANY>), dim3(grid.x, MANY / 4), dim3(256), 0, s, a);
      return;
    }
  }
  hipLaunchKernelGGL((cache8_attn_kernel<T, HD>), grid, dim3(64 * WAVES), 0, s, a);
  const int64_t cols = a.c.rows * a.rep < COLS ? a.c.rows * a.rep : COLS;
  hipLaunchKernelGGL((cache8_join_kernel<T, HD, COLS>), dim3(grid.x, (unsigned)(cols + 3) / 4), dim3(256), 0, s, a);
}
template <typename T> void launch_attn_hd(const AttnArgs &a, const Plan &p, hipStream_t s) {
  if (a.c.hd == 64) launch_attn<T, 64>(a, p, s);
  else if (a.c.hd == 128) launch_attn<T, 128>(a, p, s);
  else launch_attn<T, 256>(a, p, s);
}

bool attn_ok(const rvq_cache8 *c, int32_t dtype, int64_t rows, int32_t n_q_heads) {
  if (!rvq_cache8_ok(c) || rows < 0 || rows > INT32_MAX) return false;
  if (dtype != RVQ_F32 && dtype != RVQ_BF16 && dtype != RVQ_F16) return false;
  if (n_q_heads < c->n_kv_heads || n_q_heads > 65535 || n_q_heads % c->n_kv_heads) return false;
  return rows * (n_q_heads / c->n_kv_heads) <= INT32_MAX / 2;  // columns of a sequence
}

}  // namespace

extern "C" {

int64_t rvq_cache8_attn_workspace_bytes(const rvq_cache8 *cache, int32_t dtype, int64_t rows, int32_t n_q_heads) {
  if (!attn_ok(cache, dtype, rows, n_q_heads)) return 0;
  const int cus = attn_cus();
  const Plan p = plan_of(cus, dtype, rows, cache->n_seqs, cache->n_kv_heads, n_q_heads / cache->n_kv_heads, cache->head_dim);
  if (p.whole || rows == 0) return 16;
  return p.groups * 64 + 2 * p.groups * (p.many ? MANY : COLS) * (cache->head_dim + 2) * (int64_t)sizeof(float);
}

int rvq_cache8_attn(const rvq_cache8 *cache, const void *dQ, int32_t dtype, int64_t rows, int32_t n_q_heads,
                    int64_t ldq, int64_t hsq, const int32_t *dCu, float scale, int32_t window, int32_t sinks,
                    void *dOut, int64_t ldo, int64_t hso, void *dWorkspace, int64_t workspace_bytes, void *stream) {
  if (!attn_ok(cache, dtype, rows, n_q_heads) || !std::isfinite(scale) || window < 0 || sinks < 0) return RVQ_EINVAL;
  if (rows == 0) return RVQ_OK;
  const int hd = cache->head_dim;
  if (!rvq_cache8_pointers_ok(cache) || !rvq_aligned(dCu, 4)) return RVQ_EINVAL;
  if (!rvq_rows16_ok(dQ, dtype, rows, n_q_heads, hd, ldq, hsq) || !rvq_rows16_ok(dOut, dtype, rows, n_q_heads, hd, ldo, hso) ||
      !rvq_rows_distinct(rows, n_q_heads, hd, ldo, hso) || dQ == dOut)
    return RVQ_EINVAL;
  if (!rvq_aligned(dWorkspace, 16)) return RVQ_EINVAL;
  const int cus = attn_cus();
  if (!cus) return RVQ_EHIP;
  if (workspace_bytes < rvq_cache8_attn_workspace_bytes(cache, dtype, rows, n_q_heads)) return RVQ_EWORKSPACE;
  if (!rvq_stream_is_current((hipStream_t)stream)) return RVQ_EINVAL;
  AttnArgs a;
  a.c = view_of(cache, dCu, rows);
  a.q = dQ; a.out = dOut;
  a.ldq = ldq; a.hsq = hsq; a.ldo = ldo; a.hso = hso;
  a.rep = n_q_heads / cache->n_kv_heads;
  a.window = window; a.sinks = sinks;
  a.scale = scale * 1.44269504088896340736f;
  a.header = (int64_t *)dWorkspace;
  const Plan p = plan_of(cus, dtype, rows, cache->n_seqs, cache->n_kv_heads, a.rep, hd);
  a.part = (float *)((char *)dWorkspace + p.groups * 64);
  a.least = p.many ? 1 : WAVES;
  if (dtype == RVQ_F32) launch_attn_hd<float>(a, p, (hipStream_t)stream);
  else if (dtype == RVQ_BF16) launch_attn_hd<__bf16>(a, p, (hipStream_t)stream);
  else launch_attn_hd<_Float16>(a, p, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? RVQ_OK : RVQ_EHIP;
}

}  // extern "C"
