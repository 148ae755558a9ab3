// Attention over the paged cache of 8-bit codes, for the query tokens of a step: the kernel for few columns (single tokens), the
// joining of partial results, the choice between this kernel and the one for many columns, and the entry point.
//
// Work.  The query heads that share a kv head, times the query tokens of a sequence, are columns; an item is a
// block of columns of one (sequence, kv head), a unit one page of an item.  Units are numbered sequence by
// sequence, and every workgroup takes an equal run of them, whatever the lengths: it walks the run
// item by item, and where it holds all pages of an item it writes the rows, else a partial result (maximum, sum,
// weighted mean of the values of every column), which a second kernel joins.  The numbering needs the lengths, which only
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
//
// Bound by the codes' bytes: 131072 tokens of 8 kv heads of 128 channels are 268 MB, 51 us and 7 for the joining (5.3 TB/s; a large
// copy moves 5.2); 64 sequences of 64 to 16000 tokens 197 + 5.5 us.  A short cache is bound by the chain of one run: 2100 tokens
// take 11.8 us, of which some 7 go to finding the run, its table and the first page's way from memory, and 3.9 for the joining's launch.
// Tried and taken back: the next page's codes in registers of their own (128 channels: spills, 131072 tokens 60 -> 84 us; 64 channels
// 16.8 -> 17.5); three workgroups per CU for 64 channels (16.8 -> 16.9).
#include <algorithm>
#include <cmath>

#include "rvq_cache8_attn.h"

namespace {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float WEIGHT_BITS = 14.0f;  // weights are held as 2^14 2^(s - m)

// units (pages) of a sequence: as many for every block of its columns
__device__ __forceinline__ int64_t units_of(const AttnArgs &a, int b) {
  const Seq s = seq_of(a, b);
  return (int64_t)blocks_of(a, s.n, COLS) * a.c.heads * span_of(a, s, s.p0, s.p0 + s.n - 1).pages;
}

// The run of workgroup `w`: how many units a run has, and the sequence and place of its first one.  Every wavefront computes it
// for up to 64 sequences, a lane each, and one prefix sum gives both; more are taken by the workgroup together.
__device__ __forceinline__ bool find_run(const AttnArgs &a, int64_t w, int64_t &run, int &seq, int64_t &inside) {
  __shared__ Together<64 * WAVES, int64_t> sh;
  const int lane = threadIdx.x & 63;
  const auto run_of = [&](int64_t total) {
    const int64_t even = (total + gridDim.x - 1) / gridDim.x;
    return even > WAVES ? even : WAVES;  // a page for every wavefront
  };
  if (a.c.n_seqs <= 64) {
    const int64_t units = lane < a.c.n_seqs ? units_of(a, lane) : 0;
    if (!__any(units >= 1 << 24)) {  // 32 bits hold the sums
      const int u = (int)units;
      int sum = u;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(sum, d, 64);
        if (lane >= d) sum += o;
      }
      run = run_of(__builtin_amdgcn_readlane(sum, 63));
      const int64_t first = w * run;
      const unsigned long long past = __ballot(sum > first);
      if (!past) return false;
      seq = __ffsll(past) - 1;
      inside = first - __builtin_amdgcn_readlane(sum - u, seq);
      return true;
    }
  }
  int64_t mine = 0, total;
  for (int b = threadIdx.x; b < a.c.n_seqs; b += 64 * WAVES) mine += units_of(a, b);
  (void)scan_all<64 * WAVES, int64_t>(mine, sh, total);
  __syncthreads();
  run = run_of(total);
  return find_piece_together<64 * WAVES, int64_t>(a.c.n_seqs, w * run, [&](int i) { return units_of(a, i); }, sh, seq, inside);
}

template <typename T, int HD> struct Columns {
  static constexpr bool SPLIT = std::is_same<T, float>::value;
  static constexpr int PARTS = HD / 32;  // products of 32 channels
  f16x8 hi[PARTS], lo[SPLIT ? PARTS : 1];
  float factor;  // of a score, but for the keys' scale
  Sight sight;   // of this lane's column
};

// the elements of a lane's column as they are, on their way
template <typename T, int HD> struct RawColumns {
  static constexpr int WORDS = sizeof(T) / 2;  // 16-byte words of eight elements
  u32x4 x[HD / 32][WORDS];
  __device__ __forceinline__ RawColumns(const AttnArgs &a, const Seq &s, int head, const Block &b) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int c = b.col0 + (lane & 15), token = (int)((uint32_t)c / (uint32_t)a.rep);
    const T *q = (const T *)a.q + (int64_t)(s.row + token) * a.ldq + (int64_t)(head * a.rep + (c - token * a.rep)) * a.hsq;
#pragma unroll
    for (int m = 0; m < HD / 32; ++m)
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        x[m][i] = u32x4{0, 0, 0, 0};
        if ((lane & 15) < b.cols) x[m][i] = reinterpret_cast<const u32x4 *>(q + (m >> 1) * 64 + g * 16 + (m & 1) * 8)[i];
      }
  }
};

template <typename T, int HD>
__device__ __forceinline__ void make_columns(const AttnArgs &a, const Seq &s, const Block &b, const RawColumns<T, HD> &raw, Columns<T, HD> &k) {
  typedef Columns<T, HD> C;
  const int lane = threadIdx.x & 63;
  float x[C::PARTS][8];
  float amax = 0.0f;
#pragma unroll
  for (int m = 0; m < C::PARTS; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (C::SPLIT) x[m][i] = __uint_as_float(raw.x[m][i >> 2][i & 3]);
      else x[m][i] = (float)__builtin_bit_cast(typename Vec8<T>::type, raw.x[m][0])[i];
      amax = fmaxf(amax, fabsf(x[m][i]));
    }
  amax = fmaxf(amax, __shfl_xor(amax, 16, 64));
  amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
  int e = (int)(__float_as_uint(amax) >> 23) - 127 - 8;  // largest element to [2^8, 2^9)
  e = e < -118 ? -118 : e;
  const float down = __uint_as_float((uint32_t)(127 - e) << 23);
  k.factor = ldexpf(a.scale, e);
  const int token = (int)((uint32_t)(b.col0 + (lane & 15)) / (uint32_t)a.rep);
  k.sight = (lane & 15) < b.cols ? sight_of(a, s, s.p0 + token) : Sight{-1, -1};
#pragma unroll
  for (int m = 0; m < C::PARTS; ++m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[m][i] *= down;
    k.hi[m] = half8(x[m]);
    if constexpr (C::SPLIT) k.lo[m] = rest8(x[m], k.hi[m]);
  }
}

// the codes of a page as a lane takes them
template <int HD> struct PageCodes {
  u32x4 k[4][HD / 64], v[HD / 16];
  f32x2 scales;
  __device__ __forceinline__ void load(const AttnArgs &a, int page, int head) {
    const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    const uint8_t *kc = codes_of(a.c, page, head, 0), *vc = codes_of(a.c, page, head, 1);
    scales = *reinterpret_cast<const f32x2 *>(scale_of(a.c, page, head, 0));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < HD / 64; ++j)  // row n of tile i is token 16 (n / 4) + 4 i + n % 4
        k[i][j] = *reinterpret_cast<const u32x4 *>(kc + ((n >> 2) * 16 + i * 4 + (n & 3)) * HD + j * 64 + g * 16);
#pragma unroll
    for (int t = 0; t < HD / 16; ++t) v[t] = *reinterpret_cast<const u32x4 *>(vc + (t * 16 + n) * PAGE + g * 16);
  }
};

// one wavefront's running result of 16 columns: lane (column n, group g) holds channels 16 t + 4 g + r
template <int HD> struct State {
  f32x4 acc[HD / 16];
  float m, l, unit;  // maximum (base 2), sum of this lane's weights, scale of the accumulators
  float most;        // largest scale of values so far
};

template <typename T, int HD>
__device__ __forceinline__ void take_page(const AttnArgs &a, const Columns<T, HD> &k, State<HD> &st, PageCodes<HD> &p, int t0, bool whole) {
  typedef Columns<T, HD> C;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const f32x2 scales = p.scales;
  const float factor = k.factor * scales[0];
  float s[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x4 d = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) {
      const f16x8 x = widen8(p.k[i][j][0], p.k[i][j][1]), y = widen8(p.k[i][j][2], p.k[i][j][3]);
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
  uint32_t seen = 0;
  if (!whole) {
    seen = seen_bits(a, k.sight, t0 + g * 16);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t m = spread_bit(seen, i);
      s[i] = __uint_as_float((__float_as_uint(s[i]) & m) | (0xff800000u & ~m));  // hidden: -infinity
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
  // The accumulators' unit becomes this page's scale, but not under 2^-64 of the largest so far, and what is missing is left to the
  // weights: 2^31 weights of 2^14 times codes of 448 are 2^54, so that the accumulators stay below 2^118.  (Before the first page
  // nothing is kept and the unit is 0; a page that was never written has the scale 0.)
  st.most = fmaxf(st.most, scales[1]);
  const float unit = fmaxf(fmaxf(scales[1], st.most * 0x1p-64f), 0x1p-126f), over = 1.0f / unit;
  const float rest = scales[1] * over;
  fix *= st.unit * over;
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
      for (int i = 0; i < 4; ++i) bad |= nan_bytes(p.v[t][i]);
    bad = __ballot(bad != 0) != 0;
  }
  if (bad) {
    u32x4 ones[2];  // fp16 ones of the tokens that are seen
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i >> 2][i & 3] = (spread_bit(seen, 2 * i) & 0x3c00u) | (spread_bit(seen, 2 * i + 1) & 0x3c000000u);
#pragma unroll
    for (int t = 0; t < HD / 16; ++t) {
      u32x4 mark;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t b = nan_bytes(p.v[t][i]) >> 7;  // 1 in the place of a NaN
        mark[i] = b * 0x38u;                          // the code of 1.0
        p.v[t][i] &= ~(b * 0xffu);
      }
      f32x4 d = {0, 0, 0, 0};
      d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(mark[0], mark[1]), __builtin_bit_cast(f16x8, ones[0]), d, 0, 0, 0);
      d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(mark[2], mark[3]), __builtin_bit_cast(f16x8, ones[1]), d, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        st.acc[t][r] = __uint_as_float(d[r] > 0.0f ? 0x7fc00000u : __float_as_uint(st.acc[t][r]));
    }
  }
#pragma unroll
  for (int t = 0; t < HD / 16; ++t) {
    const f16x8 x = widen8(p.v[t][0], p.v[t][1]), y = widen8(p.v[t][2], p.v[t][3]);
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

template <typename T, int HD>
__global__ __launch_bounds__(64 * WAVES, HD == 256 ? 1 : 2) void cache8_attn_kernel(const AttnArgs a) {
  __shared__ float sh_acc[WAVES][COLS][HD + 4];
  __shared__ float sh_m[WAVES][COLS], sh_l[WAVES][COLS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, n = lane & 15;
  const int64_t w = blockIdx.x;
  int b;
  int64_t run, inside;
  if (threadIdx.x == 0) a.header[w * 8 + H_PARTS] = 0;
  if (!find_run(a, w, run, b, inside)) return;
  run = uniform(run);
  b = __builtin_amdgcn_readfirstlane(b);
  inside = uniform(inside);
  int64_t left = run;
  bool at_start = true;
  while (left > 0 && b < a.c.n_seqs) {
    const Seq s = seq_of(a, b);
    const Span span = span_of(a, s, s.p0, s.p0 + s.n - 1);
    const int blocks = blocks_of(a, s.n, COLS);
    const int64_t items = (int64_t)blocks * a.c.heads;
    int64_t item = inside / span.pages;
    int x = (int)(inside - item * span.pages);
    for (; item < items && left > 0; ++item, x = 0) {
      const int head = (int)(item / blocks);
      const Block k = block_of(a, s, (int)(item - (int64_t)head * blocks) * COLS, COLS);
      const int end = (int)min((int64_t)span.pages, x + left);
      left -= end - x;
      // This wavefront's pages are x + wave + WAVES t, t < count.  A lane reads the table for one of them, 64 at a time.
      const int mine = x + wave, count = end > mine ? (end - mine + WAVES - 1) / WAVES : 0;
      const auto first_token = [&](int t) { return span.entry(mine + WAVES * t) * PAGE; };
      const auto read_ids = [&](int t) {
        const int at = t + lane;
        return at < count && !none_sees(a, s, k, first_token(at)) ? page_of(a.c, b, span.entry(mine + WAVES * at)) : -1;
      };
      int ids = read_ids(0);
      const RawColumns<T, HD> raw(a, s, head, k);
      Columns<T, HD> c;
      State<HD> st;
#pragma unroll
      for (int t = 0; t < HD / 16; ++t) st.acc[t] = f32x4{0, 0, 0, 0};
      st.m = NEG;
      st.l = 0.0f;
      st.unit = st.most = 0.0f;
      const auto id_at = [&](int t) {
        if (t >= count) return -1;
        if (t && (t & 63) == 0) ids = read_ids(t);
        return __builtin_amdgcn_readlane(ids, t & 63);
      };
      PageCodes<HD> codes;
      int page = id_at(0);
      if (page >= 0) codes.load(a, page, head);  // on their way while the columns are made
      make_columns<T, HD>(a, s, k, raw, c);
      for (int t = 0; t < count; ++t) {
        const int t0 = first_token(t);
        if (page >= 0) take_page<T, HD>(a, c, st, codes, t0, all_see(a, s, k, t0));
        page = id_at(t + 1);
        if (page >= 0) codes.load(a, page, head);
      }
      // the wavefronts' results together: means, which are no larger than the values (the sums may pass fp32)
      st.l += __shfl_xor(st.l, 16, 64);
      st.l += __shfl_xor(st.l, 32, 64);
      if (g == 0) {
        sh_m[wave][n] = st.m;
        sh_l[wave][n] = st.l;
      }
      const float by = st.l != 0.0f ? 1.0f / st.l : 0.0f;
#pragma unroll
      for (int t = 0; t < HD / 16; ++t)
        *reinterpret_cast<f32x4 *>(&sh_acc[wave][n][t * 16 + g * 4]) = st.acc[t] * by * st.unit;
      __syncthreads();
      const int col = threadIdx.x >> 4, ch0 = (threadIdx.x & 15) * (HD / 16);
      float top = NEG, sum = 0.0f, weight[WAVES];
#pragma unroll
      for (int v = 0; v < WAVES; ++v) top = fmaxf(top, sh_m[v][col]);
#pragma unroll
      for (int v = 0; v < WAVES; ++v) {
        weight[v] = __builtin_amdgcn_exp2f(sh_m[v][col] - top) * sh_l[v][col];
        sum += weight[v];
      }
      const float over = sum != 0.0f ? 1.0f / sum : 0.0f;  // nothing seen: 0
      float o[HD / 16];
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        o[i] = 0.0f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) o[i] += (weight[v] * over) * sh_acc[v][col][ch0 + i];
      }
      const bool all = x == 0 && end == span.pages;
      if (col < k.cols) {
        if (all) {
          const int token = (int)((uint32_t)(k.col0 + col) / (uint32_t)a.rep), h = head * a.rep + (k.col0 + col - token * a.rep);
          T *out = (T *)a.out + (int64_t)(s.row + token) * a.ldo + (int64_t)h * a.hso + ch0;
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) out[i] = (T)o[i];
        } else {
          float *p = a.part + ((2 * w + (at_start ? 0 : 1)) * COLS + col) * (HD + 2);
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) p[ch0 + i] = o[i];
          if ((threadIdx.x & 15) == 0) {
            p[HD] = top;
            p[HD + 1] = sum;
          }
        }
      }
      if (x == 0 && end < span.pages && threadIdx.x == 0) {
        int64_t *hd = a.header + w * 8;
        hd[H_PARTS] = 1 + (span.pages - end + run - 1) / run;
        hd[H_FIRST] = 2 * w + (at_start ? 0 : 1);
        hd[H_ROW] = s.row;
        hd[H_COLS] = k.cols;
        hd[H_HEAD] = head;
        hd[H_COL0] = k.col0;
      }
      at_start = false;
      __syncthreads();
    }
    ++b;
    inside = 0;
  }
}

// Joins the parts of the item that begins in run blockIdx.x and goes on: the first part lies at H_FIRST, the others at the
// beginnings of the following runs.  Up to eight parts (a batch of sequences: an item meets few runs) take a wavefront per column, which
// asks for all of them at once; more (one long cache) a workgroup per column: maxima and sums are fetched together, then each
// wavefront adds up a quarter of the parts, the first few requested along with the maxima.  (64 parts of 32 columns 7.0 us, of
// which 3.9 are what the launch takes with nothing to join; by one wavefront 9.)
constexpr int MOST_GROUPS = 1024;
template <typename T, int HD, int WIDTH> __global__ __launch_bounds__(256) void cache8_join_kernel(const AttnArgs a) {
  __shared__ float sh_w[MOST_GROUPS + 1], sh_red[8];
  __shared__ float sh_o[4][HD];
  const int w = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t *hd = a.header + (int64_t)w * 8;
  const int parts = (int)hd[H_PARTS], cols = (int)hd[H_COLS], slot0 = (int)hd[H_FIRST];
  if (!parts) return;
  typedef float Out __attribute__((ext_vector_type(HD / 64)));  // a lane's channels
  const auto part = [&](int i, int c) { return a.part + ((int64_t)(i ? 2 * (w + i) : slot0) * WIDTH + c) * (HD + 2); };
  const auto values = [&](int i, int c) {
    const float *p = part(i, c) + lane * (HD / 64);
    Out o;
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) o[j] = p[j];
    return o;
  };
  const auto out_at = [&](int c) {
    const uint32_t col = (uint32_t)hd[H_COL0] + c, token = col / (uint32_t)a.rep;
    const int64_t h = hd[H_HEAD] * a.rep + (col - token * a.rep);
    return (T *)a.out + (hd[H_ROW] + token) * a.ldo + h * a.hso;
  };
  constexpr int FEW = 8;
  if (parts <= FEW) {
    for (int c = blockIdx.y * 4 + wave; c < cols; c += gridDim.y * 4) {
      Out v[FEW];
      float m[FEW], l[FEW], top = NEG, sum = 0.0f;
#pragma unroll
      for (int i = 0; i < FEW; ++i) {
        const int at = min(i, parts - 1);
        m[i] = part(at, c)[HD];
        l[i] = part(at, c)[HD + 1];
        v[i] = values(at, c);
      }
#pragma unroll
      for (int i = 0; i < FEW; ++i) top = fmaxf(top, m[i]);
#pragma unroll
      for (int i = 0; i < FEW; ++i) {
        l[i] = i < parts ? l[i] * __builtin_amdgcn_exp2f(m[i] - top) : 0.0f;
        sum += l[i];
      }
      const float over = sum != 0.0f ? 1.0f / sum : 0.0f;
      Out o = {};
#pragma unroll
      for (int i = 0; i < FEW; ++i)
        if (i < parts) o += (l[i] * over) * v[i];
      T *out = out_at(c) + lane * (HD / 64);
#pragma unroll
      for (int j = 0; j < HD / 64; ++j) out[j] = (T)o[j];
    }
    return;
  }
  if (WIDTH == MANY) {
    for (int c = blockIdx.y * 4 + wave; c < cols; c += gridDim.y * 4) {
      float top = NEG, sum = 0.0f;
      for (int i = lane; i < parts; i += 64) top = fmaxf(top, part(i, c)[HD]);
#pragma unroll
      for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
      const auto weight = [&](int i) { return __builtin_amdgcn_exp2f(part(i, c)[HD] - top) * part(i, c)[HD + 1]; };
      for (int i = lane; i < parts; i += 64) sum += weight(i);
#pragma unroll
      for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
      const float over = sum != 0.0f ? 1.0f / sum : 0.0f;
      Out o = {};
      for (int i0 = 0; i0 < parts; i0 += 64) {
        const float x = i0 + lane < parts ? weight(i0 + lane) * over : 0.0f;  // the share of a lane's part
        const int some = min(64, parts - i0);
        for (int i = 0; i < some; i += FEW) {
          Out v[FEW];
#pragma unroll
          for (int e = 0; e < FEW; ++e) v[e] = values(i0 + min(i + e, some - 1), c);
#pragma unroll
          for (int e = 0; e < FEW; ++e)
            if (i + e < some) o += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), (i + e) & 63)) * v[e];
        }
      }
      T *out = out_at(c) + lane * (HD / 64);
#pragma unroll
      for (int j = 0; j < HD / 64; ++j) out[j] = (T)o[j];
    }
    return;
  }
  for (int c = blockIdx.y; c < cols; c += gridDim.y) {
    constexpr int EARLY = 8;
    Out early[EARLY];
#pragma unroll
    for (int e = 0; e < EARLY; ++e) early[e] = values(min(wave + 4 * e, parts - 1), c);
    float top = NEG, l0 = 0.0f;
    for (int i = t; i < parts; i += 256) {
      const float *p = part(i, c) + HD;
      const float m = p[0];
      if (i == t) l0 = p[1];
      sh_w[i] = m;
      top = fmaxf(top, m);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    if (lane == 0) sh_red[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(sh_red[0], sh_red[1]), fmaxf(sh_red[2], sh_red[3]));
    float sum = 0.0f;
    for (int i = t; i < parts; i += 256) {
      const float x = __builtin_amdgcn_exp2f(sh_w[i] - top) * (i == t ? l0 : part(i, c)[HD + 1]);
      sh_w[i] = x;
      sum += x;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
    if (lane == 0) sh_red[4 + wave] = sum;
    __syncthreads();
    sum = (sh_red[4] + sh_red[5]) + (sh_red[6] + sh_red[7]);
    const float over = sum != 0.0f ? 1.0f / sum : 0.0f;
    Out o = {};
#pragma unroll
    for (int e = 0; e < EARLY; ++e)
      if (wave + 4 * e < parts) o += (sh_w[wave + 4 * e] * over) * early[e];
#pragma unroll 4
    for (int i = wave + 4 * EARLY; i < parts; i += 4) o += (sh_w[i] * over) * values(i, c);
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) sh_o[wave][lane * (HD / 64) + j] = o[j];
    __syncthreads();
    if (t < HD) {
      out_at(c)[t] = (T)((sh_o[0][t] + sh_o[1][t]) + (sh_o[2][t] + sh_o[3][t]));
    }
    __syncthreads();
  }
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
//   Up to 32 columns a sequence (on the average): the kernel for few columns, which reads a page for every 16; 16 sequences of 4000
//   tokens, us few : many, 128 channels, 16 columns 34 : 49, 32 columns 52 : 50, 36 columns (three readings) 71 : 59; 64 channels, 32
//   columns 31 : 38, 64 columns 46 : 45; 256 channels, 32 columns 106 : 126, 36 columns 145 : 130.  One kernel for all sequences of a
//   step, and those that bring nothing count: the host does not know cu (300 single tokens and a chunk of 2048, all behind 4000, take
//   1017 us, 426 and 191 in calls of their own; a chunk of 4096 in a view of 600 sequences 1506, in a view of its own 425).  fp32
//   queries always, prompts among them (three of 2000 tokens behind 2000: 1264 us, 319 in 16 bits).
//   Many columns: whole items where there is one for every workgroup that fits the chip, which shares nothing (2048 tokens behind
//   4000, us in runs : whole items 228 : 196, 16384 behind nothing 2490 : 2215); the search for an item's block goes through all
//   blocks for each item, so not beyond 4096 of them or 1024 sequences.  Fewer items: the lengths decide, on the device.
constexpr int64_t FEW_COLUMNS = 2 * COLS;
struct Plan {
  bool many;
  ItemPlan items;
  int groups;    // workgroups of equal runs
  int64_t grid;  // and all workgroups
};
Plan plan_of(int cus, int32_t dtype, int64_t rows, int n_seqs, int heads, int rep, int hd) {
  Plan p;
  const int64_t seqs = rows < n_seqs ? rows : n_seqs, cols = rows * rep;
  p.many = dtype != RVQ_F32 && cols > FEW_COLUMNS * seqs;
  const int per_cu = p.many && hd == 256 ? 1 : 2, fit = per_cu * cus / 8 * 8;  // as many for every XCD
  p.groups = fit < 8 ? 8 : fit < MOST_GROUPS ? fit : MOST_GROUPS;
  p.grid = p.groups;
  p.items = ITEMS_RUNS;
  const int64_t least = cols / MANY * heads, most = (cols / MANY + seqs) * heads;  // items
  constexpr int MOST_SEQS = 1024, MOST_BLOCKS = 4096;
  if (!p.many || n_seqs > MOST_SEQS || cols / MANY + seqs > MOST_BLOCKS) return p;
  if (least >= p.groups) {
    p.items = ITEMS_WHOLE;
    p.grid = most;
  } else if (most <= 2 * p.groups) {
    p.items = ITEMS_EITHER;
    if (most > p.grid) p.grid = most;
  }
  return p;
}

// bytes of workspace of a call
int64_t plan_bytes(const Plan &p, int hd) {
  if (p.items == ITEMS_WHOLE) return 16;
  return p.groups * (int64_t)64 + 2 * (int64_t)p.groups * (p.many ? MANY : COLS) * (hd + 2) * (int64_t)sizeof(float);
}

template <typename T, int HD> void launch_attn(const AttnArgs &a, const Plan &p, hipStream_t s) {
  const dim3 grid((unsigned)p.groups);  // of the joining kernel, and of equal runs
  if constexpr (!std::is_same<T, float>::value) {
    if (p.many) {
      rvq_launch_cache8_chunk(a, std::is_same<T, _Float16>::value, p.grid, p.items, s);
      if (p.items != ITEMS_WHOLE) hipLaunchKernelGGL((cache8_join_kernel<T, HD, MANY>), dim3(grid.x, 16), dim3(256), 0, s, a);
      return;
    }
  }
  hipLaunchKernelGGL((cache8_attn_kernel<T, HD>), grid, dim3(64 * WAVES), 0, s, a);
  const int64_t cols = a.c.rows * a.rep < COLS ? a.c.rows * a.rep : COLS;
  hipLaunchKernelGGL((cache8_join_kernel<T, HD, COLS>), dim3(grid.x, (unsigned)cols), dim3(256), 0, s, a);
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
  if (rows == 0) return 16;
  // The most that any step of up to `rows` rows takes.  Steps of one kernel take the same, or next to nothing where there is an item for
  // every workgroup: from some number of rows on, until there are too many blocks for that.  So it is the most of the largest step, the
  // smallest one, and the first one with many columns.
  const int cus = attn_cus(), heads = cache->n_kv_heads, rep = n_q_heads / heads, hd = cache->head_dim;
  const auto bytes = [&](int64_t n) { return plan_bytes(plan_of(cus, dtype, n, cache->n_seqs, heads, rep, hd), hd); };
  const int64_t first_many = rep > FEW_COLUMNS ? 1 : FEW_COLUMNS * cache->n_seqs / rep + 1;
  return std::max({bytes(1), bytes(std::min(first_many, rows)), bytes(rows)});
}

int rvq_cache8_attn(const rvq_cache8 *cache, const void *dQ, int32_t dtype, int64_t rows, int32_t n_q_heads,
                    int64_t ldq, int64_t hsq, const int32_t *dCu, float scale, int32_t window, int32_t sinks,
                    void *dOut, int64_t ldo, int64_t hso, void *dWorkspace, int64_t workspace_bytes, void *stream) {
  if (!attn_ok(cache, dtype, rows, n_q_heads) || !std::isfinite(scale * LOG2E) || window < 0 || sinks < 0) return RVQ_EINVAL;
  if (rows == 0) return RVQ_OK;
  const int hd = cache->head_dim;
  if (!rvq_cache8_pointers_ok(cache) || !rvq_aligned(dCu, 4)) return RVQ_EINVAL;
  if (!rvq_rows16_ok(dQ, dtype, rows, n_q_heads, hd, ldq, hsq) || !rvq_rows16_ok(dOut, dtype, rows, n_q_heads, hd, ldo, hso) ||
      !rvq_rows_distinct(rows, n_q_heads, hd, ldo, hso) || dQ == dOut)
    return RVQ_EINVAL;
  if (!rvq_aligned(dWorkspace, 16)) return RVQ_EINVAL;
  const int cus = attn_cus();
  if (!cus) return RVQ_EHIP;
  const Plan p = plan_of(cus, dtype, rows, cache->n_seqs, cache->n_kv_heads, n_q_heads / cache->n_kv_heads, hd);
  if (workspace_bytes < plan_bytes(p, hd)) return RVQ_EWORKSPACE;
  if (!rvq_stream_is_current((hipStream_t)stream)) return RVQ_EINVAL;
  AttnArgs a;
  a.c = view_of(cache, dCu, rows);
  a.q = dQ; a.out = dOut;
  a.ldq = ldq; a.hsq = hsq; a.ldo = ldo; a.hso = hso;
  a.rep = n_q_heads / cache->n_kv_heads;
  a.window = window; a.sinks = sinks;
  a.scale = scale * LOG2E;
  a.header = (int64_t *)dWorkspace;
  a.groups = p.groups;
  a.part = (float *)((char *)dWorkspace + (int64_t)p.groups * 64);
  if (dtype == RVQ_F32) launch_attn_hd<float>(a, p, (hipStream_t)stream);
  else if (dtype == RVQ_BF16) launch_attn_hd<__bf16>(a, p, (hipStream_t)stream);
  else launch_attn_hd<_Float16>(a, p, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? RVQ_OK : RVQ_EHIP;
}

}  // extern "C"
