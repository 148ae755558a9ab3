// Attention over the paged cache of 8-bit codes for many columns (query tokens times the heads that share a kv head): chunks of prompts.
//
// The same arithmetic as for few columns, with 32x32 products: an item has 128 columns, 32 for each wavefront, and the four
// share the page's 16 KiB of codes, which are copied to LDS a page ahead (straight from memory, 16 bytes a lane; pieces of
// a row change places so that the wavefront's reads of neighbouring rows hit different banks).  A lane holds one
// column and, of the two tiles of 32 tokens, the tokens 32 h .. 32 h + 31 (h = lane / 32): its weights are again what the
// second product takes from it.
//
// Codes become fp16 in registers, exactly, and queries are fp16 as in the kernel for few columns.  The products that take e4m3 codes
// as they are (32x32x64) need no conversion of keys, and with queries in two terms took 435 us for 470, but their
// sums are short: off by up to 2^-13 of the sum of magnitudes, where the fp16 products' are off by 2^-23 (measured on random codes).
//
// Weights are fp16, 11 bits.  The maximum that they refer to moves only where one passes fp16's range: they are held as
// 2^8 2^(s - m), so m may stay behind the true maximum by 2^7, and no maximum is taken per page, which would be two dependent
// chains over 32 scores.  They keep 11 bits down to 2^-22 of the largest, or to 2^-16 where the scales of values differ between
// pages (below; a page's by more than 2^64 from a larger one: fewer).  The sum is of the rounded weights: their roundings cancel in a mean of equal values.
//
// What bounds it is issue: per page and wavefront (128 channels) 1024 clocks of matrix instructions stand against 128
// conversions and some 4 operations, one of them an exponential of four times the length, for each of a lane's 32 scores; a probe
// of the two kinds side by side takes the longer one's time and a third of the other's.  Three sequences of 2000 to 4096 tokens behind
// up to 4000, 32 query heads on 8 kv heads of 128 channels: 455 us, 931 TFLOP/s, 69 % of what a large fp16 matrix product reaches (1345),
// both with the clock settled: the first 25 ms of such work take up to a third longer.  Sequences of 2000 tokens behind 2000, three of
// them: 64 channels 191 us, 128 319, 256 936; with a window of 1000 tokens 89, 145, 430.
// Tried and taken back (with the short sums, 435 us): the next page's scores between the exponentials (433 -> 458); s_setprio (no change);
// two pages to a barrier (431 -> 457); values turned into fp16 by one wavefront for all four, through LDS: a fifth fewer vector
// instructions and twice the reads of LDS (435 -> 475); a prescribed mix of products and weights (453 -> 456).

#include "rvq_cache8_attn.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float CHUNK_BITS = 8.0f;  // weights are held as 2^8 2^(s - m)

// The blocks of all sequences, 256 per trip, one per thread: visit(sequence, block, pages), pages = 0 for none, is called by all
// threads together until it returns true in all of them.  A block's sequence is found by bisection of the sequences' prefix sums.
struct Shared {
  int before[257], found[3];
  Together<64 * WAVES, int> wave;
  Together<64 * WAVES, int64_t> wave64;
  int64_t rest;
  int pages_like[512];
  int flags[WAVES];
};
// inclusive prefix sums over the workgroup's threads
template <typename N> __device__ __forceinline__ N scan256(N x, Together<64 * WAVES, N> &at, N &total) {
  __syncthreads();
  return scan_all(x, at, total);
}
// the 256 sequences from b0 on: their blocks, and prefix sums in `before`
__device__ __forceinline__ int count_blocks(const AttnArgs &a, Shared &sh, int b0) {
  const int t = threadIdx.x;
  int blocks;
  const int upto = scan256(b0 + t < a.c.n_seqs ? blocks_of(a, rows_of(a.c, b0 + t).n, MANY) : 0, sh.wave, blocks);
  sh.before[t + 1] = upto;
  if (t == 0) sh.before[0] = 0;
  __syncthreads();
  return blocks;
}
// block k of them: its sequence, its place there and its pages (0: there is no such block)
struct Place {
  int b, j, pages;
};
__device__ __forceinline__ Place place_of(const AttnArgs &a, const Shared &sh, int b0, int k, int blocks) {
  Place p = {0, 0, 0};
  if (k >= blocks) return p;
  int s = 0;
#pragma unroll
  for (int d = 128; d; d /= 2)
    if (sh.before[s + d] <= k) s += d;
  p.b = b0 + s;
  p.j = k - sh.before[s];
  const Seq q = seq_of(a, p.b);
  const Block x = block_of(a, q, p.j * MANY, MANY);
  p.pages = span_of(a, q, x.first, x.last).pages;
  return p;
}
template <typename Visit> __device__ __forceinline__ void walk(const AttnArgs &a, Shared &sh, Visit visit) {
  for (int b0 = 0; b0 < a.c.n_seqs; b0 += 256) {
    const int blocks = count_blocks(a, sh, b0);
    for (int k0 = 0; k0 < blocks; k0 += 256)
      if (visit(place_of(a, sh, b0, k0 + (int)threadIdx.x, blocks))) return;
    __syncthreads();
  }
}

// What a call's blocks amount to, for one kv head: pages, blocks, pages of the longest one.
struct Sums {
  int64_t pages;
  int blocks, longest;
};
__device__ __forceinline__ Sums sum_blocks(const AttnArgs &a, Shared &sh) {
  Sums s = {0, 0, 0};
  int64_t pages = 0;
  int blocks = 0, longest = 0;
  walk(a, sh, [&](const Place &p) {
    pages += p.pages;
    blocks += p.pages != 0;
    longest = max(longest, p.pages);
    return false;
  });
  (void)scan256(pages, sh.wave64, s.pages);
  (void)scan256(blocks, sh.wave, s.blocks);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) longest = max(longest, __shfl_xor(longest, d, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.wave.sums[threadIdx.x >> 6] = longest;
  __syncthreads();
  s.longest = max(max(sh.wave.sums[0], sh.wave.sums[1]), max(sh.wave.sums[2], sh.wave.sums[3]));
  return s;
}
// Pages of a workgroup's run: an equal share of all items' pages, but not under an eighth of the mean item, up to 8.  A shorter run
// costs more in its partial result (66 KB written and read for 128 columns of 128 channels, a page is 16 KB) than the others gain:
// 128 tokens behind 4000 take 90 us in runs of 5 pages and 55 in runs of 8; where items are short themselves, 9 tokens behind
// 100, runs of 8 pages take one workgroup through several items, 38 us for 18.
__device__ __forceinline__ int64_t run_length(const AttnArgs &a, const Sums &s) {
  const int64_t least = min((int64_t)8, s.pages / (8 * max(s.blocks, 1)));
  return max(max((s.pages * a.c.heads + a.groups - 1) / a.groups, least), (int64_t)1);
}
// Whether a workgroup had better take a whole item where there are fewer items than workgroups: a page of 128 channels takes some 1.45
// us where a CU has one workgroup and 2.3 where it has two (64 channels 1.1 and 1.55, 256, where there is one, 3.0); equal runs are
// shorter, but write and read their parts at some 3 TB/s and wait for the joining.  (1024 tokens, us in runs : whole items, 128
// channels, behind nothing 71 : 33, 4000 126 : 121, 30000 577 : 690; 64 channels 50 : 26, 88 : 92, 386 : 528; 256 channels 119 : 64,
// 258 : 246, 1438 : 1422.)
template <int HD> __device__ __forceinline__ bool items_whole(const AttnArgs &a, const Sums &s, int64_t run) {
  const float page1 = HD == 64 ? 1.1f : HD == 128 ? 1.45f : 3.0f, page2 = HD == 64 ? 1.55f : 2.3f;
  const int cus = a.groups / (HD == 256 ? 1 : 2), items = s.blocks * a.c.heads;
  const float runs = (float)((s.pages * a.c.heads + run - 1) / run), parts = fminf(runs + items, 2.0f * runs);
  const float whole = s.longest * (items > cus ? page2 : page1);
  const float shared = run * (runs > cus ? page2 : page1) + 8.0f + parts * (MANY * HD * 8) * (1.0f / 3e6f);
  return whole <= shared;
}

// the block that holds page `target` of all blocks' pages, and the page's place in it: found[0], found[1], rest
__device__ __forceinline__ void find_unit(const AttnArgs &a, Shared &sh, int64_t target) {
  int64_t base = 0;
  if (threadIdx.x == 0) sh.found[0] = -1;
  walk(a, sh, [&](const Place &p) {
    int64_t total;
    const int64_t at = base + scan256((int64_t)p.pages, sh.wave64, total) - p.pages;
    if (at <= target && target < at + p.pages) {
      sh.found[0] = p.b;
      sh.found[1] = p.j;
      sh.rest = target - at;
    }
    __syncthreads();
    base += total;
    return sh.found[0] >= 0;
  });
}

// Blocks by length, the longest first, to within a sixteenth: a block's class is the exponent of its pages and four more bits.
__device__ __forceinline__ int class_of(int pages) {
  const int e = 31 - __clz(pages);
  return 511 - (e * 16 + (int)(((int64_t)pages << 4) >> e) - 16);
}
// the block of that rank: found[0], found[1]; found[0] < 0: there are not so many
__device__ __forceinline__ void find_rank(const AttnArgs &a, Shared &sh, int rank) {
  const int t = threadIdx.x;
  sh.pages_like[t] = sh.pages_like[t + 256] = 0;
  if (t == 0) sh.found[0] = sh.found[2] = -1;
  Place last = {0, 0, 0};
  int trips = 0;
  walk(a, sh, [&](const Place &p) {  // (barriers of the walk come before the first count)
    if (p.pages) atomicAdd(&sh.pages_like[class_of(p.pages)], 1);
    last = p;
    ++trips;
    return false;
  });
  __syncthreads();
  const int one = sh.pages_like[2 * t], two = one + sh.pages_like[2 * t + 1];
  int total;
  const int at = scan256(two, sh.wave, total) - two;
  if (at <= rank && rank < at + two) {
    const bool second = rank >= at + one;
    sh.found[2] = 2 * t + second;
    sh.before[0] = rank - at - (second ? one : 0);
  }
  __syncthreads();
  const int cls = sh.found[2], place = sh.before[0];
  if (cls < 0) return;
  __syncthreads();  // `before` is written again
  int base = 0;
  const auto look = [&](const Place &p) {
    const int hit = p.pages && class_of(p.pages) == cls;
    const int before = base + scan256(hit, sh.wave, total) - hit;
    if (hit && before == place) {
      sh.found[0] = p.b;
      sh.found[1] = p.j;
    }
    __syncthreads();
    base += total;
    return sh.found[0] >= 0;
  };
  if (trips == 1) look(last);  // every thread still holds its block
  else walk(a, sh, look);
}

template <typename T, int HD> struct Chunk {
  static constexpr int BYTES = 2 * PAGE * HD;  // of a page and kv head
  f16x8 q[HD / 16];                            // a lane holds channels 64 c + 32 h + 8 j .. of product 4 c + j
  f32x16 acc[HD / 32];
  float factor, m, l;
  Sight sight;
};

template <typename T, int HD>
__device__ __forceinline__ void load_chunk(const AttnArgs &a, const Seq &s, int head, int col, bool valid, Chunk<T, HD> &k) {
  const int h = (threadIdx.x >> 5) & 1;
  const int token = (int)((uint32_t)col / (uint32_t)a.rep);
  float x[HD / 16][8];
  float amax = 0.0f;
  const T *q = (const T *)a.q + (int64_t)(s.row + token) * a.ldq + (int64_t)(head * a.rep + (col - token * a.rep)) * a.hsq;
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) {
    if (valid) {
      load8<T>(q + (i >> 2) * 64 + h * 32 + (i & 3) * 8, x[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) amax = not_finite(x[i][j]) ? amax : fmaxf(amax, fabsf(x[i][j]));
  }
  amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
  int e = (int)(__float_as_uint(amax) >> 23) - 127 - 8;  // largest element to [2^8, 2^9)
  e = e < -118 ? -118 : e;
  // a factor >= 0, so that the largest product is the largest score
  const float down = __uint_as_float((uint32_t)(127 - e) << 23) * (a.scale < 0.0f ? -1.0f : 1.0f);
  k.factor = ldexpf(fabsf(a.scale), e);
  k.sight = valid ? sight_of(a, s, s.p0 + token) : Sight{-1, -1};
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
}

// Where 16-byte piece c of a row lies in LDS, for keys (HD bytes a row) and values (64 bytes).  Eight lanes read a piece each
// per LDS cycle, of rows 0 1 2 3 32 33 34 35 (keys: the order of a tile's tokens) or of eight rows in turn (values); so placed, the
// eight lie in different banks.
template <int HD> __device__ __forceinline__ int key_piece(int row, int c) {
  return HD == 64 ? c ^ (((row >> 1) & 1) | ((row >> 4) & 2)) : c ^ ((row & 3) | ((row >> 3) & 4));
}
__device__ __forceinline__ int value_piece(int row, int c) { return c ^ ((row >> 1) & 3); }

// Copies a page's codes of one kv head to LDS, 1024 bytes per wavefront and step, keys first; a wavefront's own part is complete
// after vmcnt(0).  `from`: this lane's bytes of the page.
template <int HD> struct Fetch {
  static constexpr int STEPS = 2 * HD / 64;
  uint32_t from[STEPS];
  __device__ __forceinline__ Fetch() {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int at = (i * WAVES + wave) * 64 + lane;  // 16-byte piece in LDS
      if (i < HD / 64) {
        const int row = at / (HD / 16);
        from[i] = (row * (HD / 16) + key_piece<HD>(row, at % (HD / 16))) * 16;
      } else {
        const int row = (at - 4 * HD) >> 2;
        from[i] = (4 * HD + row * 4 + value_piece(row, at & 3)) * 16;
      }
    }
  }
  __device__ __forceinline__ void operator()(const uint8_t *codes, uint8_t *to) const {
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(codes + from[i]),
                                       (__attribute__((address_space(3))) void *)(to + (i * WAVES + wave) * 1024), 16, 0, 0);
  }
};

// Of the pages of a span, by their place i: those behind the sinks' that a block of columns sees anything of, [from, to), and
// those that it sees whole, [all_from, all_to).  (Pages of sinks, where there are any, count as seen in part.)
struct Range {
  int from, to, all_from, all_to;
};
__device__ __forceinline__ Range range_of(const AttnArgs &a, const Seq &s, const Block &k, const Span &span) {
  const int shift = span.sink_pages - span.begin;  // place = page + shift
  const int hide = hidden_to(a, k.first), hide_all = hidden_to(a, k.last);
  const int seen = min(k.last, s.tokens - 1), seen_by_all = min(k.first, s.tokens - 1);
  Range r;
  r.from = a.sinks > span.begin * PAGE ? span.sink_pages : max(span.sink_pages, (hide + 1) / PAGE + shift);
  r.to = max(span.sink_pages, (seen < 0 ? 0 : seen / PAGE + 1) + shift);  // (less: a window that begins behind the table's end)
  r.all_from = max(span.sink_pages, (hide_all + PAGE) / PAGE + shift);
  r.all_to = (seen_by_all + 1) / PAGE + shift;
  return r;
}

// Scale of the accumulators, the same in every lane; 0: they hold nothing yet.
struct Measure {
  float now, most;  // and the largest scale of values so far
};

// One page for this wavefront's columns.  `whole`: every column sees every token; values' codes hold no NaN otherwise.
template <typename T, int HD>
__device__ __forceinline__ void take_chunk_page(const AttnArgs &a, Chunk<T, HD> &k, const uint8_t *codes, float kscale, float vscale,
                                                Measure &unit, int t0, int whole) {
  const int lane = threadIdx.x & 63, h = lane >> 5, n = lane & 31;
  const uint8_t *kc = codes, *vc = codes + PAGE * HD;
  f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
  for (int c = 0; c < HD / 64; ++c) {
    u32x4 w[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // row n of tile i is token 32 ((n / 4) % 2) + 16 i + 4 (n / 8) + n % 4
      const int row = ((n >> 2) & 1) * 32 + i * 16 + (n >> 3) * 4 + (n & 3);
#pragma unroll
      for (int e = 0; e < 2; ++e) w[i][e] = *reinterpret_cast<const u32x4 *>(kc + row * HD + key_piece<HD>(row, 4 * c + 2 * h + e) * 16);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(w[i][j >> 1][(j & 1) * 2], w[i][j >> 1][(j & 1) * 2 + 1]), k.q[4 * c + j], s[i], 0, 0, 0);
  }
  // the values' codes are on their way while the weights are made, where registers allow it
  constexpr bool EARLY = HD <= 128;
  u32x4 v[EARLY ? HD / 32 : 1][2];
  const auto values = [&](int c, int i) {
    const int row = c * 32 + n;
    return *reinterpret_cast<const u32x4 *>(vc + row * PAGE + value_piece(row, 2 * h + i) * 16);
  };
  if constexpr (EARLY) {
#pragma unroll
    for (int c = 0; c < HD / 32; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) v[c][i] = values(c, i);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (!whole) {
    const uint32_t seen = seen_bits(a, k.sight, t0 + h * 32);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const uint32_t m = spread_bit(seen, i);
      s[i >> 4][i & 15] = __uint_as_float((__float_as_uint(s[i >> 4][i & 15]) & m) | (0xff800000u & ~m));  // hidden: -infinity
    }
  }
  const float factor = fmaxf(k.factor * kscale, 1e-37f);  // not 0, which would make a number of a hidden score
  // The accumulators' unit is a page's scale: a larger one takes over (the first page's from 0), and one that is smaller by more than
  // 2^6 does, but not under 2^-64 of the largest so far (2^31 weights below 2^16, codes of 448: the accumulators stay below 2^120).  A
  // page of a smaller scale than the unit gets weights that are as much smaller, but not in the sum of weights.
  if (__builtin_amdgcn_readfirstlane((vscale > unit.now) | (vscale < unit.now * 0x1p-6f))) {
    unit.most = uniform(fmaxf(unit.most, vscale));
    const float to = uniform(fmaxf(fmaxf(vscale, unit.most * 0x1p-64f), 0x1p-126f)), all = unit.now / to;
    unit.now = to;
#pragma unroll
    for (int c = 0; c < HD / 32; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) k.acc[c][r] *= all;
  }
  float shift = CHUNK_BITS, count = 1.0f;
  const int tiny = vscale < unit.now * 0x1p-6f;  // (a page of zeros, say) such weights may be nothing in fp16: the sum is made without
  if (vscale != unit.now && !tiny) {
    count = unit.now / vscale;
    shift -= __builtin_amdgcn_logf(count);
  }
  f16x8 w[2][2];
  float sum;
  const auto weigh = [&](int i, float ref) {  // tile i
    sum = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const f32x2 two = {__builtin_amdgcn_exp2f(fmaf(s[i][2 * j], factor, ref)), __builtin_amdgcn_exp2f(fmaf(s[i][2 * j + 1], factor, ref))};
      const f16x2 r = __builtin_convertvector(two, f16x2);
      sum = __builtin_amdgcn_fdot2(r, f16x2{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
      w[i][j >> 2][2 * j & 7] = r[0];
      w[i][j >> 2][(2 * j & 7) + 1] = r[1];
    }
  };
  const auto settle = [&](int i) {
    // A weight beyond fp16 (infinity in the sum) asks for another reference: the maximum so far.
    if (__builtin_amdgcn_readfirstlane(__ballot(__float_as_uint(sum) == 0x7f800000u) != 0)) {
      float top = s[i][0];
#pragma unroll
      for (int j = 1; j < 16; ++j) top = fmaxf(top, s[i][j]);
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      top = fmaxf(k.m, top * factor);
      const float fix = __builtin_amdgcn_exp2f(k.m - top);
      k.m = top;
      k.l *= fix;
#pragma unroll
      for (int c = 0; c < HD / 32; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) k.acc[c][r] *= fix;
      weigh(i, shift - k.m);
    }
    k.l += sum * count;
    if (__builtin_amdgcn_readfirstlane(tiny)) weigh(i, CHUNK_BITS - __builtin_amdgcn_logf(unit.now / vscale) - k.m);
  };
  const auto add = [&](int i) {
#pragma unroll
    for (int c = 0; c < HD / 32; ++c) {
      const u32x4 x = EARLY ? v[EARLY ? c : 0][i] : values(c, i);
#pragma unroll
      for (int j = 0; j < 2; ++j) k.acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(x[2 * j], x[2 * j + 1]), w[i][j], k.acc[c], 0, 0, 0);
    }
  };
  // the second tile's weights behind the first one's products (both tiles' weights first: 467 us, then, for 453)
  weigh(0, shift - k.m);
  settle(0);
  add(0);
  weigh(1, shift - k.m);
  settle(1);
  add(1);
}

// A NaN among the values' codes of a slot that some column does not see must not meet its weight of 0.  For pages that not
// every column of the workgroup sees whole: looks for one; where there is, every wavefront makes NaN of the (channel, column)
// pairs that see it (counted by a product of marks), and then the codes are taken out of the tile.  Called by all wavefronts.
template <typename T, int HD>
__device__ __forceinline__ void settle_nan(const AttnArgs &a, Chunk<T, HD> &k, uint8_t *vc, int t0, bool busy, int *flags) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, n = lane & 31;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < HD / 64; ++i) {
    const u32x4 v = *reinterpret_cast<const u32x4 *>(vc + ((i * WAVES + wave) * 64 + lane) * 16);
    any |= nan_bytes(v[0]) | nan_bytes(v[1]) | nan_bytes(v[2]) | nan_bytes(v[3]);
  }
  const int mine = __ballot(any != 0) != 0;
  if (lane == 0) flags[wave] = mine;
  __syncthreads();
  if (!__builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3])) return;
  if (busy) {
    const uint32_t seen = seen_bits(a, k.sight, t0 + h * 32);
#pragma unroll
    for (int c = 0; c < HD / 32; ++c) {
      const int row = c * 32 + n;
      f32x16 d = f32x16{};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x2 v = *reinterpret_cast<const u32x2 *>(vc + row * PAGE + value_piece(row, 2 * h + (i >> 1)) * 16 + (i & 1) * 8);
        u32x4 one;  // fp16 ones of the tokens that are seen
#pragma unroll
        for (int j = 0; j < 4; ++j)
          one[j] = (spread_bit(seen, i * 8 + 2 * j) & 0x3c00u) | (spread_bit(seen, i * 8 + 2 * j + 1) & 0x3c000000u);
        // 0x38 is the code of 1
        d = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8((nan_bytes(v[0]) >> 7) * 0x38u, (nan_bytes(v[1]) >> 7) * 0x38u),
                                                   __builtin_bit_cast(f16x8, one), d, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) k.acc[c][r] = __uint_as_float(d[r] > 0.0f ? 0x7fc00000u : __float_as_uint(k.acc[c][r]));
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < HD / 64; ++i) {
    u32x4 *at = reinterpret_cast<u32x4 *>(vc + ((i * WAVES + wave) * 64 + lane) * 16);
    u32x4 v = *at;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] &= ~((nan_bytes(v[j]) >> 7) * 0xffu);
    *at = v;
  }
  __syncthreads();
}

// ITEMS_WHOLE: a workgroup takes one item, the longest first (in the order of the blocks, three sequences of 2000 to 2500 tokens
// behind 1000 to 3300 keep the chip busy for 237 pages' time, longest first 215, of 206 that all the work takes);
// ITEMS_RUNS: an equal run of the items' pages, as in the kernel for few columns; ITEMS_EITHER: what the lengths say.
template <typename T, int HD>
__global__ __launch_bounds__(64 * WAVES, HD == 256 ? 1 : 2) void cache8_chunk_kernel(const AttnArgs a, ItemPlan items) {
  typedef Chunk<T, HD> C;
  __shared__ __align__(16) uint8_t tile[2][C::BYTES];
  __shared__ Shared sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;
  int64_t w = blockIdx.x;
  int b, head, j, x = 0;
  int64_t left, run = 1;
  Sums sums = {0, 0, 0};
  bool whole_items = items == ITEMS_WHOLE;
  if (!whole_items) {
    sums = sum_blocks(a, sh);
    if (!sums.blocks) {
      if (threadIdx.x == 0 && w < a.groups) a.header[w * 8 + H_PARTS] = 0;
      return;
    }
    run = run_length(a, sums);
    if (items == ITEMS_EITHER && items_whole<HD>(a, sums, run)) {
      whole_items = true;
      if (threadIdx.x == 0 && w < a.groups) a.header[w * 8 + H_PARTS] = 0;  // nothing to join
    } else if (w >= a.groups) {
      return;
    }
  }
  if (whole_items) {
    find_rank(a, sh, (int)(w / a.c.heads));
    if (sh.found[0] < 0) return;
    b = sh.found[0];
    j = sh.found[1];
    head = (int)(w % a.c.heads);
    left = INT32_MAX;
  } else {
    // Runs go through the blocks of one kv head after the other, and the workgroups of an XCD (every eighth) take neighbouring
    // runs: what they read together is a head or two, and stays in their L2 (16384 tokens, 8 kv heads, in runs: 2.95 -> 2.45 ms).
    const int64_t runs = (sums.pages * a.c.heads + run - 1) / run, eighth = (runs + 7) / 8;
    w = w < 8 * eighth ? w % 8 * eighth + w / 8 : w;
    if (threadIdx.x == 0) a.header[w * 8 + H_PARTS] = 0;
    if (w >= runs) return;
    head = (int)(w * run / sums.pages);
    find_unit(a, sh, w * run % sums.pages);
    b = sh.found[0];
    j = sh.found[1];
    x = (int)sh.rest;
    left = run;
  }
  b = __builtin_amdgcn_readfirstlane(b);
  head = __builtin_amdgcn_readfirstlane(head);
  j = __builtin_amdgcn_readfirstlane(j);
  x = __builtin_amdgcn_readfirstlane(x);
  bool at_start = true;
  const Fetch<HD> fetch;
  while (true) {
    const Seq s = seq_of(a, b);
    const Block k = block_of(a, s, j * MANY, MANY);
    const Span span = span_of(a, s, k.first, k.last);
    const int end = (int)min((int64_t)span.pages, x + left);
    left -= end - x;
    const int col = wave * 32 + n;
    C c;
    load_chunk<T, HD>(a, s, head, k.col0 + col, col < k.cols, c);
    Measure unit = {0.0f, 0.0f};
    // this wavefront's columns
    const bool busy = wave * 32 < k.cols;
    const Range mine = range_of(a, s, busy ? block_of(a, s, k.col0 + wave * 32, min(32, k.cols - wave * 32)) : k, span);
    const Range ours = range_of(a, s, k, span);
    const int m_from = __builtin_amdgcn_readfirstlane(mine.from), m_to = __builtin_amdgcn_readfirstlane(busy ? mine.to : 0);
    const int m_all_from = __builtin_amdgcn_readfirstlane(mine.all_from), m_all_to = __builtin_amdgcn_readfirstlane(mine.all_to);
    // the page in hand, the next one, on its way to LDS while the wavefronts work on this, and the entry behind it
    const int32_t *table = a.c.table + (int64_t)b * a.c.table_pages;
    const uint8_t *codes = codes_of(a.c, 0, head, 0);
    const float *scale = scale_of(a.c, 0, head, 0);
    const int64_t page_bytes = (int64_t)a.c.heads * C::BYTES;
    const int n_pages = (int)min(a.c.n_pages, (int64_t)INT32_MAX), sinks = span.sink_pages, behind = span.begin - sinks;
    const auto id_of = [&](int i) {
      const int entry = i < sinks ? i : i + behind;
      const int id = i < end && entry < a.c.table_pages ? table[entry] : -1;
      return id < n_pages ? id : -1;
    };
    const auto scales_of = [&](int id) { return *reinterpret_cast<const f32x2 *>(scale + (int64_t)max(id, 0) * a.c.heads * 2); };
    int page = __builtin_amdgcn_readfirstlane(id_of(x)), next = id_of(x + 1);
    f32x2 scales = scales_of(page);
    __syncthreads();  // the tiles are free
    if (page >= 0) fetch(codes + page * page_bytes, tile[0]);
    for (int i = x; i < end; ++i) {
      const int cur = (i - x) & 1;
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wavefront's part of the page has landed
      __syncthreads();
      next = __builtin_amdgcn_readfirstlane(next);
      const int after = id_of(i + 2);
      const f32x2 next_scales = scales_of(next);
      if (next >= 0) fetch(codes + next * page_bytes, tile[cur ^ 1]);
      if (page >= 0) {
        const int t0 = (i < sinks ? i : i + behind) * PAGE;
        if (i < ours.all_from || i >= ours.all_to) settle_nan<T, HD>(a, c, tile[cur] + PAGE * HD, t0, busy, sh.flags);
        if (i < m_to && (i >= m_from || i < sinks))
          take_chunk_page<T, HD>(a, c, tile[cur], uniform(scales[0]), uniform(scales[1]), unit, t0, i >= m_all_from && i < m_all_to);
      }
      page = next;
      next = after;
      scales = next_scales;
    }
    c.l += __shfl_xor(c.l, 32, 64);
    const bool all = x == 0 && end == span.pages;
    if (col < k.cols) {
      const int ch0 = h * 4;
      // the mean, which is no larger than the values (the sums may pass fp32); 0 where nothing was seen
      const float over = (__float_as_uint(c.l) << 1) != 0 ? 1.0f / c.l : 0.0f;
      if (all) {
        const int token = (int)((uint32_t)(k.col0 + col) / (uint32_t)a.rep), hq = head * a.rep + (k.col0 + col - token * a.rep);
        T *out = (T *)a.out + (int64_t)(s.row + token) * a.ldo + (int64_t)hq * a.hso + ch0;
#pragma unroll
        for (int t = 0; t < HD / 32; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            typename Vec4<T>::type o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = (T)(c.acc[t][q * 4 + r] * over * unit.now);
            *reinterpret_cast<typename Vec4<T>::type *>(out + t * 32 + q * 8) = o;
          }
      } else {
        float *p = a.part + ((2 * w + (at_start ? 0 : 1)) * MANY + col) * (HD + 2);
#pragma unroll
        for (int t = 0; t < HD / 32; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) p[t * 32 + q * 8 + ch0 + r] = c.acc[t][q * 4 + r] * over * unit.now;
        if (h == 0) {
          p[HD] = c.m;
          p[HD + 1] = c.l;
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
    if (whole_items || left <= 0) return;
    // the next item: the next block, sequence with rows, head
    x = 0;
    if (++j < blocks_of(a, s.n, MANY)) continue;
    j = 0;
    do {
      if (++b >= a.c.n_seqs) {
        b = 0;
        if (++head >= a.c.heads) return;
      }
    } while (rows_of(a.c, b).n == 0);
  }
}

}  // namespace

void rvq_launch_cache8_chunk(const AttnArgs &a, bool half, int64_t grid, ItemPlan items, hipStream_t s) {
  const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * WAVES), 0, s, a, items); };
  if (a.c.hd == 64) half ? go(cache8_chunk_kernel<_Float16, 64>) : go(cache8_chunk_kernel<__bf16, 64>);
  else if (a.c.hd == 128) half ? go(cache8_chunk_kernel<_Float16, 128>) : go(cache8_chunk_kernel<__bf16, 128>);
  else half ? go(cache8_chunk_kernel<_Float16, 256>) : go(cache8_chunk_kernel<__bf16, 256>);
}
