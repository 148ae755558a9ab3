// Attention over the paged cache of 8-bit codes for many columns (query tokens times the heads that share a kv head): chunks of prompts.
//
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

#include "rvq_cache8_attn.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float CHUNK_BITS = 8.0f, CHUNK_SLACK = 7.0f;

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
    const int64_t upto = scan256(b0 + t < a.c.n_seqs ? blocks_of(a, rows_of(a.c, b0 + t).n, MANY) : 0, sh.wave, total);
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
        const Seq q = seq_of(a, b0 + s);
        const Block x = block_of(a, q, (int)j * MANY, MANY);
        units = (int64_t)span_of(a, q, x.first, x.last).pages * a.c.heads;
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

// One page for this wavefront's columns.  `whole`: every column sees every token; values' codes hold no NaN otherwise.
template <typename T, int HD>
__device__ __forceinline__ void take_chunk_page(const AttnArgs &a, Chunk<T, HD> &k, const uint8_t *codes, float kscale, float vscale,
                                                float &unit, int t0, int whole) {
  const int lane = threadIdx.x & 63, h = lane >> 5, n = lane & 31;
  const uint8_t *kc = codes, *vc = codes + PAGE * HD;
  f32x16 s[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    // row n of tile i is token 32 ((n / 4) % 2) + 16 i + 4 (n / 8) + n % 4
    const int row = ((n >> 2) & 1) * 32 + i * 16 + (n >> 3) * 4 + (n & 3);
    u32x4 x[HD / 32];
#pragma unroll
    for (int c = 0; c < HD / 32; ++c) x[c] = *reinterpret_cast<const u32x4 *>(kc + row * HD + piece<HD / 16>(row, 2 * c + h) * 16);
    s[i] = f32x16{};
#pragma unroll
    for (int c = 0; c < HD / 32; ++c) {
      s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(x[c][0], x[c][1]), k.q[2 * c], s[i], 0, 0, 0);
      s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(x[c][2], x[c][3]), k.q[2 * c + 1], s[i], 0, 0, 0);
    }
  }
  if (!whole) {
#pragma unroll
    for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] = sees(a, k.sight, t0 + h * 32 + i) ? s[i >> 4][i & 15] : -INFINITY;
  }
  float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(fmaxf(top, s[0][i]), s[1][i]);
  top = fmaxf(top, __shfl_xor(top, 32, 64));
  const float factor = k.factor * kscale;
  top = fmaxf(k.m, top * factor);
  // (the condition is the same in every lane; it is handed over as a scalar so that the branch leaves the accumulators in place)
  const int move = (__ballot(top > k.m + CHUNK_SLACK) != 0) | (vscale > unit) | (vscale < unit * 0x1p-6f);
  if (__builtin_amdgcn_readfirstlane(move)) {
    // the accumulators' unit: this page's scale, but no more than 2^40 below the last one
    const float low = unit * 0x1p-40f, to = uniform(vscale < low ? low : vscale);
    const float fix = __builtin_amdgcn_exp2f(k.m - top), all = fix * (unit / to);
    k.m = top;
    k.l *= fix;
    unit = to;
#pragma unroll
    for (int c = 0; c < HD / 32; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) k.acc[c][r] *= all;
  }
  // a page of a smaller scale than the accumulators' unit: its weights are that much smaller, but not in the sum of weights
  float ref = CHUNK_BITS - k.m, count = 1.0f;
  if (vscale != unit) {
    count = unit / vscale;
    ref -= __builtin_amdgcn_logf(count);
  }
  float sum[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      s[i][j] = __builtin_amdgcn_exp2f(fmaf(s[i][j], factor, ref));
      sum[i] += s[i][j];
    }
  k.l += (sum[0] + sum[1]) * count;
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
#pragma unroll
  for (int c = 0; c < HD / 32; ++c) {
    const int row = c * 32 + n;
    u32x4 v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = *reinterpret_cast<const u32x4 *>(vc + row * PAGE + piece<4>(row, 2 * h + i) * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      k.acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(v[i >> 1][(i & 1) * 2], v[i >> 1][(i & 1) * 2 + 1]), w[i], k.acc[c], 0, 0, 0);
  }
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
#pragma unroll
    for (int c = 0; c < HD / 32; ++c) {
      const int row = c * 32 + n;
      f32x16 d = f32x16{};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x2 v = *reinterpret_cast<const u32x2 *>(vc + row * PAGE + piece<4>(row, 2 * h + (i >> 1)) * 16 + (i & 1) * 8);
        f16x8 one;
#pragma unroll
        for (int j = 0; j < 8; ++j) one[j] = sees(a, k.sight, t0 + h * 32 + i * 8 + j) ? (_Float16)1.0f : (_Float16)0.0f;
        // 0x38 is the code of 1
        d = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8((nan_bytes(v[0]) >> 7) * 0x38u, (nan_bytes(v[1]) >> 7) * 0x38u), one, d, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) k.acc[c][r] = d[r] > 0.0f ? __uint_as_float(0x7fc00000u) : k.acc[c][r];
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

// `whole`: a workgroup takes one item, blockIdx.x / heads counting blocks from the last of every sequence (the longest) on;
// else an equal run of the items' pages, as in the kernel for few columns.
template <typename T, int HD>
__global__ __launch_bounds__(64 * WAVES, HD == 256 ? 1 : 2) void cache8_chunk_kernel(const AttnArgs a, int whole_items) {
  typedef Chunk<T, HD> C;
  __shared__ __align__(16) uint8_t tile[2][C::BYTES];
  __shared__ WalkShared sh;
  __shared__ int flags[WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;
  const int64_t w = blockIdx.x;
  int b, head, j, x = 0;
  int64_t left, run = 1;
  if (whole_items) {
    int64_t at;
    if (!find_piece(a.c.n_seqs, w / a.c.heads, [&](int i) { return (int64_t)blocks_of(a, rows_of(a.c, i).n, MANY); }, b, at)) return;
    head = (int)(w % a.c.heads);
    j = blocks_of(a, rows_of(a.c, b).n, MANY) - 1 - (int)at;
    left = INT32_MAX;
  } else {
    if (threadIdx.x == 0) a.header[w * 8 + H_PARTS] = 0;
    const int64_t total = walk<false>(a, sh, 0), even = (total + gridDim.x - 1) / gridDim.x;
    run = even > a.least ? even : a.least;
    if (w * run >= total) return;
    walk<true>(a, sh, w * run);
    b = (int)sh.found[0];
    j = (int)sh.found[1];
    left = run;
    const Seq s = seq_of(a, b);
    const Block k = block_of(a, s, j * MANY, MANY);
    const int pages = span_of(a, s, k.first, k.last).pages;
    head = (int)(sh.found[2] / pages);
    x = (int)(sh.found[2] % pages);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  head = __builtin_amdgcn_readfirstlane(head);
  j = __builtin_amdgcn_readfirstlane(j);
  x = __builtin_amdgcn_readfirstlane(x);
  bool at_start = true;
  while (true) {
    const Seq s = seq_of(a, b);
    const Block k = block_of(a, s, j * MANY, MANY);
    const Span span = span_of(a, s, k.first, k.last);
    const int end = (int)min((int64_t)span.pages, x + left);
    left -= end - x;
    const int col = wave * 32 + n;
    C c;
    load_chunk<T, HD>(a, s, head, k.col0 + col, col < k.cols, c);
    float unit = 1.0f;  // scale of the accumulators, the same in every lane
    // this wavefront's columns
    const bool busy = wave * 32 < k.cols;
    const Block mine = busy ? block_of(a, s, k.col0 + wave * 32, min(32, k.cols - wave * 32)) : k;
    // the page in hand, the next one, on its way to LDS while the wavefronts work on this, and the entry behind it
    const auto scales_of = [&](int id) { return id >= 0 ? *reinterpret_cast<const f32x2 *>(scale_of(a.c, id, head, 0)) : f32x2{0, 0}; };
    int page = __builtin_amdgcn_readfirstlane(page_of(a.c, b, span.entry(x)));
    int next = x + 1 < end ? page_of(a.c, b, span.entry(x + 1)) : -1;
    f32x2 scales = scales_of(page);
    __syncthreads();  // the tiles are free
    if (page >= 0) fetch_page<HD>(codes_of(a.c, page, head, 0), tile[0]);
    for (int i = x; i < end; ++i) {
      const int cur = (i - x) & 1;
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wavefront's part of the page has landed
      __syncthreads();
      next = __builtin_amdgcn_readfirstlane(next);
      const int after = i + 2 < end ? page_of(a.c, b, span.entry(i + 2)) : -1;
      const f32x2 next_scales = scales_of(next);
      if (next >= 0) fetch_page<HD>(codes_of(a.c, next, head, 0), tile[cur ^ 1]);
      const int t0 = span.entry(i) * PAGE;
      if (page >= 0) {
        if (!all_see(a, s, k, t0)) settle_nan<T, HD>(a, c, tile[cur] + PAGE * HD, t0, busy, flags);
        if (busy && !none_sees(a, s, mine, t0))
          take_chunk_page<T, HD>(a, c, tile[cur], uniform(scales[0]), uniform(scales[1]), unit, t0, all_see(a, s, mine, t0));
      }
      page = next;
      next = after;
      scales = next_scales;
    }
    c.l += __shfl_xor(c.l, 32, 64);
    const bool all = x == 0 && end == span.pages;
    if (col < k.cols) {
      const int ch0 = h * 4;
      if (all) {
        const int token = (int)((uint32_t)(k.col0 + col) / (uint32_t)a.rep), hq = head * a.rep + (k.col0 + col - token * a.rep);
        T *out = (T *)a.out + (int64_t)(s.row + token) * a.ldo + (int64_t)hq * a.hso + ch0;
        const bool some = (__float_as_uint(c.l) << 1) != 0;  // else nothing was seen: 0
        const float over = some ? unit / c.l : 0.0f;
#pragma unroll
        for (int t = 0; t < HD / 32; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) out[t * 32 + q * 8 + r] = (T)(some ? c.acc[t][q * 4 + r] * over : 0.0f);
      } else {
        float *p = a.part + ((2 * w + (at_start ? 0 : 1)) * MANY + col) * (HD + 2);
#pragma unroll
        for (int t = 0; t < HD / 32; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) p[t * 32 + q * 8 + ch0 + r] = c.acc[t][q * 4 + r] * unit;
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
    // the next item: the next head, block, sequence with rows
    x = 0;
    if (++head < a.c.heads) continue;
    head = 0;
    if (++j < blocks_of(a, s.n, MANY)) continue;
    j = 0;
    do {
      if (++b >= a.c.n_seqs) return;
    } while (rows_of(a.c, b).n == 0);
  }
}

}  // namespace

void rvq_launch_cache8_chunk(const AttnArgs &a, bool half, int64_t groups, bool whole, hipStream_t s) {
  const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * WAVES), 0, s, a, (int)whole); };
  if (a.c.hd == 64) half ? go(cache8_chunk_kernel<_Float16, 64>) : go(cache8_chunk_kernel<__bf16, 64>);
  else if (a.c.hd == 128) half ? go(cache8_chunk_kernel<_Float16, 128>) : go(cache8_chunk_kernel<__bf16, 128>);
  else half ? go(cache8_chunk_kernel<_Float16, 256>) : go(cache8_chunk_kernel<__bf16, 256>);
}
