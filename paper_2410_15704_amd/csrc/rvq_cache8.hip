// The paged cache of 8-bit codes: appending a step's tokens, and reading tokens back.
//
// Both are bound by memory: 2 or 4 bytes of a row element against one byte of code.  A workgroup takes one
// page and kv head, half of its threads the keys and half the values: it holds every token of a scale, so the scale
// needs no second pass over memory and no atomics, and results do not depend on any order.  The pages of the step are
// enumerated on the device (find_piece), since only the device knows the lengths; the grid is an upper bound.
// Append of 16384 fp32 tokens of 32 kv heads of 128 channels: 153 us for 680 MB, 4.4 TB/s (a large copy 5.2: rows in, a quarter as many
// bytes of codes out, and a barrier between); four fp16 chunks of up to 1500 tokens of 8 heads 11.0 us, single tokens of 32 sequences
// 5.0 (by the kernel for a few tokens).  Read of 131072 fp16 rows of 8 heads: 205 us for 872 MB, 4.25 TB/s (two bytes written for one
// read, and a table entry per pair); 48 rows 4.9 us.
//
// Keys are stored by token, values by channel (the order in which attention feeds both to the matrix cores
// without a transposition).  A thread of the values takes four channels of 16 tokens: its reads and writes of rows are 8 or
// 16 bytes, neighbours beside each other along the row, and of codes 16 bytes of a channel; what lies between is
// a transposition of 4 x 4 bytes in registers (reading), or none (the conversion packs neighbouring tokens).
// Through LDS instead: append of the chunks 16.4 us, read of the 131072 rows 231.
// Appending takes 8 tokens a thread (16: chunks 12.3 us), reading 16.
#include <type_traits>

#include "rvq_cache8.h"

namespace {

struct MoveArgs {
  CacheView c;
  const int32_t *first;  // read: position of a sequence's first row
  char *k, *v;
  int64_t ldk, hsk, ldv, hsv;  // elements
  const float *cos, *sin;
  int rot;
};

// floor pages of n >= 1 positions from p on
__device__ __forceinline__ int64_t pages_spanned(int64_t p, int n) { return ((p + n - 1) >> 6) - (p >> 6) + 1; }

struct Span {
  int b, n;            // sequence, its rows
  int64_t row, p0;     // its first row and that row's position
  int64_t entry, page; // entry of the table and page, -1: none
  int lo, hi;          // slots of the page that the step's rows fill
};

// the step's page `at`
template <bool BACK, int THREADS> __device__ __forceinline__ bool find_span(const MoveArgs &a, int at, Span &s) {
  __shared__ Together<THREADS, int> sh;
  int inside;
  const auto first_position = [&](int b, int n) -> int64_t { return BACK ? a.first[b] : (int64_t)a.c.lengths[b] - n; };
  const auto count = [&](int b) -> int {
    const SeqRows r = rows_of(a.c, b);
    return r.n ? (int)pages_spanned(first_position(b, r.n), r.n) : 0;
  };
  if (!(a.c.n_seqs <= 64 ? find_piece<int>(a.c.n_seqs, at, count, s.b, inside)
                         : find_piece_together<THREADS, int>(a.c.n_seqs, at, count, sh, s.b, inside)))
    return false;
  const SeqRows r = rows_of(a.c, s.b);
  s.n = r.n;
  s.row = r.row;
  s.p0 = first_position(s.b, r.n);
  s.entry = (s.p0 >> 6) + inside;
  s.page = page_of(a.c, s.b, s.entry);
  const int64_t begin = s.entry * PAGE;
  s.lo = (int)(s.p0 > begin ? s.p0 - begin : 0);
  s.hi = (int)(s.p0 + r.n < begin + PAGE ? s.p0 + r.n - begin : PAGE);
  return true;
}

// Loads are made for every slot, of the nearest one that the step has, and what does not belong is dropped afterwards: a load
// under a condition would be waited for before the next one.
__device__ __forceinline__ int nearest(const Span &s, int slot) { return slot < s.lo ? s.lo : slot >= s.hi ? s.hi - 1 : slot; }

// slot of a unit -> row of the step
__device__ __forceinline__ int64_t row_of(const Span &s, int slot) { return s.row + (s.entry * PAGE + slot - s.p0); }

// codes rounded again to a larger scale
__device__ __forceinline__ uint32_t again4(uint32_t w, float ratio) {
  float v[4];
  decode4(w, v);
  return encode4_any(v[0] * ratio, v[1] * ratio, v[2] * ratio, v[3] * ratio);
}

// A thread's part of a page, 4 TOK elements.  Keys: 16 channels (unit u) of the tokens first + j PAGE 4 / TOK, j < TOK / 4.  Values:
// channels ch0 .. ch0 + 3 of tokens first .. first + TOK - 1.
template <int HD, int TOK> struct Task {
  static constexpr int HALF = 16 * HD / TOK;         // threads of the keys, and of the values
  static constexpr int STEP = HALF / (HD / 16);      // tokens between a thread's keys
  bool values;
  int first, u, ch0;
  __device__ __forceinline__ Task() {
    const int t = threadIdx.x % HALF;
    values = threadIdx.x >= HALF;
    u = t % (HD / 16);
    ch0 = t % (HD / 4) * 4;
    first = values ? t / (HD / 4) * TOK : t / (HD / 16);
  }
};
template <typename T, int HD, int LAYOUT> __global__ __launch_bounds__(4 * HD) void cache8_append_kernel(const MoveArgs a) {
  constexpr int TOK = 8, KEYS = TOK / 4, WAVES_HALF = Task<HD, TOK>::HALF / 64;
  __shared__ uint32_t wave_max[2 * WAVES_HALF];
  Span s;
  if (!find_span<false, 4 * HD>(a, blockIdx.x / a.c.heads, s) || s.page < 0) return;
  const int head = blockIdx.x % a.c.heads;
  const Task<HD, TOK> task;
  float *scale_at = scale_of(a.c, s.page, head, task.values);
  const float old = s.lo ? *scale_at : 0.0f;
  uint8_t *codes = codes_of(a.c, s.page, head, task.values);

  float x[4 * TOK];  // keys [token][16 channels], values [4 channels][token]
  const Unit<LAYOUT> unit(task.u, HD, a.rot);
  // FULL: the step fills the whole page
  const auto load = [&](auto full) {
    constexpr bool FULL = decltype(full)::value;
    const auto row_at = [&](int slot) { return row_of(s, FULL ? slot : nearest(s, slot)); };
    if (!task.values) {
      const T *src = (const T *)a.k + head * a.hsk;
      typename Raw8<T>::type va[KEYS], vb[KEYS];
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        const T *p = src + row_at(task.first + task.STEP * j) * a.ldk;
        va[j] = raw8<T>(p + unit.c0);
        vb[j] = raw8<T>(p + unit.c1);
      }
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        float p[8], q[8];
        widen<T>(va[j], p);
        widen<T>(vb[j], q);
        if (a.rot) {
          const int64_t row = row_at(task.first + task.STEP * j);
          float cs[8], sn[8];
          unit.entries(a.cos + row * (a.rot / 2), cs);
          unit.entries(a.sin + row * (a.rot / 2), sn);
          unit.rotate(p, q, cs, sn);
        }
        const int slot = task.first + task.STEP * j;
        const bool in = FULL || (slot >= s.lo && slot < s.hi);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[16 * j + i] = in ? p[i] : 0.0f;
          x[16 * j + 8 + i] = in ? q[i] : 0.0f;
        }
      }
    } else if (FULL || (task.first < s.hi && task.first + TOK > s.lo)) {
      const T *src = (const T *)a.v + head * a.hsv + task.ch0, *row0 = src + row_at(task.first) * a.ldv;
      typename Vec4<T>::type v[TOK];
#pragma unroll
      for (int i = 0; i < TOK; ++i)
        v[i] = *reinterpret_cast<const typename Vec4<T>::type *>(FULL ? row0 + i * a.ldv : src + row_at(task.first + i) * a.ldv);
#pragma unroll
      for (int i = 0; i < TOK; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[TOK * j + i] = FULL || (task.first + i >= s.lo && task.first + i < s.hi) ? (float)v[i][j] : 0.0f;
    } else {
#pragma unroll
      for (int i = 0; i < 4 * TOK; ++i) x[i] = 0.0f;
    }
  };
  if (s.lo == 0 && s.hi == PAGE) load(std::true_type());
  else load(std::false_type());
  // Largest magnitude over the workgroup's keys and over its values, as bits (they are ordered like the numbers, infinity and
  // NaN above all).  Called by all threads.
  const auto largest = [&](uint32_t mine) {
#pragma unroll
    for (int d = 32; d; d /= 2) mine = max(mine, (uint32_t)__shfl_xor((int)mine, d, 64));
    if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = mine;
    __syncthreads();  // (the first time also: every thread has read the old scale)
    uint32_t all = 0, own = 0;
#pragma unroll
    for (int w = 0; w < 2 * WAVES_HALF; ++w) {
      const uint32_t m = wave_max[w];
      all = max(all, m);
      own = (w >= WAVES_HALF) == task.values ? max(own, m) : own;
    }
    __syncthreads();
    return u32x2{all, own};
  };
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4 * TOK; ++i) bits = max(bits, __float_as_uint(x[i]) & 0x7fffffffu);
  u32x2 top = largest(bits);
  const bool finite = __builtin_amdgcn_readfirstlane(top[0]) < 0x7f800000;
  if (!finite) {  // somewhere: once more without what is not finite
    bits = 0;
#pragma unroll
    for (int i = 0; i < 4 * TOK; ++i) bits = not_finite(x[i]) ? bits : max(bits, __float_as_uint(x[i]) & 0x7fffffffu);
    top = largest(bits);
  }
  float scale = code_scale(__uint_as_float(top[1]));
  scale = s.lo ? fmaxf(scale, old) : scale;
  const bool grown = s.lo && scale > old;
  const float inverse = 1.0f / scale, ratio = grown ? old * inverse : 1.0f;
  if (threadIdx.x % task.HALF == 0) *scale_at = scale;

  uint32_t w[TOK];
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const float *p = &x[4 * i];
    if (finite) w[i] = encode4(p[0] * inverse, p[1] * inverse, p[2] * inverse, p[3] * inverse);
    else w[i] = encode4_any(p[0] * inverse, p[1] * inverse, p[2] * inverse, p[3] * inverse);
  }
  if (!task.values) {
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
      const int slot = task.first + task.STEP * j;
      if (slot < s.lo || slot >= s.hi) continue;
      *reinterpret_cast<u32x2 *>(codes + slot * HD + unit.c0) = u32x2{w[4 * j], w[4 * j + 1]};
      *reinterpret_cast<u32x2 *>(codes + slot * HD + unit.c1) = u32x2{w[4 * j + 2], w[4 * j + 3]};
    }
    if (grown)  // the page's earlier tokens
      for (int at = threadIdx.x * 16; at < s.lo * HD; at += task.HALF * 16) {
        u32x4 v = *reinterpret_cast<const u32x4 *>(codes + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = again4(v[i], ratio);
        *reinterpret_cast<u32x4 *>(codes + at) = v;
      }
    return;
  }
  // TOK slots of a channel: whole where they are all new; read and written again where old ones change; else the new bytes alone
  const int from = s.lo - task.first, to = s.hi - task.first;
  typedef uint32_t Words __attribute__((ext_vector_type(TOK / 4)));
  if (from <= 0 && to >= TOK) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      Words v;
#pragma unroll
      for (int i = 0; i < TOK / 4; ++i) v[i] = w[j * TOK / 4 + i];
      *reinterpret_cast<Words *>(codes + (task.ch0 + j) * PAGE + task.first) = v;
    }
  } else if (grown && from > 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      Words *at = reinterpret_cast<Words *>(codes + (task.ch0 + j) * PAGE + task.first);
      Words v = *at;
#pragma unroll
      for (int i = 0; i < TOK / 4; ++i) {
        const uint32_t more = again4(v[i], ratio);
        uint32_t put = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int slot = 4 * i + b;
          put |= (slot < from ? more : slot < to ? w[j * TOK / 4 + i] : v[i]) & (0xffu << (8 * b));
        }
        v[i] = put;
      }
      *at = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < TOK; ++i)
      if (i >= from && i < to)
#pragma unroll
        for (int j = 0; j < 4; ++j) codes[(task.ch0 + j) * PAGE + task.first + i] = (uint8_t)(w[j * TOK / 4 + (i >> 2)] >> (8 * (i & 3)));
  }
}

// Append where sequences bring a token or a few: the same results by a wavefront per (page, head, keys or values), four of them a
// workgroup.  It is a chain of latencies (lengths, table, rows and old scale, codes), so what counts is how many of them a CU holds:
// 20 scales at a time instead of 4.  A lane takes neighbouring channels, N tokens at a time with all loads before the first product (8
// tokens: 512 sequences 13.3 -> 15.7 us, fewer wavefronts fit); a page of more tokens than N is read twice.
template <typename T, int HD, int LAYOUT> __global__ __launch_bounds__(256) void cache8_append_few_kernel(const MoveArgs a) {
  constexpr int C = HD / 64, N = HD == 256 ? 2 : 4;
  const int pairs = (a.c.heads + 1) / 2, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Span s;
  if (!find_span<false, 256>(a, blockIdx.x / pairs, s) || s.page < 0) return;
  const int head = (int)(blockIdx.x % pairs) * 2 + (wave >> 1);
  const bool values = wave & 1;
  if (head >= a.c.heads) return;
  float *scale_at = scale_of(a.c, s.page, head, values);
  const float old = s.lo ? *scale_at : 0.0f;
  uint8_t *codes = codes_of(a.c, s.page, head, values);
  const T *src = values ? (const T *)a.v + head * a.hsv : (const T *)a.k + head * a.hsk;
  const int64_t ld = values ? a.ldv : a.ldk;
  const int half = values ? 0 : a.rot / 2;
  // the channel that each of the lane's is turned with (itself: none) and the pair's entry of the tables
  int partner[C], pair[C];
  bool first[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int c = lane * C + j;
    first[j] = LAYOUT == RVQ_ROPE_HALVES ? c < half : !(c & 1);
    partner[j] = c >= 2 * half ? c : LAYOUT == RVQ_ROPE_HALVES ? (first[j] ? c + half : c - half) : c ^ 1;
    pair[j] = c >= 2 * half ? 0 : LAYOUT == RVQ_ROPE_HALVES ? min(c, partner[j]) : c >> 1;
  }
  float x[N][C], top = 0.0f;
  const auto load = [&](int slot0) {  // N tokens from slot0 on, and their largest magnitude
    typedef T Own __attribute__((ext_vector_type(C)));
    Own own[N];
    T other[N][C];
    float cs[N][C], sn[N][C];
#pragma unroll
    for (int i = 0; i < N; ++i) own[i] = *reinterpret_cast<const Own *>(src + row_of(s, nearest(s, slot0 + i)) * ld + lane * C);
    if (half) {  // all loads before the first product
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < C; ++j) {
          const int64_t row = row_of(s, nearest(s, slot0 + i));
          other[i][j] = src[row * ld + partner[j]];
          cs[i][j] = a.cos[row * half + pair[j]];
          sn[i][j] = a.sin[row * half + pair[j]];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < C; ++j) x[i][j] = (float)own[i][j];
    if (half) {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < C; ++j) {
          const float y = (float)other[i][j];
          float u = first[j] ? x[i][j] : y, v = first[j] ? y : x[i][j];
          rotate_pair(u, v, cs[i][j], sn[i][j]);
          x[i][j] = partner[j] == lane * C + j ? x[i][j] : first[j] ? u : v;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < C; ++j) top = not_finite(x[i][j]) ? top : fmaxf(top, fabsf(x[i][j]));
  };
  for (int slot0 = s.lo; slot0 < s.hi; slot0 += N) load(slot0);
#pragma unroll
  for (int d = 32; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
  float scale = code_scale(top);
  scale = s.lo ? fmaxf(scale, old) : scale;
  const float inverse = 1.0f / scale;
  if (lane == 0) *scale_at = scale;
  if (s.lo && scale > old) {  // the page's earlier tokens
    const float ratio = old * inverse;
    const int pieces = values ? HD * PAGE / 16 : s.lo * HD / 16;
    for (int i = lane; i < pieces; i += 64) {
      const int first = values ? i % (PAGE / 16) * 16 : 0, held = values ? s.lo - first : 16;  // bytes of the piece that change
      if (held <= 0) continue;
      u32x4 v = *reinterpret_cast<const u32x4 *>(codes + i * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int n = held - 4 * j;
        const uint32_t mask = n <= 0 ? 0u : n >= 4 ? 0xffffffffu : (1u << (8 * n)) - 1u;
        v[j] = (again4(v[j], ratio) & mask) | (v[j] & ~mask);
      }
      *reinterpret_cast<u32x4 *>(codes + i * 16) = v;
    }
    __threadfence_block();  // some of these bytes are written once more below, by other lanes
  }
  for (int slot0 = s.lo; slot0 < s.hi; slot0 += N) {
    if (s.hi - s.lo > N) load(slot0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (slot0 + i >= s.hi) break;
      float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < C; ++j) y[j] = x[i][j] * inverse;
      const uint32_t w = encode4_any(y[0], y[1], y[2], y[3]);
      if (values) {
#pragma unroll
        for (int j = 0; j < C; ++j) codes[(lane * C + j) * PAGE + slot0 + i] = (uint8_t)(w >> (8 * j));
      } else {
        typedef std::conditional_t<C == 1, uint8_t, std::conditional_t<C == 2, uint16_t, uint32_t>> Word;
        *reinterpret_cast<Word *>(codes + (slot0 + i) * HD + lane * C) = (Word)w;
      }
    }
  }
}

template <typename T, int HD, int LAYOUT> __global__ __launch_bounds__(2 * HD) void cache8_read_kernel(const MoveArgs a) {
  Span s;
  if (!find_span<true, 2 * HD>(a, blockIdx.x / a.c.heads, s)) return;
  const int head = blockIdx.x % a.c.heads;
  const Task<HD, 16> task;
  T *dst = (T *)(task.values ? a.v : a.k);
  if (!dst) return;
  dst += head * (task.values ? a.hsv : a.hsk);
  // slots that hold a token of the sequence
  const int64_t end = (int64_t)a.c.lengths[s.b] - s.entry * PAGE;
  const int held = s.page < 0 ? 0 : (int)(end < 0 ? 0 : end > PAGE ? PAGE : end);
  const uint8_t *codes = codes_of(a.c, s.page < 0 ? 0 : s.page, head, task.values);
  const float scale = s.page < 0 ? 0.0f : *scale_of(a.c, s.page, head, task.values);
  // FULL: the step takes the whole page, and all of it is there
  const auto move_page = [&](auto full) {
    constexpr bool FULL = decltype(full)::value;
    const auto wanted = [&](int slot) { return FULL || (slot >= s.lo && slot < s.hi); };
    const auto there = [&](int slot) { return FULL || slot < held; };
    if (!task.values) {
      const Unit<LAYOUT> unit(task.u, HD, a.rot);
      u32x2 w[4][2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint8_t *at = codes + (task.first + 16 * j) * HD;
        w[j][0] = *reinterpret_cast<const u32x2 *>(at + unit.c0);
        w[j][1] = *reinterpret_cast<const u32x2 *>(at + unit.c1);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int slot = task.first + 16 * j;
        if (!wanted(slot)) continue;
        const int64_t row = row_of(s, slot);
        float v[2][8];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float t[4];
            decode4(w[j][e][i], t);
#pragma unroll
            for (int m = 0; m < 4; ++m) v[e][4 * i + m] = there(slot) ? t[m] * scale : 0.0f;
          }
        if (a.rot) {
          float cs[8], sn[8];
          unit.entries(a.cos + row * (a.rot / 2), cs);
          unit.entries(a.sin + row * (a.rot / 2), sn);
#pragma unroll
          for (int i = 0; i < 8; ++i) sn[i] = -sn[i];
          unit.rotate(v[0], v[1], cs, sn);
          // Tables of an amplitude other than 1 scaled the pairs by it twice, here and when they were stored.  (Entries that are rounded
          // to fp32 differ from 1 by 2^-23 in cos^2 + sin^2, and its sum here by as much: no amplitude.)
          float size[8];
          bool scaled = false;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            size[i] = fmaf(cs[i], cs[i], sn[i] * sn[i]);
            scaled |= fabsf(size[i] - 1.0f) > 0x1p-22f;
          }
          if (__any(scaled))
            unit.each(v[0], v[1], [&](float &x, float &y, int i) {
              const float by = fabsf(size[i] - 1.0f) > 0x1p-22f ? 1.0f / size[i] : 1.0f;
              x *= by;
              y *= by;
            });
        }
        T *p = dst + row * a.ldk;
        store8<T>(p + unit.c0, v[0]);
        store8<T>(p + unit.c1, v[1]);
      }
      return;
    }
    if (!FULL && (task.first >= s.hi || task.first + 16 <= s.lo)) return;
    u32x4 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const u32x4 *>(codes + (task.ch0 + j) * PAGE + task.first);
    T *row0 = dst + row_of(s, task.first) * a.ldv + task.ch0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // four channels by four tokens, turned
      const uint32_t lo01 = __builtin_amdgcn_perm(w[1][i], w[0][i], 0x05010400), lo23 = __builtin_amdgcn_perm(w[3][i], w[2][i], 0x05010400);
      const uint32_t hi01 = __builtin_amdgcn_perm(w[1][i], w[0][i], 0x07030602), hi23 = __builtin_amdgcn_perm(w[3][i], w[2][i], 0x07030602);
      const uint32_t turned[4] = {__builtin_amdgcn_perm(lo23, lo01, 0x05040100), __builtin_amdgcn_perm(lo23, lo01, 0x07060302),
                                  __builtin_amdgcn_perm(hi23, hi01, 0x05040100), __builtin_amdgcn_perm(hi23, hi01, 0x07060302)};
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const int slot = task.first + 4 * i + m;
        if (!wanted(slot)) continue;
        float t[4];
        decode4(turned[m], t);
        typename Vec4<T>::type v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (T)(there(slot) ? t[j] * scale : 0.0f);
        *reinterpret_cast<typename Vec4<T>::type *>(row0 + (4 * i + m) * a.ldv) = v;
      }
    }
  };
  if (s.lo == 0 && s.hi == PAGE && held == PAGE) move_page(std::true_type());
  else move_page(std::false_type());
}

// pages that `rows` rows of n_seqs sequences can span: floor((n + 62) / 64) + 1 for each of n >= 1 rows
int64_t most_pages(int64_t rows, int n_seqs) {
  const int64_t seqs = rows < n_seqs ? rows : n_seqs, most = (rows + 62 * seqs) / PAGE + seqs;
  return most < rows ? most : rows;
}

enum Move { READ, APPEND, APPEND_FEW };
template <Move WHAT, typename T, int HD, int LAYOUT> void launch_move(const MoveArgs &a, dim3 grid, hipStream_t s) {
  if constexpr (WHAT == READ) hipLaunchKernelGGL((cache8_read_kernel<T, HD, LAYOUT>), grid, dim3(2 * HD), 0, s, a);
  else if constexpr (WHAT == APPEND) hipLaunchKernelGGL((cache8_append_kernel<T, HD, LAYOUT>), grid, dim3(4 * HD), 0, s, a);
  else hipLaunchKernelGGL((cache8_append_few_kernel<T, HD, LAYOUT>), grid, dim3(256), 0, s, a);
}
template <Move WHAT, typename T, int HD> void launch_move_layout(const MoveArgs &a, int layout, dim3 grid, hipStream_t s) {
  if (layout == RVQ_ROPE_HALVES) launch_move<WHAT, T, HD, RVQ_ROPE_HALVES>(a, grid, s);
  else launch_move<WHAT, T, HD, RVQ_ROPE_ADJACENT>(a, grid, s);
}
template <Move WHAT, typename T> void launch_move_hd(const MoveArgs &a, int layout, dim3 grid, hipStream_t s) {
  if (a.c.hd == 64) launch_move_layout<WHAT, T, 64>(a, layout, grid, s);
  else if (a.c.hd == 128) launch_move_layout<WHAT, T, 128>(a, layout, grid, s);
  else launch_move_layout<WHAT, T, 256>(a, layout, grid, s);
}
template <Move WHAT> int move(const MoveArgs &a, int layout, int32_t dtype, hipStream_t s) {
  // the heads of a page beside each other: their rows are neighbours in memory, and they read the same tables
  const int64_t blocks = most_pages(a.c.rows, a.c.n_seqs) * a.c.heads;
  if (blocks > INT32_MAX) return RVQ_EINVAL;
  const dim3 grid((unsigned)(WHAT == APPEND_FEW ? blocks / a.c.heads * ((a.c.heads + 1) / 2) : blocks));
  if (dtype == RVQ_F32) launch_move_hd<WHAT, float>(a, layout, grid, s);
  else if (dtype == RVQ_BF16) launch_move_hd<WHAT, __bf16>(a, layout, grid, s);
  else launch_move_hd<WHAT, _Float16>(a, layout, grid, s);
  return hipGetLastError() == hipSuccess ? RVQ_OK : RVQ_EHIP;
}

// what append and read check alike; rows >= 0
bool move_ok(const rvq_cache8 *c, int32_t dtype, int64_t rows, const int32_t *dCu, const float *dCos, const float *dSin,
             int32_t rot, int32_t layout) {
  if (!rvq_cache8_ok(c) || rows < 0 || rows > INT32_MAX) return false;
  if (dtype != RVQ_F32 && dtype != RVQ_BF16 && dtype != RVQ_F16) return false;
  if (layout != RVQ_ROPE_ADJACENT && layout != RVQ_ROPE_HALVES) return false;
  if (!dCos != !dSin || !dCos != (rot == 0)) return false;
  if (rot < 0 || rot > c->head_dim || rot % 16) return false;
  if (rot && (!rvq_aligned(dCos, 16) || !rvq_aligned(dSin, 16))) return false;
  return rows == 0 || (rvq_cache8_pointers_ok(c) && rvq_aligned(dCu, 4));
}

}  // namespace

extern "C" {

int rvq_cache8_append(const rvq_cache8 *cache, const void *dK, const void *dV, int32_t dtype, int64_t rows,
                      int64_t ldk, int64_t hsk, int64_t ldv, int64_t hsv, const int32_t *dCu,
                      const float *dCos, const float *dSin, int32_t rot, int32_t layout, void *stream) {
  if (!move_ok(cache, dtype, rows, dCu, dCos, dSin, rot, layout)) return RVQ_EINVAL;
  if (rows == 0) return RVQ_OK;
  const int heads = cache->n_kv_heads, hd = cache->head_dim;
  if (!rvq_rows16_ok(dK, dtype, rows, heads, hd, ldk, hsk) || !rvq_rows16_ok(dV, dtype, rows, heads, hd, ldv, hsv)) return RVQ_EINVAL;
  if (!rvq_stream_is_current((hipStream_t)stream)) return RVQ_EINVAL;
  MoveArgs a = {view_of(cache, dCu, rows), nullptr, (char *)dK, (char *)dV, ldk, hsk, ldv, hsv, dCos, dSin, rot};
  // Up to 512 channels of new tokens a sequence, on the average: a wavefront a scale (us, a workgroup a scale : a wavefront; 8 heads
  // of 128 channels, 32 sequences, a token each 5.8 : 4.5, 512 sequences 43 : 13, of 4 tokens 56 : 21, of 8 62 : 34, but 4 sequences of
  // 8 tokens 5.8 : 6.8 and 64 of 16 11 : 15; 500 single tokens beside a chunk of 1500 53 : 38).
  if (rows * hd <= 512 * (int64_t)cache->n_seqs) return move<APPEND_FEW>(a, layout, dtype, (hipStream_t)stream);
  return move<APPEND>(a, layout, dtype, (hipStream_t)stream);
}

int rvq_cache8_read(const rvq_cache8 *cache, const int32_t *dCu, const int32_t *dFirst, int64_t rows,
                    const float *dCos, const float *dSin, int32_t rot, int32_t layout, int32_t dtype, void *dK,
                    int64_t ldk, int64_t hsk, void *dV, int64_t ldv, int64_t hsv, void *stream) {
  if (!move_ok(cache, dtype, rows, dCu, dCos, dSin, rot, layout)) return RVQ_EINVAL;
  if (rows == 0 || (!dK && !dV)) return RVQ_OK;
  const int heads = cache->n_kv_heads, hd = cache->head_dim;
  if (!rvq_aligned(dFirst, 4)) return RVQ_EINVAL;
  if (dK && (!rvq_rows16_ok(dK, dtype, rows, heads, hd, ldk, hsk) || !rvq_rows_distinct(rows, heads, hd, ldk, hsk))) return RVQ_EINVAL;
  if (dV && (!rvq_rows16_ok(dV, dtype, rows, heads, hd, ldv, hsv) || !rvq_rows_distinct(rows, heads, hd, ldv, hsv))) return RVQ_EINVAL;
  if (!rvq_stream_is_current((hipStream_t)stream)) return RVQ_EINVAL;
  MoveArgs a = {view_of(cache, dCu, rows), dFirst, (char *)dK, (char *)dV, ldk, hsk, ldv, hsv, dCos, dSin, rot};
  return move<READ>(a, layout, dtype, (hipStream_t)stream);
}

}  // extern "C"
