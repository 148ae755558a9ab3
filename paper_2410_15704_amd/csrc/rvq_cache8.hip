// The paged cache of 8-bit codes: appending a step's tokens, and reading tokens back.
//
// Both are bound by memory: 2 or 4 bytes of a row element against one byte of code.  A workgroup takes one
// page and kv head, keys or values: it holds every token of a scale, so the scale needs no second pass over
// memory and no atomics, and results do not depend on any order.  The pages of the step are enumerated on the
// device (find_piece), since only the device knows the lengths; the grid is an upper bound.
//
// Keys are stored by token, values by channel (the order in which attention feeds both to the matrix cores
// without a transposition), so the values' tile is turned in LDS here, once per token instead of once per reading.
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

template <bool READ> __device__ __forceinline__ bool find_span(const MoveArgs &a, Span &s) {
  int64_t inside;
  const auto first_position = [&](int b, int n) -> int64_t { return READ ? a.first[b] : (int64_t)a.c.lengths[b] - n; };
  const auto count = [&](int b) -> int64_t {
    const SeqRows r = rows_of(a.c, b);
    return r.n ? pages_spanned(first_position(b, r.n), r.n) : 0;
  };
  if (!find_piece(a.c.n_seqs, blockIdx.x, count, s.b, inside)) return false;
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

// slot of a unit -> row of the step
__device__ __forceinline__ int64_t row_of(const Span &s, int slot) { return s.row + (s.entry * PAGE + slot - s.p0); }

// 16 codes rounded again to a larger scale
__device__ __forceinline__ uint32_t again4(uint32_t w, float ratio) {
  float v[4];
  decode4(w, v);
  return encode4_any(v[0] * ratio, v[1] * ratio, v[2] * ratio, v[3] * ratio);
}

template <typename T, int HD, int LAYOUT> __global__ __launch_bounds__(256) void cache8_append_kernel(const MoveArgs a) {
  constexpr int UNITS = HD / 16, PER = PAGE * UNITS / 256, LDR = HD + 16;
  __shared__ float wave_max[4];
  __shared__ __align__(16) uint8_t tile[PAGE * LDR];
  Span s;
  if (!find_span<false>(a, s) || s.page < 0) return;
  const int head = blockIdx.y >> 1, values = blockIdx.y & 1;
  const T *src = (const T *)(values ? a.v : a.k) + head * (values ? a.hsv : a.hsk);
  const int64_t ld = values ? a.ldv : a.ldk;
  const int rot = values ? 0 : a.rot;
  float *scale_at = scale_of(a.c, s.page, head, values);
  const float old = s.lo ? *scale_at : 0.0f;

  float x[PER][16];
  float amax = 0.0f;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int id = j * 256 + (int)threadIdx.x, slot = id / UNITS, u = id % UNITS;
    if (slot < s.lo || slot >= s.hi) continue;
    int c0, c1;
    unit_channels<LAYOUT>(u, rot, c0, c1);
    const int64_t row = row_of(s, slot);
    const T *p = src + row * ld;
    float va[8], vb[8];
    load8<T>(p + c0, va);
    load8<T>(p + c1, vb);
    if (16 * u < rot) {
      float cs[8], sn[8];
      load8<float>(a.cos + row * (rot / 2) + 8 * u, cs);
      load8<float>(a.sin + row * (rot / 2) + 8 * u, sn);
      rotate_unit<LAYOUT>(va, vb, cs, sn);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[j][i] = va[i];
      x[j][8 + i] = vb[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) amax = not_finite(x[j][i]) ? amax : fmaxf(amax, fabsf(x[j][i]));
  }
#pragma unroll
  for (int d = 32; d; d /= 2) amax = fmaxf(amax, __shfl_xor(amax, d, 64));
  if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = amax;
  __syncthreads();  // also: every thread has read the old scale
  amax = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
  float scale = code_scale(amax);
  scale = s.lo ? fmaxf(scale, old) : scale;
  const bool grown = s.lo && scale > old;
  const float inverse = 1.0f / scale, ratio = grown ? old * inverse : 1.0f;
  if (threadIdx.x == 0) *scale_at = scale;

  uint8_t *codes = codes_of(a.c, s.page, head, values);
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int id = j * 256 + (int)threadIdx.x, slot = id / UNITS, u = id % UNITS;
    if (slot < s.lo || slot >= s.hi) continue;
    int c0, c1;
    unit_channels<LAYOUT>(u, rot, c0, c1);
    u32x2 w0, w1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float *p = &x[j][4 * i], *q = &x[j][8 + 4 * i];
      w0[i] = encode4_any(p[0] * inverse, p[1] * inverse, p[2] * inverse, p[3] * inverse);
      w1[i] = encode4_any(q[0] * inverse, q[1] * inverse, q[2] * inverse, q[3] * inverse);
    }
    uint8_t *to = values ? tile + slot * LDR : codes + slot * HD;
    *reinterpret_cast<u32x2 *>(to + c0) = w0;
    *reinterpret_cast<u32x2 *>(to + c1) = w1;
  }
  if (!values) {
    if (grown)  // the page's earlier tokens
      for (int at = threadIdx.x * 16; at < s.lo * HD; at += 256 * 16) {
        u32x4 w = *reinterpret_cast<const u32x4 *>(codes + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = again4(w[i], ratio);
        *reinterpret_cast<u32x4 *>(codes + at) = w;
      }
    return;
  }
  __syncthreads();
  // a thread writes 16 slots of one channel: whole where they are all new, else what is new, or what is old and changes
  for (int id = threadIdx.x; id < HD * 4; id += 256) {
    const int c = id >> 2, s0 = (id & 3) * 16;
    uint8_t *to = codes + c * PAGE + s0;
    const bool any_new = s0 < s.hi && s0 + 16 > s.lo, any_old = s0 < s.lo;
    if (!any_new && !(any_old && grown)) continue;
    u32x4 w = {0, 0, 0, 0};
    const bool all_new = s0 >= s.lo && s0 + 16 <= s.hi;
    if (!all_new) w = *reinterpret_cast<const u32x4 *>(to);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t was = w[i], more = grown ? again4(was, ratio) : was;
      uint32_t put = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int slot = s0 + 4 * i + j;
        const uint32_t from = slot < s.lo ? more >> (8 * j) : slot < s.hi ? tile[slot * LDR + c] : was >> (8 * j);
        put |= (from & 0xffu) << (8 * j);
      }
      w[i] = put;
    }
    *reinterpret_cast<u32x4 *>(to) = w;
  }
}

template <typename T, int HD, int LAYOUT> __global__ __launch_bounds__(256) void cache8_read_kernel(const MoveArgs a) {
  constexpr int UNITS = HD / 16, PER = PAGE * UNITS / 256, LDR = HD + 16;
  __shared__ __align__(16) uint8_t tile[PAGE * LDR];
  Span s;
  if (!find_span<true>(a, s)) return;
  const int head = blockIdx.y >> 1, values = blockIdx.y & 1;
  T *dst = (T *)(values ? a.v : a.k);
  if (!dst) return;
  dst += head * (values ? a.hsv : a.hsk);
  const int64_t ld = values ? a.ldv : a.ldk;
  const int rot = values ? 0 : a.rot;
  // slots that hold a token of the sequence
  const int64_t end = (int64_t)a.c.lengths[s.b] - s.entry * PAGE;
  const int held = s.page < 0 ? 0 : (int)(end < 0 ? 0 : end > PAGE ? PAGE : end);
  const uint8_t *codes = s.page < 0 ? nullptr : codes_of(a.c, s.page, head, values);
  const float scale = s.page < 0 ? 0.0f : *scale_of(a.c, s.page, head, values);
  if (values && held) {
    for (int id = threadIdx.x; id < HD * 4; id += 256) {
      const int c = id >> 2, s0 = (id & 3) * 16;
      if (s0 >= s.hi || s0 + 16 <= s.lo) continue;
      const u32x4 w = *reinterpret_cast<const u32x4 *>(codes + c * PAGE + s0);
#pragma unroll
      for (int i = 0; i < 16; ++i) tile[(s0 + i) * LDR + c] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int id = j * 256 + (int)threadIdx.x, slot = id / UNITS, u = id % UNITS;
    if (slot < s.lo || slot >= s.hi) continue;
    int c0, c1;
    unit_channels<LAYOUT>(u, rot, c0, c1);
    const int64_t row = row_of(s, slot);
    float va[8] = {}, vb[8] = {};
    if (slot < held) {
      const uint8_t *from = values ? tile + slot * LDR : codes + slot * HD;
      const u32x2 w0 = *reinterpret_cast<const u32x2 *>(from + c0), w1 = *reinterpret_cast<const u32x2 *>(from + c1);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float t[4];
        decode4(w0[i], t);
#pragma unroll
        for (int m = 0; m < 4; ++m) va[4 * i + m] = t[m] * scale;
        decode4(w1[i], t);
#pragma unroll
        for (int m = 0; m < 4; ++m) vb[4 * i + m] = t[m] * scale;
      }
      if (16 * u < rot) {
        float cs[8], sn[8];
        load8<float>(a.cos + row * (rot / 2) + 8 * u, cs);
        load8<float>(a.sin + row * (rot / 2) + 8 * u, sn);
#pragma unroll
        for (int i = 0; i < 8; ++i) sn[i] = -sn[i];
        rotate_unit<LAYOUT>(va, vb, cs, sn);
      }
    }
    T *p = dst + row * ld;
    store8<T>(p + c0, va);
    store8<T>(p + c1, vb);
  }
}

// pages that `rows` rows of n_seqs sequences can span: floor((n + 62) / 64) + 1 for each of n >= 1 rows
int64_t most_pages(int64_t rows, int n_seqs) {
  const int64_t seqs = rows < n_seqs ? rows : n_seqs, most = (rows + 62 * seqs) / PAGE + seqs;
  return most < rows ? most : rows;
}

template <bool READ, typename T, int HD> void launch_move(const MoveArgs &a, int layout, dim3 grid, hipStream_t s) {
  if (layout == RVQ_ROPE_HALVES) {
    if (READ) hipLaunchKernelGGL((cache8_read_kernel<T, HD, RVQ_ROPE_HALVES>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cache8_append_kernel<T, HD, RVQ_ROPE_HALVES>), grid, dim3(256), 0, s, a);
  } else {
    if (READ) hipLaunchKernelGGL((cache8_read_kernel<T, HD, RVQ_ROPE_ADJACENT>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cache8_append_kernel<T, HD, RVQ_ROPE_ADJACENT>), grid, dim3(256), 0, s, a);
  }
}
template <bool READ, typename T> void launch_move_hd(const MoveArgs &a, int layout, dim3 grid, hipStream_t s) {
  if (a.c.hd == 64) launch_move<READ, T, 64>(a, layout, grid, s);
  else if (a.c.hd == 128) launch_move<READ, T, 128>(a, layout, grid, s);
  else launch_move<READ, T, 256>(a, layout, grid, s);
}
template <bool READ> int move(const MoveArgs &a, int layout, int32_t dtype, hipStream_t s) {
  const int64_t blocks = most_pages(a.c.rows, a.c.n_seqs);
  const dim3 grid((unsigned)blocks, 2 * a.c.heads);
  if (dtype == RVQ_F32) launch_move_hd<READ, float>(a, layout, grid, s);
  else if (dtype == RVQ_BF16) launch_move_hd<READ, __bf16>(a, layout, grid, s);
  else launch_move_hd<READ, _Float16>(a, layout, grid, s);
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
  return move<false>(a, layout, dtype, (hipStream_t)stream);
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
  return move<true>(a, layout, dtype, (hipStream_t)stream);
}

}  // extern "C"
