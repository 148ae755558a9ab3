// Rotary position tables, and the rotation of head vectors (queries).
//
// Both are bound by memory: a table entry costs an fp64 angle once per step, the rotation three
// operations per element that is read and written once.  16384 tokens of 32 heads of 128 channels, 64 of them rotated, fp16,
// tables included: 58 us for 273 MB, 4.7 TB/s of the 5.2 that a large copy reaches.  64 tokens: 3.1 us for the tables, 3.2 for the
// rotation, which are launches.  Rows of any stride or width go a pair a thread: 16384 tokens of 32 fp16 heads 120 us, where aligned
// ones of whole groups take 43.  Stores past the caches would gain some (58 -> 55 us) and cost the next call, which reads these rows.
#include <algorithm>
#include <cmath>

#include "rvq_rows.h"

namespace {

struct TableArgs {
  const int64_t *pos;
  int64_t N;
  int half;  // rot / 2
  double log2_base, factor, orig_len, alpha, beta, amplitude;
  float *cos, *sin;
};

// A thread keeps one frequency and walks over tokens.  The angle is a 64-bit product taken in quarter
// turns; what is left of it after the nearest whole quarter, at most an eighth of a turn, is exact in 64
// bits and goes to the fp32 sine and cosine rounded once: |error| <= 2^-25 + pos 2^-52 + theirs.
__global__ void rope_tables_kernel(const TableArgs a) {
  const int64_t step = (int64_t)gridDim.x * blockDim.x;
  const int64_t total = a.N * a.half;
  int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= total) return;
  const int64_t dn = step / a.half;  // the launch makes step a multiple of half
  int64_t n = at / a.half;
  const int i = (int)(at - n * a.half);
  double theta = exp2(a.log2_base * (-(double)i / a.half));
  if (a.factor != 1.0) {
    double g = 0.0;
    if (a.orig_len > 0.0) {
      g = (a.orig_len * theta * 0.15915494309189533577 - a.alpha) / (a.beta - a.alpha);
      g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
    }
    theta = g * theta + (1.0 - g) * theta / a.factor;
  }
  const float amp = (float)a.amplitude;
  for (; n < a.N; n += dn, at += step) {
    const double quarters = ((double)a.pos[n] * theta) * 0.63661977236758134308;
    const double whole = rint(quarters);
    float s, c;
    sincospif((float)(quarters - whole) * 0.5f, &s, &c);
    const int k = (int)(whole - 4.0 * rint(whole * 0.25)) & 3;
    const float s2 = (k & 1) ? c : s, c2 = (k & 1) ? s : c;
    a.cos[at] = amp * ((k == 1 || k == 2) ? -c2 : c2);
    a.sin[at] = amp * ((k & 2) ? -s2 : s2);
  }
}

struct RopeArgs {
  const void *x;
  void *out;
  const float *cos, *sin;
  int64_t N, ldx, hsx, ldo, hso;
  int heads, hd, rot;
};

// 16 channels per thread and head, 32 or 64 bytes; the threads of a row are units of head groups, a thread takes
// every hgroups-th head, so its table entries are fetched once.
template <typename T, int LAYOUT>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a, int hgroups, int rows_per_block) {
  const int units = a.hd / 16, tpr = units * hgroups;
  const int r = threadIdx.x / tpr, t = threadIdx.x - r * tpr;
  if (r >= rows_per_block) return;
  const int h0 = t / units, u = t - h0 * units;
  const Unit<LAYOUT> unit(u, a.hd, a.rot);
  for (int64_t n = (int64_t)blockIdx.x * rows_per_block + r; n < a.N; n += (int64_t)gridDim.x * rows_per_block) {
    float cs[8], sn[8];
    unit.entries(a.cos + n * (a.rot / 2), cs);
    unit.entries(a.sin + n * (a.rot / 2), sn);
    for (int h = h0; h < a.heads; h += hgroups) {
      const T *x = (const T *)a.x + n * a.ldx + h * a.hsx;
      T *o = (T *)a.out + n * a.ldo + h * a.hso;
      float p[8], q[8];
      load8<T>(x + unit.c0, p);
      load8<T>(x + unit.c1, q);
      unit.rotate(p, q, cs, sn);
      store8<T>(o + unit.c0, p);
      store8<T>(o + unit.c1, q);
    }
  }
}

// rows of any stride, alignment and width: a pair, or a channel that does not rotate, per thread and step
template <typename T>
__global__ void rope_any_kernel(const RopeArgs a, int layout) {
  const int pairs = a.rot / 2, per_head = pairs + a.hd - a.rot;
  const int64_t total = a.N * a.heads * per_head, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; at < total; at += step) {
    const int64_t row = at / per_head, n = row / a.heads;
    const int i = (int)(at - row * per_head), h = (int)(row - n * a.heads);
    const T *x = (const T *)a.x + n * a.ldx + h * a.hsx;
    T *o = (T *)a.out + n * a.ldo + h * a.hso;
    if (i < pairs) {
      const int c0 = layout == RVQ_ROPE_HALVES ? i : 2 * i, c1 = layout == RVQ_ROPE_HALVES ? i + pairs : 2 * i + 1;
      float p = (float)x[c0], q = (float)x[c1];
      rotate_pair(p, q, a.cos[n * pairs + i], a.sin[n * pairs + i]);
      o[c0] = (T)p;
      o[c1] = (T)q;
    } else {
      o[i + pairs] = x[i + pairs];
    }
  }
}

template <typename T> void launch_rope(const RopeArgs &a, int layout, bool whole, hipStream_t s) {
  if (whole) {
    const int units = a.hd / 16;
    const int hgroups = a.heads < 256 / units ? a.heads : 256 / units;
    const int rows = 256 / (units * hgroups);
    const int64_t blocks = (a.N + rows - 1) / rows;
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
    if (layout == RVQ_ROPE_HALVES)
      hipLaunchKernelGGL((rope_kernel<T, RVQ_ROPE_HALVES>), grid, dim3(256), 0, s, a, hgroups, rows);
    else
      hipLaunchKernelGGL((rope_kernel<T, RVQ_ROPE_ADJACENT>), grid, dim3(256), 0, s, a, hgroups, rows);
    return;
  }
  const int64_t blocks = (a.N * a.heads * (a.hd - a.rot / 2) + 255) / 256;
  hipLaunchKernelGGL((rope_any_kernel<T>), dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), dim3(256), 0, s, a, layout);
}

bool of_align(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

extern "C" {

int rvq_rope_tables(const int64_t *dPositions, int64_t N, int32_t rot, double base, double factor,
                    double orig_len, double alpha, double beta, double amplitude, float *dCos, float *dSin,
                    void *stream) {
  if (N < 0 || rot < 2 || (rot & 1) || rot > 65536) return RVQ_EINVAL;
  if (!(base > 0.0) || !(factor > 0.0) || !(orig_len >= 0.0) || !std::isfinite(base) || !std::isfinite(factor) ||
      !std::isfinite(orig_len) || !std::isfinite((float)amplitude))
    return RVQ_EINVAL;
  if (orig_len > 0.0 && !(std::isfinite(alpha) && std::isfinite(beta) && alpha < beta)) return RVQ_EINVAL;
  if (N == 0) return RVQ_OK;
  if (!dPositions || !dCos || !dSin || !of_align(dPositions, 8) || !of_align(dCos, 4) || !of_align(dSin, 4)) return RVQ_EINVAL;
  if (N > (INT64_MAX / 8) / rot) return RVQ_EINVAL;
  if (!rvq_stream_is_current((hipStream_t)stream)) return RVQ_EINVAL;
  TableArgs a;
  a.pos = dPositions; a.N = N; a.half = rot / 2;
  a.log2_base = std::log2(base);
  a.factor = factor; a.orig_len = orig_len; a.alpha = alpha; a.beta = beta; a.amplitude = amplitude;
  a.cos = dCos; a.sin = dSin;
  // whole multiples of `half` threads, so that a thread stays with its frequency; about four tokens each where
  // there are enough of them (the frequency costs as much as several angles)
  const int64_t total = N * a.half;
  int64_t blocks = (total + 1023) / 1024;
  blocks = blocks < 1 ? 1 : blocks > 4096 ? 4096 : blocks;
  const int64_t unit = a.half / std::__gcd((int64_t)a.half, (int64_t)256);  // blocks that hold whole tokens
  blocks = (blocks + unit - 1) / unit * unit;
  hipLaunchKernelGGL(rope_tables_kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, a);
  return hipGetLastError() == hipSuccess ? RVQ_OK : RVQ_EHIP;
}

int rvq_rope(const void *dX, int32_t dtype, int64_t N, int32_t n_heads, int32_t head_dim, int32_t rot,
             int32_t layout, int64_t ldx, int64_t hsx, const float *dCos, const float *dSin, void *dOut,
             int64_t ldo, int64_t hso, void *stream) {
  if (dtype != RVQ_F32 && dtype != RVQ_BF16 && dtype != RVQ_F16) return RVQ_EINVAL;
  if (layout != RVQ_ROPE_ADJACENT && layout != RVQ_ROPE_HALVES) return RVQ_EINVAL;
  if (N < 0 || n_heads < 1 || n_heads > 65535 || head_dim < 2 || head_dim > 65536) return RVQ_EINVAL;
  if (rot < 2 || (rot & 1) || rot > head_dim) return RVQ_EINVAL;
  if (ldx < 0 || hsx < 0 || ldo < 0 || hso < 0) return RVQ_EINVAL;
  if (N == 0) return RVQ_OK;
  const size_t e = dtype == RVQ_F32 ? 4 : 2;
  if (!dX || !dOut || !dCos || !dSin || !of_align(dX, e) || !of_align(dOut, e) || !of_align(dCos, 4) || !of_align(dSin, 4))
    return RVQ_EINVAL;
  if (!rvq_rows_fit(N, n_heads, head_dim, ldx, hsx) || !rvq_rows_fit(N, n_heads, head_dim, ldo, hso) ||
      !rvq_rows_distinct(N, n_heads, head_dim, ldo, hso))
    return RVQ_EINVAL;
  if (dX == dOut && (ldx != ldo || hsx != hso)) return RVQ_EINVAL;
  if (!rvq_stream_is_current((hipStream_t)stream)) return RVQ_EINVAL;
  RopeArgs a;
  a.x = dX; a.out = dOut; a.cos = dCos; a.sin = dSin;
  a.N = N; a.ldx = ldx; a.hsx = hsx; a.ldo = ldo; a.hso = hso;
  a.heads = n_heads; a.hd = head_dim; a.rot = rot;
  const int64_t any = ldx | hsx | ldo | hso;
  const bool whole = of_align(dX, 16) && of_align(dOut, 16) && of_align(dCos, 16) && of_align(dSin, 16) &&
                     (any * (int64_t)e) % 16 == 0 && rot % 16 == 0 && head_dim % 16 == 0 && head_dim <= 1024;
  hipStream_t s = (hipStream_t)stream;
  if (dtype == RVQ_F32) launch_rope<float>(a, layout, whole, s);
  else if (dtype == RVQ_BF16) launch_rope<__bf16>(a, layout, whole, s);
  else launch_rope<_Float16>(a, layout, whole, s);
  return hipGetLastError() == hipSuccess ? RVQ_OK : RVQ_EHIP;
}

}  // extern "C"
