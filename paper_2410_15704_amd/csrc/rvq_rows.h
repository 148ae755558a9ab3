// Moving and rotating rows of fp32 / bf16 / fp16 elements in groups of eight (device code shared by the
// rotation and by the cache of 8-bit codes).
#pragma once

#include "rvq_internal.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Vec4 {
  typedef T type __attribute__((ext_vector_type(4)));
};
template <typename T> struct Vec8;
template <> struct Vec8<__bf16> { typedef bf16x8 type; };
template <> struct Vec8<_Float16> { typedef f16x8 type; };

// eight neighbouring elements as they are (16-byte aligned), and as floats
template <typename T> struct Raw8 { typedef typename Vec8<T>::type type; };
template <> struct Raw8<float> {
  struct type { f32x4 a, b; };
};
template <typename T> __device__ __forceinline__ typename Raw8<T>::type raw8(const T *p) {
  return *reinterpret_cast<const typename Raw8<T>::type *>(p);
}
template <typename T> __device__ __forceinline__ void widen(const typename Raw8<T>::type &x, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
}
template <> __device__ __forceinline__ void widen<float>(const Raw8<float>::type &x, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = x.a[i]; v[4 + i] = x.b[i]; }
}
// eight neighbouring elements, 16-byte aligned
template <typename T> __device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
  const typename Vec8<T>::type x = *reinterpret_cast<const typename Vec8<T>::type *>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
}
template <> __device__ __forceinline__ void load8<float>(const float *p, float (&v)[8]) {
  const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
// one rounding to nearest even
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
  typename Vec8<T>::type x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (T)v[i];
  *reinterpret_cast<typename Vec8<T>::type *>(p) = x;
}
template <> __device__ __forceinline__ void store8<float>(float *p, const float (&v)[8]) {
  f32x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) { a[i] = v[i]; b[i] = v[4 + i]; }
  reinterpret_cast<f32x4 *>(p)[0] = a;
  reinterpret_cast<f32x4 *>(p)[1] = b;
}

// One pair in fp32, right to about a unit of the result's last place: what the first product's rounding lost is added again
// (a difference of products would otherwise lose as many places as it cancels, and a code of three bits behind the leading one,
// whatever its size, sees that).  Written out so that every kernel rounds alike; the empty statements keep the compiler from
// taking a conversion to a 16-bit type into the last addition (fp16 would then skip the fp32 rounding).
__device__ __forceinline__ void rotate_pair(float &a, float &b, float c, float s) {
  const float x = a, y = b;
  const float ys = y * s, yc = y * c;
  // (where a product is infinite, what it lost is no number: any finite one will do, and the median of three gives one)
  constexpr float MOST = 3.402823466e38f;
  const float lost_s = __builtin_amdgcn_fmed3f(fmaf(-y, s, ys), -MOST, MOST), lost_c = __builtin_amdgcn_fmed3f(fmaf(y, c, -yc), -MOST, MOST);
  a = fmaf(x, c, -ys) + lost_s;
  b = fmaf(x, s, yc) + lost_c;
  asm("" : "+v"(a));
  asm("" : "+v"(b));
}

// A unit of a head is 16 channels whose rotation needs nothing else: two groups of eight that begin at c0 and c1.
//   adjacent pairs  the u-th group of each half of the head, four pairs in each: the groups of neighbouring units lie beside
//                   each other in memory
//   halves          the u-th groups of the two halves of what rotates, eight pairs; then 16 neighbouring channels of the rest
// Both need rot and the head's channels in multiples of 16.
template <int LAYOUT> struct Unit {
  int c0, c1, u;
  bool turn0, turn1;
  __device__ __forceinline__ Unit(int unit, int hd, int rot) : u(unit) {
    if (LAYOUT == RVQ_ROPE_HALVES) {
      const bool turns = 16 * u < rot;
      c0 = turns ? 8 * u : 16 * u;
      c1 = c0 + (turns ? rot / 2 : 8);
      turn0 = turn1 = turns;
    } else {
      c0 = 8 * u;
      c1 = hd / 2 + 8 * u;
      turn0 = c0 < rot;
      turn1 = c1 < rot;
    }
  }
  // the entries of a row of tables [.][rot / 2]
  __device__ __forceinline__ void entries(const float *row, float (&e)[8]) const {
    const int p0 = LAYOUT == RVQ_ROPE_HALVES ? 8 * u : c0 / 2, p1 = LAYOUT == RVQ_ROPE_HALVES ? 8 * u + 4 : c1 / 2;
    // (of a unit that does not turn: the first entries, not used; a load under a condition costs more)
    const f32x4 a = *reinterpret_cast<const f32x4 *>(row + (turn0 ? p0 : 0)), b = *reinterpret_cast<const f32x4 *>(row + (turn1 ? p1 : 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) { e[i] = a[i]; e[4 + i] = b[i]; }
  }
  // pair(first channel, second, entry) for every pair that turns
  template <typename Pair> __device__ __forceinline__ void each(float (&a)[8], float (&b)[8], Pair pair) const {
    if constexpr (LAYOUT == RVQ_ROPE_HALVES) {
      if (!turn0) return;
#pragma unroll
      for (int i = 0; i < 8; ++i) pair(a[i], b[i], i);
    } else {
      if (turn0)
#pragma unroll
        for (int i = 0; i < 4; ++i) pair(a[2 * i], a[2 * i + 1], i);
      if (turn1)
#pragma unroll
        for (int i = 0; i < 4; ++i) pair(b[2 * i], b[2 * i + 1], 4 + i);
    }
  }
  __device__ __forceinline__ void rotate(float (&a)[8], float (&b)[8], const float (&cs)[8], const float (&sn)[8]) const {
    each(a, b, [&](float &x, float &y, int i) { rotate_pair(x, y, cs[i], sn[i]); });
  }
};

}  // namespace
