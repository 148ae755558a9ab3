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

// A unit of a head is 16 channels whose rotation needs nothing else: two groups of eight that begin at c0
// and c1.  Units below rot / 16 hold the pairs 8 u .. 8 u + 7, the others are channels that do not rotate.
template <int LAYOUT> __device__ __forceinline__ void unit_channels(int u, int rot, int &c0, int &c1) {
  if (LAYOUT == RVQ_ROPE_HALVES && 16 * u < rot) {
    c0 = 8 * u;
    c1 = rot / 2 + 8 * u;
  } else {
    c0 = 16 * u;
    c1 = c0 + 8;
  }
}

// One pair in fp32: a product, then a multiply-add, written out so that every kernel rounds alike; the empty statements
// keep the compiler from taking the conversion to a 16-bit type into the multiply-add (fp16 would then skip the fp32 rounding).
__device__ __forceinline__ void rotate_pair(float &a, float &b, float c, float s) {
  const float x = a, y = b;
  a = fmaf(x, c, -(y * s));
  b = fmaf(x, s, y * c);
  asm("" : "+v"(a));
  asm("" : "+v"(b));
}

// the rotation of a unit
template <int LAYOUT>
__device__ __forceinline__ void rotate_unit(float (&a)[8], float (&b)[8], const float (&cs)[8], const float (&sn)[8]) {
  if constexpr (LAYOUT == RVQ_ROPE_HALVES) {
#pragma unroll
    for (int i = 0; i < 8; ++i) rotate_pair(a[i], b[i], cs[i], sn[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      rotate_pair(a[2 * i], a[2 * i + 1], cs[i], sn[i]);
      rotate_pair(b[2 * i], b[2 * i + 1], cs[4 + i], sn[4 + i]);
    }
  }
}

}  // namespace
