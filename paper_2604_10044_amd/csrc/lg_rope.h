// lg_rope.h -- the rotation of a head's values in 16-byte pieces, for the kernels that append (lg_rope.hip,
// lg_fp4_append.hip).
#pragma once

#include "lg_paged_internal.h"

namespace lg {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};
template <>
struct Elem<__bf16> {
  static __device__ __forceinline__ float get(__bf16 x) { return (float)x; }
  static __device__ __forceinline__ __bf16 put(float x) { return (__bf16)x; }  // to nearest, ties to even
};

template <typename T>
union Piece {  // 16 bytes of a head
  u32x4_t u;
  T e[16 / sizeof(T)];
};

enum { kRopeHalf = 0, kRopePairs = 1, kRopeAny = 2 };

// One unit of work on a head: M = kRopeHalf: the pieces at 16 u bytes of both halves of the rotated part,
// or a piece behind it; kRopePairs: a piece; kRopeAny (rotated parts that are no whole pieces): a pair of
// values, or a value behind the rotated part. A pair is read and written by one thread, so dst may be src.
template <typename T, int M, bool ILV>
__device__ __forceinline__ void rope_unit(const T* src, T* dst, int u, int rot, const float* cs) {
  constexpr int E = 16 / sizeof(T);
  const int half = rot / 2;
  const float* sn = cs + 64;
  if constexpr (M == kRopeHalf) {
    Piece<T> x, y;
    if (u * E < half) {
      x.u = *(const u32x4_t*)(src + u * E);
      y.u = *(const u32x4_t*)(src + half + u * E);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float a = Elem<T>::get(x.e[e]), b = Elem<T>::get(y.e[e]);
        const float c = cs[u * E + e], s = sn[u * E + e];
        x.e[e] = Elem<T>::put(a * c - b * s);
        y.e[e] = Elem<T>::put(b * c + a * s);
      }
      *(u32x4_t*)(dst + u * E) = x.u;
      *(u32x4_t*)(dst + half + u * E) = y.u;
    } else {
      *(u32x4_t*)(dst + half + u * E) = *(const u32x4_t*)(src + half + u * E);
    }
  } else if constexpr (M == kRopePairs) {
    Piece<T> x;
    x.u = *(const u32x4_t*)(src + u * E);
    if (u * E < rot) {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float a = Elem<T>::get(x.e[e]), b = Elem<T>::get(x.e[e + 1]);
        const float c = cs[(u * E + e) / 2], s = sn[(u * E + e) / 2];
        x.e[e] = Elem<T>::put(a * c - b * s);
        x.e[e + 1] = Elem<T>::put(b * c + a * s);
      }
    }
    *(u32x4_t*)(dst + u * E) = x.u;
  } else if (u < half) {
    const int i = ILV ? 2 * u : u, j = ILV ? 2 * u + 1 : u + half;
    const float a = Elem<T>::get(src[i]), b = Elem<T>::get(src[j]);
    dst[i] = Elem<T>::put(a * cs[u] - b * sn[u]);
    dst[j] = Elem<T>::put(b * cs[u] + a * sn[u]);
  } else {
    dst[half + u] = src[half + u];
  }
}

}  // namespace lg
