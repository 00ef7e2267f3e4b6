// Rows in pieces of 16 bytes that begin at any element: a global load or store of four words needs no more than its element's
// alignment on this machine, so rows of odd widths and slices of odd sizes take the same wide accesses as aligned ones, and only the
// last piece of a row that it does not fill goes element by element.
#pragma once
#include "common.h"

namespace hfta {

typedef uint32_t piece_u4 __attribute__((ext_vector_type(4), aligned(2)));

template <typename T> struct Piece16 {
  static constexpr int N = 16 / (int)sizeof(T);
  static __device__ __forceinline__ void load(float (&x)[N], const T* p) { values(x, *reinterpret_cast<const piece_u4*>(p)); }
  // the first n elements; zeros behind them
  static __device__ __forceinline__ void load(float (&x)[N], const T* p, int n) {
    if (n >= N) return load(x, p);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = e < n ? Elem<T>::load(p + e) : 0.f;
  }
  // the same in two steps: what memory holds, and its values
  static __device__ __forceinline__ piece_u4 raw(const T* p, int n) {
    if (n >= N) return *reinterpret_cast<const piece_u4*>(p);
    union { piece_u4 u; T e[N]; } v;
    v.u = piece_u4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) v.e[e] = p[e];
    return v.u;
  }
  static __device__ __forceinline__ void values(float (&x)[N], piece_u4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
      } else {
        x[i] = __uint_as_float(v[i]);
      }
    }
  }
  static __device__ __forceinline__ void store(T* p, const float (&x)[N]) {
    piece_u4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) v[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
      else v[i] = __float_as_uint(x[i]);
    }
    *reinterpret_cast<piece_u4*>(p) = v;
  }
  static __device__ __forceinline__ void store(T* p, const float (&x)[N], int n) {
    if (n >= N) return store(p, x);
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) Elem<T>::store(p + e, x[e]);
  }
};

}  // namespace hfta
