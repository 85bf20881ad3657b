// Rows of fp32 or bf16 features, moved four at a time (VEC: rows are aligned for it) or one by one.
#pragma once
#include "mrt_bf16_tiles.hpp"

namespace mrt {
namespace {

// ---- rows of four features -------------------------------------------------------------------
template <typename T> struct Quad;
template <> struct Quad<float> {
  typedef f32x4 raw;
  static __device__ inline f32x4 widen(raw x) { return x; }
  static __device__ inline float one(float x) { return x; }
};
template <> struct Quad<u16> {
  typedef __attribute__((ext_vector_type(4))) u16 raw;
  static __device__ inline float one(u16 x) { return __uint_as_float((uint32_t)x << 16); }
  static __device__ inline f32x4 widen(raw x) { return f32x4{one(x[0]), one(x[1]), one(x[2]), one(x[3])}; }
};
// features v .. v + 3 of the row at p (the load itself is unconditional); from d on they are zeros, where
// rows are moved by four only once blank4 has seen them
template <bool VEC, typename T>
__device__ inline f32x4 ld4(const T* p, int v, int d) {
  f32x4 x;
  if constexpr (VEC) {
    x = Quad<T>::widen(*(const typename Quad<T>::raw*)(p + (v < d ? v : 0)));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float one = Quad<T>::one(p[v + e < d ? v + e : 0]);
      x[e] = v + e < d ? one : 0.f;
    }
  }
  return x;
}
template <bool VEC>
__device__ inline f32x4 blank4(f32x4 x, int v, int d) {
  return VEC && v >= d ? f32x4{0.f, 0.f, 0.f, 0.f} : x;
}
template <bool VEC>
__device__ inline void st4(float* p, f32x4 x, int v, int d) {
  if constexpr (VEC) {
    if (v < d) *(f32x4*)(p + v) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (v + e < d) p[v + e] = x[e];
  }
}
template <bool VEC>
__device__ inline void st4(u16* p, f32x4 x, int v, int d) {
  if constexpr (VEC) {
    typedef typename Quad<u16>::raw raw;
    if (v < d) *(raw*)(p + v) = raw{f2bf(x[0]), f2bf(x[1]), f2bf(x[2]), f2bf(x[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (v + e < d) p[v + e] = f2bf(x[e]);
  }
}

}  // namespace
}  // namespace mrt
