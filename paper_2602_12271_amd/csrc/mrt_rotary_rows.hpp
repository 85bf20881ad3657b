// What the kernels of rotary positions share: rows in runs of a few elements, the turns of the pairs.
#pragma once
#include "mrt_internal.hpp"

#include <cmath>

namespace mrt {

namespace {

constexpr int kMostPairs = 128;

// (runs of eight fp32 numbers are two accesses of 16 bytes)
template <typename T, int V> struct Run {
  typedef __attribute__((ext_vector_type(V), aligned(V * sizeof(T) < 16 ? V * sizeof(T) : 16))) T type;
};
template <typename T> struct Run<T, 1> { typedef T type; };

template <typename T, int V>
__device__ inline void load_run(const T* at, float (&x)[V]) {
  const typename Run<T, V>::type v = *(const typename Run<T, V>::type*)at;
  if constexpr (V == 1) x[0] = (float)v;
  else {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = (float)v[e];
  }
}
template <typename T, int V>
__device__ inline void store_run(T* at, const float (&x)[V]) {
  typename Run<T, V>::type v;
  if constexpr (V == 1) v = (T)x[0];
  else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = (T)x[e];
  }
  *(typename Run<T, V>::type*)at = v;
}

// turns[p]: of pair p, per position; negative for the inverse
inline void rotary_turns(const mrt_rotary& r, bool inverse, double* turns) {
  // powers of the ladder's ratio in 64 significant bits: a product a pair instead of a pow
  const long double turn = (inverse ? -0.5L : 0.5L) / 3.14159265358979323846264338327950288L;
  const int pairs = r.pairs[0] + r.pairs[1] + r.pairs[2];
  for (int axis = 0, p = 0; axis < 3; ++axis) {
    const int count = r.ladder == MRT_ROTARY_SHARED ? pairs : r.pairs[axis];
    if (r.pairs[axis] == 0) continue;
    const long double ratio = powl((long double)r.theta, -1.0L / count);
    long double at = r.ladder == MRT_ROTARY_SHARED ? turn * powl(ratio, p) : turn;
    for (int i = 0; i < r.pairs[axis]; ++i, at *= ratio) turns[p++] = (double)at;
  }
}

}  // namespace

}  // namespace mrt
