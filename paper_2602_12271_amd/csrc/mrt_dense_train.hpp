// What the kernels of the dense attention's backward pass share: geometry, visibility, units of work.
#pragma once
#include "mrt_internal.hpp"

#include <algorithm>
#include <cmath>

namespace mrt {

// Geometry of one backward call, by value to every kernel.
//
//   S = scale Q K^T      P = exp(S - lse)      dV = P^T dO
//   dP = dO V^T          dS = P (dP - delta)   dQ = scale dS K      dK = scale dS^T Q
//
// with lse the logarithm of the sum of a row's exponentials (of the forward call) and
// delta = sum over features of dO O = sum over keys of P dP.
struct DenseBwd {
  const void *Q, *K, *V, *O, *dO;
  void *dQ, *dK, *dV;
  const float* lse;      // [batch][heads][Nq], natural logarithm; -inf: a row that sees no key
  float* stats;          // [batch][heads][ceil(Nq / 32)][2][32]: -log2(e) lse, -delta (the launch of the queries writes them)
  float *pq, *pk, *pv;   // parts of dQ [part][batch heads][Nq][d], of dK and dV [part][batch kv_heads][Nkv][d]
  mrt_strides q, k, v, o, dout, dq, dk, dv;
  const int* kv_len;     // [batch] or null
  int H, KH, group;      // heads, heads of K and V, heads that share one of them
  int B, d;
  int Nq, Nkv, hw;
  int cc, qoff;          // frames per causal chunk (0: no mask), absolute frame of query frame 0
  int parts_q, parts_kv; // workgroups that share the keys of a query tile, the queries of a key tile
  float scale;
};

// Geometry of a forward call that keeps its row statistics (fp32 products).
struct DenseFwd {
  const void *Q, *K, *V;
  void* O;
  float* lse;
  float* po;             // parts: [part][batch heads][Nq][d] sums of weighted values,
  float2* ml;            //        [part][batch heads][Nq] softmax reference (base 2) and sum of weights
  mrt_strides q, k, v, o;
  const int* kv_len;
  int H, KH, group, B, d;
  int Nq, Nkv, hw;
  int cc, qoff;
  int parts;
  float scale;
};

template <typename P>
__device__ inline int dense_keys(const P& p, int b) {
  if (!p.kv_len) return p.Nkv;
  const int n = p.kv_len[b];
  return n < 0 ? 0 : n < p.Nkv ? n : p.Nkv;
}
// Keys query q sees, a prefix of the `keys` that its sequence has.
template <typename P>
__host__ __device__ inline int dense_last_key(const P& p, int q, int keys) {
  if (p.cc == 0) return keys;
  const long long lim = (long long)((p.qoff + q / p.hw) / p.cc + 1) * p.cc * p.hw;
  return lim < keys ? (int)lim : keys;
}
// Keys that some query of the sequence sees: what the others hold shows nowhere.
__device__ inline int dense_seen_keys(const DenseBwd& p, int b) { return dense_last_key(p, p.Nq - 1, dense_keys(p, b)); }
// First query that sees key k (Nq or more: none).
__host__ __device__ inline int dense_first_query(const DenseBwd& p, int k) {
  if (p.cc == 0) return 0;
  const long long frame = (long long)(k / p.hw / p.cc) * p.cc - p.qoff;
  const long long q = frame * p.hw;
  return q <= 0 ? 0 : q < p.Nq ? (int)q : p.Nq;
}

// Workgroups that share the keys of a query tile, and the queries of a key tile.
struct DenseBwdShape {
  int parts_q, parts_kv;
  bool sums_q;           // dQ is summed from parts, even from one
};

// How many workgroups share the streamed rows of a tile: as many as promise the least time by this model.  A step takes t
// microseconds where a compute unit has one workgroup, 1.5 t where it has two (under a mask a long one and one of mean
// length); a join costs a launch and the parts' bytes.
constexpr long long kMostPartElements = 1 << 27;      // of all parts together
struct DenseShare {
  int parts;
  double us;
};
inline DenseShare dense_share(long long rows, int tile, long long heads, int d, double t, double first, double last, int arrays) {
  const double cus = compute_units(), longest = std::max(first, last), mean = 0.5 * (first + last);
  const long long tiles = (rows + tile - 1) / tile * heads, elements = rows * heads * d * arrays;
  auto time = [&](int parts) {
    const double each = tiles * parts / cus, pairs = std::floor(each / 2), rest = each - 2 * pairs;
    const double rounds = 1.5 * pairs + (rest > 1 ? 1.5 : rest > 0 ? 1.0 : 0.0);
    const double alone = std::ceil(longest / parts), beside = rounds < 1.5 ? alone : 0.75 * (alone + std::ceil(mean / parts));
    const double steps = std::max(beside, rounds > 1.5 ? (mean / parts + 1) * rounds : 0.0);
    return steps * t + (parts > 1 ? 4.0 + 1.3e-6 * elements * parts : 0.0);
  };
  int best = 1;
  double least = time(1) * 0.95;      // (sharing has to promise 5 %)
  for (int parts = 2; parts <= 32 && 2 * parts <= longest && elements * parts <= kMostPartElements; ++parts) {
    const double us = time(parts);
    if (us < least) { least = us; best = parts; }
  }
  return {best, time(best)};
}
// tile: rows of a workgroup; step: streamed rows; tq, tkv: microseconds a step takes
inline DenseBwdShape dense_bwd_shape(const DenseBwd& p, int tile, int step, double tq, double tkv) {
  auto steps = [&](long long n) { return (double)((n + step - 1) / step); };
  auto keys = [&](long long q) { return steps(dense_last_key(p, (int)std::min<long long>(q, p.Nq - 1), p.Nkv)); };
  auto queries = [&](long long k) { return steps((long long)(p.Nq - dense_first_query(p, (int)std::min<long long>(k, p.Nkv - 1))) * p.group); };
  DenseBwdShape shape;
  shape.parts_q = dense_share(p.Nq, tile, (long long)p.B * p.H, p.d, tq, keys(tile - 1), keys(p.Nq - 1), 1).parts;
  shape.parts_kv = dense_share(p.Nkv, tile, (long long)p.B * p.KH, p.d, tkv, queries(0), queries((p.Nkv - 1) / tile * (long long)tile), 2).parts;
  shape.sums_q = shape.parts_q > 1;
  return shape;
}

DenseBwdShape bf16_dense_bwd_shape(const DenseBwd& p);
hipError_t launch_bf16_dense_bwd(const DenseBwd& p, hipStream_t s);
DenseBwdShape f32_dense_bwd_shape(const DenseBwd& p);
// whether rows move as quads (elements of `bytes`)
bool f32_dense_fwd_quads(const DenseFwd& p, size_t bytes);
// fp32 forward calls: workgroups that share a tile's keys, 0 where launch_f32_dense_save takes less time
int f32_dense_fwd_parts(const DenseFwd& p);
hipError_t launch_f32_dense_fwd(const DenseFwd& p, int dtype, hipStream_t s);
hipError_t launch_f32_dense_bwd(const DenseBwd& p, int dtype, hipStream_t s);
// sums the parts of dQ, or of dK and dV, into the gradients (`dtype`)
hipError_t launch_dense_bwd_join(const DenseBwd& p, bool kv, int dtype, hipStream_t s);

}  // namespace mrt
