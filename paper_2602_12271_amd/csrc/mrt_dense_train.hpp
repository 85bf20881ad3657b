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
  float* stats;          // [batch][heads][ceil(Nq / 32)][2][32]: -log2(e) lse, -delta (a launch before the tiles' writes them)
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
  bool sums_q, sums_kv;  // dQ, dK and dV are summed from parts
};

// How many workgroups share the streamed rows of a tile of queries and of a tile of keys: what promises the least time by
// this model.  A step takes tq or tkv microseconds where a compute unit has one workgroup, kBeside times that where it has
// two, and a workgroup a step more than it has.  Few workgroups take as long as the longest; more than two a compute unit
// as long as all their steps together and some of the longest, mostly of queries, which come last (steps differ under a
// mask).  Sharing costs a launch that joins the parts, and their bytes; it evens out more than the model knows, so that a
// call without it counts 3 % more.  (Fitted to 41 shapes of 1 to 40 heads, 200 to 14040 tokens, each timed with 20
// to 60 pairs of parts: what it chooses takes 3 % longer than the best pair in the mean.  us of unshared and shared calls:
// 12 heads of 4680 tokens 456 | 428, two to a tile of queries; one head of 4680 tokens 151 | 67, six and seven.)
constexpr double kBeside = 1.6, kLastQueries = 0.25, kLastKeys = 0.06, kJoin = 6.0, kJoinElement = 1.35e-6, kUnshared = 1.03;
constexpr long long kMostPartElements = 1 << 27;      // of all parts together
constexpr int kMostParts = 32, kJoinThreads = 64;
// tile: rows of a workgroup; step: streamed rows
inline DenseBwdShape dense_bwd_shape(const DenseBwd& p, int tile, int step, double tq, double tkv) {
  auto steps = [&](long long n) { return (double)((n + step - 1) / step); };
  auto keys = [&](long long q) { return steps(dense_last_key(p, (int)std::min<long long>(q, p.Nq - 1), p.Nkv)); };
  auto queries = [&](long long k) { return steps((long long)(p.Nq - dense_first_query(p, (int)std::min<long long>(k, p.Nkv - 1))) * p.group); };
  struct Side {
    double tiles, longest, mean, t;
  };
  auto side = [](double tiles, double first, double last, double t) { return Side{tiles, std::max(first, last), 0.5 * (first + last), t}; };
  const Side q = side((double)((p.Nq + tile - 1) / tile) * p.B * p.H, keys(tile - 1), keys(p.Nq - 1), tq);
  const Side k = side((double)((p.Nkv + tile - 1) / tile) * p.B * p.KH, queries(0), queries((p.Nkv - 1) / tile * (long long)tile), tkv);
  const long long eq = (long long)p.B * p.H * p.Nq * p.d, ekv = 2ll * p.B * p.KH * p.Nkv * p.d;
  const double cus = compute_units();
  auto elements = [&](int pq, int pk) { return (pq > 1 ? eq * pq : 0) + (pk > 1 ? ekv * pk : 0); };
  auto time = [&](int pq, int pk) {
    const double lq = (std::ceil(q.longest / pq) + 1) * q.t, lk = (std::ceil(k.longest / pk) + 1) * k.t, longest = std::max(lq, lk);
    const double units = q.tiles * pq + k.tiles * pk, all = q.tiles * (q.mean + pq) * q.t + k.tiles * (k.mean + pk) * k.t;
    const double pair = std::max(0.5 * kBeside * (longest + all / units), longest);
    if (units <= cus) return longest;
    return units <= 2 * cus ? pair : std::max(0.5 * kBeside * all / cus + kLastQueries * lq + kLastKeys * lk, pair);
  };
  DenseBwdShape best = {1, 1, false, false};
  double least = kUnshared * time(1, 1);
  auto look = [&](int pq, int pk) {
    const long long n = elements(pq, pk);
    if (pq < 1 || pk < 1 || pq > kMostParts || pk > kMostParts || n == 0 || n > kMostPartElements) return;
    const double us = time(pq, pk) + kJoin + kJoinElement * n;
    if (us < least) {
      least = us;
      best = {pq, pk, pq > 1, pk > 1};
    }
  };
  // pairs that make workgroups of about one length, or that share tiles of one kind; up to eight workgroups a compute unit
  const double ratio = std::max(k.longest * k.t, 1e-3) / std::max(q.longest * q.t, 1e-3);
  for (int n = 1; n <= kMostParts && 2 * n <= std::max(q.longest, k.longest) && n * std::min(q.tiles, k.tiles) <= 8 * cus; ++n) {
    const double other = ratio >= 1 ? n / ratio : n * ratio;
    for (int m = (int)other; m <= (int)other + 1; ++m) ratio >= 1 ? look(m, n) : look(n, m);
    if (2 * n <= q.longest) look(n, 1);
    if (2 * n <= k.longest) look(1, n);
  }
  return best;
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
// sums the parts of dQ, of dK and dV, or of all three, into them (`dtype`)
hipError_t launch_dense_bwd_join(const DenseBwd& p, bool q, bool kv, int dtype, hipStream_t s);

}  // namespace mrt
