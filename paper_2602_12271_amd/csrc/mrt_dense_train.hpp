// What the kernels of the dense attention's backward pass share: geometry, visibility, units of work.
#pragma once
#include "mrt_internal.hpp"

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

__device__ inline int dense_keys(const DenseBwd& p, int b) {
  if (!p.kv_len) return p.Nkv;
  const int n = p.kv_len[b];
  return n < 0 ? 0 : n < p.Nkv ? n : p.Nkv;
}
// Keys query q sees, a prefix of the `keys` that its sequence has.
__host__ __device__ inline int dense_last_key(const DenseBwd& p, int q, int keys) {
  if (p.cc == 0) return keys;
  const long long lim = (long long)((p.qoff + q / p.hw) / p.cc + 1) * p.cc * p.hw;
  return lim < keys ? (int)lim : keys;
}
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
};
DenseBwdShape bf16_dense_bwd_shape(const DenseBwd& p);
hipError_t launch_bf16_dense_bwd(const DenseBwd& p, hipStream_t s);
DenseBwdShape f32_dense_bwd_shape(const DenseBwd& p);
hipError_t launch_f32_dense_bwd(const DenseBwd& p, int dtype, hipStream_t s);
// sums the parts of dQ, or of dK and dV, into the gradients (`dtype`)
hipError_t launch_dense_bwd_join(const DenseBwd& p, bool kv, int dtype, hipStream_t s);

}  // namespace mrt
